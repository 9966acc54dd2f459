// Shared by the kernels on a paged sequence cache (gfx950): where a page lies, and its 8-bit form.
//
// A page holds 2^shift rows (16 to 256) of every key/value head: row s of head g of page i lies at ((i * Hk + g) << shift) + s.  A wave's
// load takes 4 to 16 adjacent rows, which never leave a page, so that a page's number is uniform over the wave and its rows are read
// through a buffer of its own, whose size is what the sequence has filled of the page: rows behind that, and pages that the
// table does not give, read as zeros and fetch nothing.
//
// 8 bits: e4m3 codes with a power-of-two scale per 32 channels of a row, stored as its exponent + 127.  e = the least exponent, -100 or
// more, with max |x| <= 448 * 2^e; a code stands for code * 2^e, a number that bf16 holds exactly.  Rounding x * 2^-e to
// e4m3 (nearest even) is the only rounding: off by 2^-4 of the value at most, or 2^-10 * 2^e for values below 2^-6 * 2^e.
#pragma once
#include "moda_decode_fold.h"
#include "moda_launch.h"

namespace moda {

constexpr int kBlock = 32;              // channels that share a scale
constexpr int kScaleBias = 127;         // a scale byte less this: the exponent
constexpr int kLeastByte = 127 - 100;   // (below, values would leave bf16's normal range)
constexpr int kMostByte = 247;          // that of the largest finite bf16 values: codes above 240 would stand for 2^128
constexpr unsigned kBufferFlags = 0x00020000;  // raw buffer, 32-bit untyped data

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_buffer(const void* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, bytes, kBufferFlags);
}

// 2^(byte - 127) for a byte of 1 or more.
__device__ __forceinline__ float scale_of(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }

// Channels 2 i, 2 i + 1 of four codes in a dword, as bf16 (exact) or fp32.
template <bool HI>
__device__ __forceinline__ uint32_t codes_bf16(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
}
template <bool HI>
__device__ __forceinline__ f32x2 codes_f32(uint32_t codes, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, HI);
}

// Sums over a wave's lanes up to and with the own one, of non-negative numbers (in registers: a shuffle through LDS takes ten times as long).
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_or_zero(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int row_scan(int x) {  // over the lanes of a row of 16
  x += dpp_or_zero<0x111, 0xf>(x);  // row_shr:1
  x += dpp_or_zero<0x112, 0xf>(x);
  x += dpp_or_zero<0x114, 0xf>(x);
  x += dpp_or_zero<0x118, 0xf>(x);
  return x;
}
__device__ __forceinline__ int wave_scan(int x) {
  x = row_scan(x);
  x += dpp_or_zero<0x142, 0xa>(x);  // row_bcast:15 to rows 1 and 3
  x += dpp_or_zero<0x143, 0xc>(x);  // row_bcast:31 to rows 2 and 3
  return x;
}

// The largest of a wave's numbers, in its last lane.
__device__ __forceinline__ unsigned wave_max(unsigned x) {
  x = max(x, (unsigned)dpp_or_zero<0x111, 0xf>((int)x));
  x = max(x, (unsigned)dpp_or_zero<0x112, 0xf>((int)x));
  x = max(x, (unsigned)dpp_or_zero<0x114, 0xf>((int)x));
  x = max(x, (unsigned)dpp_or_zero<0x118, 0xf>((int)x));
  x = max(x, (unsigned)dpp_or_zero<0x142, 0xa>((int)x));
  return max(x, (unsigned)dpp_or_zero<0x143, 0xc>((int)x));
}

// The physical page of logical page i of a sequence whose row of the table is `table`; -1: none.
__device__ __forceinline__ int page_at(const int* table, int i, int n_pages) {
  const int id = table[i];
  return (unsigned)id < (unsigned)n_pages ? id : -1;
}

}  // namespace moda
