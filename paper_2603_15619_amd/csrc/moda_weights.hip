// The attention weight that every key of a prompt has gathered:
//     W[b,g,j] = sum over the heads h of g and the queries t that see j of exp(scale <q_t, k_j> - LSE_t).
// The LSE is known, so there is no running reference: one matrix product, one exponential and one addition per pair.
// A wave owns 32 keys (rows of S = K Q^T, fragments in registers) and walks all queries of all heads of its group, 32
// at a time: a lane's column is one query, whose LSE it holds, and its 16 scores belong to 16 keys, whose sums
// it keeps in fp32 registers.  The 32 columns are added once, at the end: no atomics, one order.
#include <algorithm>

#include "moda_launch.h"
#include "moda_tile.h"

namespace moda {

constexpr int kWtWaves = 4;
constexpr int kWtKeys = kWtWaves * 32;  // keys of a workgroup

// Fragments of 32 rows for S = K Q^T.  bf16: v_mfma_f32_32x32x16_bf16, lane l holds channels 16 i + 8 (l / 32) .. + 7 of
// row l % 32.  fp32: v_mfma_f32_32x32x2_f32, four at a time; which channel stands at which place of the contraction
// is free as long as both operands agree, so a lane takes channels 8 i + 4 (l / 32) .. + 3.
template <int D, bool F32>
struct RowFrag {
  static constexpr int kN = F32 ? D / 8 : D / 16;
  static constexpr int RB = D * (F32 ? 4 : 2);
  u32x4 x[kN];
  __device__ __forceinline__ void load(const char* row, int hi) {
#pragma unroll
    for (int i = 0; i < kN; ++i) x[i] = *(const u32x4*)(row + i * 32 + hi * 16);
  }
};
template <int D, bool F32>
__device__ __forceinline__ f32x16 product(const RowFrag<D, F32>& k, const RowFrag<D, F32>& q) {
  f32x16 s;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
  for (int i = 0; i < RowFrag<D, F32>::kN; ++i) {
    if constexpr (F32) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(float, (unsigned)k.x[i][c]),
                                                 __builtin_bit_cast(float, (unsigned)q.x[i][c]), s, 0, 0, 0);
    } else {
      s = mfma_bf16(__builtin_bit_cast(bf16x8, k.x[i]), __builtin_bit_cast(bf16x8, q.x[i]), s);
    }
  }
  return s;
}

template <int D, bool F32>
__global__ __launch_bounds__(kWtWaves * 64) void moda_weights_kernel(WeightsParams p, int n_tiles) {
  constexpr int RB = RowFrag<D, F32>::RB;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, hi = lane >> 5;
  const int bg = blockIdx.x / n_tiles, b = bg / p.Hk, g = bg - b * p.Hk, G = p.Hq / p.Hk;
  const int len = p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
  const int key0 = (blockIdx.x % n_tiles) * kWtKeys + wave * 32;
  if (key0 >= len) return;
  const int first = max(0, len - p.window);
  const int t0 = p.causal ? max(first, key0) : first;  // first query that sees a key of this wave
  RowFrag<D, F32> kf;
  kf.load((const char*)p.K + ((size_t)bg * p.T_alloc + min(key0 + l32, len - 1)) * RB, hi);
  float acc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
  for (int h = g * G; h < g * G + G; ++h) {
    const char* qb = (const char*)p.Q + ((size_t)b * p.Hq + h) * p.T * RB;
    const float* lse = p.LSE + ((size_t)b * p.Hq + h) * p.T;
    for (int q0 = t0; q0 < len; q0 += 32) {
      const int t = q0 + l32, tc = min(t, len - 1);
      RowFrag<D, F32> qf;
      qf.load(qb + (size_t)tc * RB, hi);
      const float x = lse[tc];
      // a query that sees nothing has LSE -inf and logits -inf
      const float lse2 = x == -INFINITY ? INFINITY : x * 1.4426950408889634f;
      const f32x16 s = product(kf, qf);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = key0 + (i >> 2) * 8 + hi * 4 + (i & 3);
        const bool seen = t < len && (!p.causal || t >= key);
        acc[i] += seen ? fast_exp2(s[i] * p.scale_log2 - lse2) : 0.f;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
#pragma unroll
    for (int x = 1; x < 32; x *= 2) acc[i] += __shfl_xor(acc[i], x);
  }
  float w = 0.f;  // lane l32 = i of each half stores key i
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (l32 == i) w = acc[i];
  const int key = key0 + (l32 >> 2) * 8 + hi * 4 + (l32 & 3);
  if (l32 < 16 && key < len) {
    const size_t at = (size_t)bg * p.T_alloc + key;
    p.w_out[at] = (p.w_in ? p.w_in[at] : 0.f) + w;
  }
}

size_t weights_workspace_bytes(const WeightsParams&, int, bool) { return 0; }

hipError_t launch_weights(const WeightsParams& p, int d, bool f32, void*, hipStream_t stream) {
  const int tiles = (p.T + kWtKeys - 1) / kWtKeys;
  const long long blocks = (long long)p.B * p.Hk * tiles;
  if (!grid_ok(blocks, kWtWaves * 64)) return kGridTooLarge;
  return launch_kernel(d == 128 ? (f32 ? moda_weights_kernel<128, true> : moda_weights_kernel<128, false>)
                                : (f32 ? moda_weights_kernel<64, true> : moda_weights_kernel<64, false>),
                       dim3((unsigned)blocks), dim3(kWtWaves * 64), stream, p, tiles);
}

}  // namespace moda
