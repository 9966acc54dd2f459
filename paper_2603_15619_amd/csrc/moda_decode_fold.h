// Folding the softmax states of a wave's groups of lanes, for the decoding kernels: a group of d/8 lanes holds the
// state of the key rows that it walks (reference, normaliser, eight output channels per lane).
#pragma once
#include "moda_common.h"

namespace moda {

// Two registers of which one's lanes 32.. and the other's lanes ..31 change places, added; the same with odd and even
// rows of 16 lanes.
__device__ __forceinline__ float swap_add32(float a, float b) {
  auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(int, a), __builtin_bit_cast(int, b), false, false);
  return __builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]);
}
__device__ __forceinline__ float swap_add16(float a, float b) {
  auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(int, a), __builtin_bit_cast(int, b), false, false);
  return __builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]);
}
// Sum and maximum over a wave's groups of LPR lanes: every lane gets that of the lanes at its place.
template <int LPR>
__device__ __forceinline__ float groups_sum(float x) {
  if (LPR <= 8) x += dpp_mov<0x128>(x);  // row_ror:8
  if (LPR == 4) x += dpp_mov<0x124>(x);  // row_ror:4
  return pair_sum(swap_add16(x, x));
}
template <int LPR>
__device__ __forceinline__ float groups_max(float x) {
  if (LPR <= 8) x = fmaxf(x, dpp_mov<0x128>(x));
  if (LPR == 4) x = fmaxf(x, dpp_mov<0x124>(x));
  const int i = __builtin_bit_cast(int, x);
  auto r = __builtin_amdgcn_permlane16_swap(i, i, false, false);
  return pair_max(fmaxf(__builtin_bit_cast(float, (int)r[0]), __builtin_bit_cast(float, (int)r[1])));
}

// A wave's state of one head, of its groups of LPR lanes (their references, normalisers, eight channels each), folded and
// written to red[0 .. D) (channels), red[D] (reference), red[D + 1] (normaliser).  Every exchange halves the channels that a
// lane holds.
template <int D>
__device__ __forceinline__ void fold_groups(float m, float l, const float (&o)[8], float c2, int lane, float* red) {
  constexpr int LPR = D / 8;
  const float mm = groups_max<LPR>(m);
  const float f = m == -INFINITY ? 0.f : fast_exp2((m - mm) * c2);
  const float ll = groups_sum<LPR>(l * f);
  float half[4], quarter[2];
#pragma unroll
  for (int k = 0; k < 4; ++k) half[k] = swap_add32(o[k] * f, o[k + 4] * f);  // lanes < 32: channel k, others k + 4
#pragma unroll
  for (int k = 0; k < 2; ++k) {  // even rows of 16 lanes: channel k, odd ones k + 2 of those
    quarter[k] = swap_add16(half[k], half[k + 2]);
    if (LPR == 8) quarter[k] += dpp_mov<0x128>(quarter[k]);
  }
  if ((lane & 15) < LPR)
    *(f32x2*)&red[lane % LPR * 8 + (lane >> 5) * 4 + ((lane >> 4) & 1) * 2] = (f32x2){quarter[0], quarter[1]};
  if (lane == 0) *(f32x2*)&red[D] = (f32x2){mm, ll};
}

// The same of groups of D / 16 lanes, sixteen channels per lane.
template <int D>
__device__ __forceinline__ void fold_groups(float m, float l, const float (&o)[16], float c2, int lane, float* red) {
  constexpr int LPR = D / 16;
  const float mm = groups_max<LPR>(m);
  const float f = m == -INFINITY ? 0.f : fast_exp2((m - mm) * c2);
  const float ll = groups_sum<LPR>(l * f);
  float half[8];
  f32x4 quarter;
#pragma unroll
  for (int k = 0; k < 8; ++k) half[k] = swap_add32(o[k] * f, o[k + 8] * f);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float x = swap_add16(half[k], half[k + 4]);
    x += dpp_mov<0x128>(x);
    if (LPR == 4) x += dpp_mov<0x124>(x);
    quarter[k] = x;
  }
  float* to = red + lane % LPR * 16 + (lane >> 5) * 8 + ((lane >> 4) & 1) * 4;  // (D + 2 floats a state: 8-byte aligned)
  if ((lane & 15) < LPR) {
    *(f32x2*)to = (f32x2){quarter[0], quarter[1]};
    *(f32x2*)(to + 2) = (f32x2){quarter[2], quarter[3]};
  }
  if (lane == 0) *(f32x2*)&red[D] = (f32x2){mm, ll};
}

// (reference, normaliser) of query j's waves, whose states lie in red as fold_groups writes them, and channel ch's sum.
template <int D, int GT, int WAVES>
__device__ __forceinline__ f32x2 fold_rows(const float* red, int j, int ch, float c2, float& oo) {
  float mm = -INFINITY, ll = 0.f;
  oo = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) mm = fmaxf(mm, red[(w * GT + j) * (D + 2) + D]);
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const float* x = red + (w * GT + j) * (D + 2);
    const float f = x[D] == -INFINITY ? 0.f : fast_exp2((x[D] - mm) * c2);
    ll += f * x[D + 1];
    oo += f * x[ch];
  }
  return (f32x2){mm, ll};
}

// Rows of sequence i that `lengths` (null: all) gives.
__device__ __forceinline__ int filled(const int* lengths, int i, int most) {
  return lengths ? min(max(lengths[i], 0), most) : most;
}

}  // namespace moda
