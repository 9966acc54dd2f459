// The attention weight that every key of a prompt has gathered:
//     W[b,g,j] = sum over the heads h of g and the queries t that see j of exp(scale <q_t, k_j> - LSE_t).
// The LSE is known, so there is no running reference: one matrix product, one exponential and one addition per pair.
// A wave owns 32 or 64 keys (rows of S = K Q^T, fragments in registers) and walks queries of the heads of its
// group: a lane's column is one query, whose LSE it holds, and its 16 scores belong to 16 keys, whose sums
// it keeps in fp32 registers.  The 32 columns are added once, at the end.  Where key tiles are few, the queries
// of a tile are dealt out to several workgroups, whose sums a second kernel adds: no atomics, one order.
#include <algorithm>

#include "moda_launch.h"
#include "moda_tile.h"

namespace moda {

constexpr int kWtWaves = 4;
constexpr int kWtKeys = kWtWaves * 32;  // keys of a workgroup

// ---------------------------------------------------------------- fp32
// v_mfma_f32_32x32x2_f32: which channel stands at which place of the contraction is free as long as both operands
// agree, so lane l takes channels 8 i + 4 (l / 32) .. + 3 of row l % 32 in one load, for four instructions.
template <int D>
struct RowF32 {
  f32x4 x[D / 8];
  __device__ __forceinline__ void load(const float* row, int hi) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) x[i] = *(const f32x4*)(row + i * 8 + hi * 4);
  }
};

template <int D>
__global__ __launch_bounds__(kWtWaves * 64) void moda_weights_f32_kernel(WeightsParams p, int n_tiles) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, hi = lane >> 5;
  const int bg = blockIdx.x / n_tiles, b = bg / p.Hk, g = bg - b * p.Hk, G = p.Hq / p.Hk;
  const int len = p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
  const int key0 = (blockIdx.x % n_tiles) * kWtKeys + wave * 32;
  if (key0 >= len) return;
  const int first = max(0, len - p.window);
  const int t0 = p.causal ? max(first, key0) : first;  // first query that sees a key of this wave
  RowF32<D> kf;
  kf.load((const float*)p.K + ((size_t)bg * p.T_alloc + min(key0 + l32, len - 1)) * D, hi);
  float acc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
  for (int h = g * G; h < g * G + G; ++h) {
    const size_t head = ((size_t)b * p.Hq + h) * p.T;
    for (int q0 = t0; q0 < len; q0 += 32) {
      const int t = q0 + l32, tc = min(t, len - 1);
      RowF32<D> qf;
      qf.load((const float*)p.Q + (head + tc) * D, hi);
      const float x = p.LSE[head + tc];
      // a query behind the end counts nothing; one that sees nothing has LSE -inf and logits -inf
      const float lse2 = x == -INFINITY ? INFINITY : x * 1.4426950408889634f;
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 8; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.x[i][c], qf.x[i][c], s, 0, 0, 0);
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

// ---------------------------------------------------------------- bf16
constexpr int kWbWaves = 4, kWbKeys = kWbWaves * 64, kWbQueries = 64;

// exp2(s c2 - lse2) of a 32 x 32 block, added to its keys' sums.  EDGE: not every query of the block sees every key; key i of
// the lane counts if ahead + i <= 0.
template <bool EDGE>
__device__ __forceinline__ void add_block(float (&acc)[16], const f32x16& s, float c2, float lse2, int ahead) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float e = fast_exp2(__builtin_fmaf(s[i], c2, -lse2));
    acc[i] += !EDGE || ahead + (i >> 2) * 8 + (i & 3) <= 0 ? e : 0.f;
  }
}

template <int D>
__global__ __launch_bounds__(kWbWaves * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))
void moda_weights_bf16_kernel(WeightsParams p, int n_tiles, int n_split, int head_group, float* ws) {
  using Tl = Tile<D>;
  constexpr int RB = D * 2, kStage = Tl::kBytes + 256;  // 64 queries, their LSE
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * kStage + 512];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, hi = lane >> 5;
  const int G = p.Hq / p.Hk;
  int bg, pos;
  head_blocked_id(blockIdx.x, p.B * p.Hk, n_tiles * n_split, bg, pos, head_group);
  const int tile = pos / n_split, split = pos % n_split;
  const int b = bg / p.Hk, g = bg - b * p.Hk;
  const int len = p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
  if (tile * kWbKeys >= len) return;
  const int key0 = tile * kWbKeys + wave * 64;  // (may lie behind the sequence: nothing is stored then)
  const int first = max(0, len - p.window);
  const int t0 = p.causal ? max(first, tile * kWbKeys) : first;  // first query that sees a key of the tile
  const int nq = (len - t0 + kWbQueries - 1) / kWbQueries;       // tiles of queries per head, >= 1
  const long long units = (long long)nq * G;
  const int u0 = (int)(units * split / n_split), u1 = (int)(units * (split + 1) / n_split);

  bf16x8 kf[2][Tl::kDSteps];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const char* row = (const char*)p.K + ((size_t)bg * p.T_alloc + min(key0 + kb * 32 + l32, len - 1)) * RB + hi * 16;
#pragma unroll
    for (int st = 0; st < Tl::kDSteps; ++st) kf[kb][st] = *(const bf16x8*)(row + st * 32);
  }
  float acc[2][16];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[kb][i] = 0.f;

  TileLoader<D, kWbWaves> loader;
  loader.init(wave, lane);
  FragAddr<D> fa;
  fa.init(lane);
  const unsigned smem_addr = (unsigned)(size_t)(lds_ptr)smem;
  // rows from the sequence's length on lie outside the buffers: they read as zeros
  int h_next = g * G + u0 / nq, qi_next = u0 % nq;
  auto issue = [&](int stage) {
    const size_t head = (size_t)b * p.Hq + h_next;
    const int q0 = t0 + qi_next * kWbQueries;
    loader.issue(make_tile_buffer((const char*)p.Q + head * p.T * RB, (unsigned)len * (unsigned)RB), q0, smem_addr + stage * kStage);
    if (wave == 0)
      copy4(make_tile_buffer(p.LSE + head * p.T, (unsigned)len * 4u), lane * 4, q0 * 4, smem_addr + stage * kStage + Tl::kBytes);
    if (++qi_next == nq) {
      qi_next = 0;
      ++h_next;
    }
  };
  if (u0 < u1) issue(0);
  int qi = u0 % nq;
  for (int u = u0; u < u1; ++u) {
    const int stage = (u - u0) & 1;
    const unsigned q_tile = smem_addr + stage * kStage;
    wait_copies();
    __syncthreads();  // the tile is there, and everybody is done with the other one
    if (u + 1 < u1) issue(stage ^ 1);
    const int q0 = t0 + qi * kWbQueries;
    if (++qi == nq) qi = 0;
    if (p.causal && q0 + kWbQueries <= key0) continue;  // (uniform) no query of the tile sees a key of this wave
    const bool edge = (p.causal && q0 < key0 + 63) || q0 + kWbQueries > len;  // (uniform)
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      const float x = *(const float __attribute__((address_space(3)))*)(size_t)(q_tile + Tl::kBytes + (qb * 32 + l32) * 4);
      const int t = q0 + qb * 32 + l32;
      // a query that sees nothing has LSE -inf and logits -inf
      const float lse2 = x == -INFINITY ? INFINITY : x * 1.4426950408889634f;
      f32x16 s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
      for (int st = 0; st < Tl::kDSteps; ++st) {
        const bf16x8 qf = FragAddr<D>::row_frag((unsigned)xor_here((int)(fa.row + q_tile), st << 5), qb, 0);
        s[0] = mfma_bf16(kf[0][st], qf, s[0]);
        s[1] = mfma_bf16(kf[1][st], qf, s[1]);
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        if (edge) add_block<true>(acc[kb], s[kb], p.scale_log2, lse2, t >= len ? 1 : p.causal ? key0 + kb * 32 + hi * 4 - t : -32);
        else add_block<false>(acc[kb], s[kb], p.scale_log2, lse2, 0);
      }
    }
  }
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    float w = 0.f;  // lane l32 = i of each half stores key i
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float a = group_sum<16>(acc[kb][i]);
      const int x = __builtin_bit_cast(int, a);
      auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
      a = __builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]);
      if (l32 == i) w = a;
    }
    const int key = key0 + kb * 32 + (l32 >> 2) * 8 + hi * 4 + (l32 & 3);
    if (l32 < 16 && key < len) {
      const size_t at = (size_t)bg * p.T_alloc + key;
      if (n_split == 1) p.w_out[at] = (p.w_in ? p.w_in[at] : 0.f) + w;
      else ws[((size_t)split * p.B * p.Hk + bg) * p.T + key] = w;
    }
  }
}

// The splits' sums, in their order.
__global__ __launch_bounds__(256) void moda_weights_add_kernel(WeightsParams p, int n_split, int n_chunks, const float* ws) {
  const int bg = blockIdx.x / n_chunks, j = (blockIdx.x % n_chunks) * 256 + threadIdx.x, b = bg / p.Hk;
  if (j >= (p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T)) return;
  const size_t at = (size_t)bg * p.T_alloc + j;
  float w = 0.f;
  for (int s = 0; s < n_split; ++s) w += ws[((size_t)s * p.B * p.Hk + bg) * p.T + j];
  p.w_out[at] = (p.w_in ? p.w_in[at] : 0.f) + w;
}

// Workgroups that share a tile's queries: enough for a few rounds of the 512 that the chip holds, of at least
// kLeastUnits tiles of queries each (of the longest walk).
constexpr int kLeastUnits = 8;
static int splits(const WeightsParams& p) {
  const long long tiles = (long long)p.B * p.Hk * ((p.T + kWbKeys - 1) / kWbKeys);
  const long long units = (long long)(p.Hq / p.Hk) * ((std::min(p.window, p.T) + kWbQueries - 1) / kWbQueries);
  const long long want = std::min((2048 + tiles - 1) / tiles, (units + kLeastUnits - 1) / kLeastUnits);
  return (int)std::max(1ll, std::min(want, 256ll));
}

size_t weights_workspace_bytes(const WeightsParams& p, int, bool f32) {
  const int n = f32 ? 1 : splits(p);
  return n > 1 ? (size_t)n * p.B * p.Hk * p.T * sizeof(float) : 0;
}

hipError_t launch_weights(const WeightsParams& p, int d, bool f32, void* workspace, hipStream_t stream) {
  const long long groups = (long long)p.B * p.Hk;
  if (f32) {
    const int tiles = (p.T + kWtKeys - 1) / kWtKeys;
    if (!grid_ok(groups * tiles, kWtWaves * 64)) return kGridTooLarge;
    return launch_kernel(d == 128 ? moda_weights_f32_kernel<128> : moda_weights_f32_kernel<64>, dim3((unsigned)(groups * tiles)),
                         dim3(kWtWaves * 64), stream, p, tiles);
  }
  const int tiles = (p.T + kWbKeys - 1) / kWbKeys, n = splits(p), chunks = (p.T + 255) / 256;
  if (!grid_ok(groups * tiles * n, kWbWaves * 64) || !grid_ok(groups * chunks, 256)) return kGridTooLarge;
  // heads that a die walks together: as many as have their queries (of all heads of the group) in its 4 MB L2
  int hg = 0;
  if (groups % 8 == 0) {
    const long long fit = (4ll << 20) / ((long long)p.Hq / p.Hk * p.T * d * 2);
    for (hg = 1; hg * 2 <= fit && groups / 8 % (hg * 2) == 0;) hg *= 2;
  }
  hipError_t e = launch_kernel(d == 128 ? moda_weights_bf16_kernel<128> : moda_weights_bf16_kernel<64>,
                               dim3((unsigned)(groups * tiles * n)), dim3(kWbWaves * 64), stream, p, tiles, n, hg, (float*)workspace);
  if (e == hipSuccess && n > 1)
    e = launch_kernel(moda_weights_add_kernel, dim3((unsigned)(groups * chunks)), dim3(256), stream, p, n, chunks, (const float*)workspace);
  return e;
}

}  // namespace moda
