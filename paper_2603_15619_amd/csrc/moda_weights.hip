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

// Sum of acc[i] over the 32 columns (lanes of a half); lane l32 = i of each half gets that of row i.
__device__ __forceinline__ float columns_sum(const float (&acc)[16], int l32) {
  float w = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float a = group_sum<16>(acc[i]);
    const int x = __builtin_bit_cast(int, a);
    auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    a = __builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]);
    if (l32 == i) w = a;
  }
  return w;
}

__device__ __forceinline__ void store_sum(const WeightsParams& p, float* ws, int n_split, int split, int bg, int key, float w) {
  const size_t at = (size_t)bg * p.T_alloc + key;
  if (n_split == 1) p.w_out[at] = (p.w_in ? p.w_in[at] : 0.f) + w;
  else ws[((size_t)split * p.B * p.Hk + bg) * p.T + key] = w;
}

// ---------------------------------------------------------------- fp32
// v_mfma_f32_32x32x2_f32: which channel stands at which place of the contraction is free as long as both operands
// agree, so lane l takes channels 8 i + 4 (l / 32) .. + 3 of row l % 32 in one load, for four instructions.  The four waves
// of a workgroup share its 32 keys and take blocks of 32 queries in turn, the next block's rows in flight.
constexpr int kWfWaves = 4, kWfKeys = 32;

template <int D>
struct RowF32 {
  f32x4 x[D / 8];
  __device__ __forceinline__ void load(const float* row, int hi) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) x[i] = *(const f32x4*)(row + i * 8 + hi * 4);
  }
};

template <int D>
__global__ __launch_bounds__(kWfWaves * 64, 2) void moda_weights_f32_kernel(WeightsParams p, int n_split, float* ws) {
  __shared__ float red[kWfWaves][32];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hi = lane >> 5;
  const int groups = p.B * p.Hk, G = p.Hq / p.Hk;
  const int split = blockIdx.x % n_split, bg = blockIdx.x / n_split % groups, tile = blockIdx.x / n_split / groups;  // (heavy tiles first)
  const int b = bg / p.Hk, g = bg - b * p.Hk;
  const int len = p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
  const int key0 = tile * kWfKeys;
  if (key0 >= len) return;
  const int first = max(0, len - p.window);
  const int t0 = p.causal ? max(first, key0) : first;  // first query that sees a key of the tile
  const int nq = (len - t0 + 31) / 32;
  const long long units = (long long)nq * G;  // blocks of 32 queries: a wave takes every fourth of the workgroup's
  const int u0 = (int)(units * split / n_split), u1 = (int)(units * (split + 1) / n_split);
  RowF32<D> kf, next;
  kf.load((const float*)p.K + ((size_t)bg * p.T_alloc + min(key0 + l32, len - 1)) * D, hi);
  float acc[16], x = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
  auto load = [&](int u) {
    const size_t row = ((size_t)b * p.Hq + g * G + u / nq) * p.T + min(t0 + u % nq * 32 + l32, len - 1);
    next.load((const float*)p.Q + row * D, hi);
    x = p.LSE[row];
  };
  if (u0 + wave < u1) load(u0 + wave);
  for (int u = u0 + wave; u < u1; u += kWfWaves) {
    const int t = t0 + u % nq * 32 + l32;
    const RowF32<D> qf = next;
    // a query that sees nothing has LSE -inf and logits -inf
    const float lse2 = x == -INFINITY ? INFINITY : x * 1.4426950408889634f;
    if (u + kWfWaves < u1) load(u + kWfWaves);  // (uniform)
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
  float w = columns_sum(acc, l32);
  if (l32 < 16) red[wave][(l32 >> 2) * 8 + hi * 4 + (l32 & 3)] = w;
  __syncthreads();
  if (tid < 32 && key0 + tid < len) {
    w = 0.f;
#pragma unroll
    for (int i = 0; i < kWfWaves; ++i) w += red[i][tid];
    store_sum(p, ws, n_split, split, bg, key0 + tid, w);
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
__global__ __launch_bounds__(kWbWaves * 64) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2, D == 64 ? 3 : 2)))
void moda_weights_bf16_kernel(WeightsParams p, int n_tiles, int n_split, int head_group, float* ws) {
  using Tl = Tile<D>;
  constexpr int RB = D * 2, kStage = Tl::kBytes + 256;  // 64 queries, their LSE
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * kStage];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hi = lane >> 5;
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

  f32x16 zero;
#pragma unroll
  for (int i = 0; i < 16; ++i) zero[i] = 0.f;

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
  // The scores of a block and, between its matrix instructions, the sums of the block before it: the matrix pipe works on while the
  // vector ALUs do 16 / kDSteps of those scores per instruction.  (Blocks of scores first, then their sums, two waves per SIMD:
  // B=8 H=16 T=4096 d=128 309 us / so 302; Hq=64 Hk=8 T=16384 d=64 1453 / 1365, of that 1398 with two waves.  Carrying the last
  // block over to the next tile costs registers and gains nothing: 309, 1441.)
  auto product_beside = [&](const bf16x8 (&k)[Tl::kDSteps], const bf16x8 (&q)[Tl::kDSteps], float (&sum)[16], const f32x16& old, float z) {
    constexpr int kPer = 16 / Tl::kDSteps;
    f32x16 s = zero;
#pragma unroll
    for (int st = 0; st < Tl::kDSteps; ++st) {
      s = mfma_bf16(k[st], q[st], s);
#pragma unroll
      for (int i = st * kPer; i < (st + 1) * kPer; ++i) sum[i] += fast_exp2(__builtin_fmaf(old[i], p.scale_log2, -z));
      __builtin_amdgcn_sched_barrier(0);
    }
    return s;
  };
  if (u0 < u1) issue(0);
  int qi = u0 % nq, stage = 0;
  for (int u = u0; u < u1; ++u) {
    const unsigned q_tile = smem_addr + stage * kStage;
    wait_copies();
    __syncthreads();  // the tile is there, and everybody is done with the one before it, whose stage is free
    stage ^= 1;
    if (u + 1 < u1) issue(stage);
    const int q0 = t0 + qi * kWbQueries;
    if (++qi == nq) qi = 0;
    if (p.causal && q0 + kWbQueries <= key0) continue;  // (uniform) no query of the tile sees a key of this wave
    const bool edge = (p.causal && q0 < key0 + 63) || q0 + kWbQueries > len;  // (uniform)
    const unsigned q_row = fa.row + q_tile;
    auto lse2_of = [&](int qb) {
      const float x = *(const float __attribute__((address_space(3)))*)(size_t)(q_tile + Tl::kBytes + (qb * 32 + l32) * 4);
      return x == -INFINITY ? INFINITY : x * 1.4426950408889634f;  // a query that sees nothing: its logits are -inf as well
    };
    auto query_frag = [&](int qb, int st) { return FragAddr<D>::row_frag((unsigned)xor_here((int)q_row, st << 5), qb, 0); };
    if (!edge) {
      const float z[2] = {lse2_of(0), lse2_of(1)};
      bf16x8 qf[2][Tl::kDSteps];
#pragma unroll
      for (int qb = 0; qb < 2; ++qb)
#pragma unroll
        for (int st = 0; st < Tl::kDSteps; ++st) qf[qb][st] = query_frag(qb, st);
      f32x16 before = zero;
#pragma unroll
      for (int st = 0; st < Tl::kDSteps; ++st) before = mfma_bf16(kf[0][st], qf[0][st], before);
#pragma unroll
      for (int blk = 1; blk < 4; ++blk)  // (queries blk / 2, keys blk % 2), beside the sums of the block before
        before = product_beside(kf[blk & 1], qf[blk >> 1], acc[(blk + 1) & 1], before, z[(blk - 1) >> 1]);
      add_block<false>(acc[1], before, p.scale_log2, z[1], 0);
    } else {
#pragma unroll 1
      for (int qb = 0; qb < 2; ++qb) {
        const int t = q0 + qb * 32 + l32;
        const float z = lse2_of(qb);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          f32x16 s = zero;
#pragma unroll
          for (int st = 0; st < Tl::kDSteps; ++st) s = mfma_bf16(kf[kb][st], query_frag(qb, st), s);
          add_block<true>(acc[kb], s, p.scale_log2, z, t >= len ? 1 : p.causal ? key0 + kb * 32 + hi * 4 - t : -32);
        }
      }
    }
  }
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const float w = columns_sum(acc[kb], l32);
    const int key = key0 + kb * 32 + (l32 >> 2) * 8 + hi * 4 + (l32 & 3);
    if (l32 < 16 && key < len) store_sum(p, ws, n_split, split, bg, key, w);
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

// Workgroups that share a tile's queries: enough for a few rounds of the 512 that the chip holds, of at least kLeastUnits
// tiles of queries each (of the longest walk).
constexpr int kLeastUnits = 8;
static int splits(const WeightsParams& p, bool f32) {
  const int keys = f32 ? kWfKeys : kWbKeys, queries = f32 ? 32 : kWbQueries;
  const long long tiles = (long long)p.B * p.Hk * ((p.T + keys - 1) / keys);
  const long long units = (long long)(p.Hq / p.Hk) * ((std::min(p.window, p.T) + queries - 1) / queries);
  const long long want = std::min((2048 + tiles - 1) / tiles, (units + kLeastUnits - 1) / kLeastUnits);
  return (int)std::max(1ll, std::min(want, 256ll));
}

size_t weights_workspace_bytes(const WeightsParams& p, int, bool f32) {
  const int n = splits(p, f32);
  return n > 1 ? (size_t)n * p.B * p.Hk * p.T * sizeof(float) : 0;
}

hipError_t launch_weights(const WeightsParams& p, int d, bool f32, void* workspace, hipStream_t stream) {
  const long long groups = (long long)p.B * p.Hk;
  const int keys = f32 ? kWfKeys : kWbKeys, tiles = (p.T + keys - 1) / keys, n = splits(p, f32), chunks = (p.T + 255) / 256;
  if (!grid_ok(groups * tiles * n, kWbWaves * 64) || !grid_ok(groups * chunks, 256)) return kGridTooLarge;
  const dim3 grid((unsigned)(groups * tiles * n)), block(kWbWaves * 64);
  static_assert(kWfWaves == kWbWaves, "one block size");
  // key/value heads that a die walks together: with more of them their heavy first tiles start together and the light ones are left
  // for the end, with fewer their queries stay in its 4 MB L2.  16 MB of queries: B=8 H=16 T=4096 d=128 338 us, 4 MB 344, 1 MB 390.
  int hg = 0;
  if (groups % 8 == 0) {
    const long long fit = (16ll << 20) / ((long long)p.Hq / p.Hk * p.T * d * 2);
    for (hg = 1; hg * 2 <= fit && groups / 8 % (hg * 2) == 0;) hg *= 2;
  }
  hipError_t e;
  if (f32) e = launch_kernel(d == 128 ? moda_weights_f32_kernel<128> : moda_weights_f32_kernel<64>, grid, block, stream, p, n, (float*)workspace);
  else e = launch_kernel(d == 128 ? moda_weights_bf16_kernel<128> : moda_weights_bf16_kernel<64>, grid, block, stream, p, tiles, n, hg, (float*)workspace);
  if (e == hipSuccess && n > 1)
    e = launch_kernel(moda_weights_add_kernel, dim3((unsigned)(groups * chunks)), dim3(256), stream, p, n, chunks, (const float*)workspace);
  return e;
}

}  // namespace moda
