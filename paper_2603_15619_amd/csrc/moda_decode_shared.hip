// Decoding step of a batch whose sequences share prefixes and differ in length, with the attention weight of every row of
// the own caches added to an accumulator where the caller keeps one.
//
// With the logits x_c = scale <q, k_c> of a token's prefix rows, own rows and slots,
//     m = max x,  l = sum exp(x_c - m),  O = (1/l) sum exp(x_c - m) v_c,  LSE = m + ln l,
//     weights_out[j] = weights_in[j] + sum over the heads of a group of exp(x_j - LSE).
// (m, l, unnormalised O) of disjoint sets of rows merge exactly, so the rows are cut into slices over workgroups, whose
// states go to the workspace in fp32, and a second kernel merges them.  Where weights are asked for, the own
// rows' logits go there too (4 bytes per row and head, where a row of K and V is 4 d), since no slice knows the LSE.
#include <algorithm>

#include "moda_decode_fold.h"
#include "moda_launch.h"

namespace moda {

constexpr int kShWaves = 4;

__device__ __forceinline__ int filled(const int* lengths, int i, int most) {
  return lengths ? min(max(lengths[i], 0), most) : most;
}

// One workgroup = (batch, key/value head, chunk of GT query heads, slice): slices of the prefix, of the own cache, the slots.
// A lane owns 8 channels, d/8 lanes a row, as in moda_decode_partial_kernel.
template <int D, int GT>
__global__ __launch_bounds__(kShWaves * 64) void moda_shared_rows_kernel(SharedParams p) {
  constexpr int LPR = D / 8, RPS = 64 / LPR, RB = D * 2;
  __shared__ __attribute__((aligned(16))) float red[kShWaves][GT][D + 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int rg = lane / LPR, l16 = lane % LPR;
  const int G = p.Hq / p.Hk;
  const int n_gc = (G + GT - 1) / GT;
  int id = blockIdx.x;
  const int slice = id % p.n_slices;
  id /= p.n_slices;
  const int gc = id % n_gc, bg = id / n_gc;
  const int b = bg / p.Hk, g = bg - b * p.Hk;
  const int h0 = g * G + gc * GT;
  const float c2 = p.scale_log2;

  // the slice's rows [k_begin, k_end) of a slab
  const char *Kb, *Vb;
  int k_begin, k_end;
  const bool own = slice >= p.n_prefix && slice < p.n_prefix + p.n_own;
  if (slice < p.n_prefix) {
    const int x = b / (p.B / p.Np);
    const size_t slab = ((size_t)x * p.Hk + g) * p.P_alloc * RB;
    Kb = (const char*)p.Kp + slab;
    Vb = (const char*)p.Vp + slab;
    k_begin = slice * p.prefix_per;
    k_end = min(filled(p.prefix_lengths, x, p.P), k_begin + p.prefix_per);
  } else if (own) {
    const size_t slab = (size_t)bg * p.T_alloc * RB;
    Kb = (const char*)p.Ks + slab;
    Vb = (const char*)p.Vs + slab;
    k_begin = (slice - p.n_prefix) * p.own_per;
    k_end = min(filled(p.lengths, b, p.T), k_begin + p.own_per);
  } else {
    const size_t slab = (size_t)bg * p.depth_alloc * RB;
    Kb = (const char*)p.Kd + slab;
    Vb = (const char*)p.Vd + slab;
    k_begin = 0;
    k_end = p.depth_count;
  }
  float* scores = own && p.w_out ? p.scores + ((size_t)b * p.Hq + h0) * p.T : nullptr;

  u32x4 q[GT];
  float m[GT], l[GT], o[GT][8];
#pragma unroll
  for (int j = 0; j < GT; ++j) {
    const int h = min(h0 + j, g * G + G - 1);  // heads past the group repeat the last one; never stored
    q[j] = *(const u32x4*)((const char*)p.Q + ((size_t)b * p.Hq + h) * RB + l16 * 16);
    m[j] = -INFINITY;
    l[j] = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) o[j][k] = 0.f;
  }
  constexpr int STEP = kShWaves * RPS;
  for (int key = k_begin + wave * RPS + rg; key - rg < k_end; key += STEP) {  // (uniform over a wave)
    const bool in = key < k_end;
    const size_t at = (size_t)min(key, k_end - 1) * RB + l16 * 16;
    const u32x4 kv = *(const u32x4*)(Kb + at);
    u32x4 vv = *(const u32x4*)(Vb + at);
    if (!in) vv = (u32x4){0u, 0u, 0u, 0u};  // (weight zero, which an infinite value would turn into NaN)
#pragma unroll
    for (int j = 0; j < GT; ++j) {
      float a = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) a = dot2_bf16(q[j][k], kv[k], a);
      a = group_sum<LPR>(a);
      if (scores && in && l16 == 0 && h0 + j < g * G + G) scores[(size_t)j * p.T + key] = a;
      a = in ? a : -INFINITY;
      const float mn = fmaxf(m[j], a);
      const float ref = mn == -INFINITY ? 0.f : mn;
      const float al = fast_exp2((m[j] - ref) * c2), pw = fast_exp2((a - ref) * c2);
      m[j] = mn;
      l[j] = l[j] * al + pw;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        o[j][2 * k] = o[j][2 * k] * al + pw * bf16_lo(vv[k]);
        o[j][2 * k + 1] = o[j][2 * k + 1] * al + pw * bf16_hi(vv[k]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < GT; ++j) fold_groups<D>(m[j], l[j], o[j], c2, lane, red[wave][j]);
  __syncthreads();
  for (int t = tid; t < GT * D; t += kShWaves * 64) {
    const int j = t / D, ch = t % D;
    if (h0 + j >= g * G + G) continue;
    float mm = -INFINITY, ll = 0.f, oo = 0.f;
#pragma unroll
    for (int w = 0; w < kShWaves; ++w) mm = fmaxf(mm, red[w][j][D]);
#pragma unroll
    for (int w = 0; w < kShWaves; ++w) {
      const float mi = red[w][j][D];
      const float f = mi == -INFINITY ? 0.f : fast_exp2((mi - mm) * c2);
      ll += f * red[w][j][D + 1];
      oo += f * red[w][j][ch];
    }
    float* dst = p.ws + (((size_t)b * p.Hq + h0 + j) * p.n_slices + slice) * (D + 2);
    dst[ch] = oo;
    if (ch == 0) {
      dst[D] = mm;
      dst[D + 1] = ll;
    }
  }
}

// Thread = channel of one (batch, query head): folds its slices.
template <int D>
__global__ __launch_bounds__(D) void moda_shared_merge_kernel(SharedParams p) {
  const int ch = threadIdx.x, bh = blockIdx.x;
  const float c2 = p.scale_log2;
  const float* ws = p.ws + (size_t)bh * p.n_slices * (D + 2);
  float mm = -INFINITY, ll = 0.f, oo = 0.f;
  for (int s = 0; s < p.n_slices; ++s) {
    const float* w = ws + (size_t)s * (D + 2);
    const float mn = fmaxf(mm, w[D]);
    const float al = mm == -INFINITY ? 0.f : fast_exp2((mm - mn) * c2), f = w[D] == -INFINITY ? 0.f : fast_exp2((w[D] - mn) * c2);
    mm = mn;
    ll = ll * al + f * w[D + 1];
    oo = oo * al + f * w[ch];
  }
  const bool none = ll == 0.f;  // nothing seen, or nothing that has weight
  ((__bf16*)p.O)[(size_t)bh * D + ch] = (__bf16)(none ? 0.f : oo / ll);
  if (ch == 0) p.LSE[bh] = none ? -INFINITY : mm * p.scale + __logf(ll);
}

// weights_out = weights_in + the heads' weights: thread = row of one (batch, key/value head).
__global__ __launch_bounds__(256) void moda_shared_weights_kernel(SharedParams p, int n_chunks) {
  const int bg = blockIdx.x / n_chunks, j = (blockIdx.x % n_chunks) * 256 + threadIdx.x;
  const int b = bg / p.Hk, g = bg - b * p.Hk, G = p.Hq / p.Hk;
  if (j >= filled(p.lengths, b, p.T)) return;
  const size_t at = (size_t)bg * p.T_alloc + j;
  float w = p.w_in ? p.w_in[at] : 0.f;
  for (int h = 0; h < G; ++h) {
    const size_t bh = (size_t)b * p.Hq + g * G + h;
    const float lse = p.LSE[bh];
    if (lse != -INFINITY) w += fast_exp2(p.scores[bh * p.T + j] * p.scale_log2 - lse * 1.4426950408889634f);
  }
  p.w_out[at] = w;
}

// ---------------------------------------------------------------- the cut into slices
static int heads_per_chunk(int G) { return G >= 3 ? 4 : G >= 2 ? 2 : 1; }

static void plan(SharedParams& p) {
  const long long groups = (long long)p.B * p.Hk;
  const int want = (int)std::max(1ll, 2048 / groups);
  auto cut = [&](int rows, int& n, int& per) {
    n = std::min(want, (rows + 255) / 256);
    per = n ? ((rows + n - 1) / n + 31) / 32 * 32 : 0;
    n = n ? (rows + per - 1) / per : 0;
  };
  cut(p.P, p.n_prefix, p.prefix_per);
  cut(p.T, p.n_own, p.own_per);
  p.n_slices = p.n_prefix + p.n_own + (p.depth_count > 0 ? 1 : 0);
}

static size_t state_bytes(const SharedParams& p, int d) {
  return ((size_t)p.B * p.Hq * p.n_slices * (d + 2) * sizeof(float) + 15) / 16 * 16;
}

size_t decode_shared_workspace_bytes(const SharedParams& dims, int d, bool with_weights) {
  SharedParams p = dims;
  plan(p);
  const size_t bytes = state_bytes(p, d) + (with_weights ? (size_t)p.B * p.Hq * p.T * sizeof(float) : 0);
  return std::max<size_t>(bytes, 16);
}

template <int D>
static hipError_t launch_d(const SharedParams& p, hipStream_t stream) {
  const int G = p.Hq / p.Hk, gt = heads_per_chunk(G);
  const long long blocks = (long long)p.B * p.Hk * ((G + gt - 1) / gt) * p.n_slices;
  const long long heads = (long long)p.B * p.Hq;
  const int chunks = (p.T + 255) / 256;
  const long long w_blocks = (long long)p.B * p.Hk * chunks;
  const bool weights = p.w_out && p.T > 0;
  if ((blocks > 0 && !grid_ok(blocks, kShWaves * 64)) || !grid_ok(heads, D) || (weights && !grid_ok(w_blocks, 256)))
    return kGridTooLarge;
  hipError_t e = hipSuccess;
  if (blocks > 0)
    e = launch_kernel(gt == 4 ? moda_shared_rows_kernel<D, 4> : gt == 2 ? moda_shared_rows_kernel<D, 2> : moda_shared_rows_kernel<D, 1>,
                      dim3((unsigned)blocks), dim3(kShWaves * 64), stream, p);
  if (e == hipSuccess) e = launch_kernel(moda_shared_merge_kernel<D>, dim3((unsigned)heads), dim3(D), stream, p);
  if (e == hipSuccess && weights)
    e = launch_kernel(moda_shared_weights_kernel, dim3((unsigned)w_blocks), dim3(256), stream, p, chunks);
  return e;
}

hipError_t launch_decode_shared(SharedParams p, int d, void* workspace, hipStream_t stream) {
  plan(p);
  p.ws = (float*)workspace;
  p.scores = (float*)((char*)workspace + state_bytes(p, d));
  return d == 128 ? launch_d<128>(p, stream) : launch_d<64>(p, stream);
}

}  // namespace moda
