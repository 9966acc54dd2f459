// The choice of pages for a decoding step that reads only some of them.
//
// With the bounds lo_c <= k_c <= hi_c of a page's keys and the queries q of a group's heads, the group's logits (before the scale) on
// any row of the page add up to at most
//     score = sum over c of up_c hi_c + down_c lo_c,   up_c = sum over the heads of max(q_c, 0),  down_c = that of min(q_c, 0):
// 2 d products per page, however many heads.  The first and the last pages stay, then the pages of the largest scores.  Scores
// are formed in 64 bits: products of bf16 numbers are exact there and their sums all but so, so that the order of the sums does not decide
// between pages of nearly the same score (in fp32 it would, at 2^-24 of the largest term).
// Two kernels: scores, as integers of the same order, to the workspace; then per (sequence, key/value head) the least key that is
// kept, by histograms of 8 bits of the candidates' keys, and the pages at or above it in ascending order.
#include "moda_pages.h"

namespace moda {

typedef unsigned long long u64;

// Orders as the score does; a NaN above all numbers, below the pages that stay anyway; 0: no page.
constexpr u64 kStays = ~0ull, kNaNKey = ~0ull - 1;
__device__ __forceinline__ u64 score_key(double s) {
  const u64 u = __builtin_bit_cast(u64, s + 0.0);
  return s != s ? kNaNKey : u ^ ((u >> 63) ? ~0ull : 1ull << 63);
}

__device__ __forceinline__ int pages_filled(const SelectParams& p, int b) {
  return (filled(p.lengths, b, p.T) + (1 << p.shift) - 1) >> p.shift;
}

// A page's bounds are read by D / 4 lanes, eight channels each: half of them hold lo, half hi.
template <int D>
__global__ __launch_bounds__(256) void moda_page_score_kernel(SelectParams p, int per_wave, int chunks) {
  constexpr int LPP = D / 4, PPI = 64 / LPP, RB = D * 2, kU = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane % LPP, G = p.Hq / p.Hk;
  const int bg = blockIdx.x / chunks, b = bg / p.Hk, g = bg - b * p.Hk;
  const int n = pages_filled(p, b), begin = ((blockIdx.x - bg * chunks) * 4 + wave) * per_wave, end = min(n, begin + per_wave);
  if (begin >= end) return;
  const bool high = l >= LPP / 2;
  const int at = l % (LPP / 2) * 16;
  double q[8] = {};
  for (int h = 0; h < G; ++h) {
    const u32x4 x = *(const u32x4*)((const char*)p.Q + ((size_t)b * p.Hq + g * G + h) * RB + at);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float f = i % 2 ? bf16_hi(x[i / 2]) : bf16_lo(x[i / 2]);
      // (a NaN query counts on both sides)
      q[i] += f != f || (high ? f > 0.f : f < 0.f) ? (double)f : 0.0;
    }
  }
  const int* table = p.table + (size_t)b * p.max_pages;
  u64* keys = p.keys + (size_t)bg * p.cols;
  for (int i0 = begin; i0 < end; i0 += kU * PPI) {
    int id[kU];
    u32x4 x[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int i = i0 + u * PPI + lane / LPP;
      id[u] = i < end ? page_at(table, i, p.n_pages) : -1;
    }
#pragma unroll
    for (int u = 0; u < kU; ++u)
      x[u] = *(const u32x4*)((const char*)p.bounds + ((size_t)max(id[u], 0) * p.Hk + g) * 2 * RB + (high ? RB : 0) + at);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      double s = 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) s = __builtin_fma(q[i], (double)(i % 2 ? bf16_hi(x[u][i / 2]) : bf16_lo(x[u][i / 2])), s);
#pragma unroll
      for (int k = 1; k < LPP; k *= 2) s += __shfl_xor(s, k);
      const int i = i0 + u * PPI + lane / LPP;
      if (l == 0 && i < end) keys[i] = id[u] < 0 ? 0ull : i < p.first || i >= n - p.recent ? kStays : score_key(s);
    }
  }
}

template <int NT>
__global__ __launch_bounds__(NT) void moda_page_choose_kernel(SelectParams p) {
  constexpr int NW = NT / 64;
  __shared__ int hist[256];
  __shared__ int found[2];  // digit, candidates above it
  __shared__ int count[NW][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x / p.Hk, n = pages_filled(p, b);
  const u64* keys = p.keys + (size_t)blockIdx.x * p.cols;
  int* out = p.pages + (size_t)blockIdx.x * p.keep;
  // the least key that is kept: `prefix` its digits so far, `need` how many of the candidates (keys with these digits) are kept
  u64 prefix = 0;
  int need = p.keep, shift = 64;
  bool all = n <= p.keep;  // of the candidates
  while (!all && shift > 0) {  // (uniform)
    for (int i = tid; i < 256; i += NT) hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += NT) {
      const u64 k = keys[i];
      if (k != 0 && (shift == 64 || k >> shift == prefix)) atomicAdd(&hist[(int)(k >> (shift - 8)) & 255], 1);
    }
    __syncthreads();
    if (wave == 0) {  // four digits a lane, from the largest down
      int c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += c[i] = hist[255 - lane * 4 - i];
      int above = sum;
#pragma unroll
      for (int x = 1; x < 64; x *= 2) {
        const int y = __shfl_up(above, x);
        if (lane >= x) above += y;
      }
      const int total = __shfl(above, 63);
      above -= sum;
      if (total <= need) {
        if (lane == 0) found[0] = -1;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (above < need && above + c[i] >= need) {
            found[0] = 255 - lane * 4 - i;
            found[1] = above;
          }
          above += c[i];
        }
      }
    }
    __syncthreads();
    const int digit = found[0];
    if (digit < 0) {
      all = true;
    } else {
      need -= found[1];
      prefix = prefix << 8 | (u64)digit;
      shift -= 8;
      all = hist[digit] == need;
    }
    __syncthreads();
  }
  // Every key above the candidates is kept, and the first `need` candidates (all: every one).
  int before = 0, equal_before = 0;
  for (int i0 = 0; i0 < n; i0 += NT) {  // (uniform)
    const u64 k = i0 + tid < n ? keys[i0 + tid] : 0;
    const u64 top = shift == 64 ? 0 : k >> shift;
    const bool equal = k != 0 && top == prefix, more = k != 0 && top > prefix;
    const u64 mask_e = __builtin_amdgcn_ballot_w64(equal), mask_m = __builtin_amdgcn_ballot_w64(more);
    if (lane == 0) {
      count[wave][0] = __builtin_popcountll(mask_m);
      count[wave][1] = __builtin_popcountll(mask_e);
    }
    __syncthreads();
    int m = before, e = equal_before;
    for (int w = 0; w < NW; ++w) {
      if (w < wave) {
        m += count[w][0];
        e += count[w][1];
      }
      before += count[w][0];
      equal_before += count[w][1];
    }
    const u64 below = (1ull << lane) - 1;
    m += __builtin_popcountll(mask_m & below);
    e += __builtin_popcountll(mask_e & below);
    const int most = all ? 0x7fffffff : need;
    if (more || (equal && e < most)) out[m + min(e, most)] = i0 + tid;
    __syncthreads();
  }
  const int kept = before + (all ? equal_before : min(equal_before, need));
  for (int i = kept + tid; i < p.keep; i += NT) out[i] = -1;
}

static int columns(const SelectParams& p) { return (int)(((long long)p.T + (1 << p.shift) - 1) >> p.shift); }

size_t select_workspace_bytes(const SelectParams& p) { return (size_t)p.B * p.Hk * columns(p) * sizeof(u64); }

hipError_t launch_select(SelectParams p, int d, void* workspace, hipStream_t stream) {
  p.cols = columns(p);
  p.keys = (u64*)workspace;
  const long long groups = (long long)p.B * p.Hk;
  const int per_wave = 32, chunks = (p.cols + 4 * per_wave - 1) / (4 * per_wave);
  if (!grid_ok(groups, 1024) || (chunks > 0 && !grid_ok(groups * chunks, 256))) return kGridTooLarge;
  if (chunks > 0) {
    const hipError_t e = launch_kernel(d == 128 ? moda_page_score_kernel<128> : moda_page_score_kernel<64>, dim3((unsigned)(groups * chunks)),
                                       dim3(256), stream, p, per_wave, chunks);
    if (e != hipSuccess) return e;
  }
  return launch_kernel(moda_page_choose_kernel<1024>, dim3((unsigned)groups), dim3(1024), stream, p);
}

}  // namespace moda
