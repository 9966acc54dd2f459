// The choice of pages for a decoding step that reads only some of them.
//
// With the bounds lo_c <= k_c <= hi_c of a page's keys and the queries q of a group's heads, the group's logits (before the scale) on
// any row of the page add up to at most
//     score = sum over c of up_c hi_c + down_c lo_c,   up_c = sum over the heads of max(q_c, 0),  down_c = that of min(q_c, 0):
// 2 d products per page, however many heads.  The first and the last pages stay, then the pages of the largest scores.  Scores
// are formed in 64 bits: products of bf16 numbers are exact there and their sums all but so, so that the order of the sums does not decide
// between pages of nearly the same score (in fp32 it would, at 2^-24 of the largest term).
//
// Scores: a wave reads the bounds of 16 pages (d = 64: 32) with 8 loads in flight, eight channels per lane, and folds the 8 partial sums of
// a lane and its neighbours so that every exchange halves what a lane holds: 9 additions in 64 bits (d = 64: 8) for 8 loads.  A score becomes a
// 64-bit integer of the same order.  The choice: the least key that is kept lies in a range of keys, at first from the least to the
// largest; a histogram of 1024 parts of the range narrows it until all candidates in it are kept or are equal (then the lowest
// pages are).  Kept pages are counted off in ascending order.
// Few pages per (sequence, key/value head): one workgroup of 16 waves does both, keys in LDS; more: two kernels, keys in the workspace.
#include <algorithm>

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

template <int CTRL>
__device__ __forceinline__ double dpp_mov(double x) {
  const u64 u = __builtin_bit_cast(u64, x);
  const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)(unsigned)u, CTRL, 0xf, 0xf, false);
  const unsigned hi = __builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), CTRL, 0xf, 0xf, false);
  return __builtin_bit_cast(double, (u64)hi << 32 | lo);
}
// Two values of which each lane keeps one, a where `second` is not set, summed with what the lane's partner has of it.
template <int CTRL>
__device__ __forceinline__ double halve(double a, double b, bool second) {
  return (second ? b : a) + dpp_mov<CTRL>(second ? a : b);
}
// ... the partner in the row of 16 lanes beside; odd rows keep b
__device__ __forceinline__ double halve_rows(double a, double b) {
  const u64 x = __builtin_bit_cast(u64, a), y = __builtin_bit_cast(u64, b);
  auto lo = __builtin_amdgcn_permlane16_swap((unsigned)x, (unsigned)y, false, false);
  auto hi = __builtin_amdgcn_permlane16_swap((unsigned)(x >> 32), (unsigned)(y >> 32), false, false);
  return __builtin_bit_cast(double, (u64)hi[0] << 32 | (unsigned)lo[0]) + __builtin_bit_cast(double, (u64)hi[1] << 32 | (unsigned)lo[1]);
}

// The scores of one (sequence, key/value head).  A page's bounds are read by D / 4 lanes, eight channels each: half of them hold lo, half hi.
template <int D>
struct Scorer {
  static constexpr int LPP = D / 4, PPI = 64 / LPP, kLoads = 8, kPages = kLoads * PPI, RB = D * 2;  // pages of a load, of a batch
  double q[8];
  const int* table;
  const char* bounds;
  int n, lane;
  size_t page_bytes;
  u32x4 x[kLoads];
  int id;  // lane i: page i of the batch
  __device__ __forceinline__ void init(const SelectParams& p, int b, int g, int n_) {
    n = n_;
    lane = threadIdx.x & 63;
    table = p.table + (size_t)b * p.max_pages;
    page_bytes = (size_t)p.Hk * 2 * RB;
    bounds = (const char*)p.bounds + (size_t)g * 2 * RB + lane % LPP * 16;  // (lo, then hi: D / 4 pieces of 16 bytes)
  }
  // Pages first .. first + kPages - 1 are asked for; those behind the n-th and missing ones repeat page 0 of the pool.
  __device__ __forceinline__ void load(const SelectParams& p, int first) {
    id = lane < kPages && first + lane < n ? page_at(table, first + lane, p.n_pages) : -1;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) x[u] = *(const u32x4*)(bounds + (size_t)max(__shfl(id, u * PPI + lane / LPP), 0) * page_bytes);
  }
  __device__ __forceinline__ void query(const SelectParams& p, int b, int g) {
    const int G = p.Hq / p.Hk;
    const bool high = lane % LPP >= LPP / 2;
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = 0.0;
    const char* at = (const char*)p.Q + ((size_t)b * p.Hq + g * G) * RB + lane % (LPP / 2) * 16;
#pragma unroll 2
    for (int h = 0; h < G; ++h) {
      const u32x4 y = *(const u32x4*)(at + (size_t)h * RB);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float f = i % 2 ? bf16_hi(y[i / 2]) : bf16_lo(y[i / 2]);
        // (a NaN query counts on both sides)
        q[i] += f != f || (high ? f > 0.f : f < 0.f) ? (double)f : 0.0;
      }
    }
  }
  // The page of the batch whose key the lane holds (d = 128: four lanes hold it, d = 64: two, of which one stores it).
  __device__ __forceinline__ int page() const {
    const int u = D == 128 ? ((lane >> 4) & 1) * 4 + ((lane >> 3) & 1) * 2 + ((lane >> 2) & 1) : ((lane >> 3) & 1) * 4 + ((lane >> 2) & 1) * 2 + ((lane >> 1) & 1);
    return u * PPI + lane / LPP;
  }
  __device__ __forceinline__ bool stores() const { return lane % (D / 32) == 0; }
  // The key of that page, of the batch that was asked for.
  __device__ __forceinline__ u64 key(const SelectParams& p, int first) const {
    auto part = [&](int u) {
      double s = 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) s = __builtin_fma(q[i], (double)(i % 2 ? bf16_hi(x[u][i / 2]) : bf16_lo(x[u][i / 2])), s);
      return s;
    };
    double s4[4], s2[2], r;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      s4[k] = D == 128 ? halve_rows(part(k), part(k + 4)) : halve<0x128>(part(k), part(k + 4), lane & 8);  // row_ror:8
      __builtin_amdgcn_sched_barrier(0);  // (one pair at a time: the registers hold 16 waves)
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
      s2[k] = D == 128 ? halve<0x128>(s4[k], s4[k + 2], lane & 8) : halve<0x141>(s4[k], s4[k + 2], lane & 4);  // row_half_mirror
    r = D == 128 ? halve<0x141>(s2[0], s2[1], lane & 4) : halve<0x4E>(s2[0], s2[1], lane & 2);                 // quad_perm [2,3,0,1]
    if (D == 128) r += dpp_mov<0x4E>(r);
    r += dpp_mov<0xB1>(r);  // quad_perm [1,0,3,2]
    const int i = first + page();
    return __shfl(id, page()) < 0 ? 0ull : i < p.first || i >= n - p.recent ? kStays : score_key(r);
  }
};

// ---------------------------------------------------------------- the choice
// Of n keys (0: no page) the pages of the largest, p.keep of them, to out in ascending order, -1 behind them.  key(i): page i's.
constexpr int kParts = 1024;
template <int NT>
struct Choice {
  int hist[kParts];
  unsigned least, most;  // upper halves of the keys that compete
  int stay, compete;
  int part, above, in;
  int count[NT / 64][2];
};
template <int NT, class Key>
__device__ __forceinline__ void choose(Choice<NT>& c, Key&& key, int n, int keep, int* out) {
  constexpr int NW = NT / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto competes = [](u64 k) { return k != 0 && k != kStays; };
  // Pages with keys above `hi` are kept, and `need` of those in [lo, hi]: the lowest, or (all) every one.
  u64 lo = 1, hi = kNaNKey;
  int need = keep;
  bool all = n <= keep;
  if (!all) {  // (uniform)
    if (tid == 0) {
      c.least = ~0u;
      c.most = 0;
      c.stay = c.compete = 0;
    }
    __syncthreads();
    unsigned least = ~0u, most = 0;
    int stay = 0, compete = 0;
    for (int i = tid; i < n; i += NT) {
      const u64 k = key(i);
      if (competes(k)) {
        least = min(least, (unsigned)(k >> 32));
        most = max(most, (unsigned)(k >> 32));
        ++compete;
      }
      stay += k == kStays;
    }
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
      least = min(least, (unsigned)__shfl_xor((int)least, x));
      most = max(most, (unsigned)__shfl_xor((int)most, x));
      stay += __shfl_xor(stay, x);
      compete += __shfl_xor(compete, x);
    }
    if (lane == 0) {
      atomicMin(&c.least, least);
      atomicMax(&c.most, most);
      atomicAdd(&c.stay, stay);
      atomicAdd(&c.compete, compete);
    }
    __syncthreads();
    lo = (u64)c.least << 32;
    hi = (u64)c.most << 32 | 0xffffffffu;
    need = keep - c.stay;
    all = c.compete <= need;
    if (need <= 0) {  // (the pages that stay fill the list)
      all = false;
      lo = hi = kStays;
      need = keep;
    }
  }
  while (!all && lo < hi) {  // (uniform)
    const int shift = max(54 - __builtin_clzll(hi - lo), 0);  // so that (hi - lo) >> shift is below 1024
    for (int i = tid; i < kParts; i += NT) c.hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += NT) {
      const u64 k = key(i);
      if (competes(k) && k >= lo && k <= hi) atomicAdd(&c.hist[(int)((k - lo) >> shift)], 1);
    }
    __syncthreads();
    if (wave == 0) {  // 16 parts a lane, from the largest down
      constexpr int kPer = kParts / 64;
      int h[kPer], sum = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) sum += h[i] = c.hist[kParts - 1 - lane * kPer - i];
      int above = sum;
#pragma unroll
      for (int x = 1; x < 64; x *= 2) {
        const int y = __shfl_up(above, x);
        if (lane >= x) above += y;
      }
      above -= sum;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (above < need && above + h[i] >= need) {
          c.part = kParts - 1 - lane * kPer - i;
          c.above = above;
          c.in = h[i];
        }
        above += h[i];
      }
    }
    __syncthreads();
    need -= c.above;
    all = c.in == need;
    lo += (u64)c.part << shift;
    if (hi - lo >= 1ull << shift) hi = lo + ((1ull << shift) - 1);
    __syncthreads();
  }
  int before = 0, equal_before = 0;
  const int most = all ? 0x7fffffff : need;
  for (int i0 = 0; i0 < n; i0 += NT) {  // (uniform)
    const u64 k = i0 + tid < n ? key(i0 + tid) : 0;
    const bool more = k > hi, in = k >= lo && !more;
    const u64 mask_e = __builtin_amdgcn_ballot_w64(in), mask_m = __builtin_amdgcn_ballot_w64(more);
    if (lane == 0) {
      c.count[wave][0] = __builtin_popcountll(mask_m);
      c.count[wave][1] = __builtin_popcountll(mask_e);
    }
    __syncthreads();
    int m = before, e = equal_before;
    for (int w = 0; w < NW; ++w) {
      const int cm = c.count[w][0], ce = c.count[w][1];
      if (w < wave) {
        m += cm;
        e += ce;
      }
      before += cm;
      equal_before += ce;
    }
    const u64 below = (1ull << lane) - 1;
    m += __builtin_popcountll(mask_m & below);
    e += __builtin_popcountll(mask_e & below);
    if (more || (in && e < most)) out[m + min(e, most)] = i0 + tid;
    __syncthreads();
  }
  const int kept = before + min(equal_before, most);
  for (int i = kept + tid; i < keep; i += NT) out[i] = -1;
}

// ---------------------------------------------------------------- kernels
constexpr int kOnePages = 4096;  // of one (sequence, key/value head) in one kernel
template <int D>
__global__ __launch_bounds__(1024) void moda_page_select_kernel(SelectParams p) {
  __shared__ u64 keys[kOnePages];
  __shared__ Choice<1024> c;
  const int b = blockIdx.x / p.Hk, g = blockIdx.x - b * p.Hk, n = pages_filled(p, b);
  Scorer<D> s;
  s.init(p, b, g, n);
  int first = (threadIdx.x >> 6) * s.kPages;
  if (first < n && n > p.keep) {  // (uniform over a wave)
    s.load(p, first);
    s.query(p, b, g);
    while (true) {
      const u64 k = s.key(p, first);
      if (s.stores() && first + s.page() < n) keys[first + s.page()] = k;
      first += 16 * s.kPages;
      if (first >= n) break;
      s.load(p, first);
    }
  } else if (n <= p.keep) {  // all pages there are
    for (int i = threadIdx.x; i < n; i += 1024) keys[i] = page_at(s.table, i, p.n_pages) < 0 ? 0ull : kStays;
  }
  __syncthreads();
  choose<1024>(c, [&](int i) { return keys[i]; }, n, p.keep, p.pages + (size_t)blockIdx.x * p.keep);
}

template <int D>
__global__ __launch_bounds__(256) void moda_page_score_kernel(SelectParams p, int batches, int chunks) {
  const int bg = blockIdx.x / chunks, b = bg / p.Hk, g = bg - b * p.Hk, n = pages_filled(p, b);
  Scorer<D> s;
  int first = ((blockIdx.x - bg * chunks) * 4 + (threadIdx.x >> 6)) * batches * s.kPages;
  const int end = min(n, first + batches * s.kPages);
  if (first >= end) return;
  s.init(p, b, g, n);
  u64* keys = p.keys + (size_t)bg * p.cols;
  s.load(p, first);
  s.query(p, b, g);
  while (true) {
    const u64 k = s.key(p, first);
    if (s.stores() && first + s.page() < n) keys[first + s.page()] = k;
    first += s.kPages;
    if (first >= end) break;
    s.load(p, first);
  }
}
__global__ __launch_bounds__(1024) void moda_page_choose_kernel(SelectParams p) {
  __shared__ Choice<1024> c;
  const u64* keys = p.keys + (size_t)blockIdx.x * p.cols;
  choose<1024>(c, [&](int i) { return keys[i]; }, pages_filled(p, blockIdx.x / p.Hk), p.keep, p.pages + (size_t)blockIdx.x * p.keep);
}

static int columns(const SelectParams& p) { return (int)(((long long)p.T + (1 << p.shift) - 1) >> p.shift); }

static bool in_one(const SelectParams& p) { return columns(p) <= kOnePages; }

size_t select_workspace_bytes(const SelectParams& p) { return (size_t)p.B * p.Hk * columns(p) * sizeof(u64); }

hipError_t launch_select(SelectParams p, int d, void* workspace, hipStream_t stream) {
  p.cols = columns(p);
  p.keys = (u64*)workspace;
  const long long groups = (long long)p.B * p.Hk;
  if (!grid_ok(groups, 1024)) return kGridTooLarge;
  if (in_one(p))
    return launch_kernel(d == 128 ? moda_page_select_kernel<128> : moda_page_select_kernel<64>, dim3((unsigned)groups), dim3(1024), stream, p);
  // a wave takes several batches of pages where there are more than 16 waves a compute unit
  const int per_batch = 8 * 256 / d;
  const long long all = groups * ((p.cols + per_batch - 1) / per_batch);
  const int batches = (int)std::min(8ll, std::max(1ll, all / 4096));
  const int chunks = (p.cols + 4 * batches * per_batch - 1) / (4 * batches * per_batch);
  if (!grid_ok(groups * chunks, 256)) return kGridTooLarge;
  const hipError_t e = launch_kernel(d == 128 ? moda_page_score_kernel<128> : moda_page_score_kernel<64>, dim3((unsigned)(groups * chunks)),
                                     dim3(256), stream, p, batches, chunks);
  if (e != hipSuccess) return e;
  return launch_kernel(moda_page_choose_kernel, dim3((unsigned)groups), dim3(1024), stream, p);
}

}  // namespace moda
