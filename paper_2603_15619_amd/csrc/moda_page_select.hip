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
// largest; a histogram of 256 or 1024 parts of the range narrows it until all candidates in it are kept or are equal (then the lowest
// pages are).  Kept pages are counted off in ascending order.
// Few pages per (sequence, key/value head), or many such: a workgroup does both, keys in LDS; else two kernels, keys in the workspace.
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
  // The lane's queries from those of the workgroup, [lo, hi][d].
  __device__ __forceinline__ void query(const double* sums) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = sums[lane % LPP * 8 + i];
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

// The sums of a group's queries that bounds are multiplied by: down_c, then up_c.  A thread has one of them.
template <int D, int THREADS>
__device__ __forceinline__ void query_sums(const SelectParams& p, int b, int g, double* sums) {
  const int G = p.Hq / p.Hk, t = threadIdx.x;
  static_assert(THREADS >= 2 * D, "a thread per sum");
  if (t >= 2 * D) return;
  const bool high = t >= D;
  const unsigned short* at = (const unsigned short*)p.Q + ((size_t)b * p.Hq + g * G) * D + t % D;
  double q = 0.0;
  for (int h0 = 0; h0 < G; h0 += 8) {
    unsigned short y[8];
#pragma unroll
    for (int h = 0; h < 8; ++h) y[h] = at[(size_t)min(h0 + h, G - 1) * D];
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      if (h0 + h >= G) break;  // (uniform)
      const float f = bf16_lo(y[h]);
      // (a NaN query counts on both sides)
      q += f != f || (high ? f > 0.f : f < 0.f) ? (double)f : 0.0;
    }
  }
  sums[t] = q;
}

// ---------------------------------------------------------------- the choice
constexpr int kPer = 4;  // keys of a thread
// ... by a workgroup of so many threads, each of which has a part of the histogram
template <int THREADS>
struct Choice {
  static constexpr int kWaves = THREADS / 64, kChunk = kPer * THREADS;
  int hist[THREADS];
  unsigned least, most;  // upper halves of the keys that compete, the least one's bits turned round
  int stay, compete;
  int part, above, in;
  int count[kPer * kWaves];
};
__device__ __forceinline__ bool competes(u64 k) { return k != 0 && k != kStays; }

// Before the keys are formed: an empty histogram, nothing seen.
template <int THREADS>
__device__ __forceinline__ void choice_start(Choice<THREADS>& c) {
  c.hist[threadIdx.x] = 0;
  if (threadIdx.x == 0) {
    c.least = c.most = 0;
    c.stay = c.compete = 0;
  }
}
// What a thread has seen of the keys; flush: the workgroup gets to know it.
struct Seen {
  unsigned least = 0, most = 0;
  int stay = 0, compete = 0;
  __device__ __forceinline__ void add(u64 k) {
    if (competes(k)) {
      least = max(least, ~(unsigned)(k >> 32));
      most = max(most, (unsigned)(k >> 32));
      ++compete;
    }
    stay += k == kStays;
  }
  template <int THREADS>
  __device__ __forceinline__ void flush(Choice<THREADS>& c) const {
    const unsigned a = wave_max(least), z = wave_max(most);
    const int s = wave_scan(stay), n = wave_scan(compete);
    if ((threadIdx.x & 63) == 63) {
      atomicMax(&c.least, a);
      atomicMax(&c.most, z);
      atomicAdd(&c.stay, s);
      atomicAdd(&c.compete, n);
    }
  }
};

// Of n keys (0: no page), all seen, the pages of the largest, `keep` of them, to out in ascending order, -1 behind them.  keys: in LDS (LDS: at
// most kChunk of them, which then stay in registers) or in memory.  A pass takes kChunk keys at a time, kPer a thread.
template <bool LDS, int THREADS>
__device__ __forceinline__ void choose(Choice<THREADS>& c, const u64* keys, int n, int keep, int* out) {
  constexpr int kWaves = Choice<THREADS>::kWaves, kChunk = Choice<THREADS>::kChunk;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  u64 held[kPer];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) held[j] = i0 + j * THREADS + tid < n ? keys[i0 + j * THREADS + tid] : 0;
  };
  if (LDS) fetch(0);
  // Pages with keys above `hi` are kept, and `need` of those in [lo, hi]: the lowest, or (all) every one.
  u64 lo = (u64)~c.least << 32, hi = (u64)c.most << 32 | 0xffffffffu;
  int need = keep - c.stay;
  bool all = c.compete <= need;
  if (need <= 0) {  // the pages that stay fill the list
    all = false;
    lo = hi = kStays;
    need = keep;
  }
  while (!all && lo < hi) {  // (uniform)
    const int shift = max(64 - __builtin_ctz(THREADS) - __builtin_clzll(hi - lo), 0);  // so that (hi - lo) >> shift is below THREADS
    for (int i0 = 0; i0 < n; i0 += kChunk) {
      if (!LDS) fetch(i0);
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (competes(held[j]) && held[j] >= lo && held[j] <= hi) atomicAdd(&c.hist[(int)((held[j] - lo) >> shift)], 1);
    }
    __syncthreads();
    // a part a thread, from the largest down; the parts are empty again behind
    const int h = c.hist[THREADS - 1 - tid], to = wave_scan(h);
    c.hist[THREADS - 1 - tid] = 0;
    if (lane == 63) c.count[wave] = to;
    __syncthreads();
    const int of_wave = c.count[lane % kWaves], up_to = row_scan(of_wave);
    const int above = __builtin_amdgcn_readlane(up_to - of_wave, wave) + to - h;
    if (above < need && above + h >= need) {
      c.part = THREADS - 1 - tid;
      c.above = above;
      c.in = h;
    }
    __syncthreads();
    need -= c.above;
    all = c.in == need;
    lo += (u64)c.part << shift;
    if (hi - lo >= 1ull << shift) hi = lo + ((1ull << shift) - 1);
  }
  // Counted off: (kept for sure, candidates) of 64 keys each as one number, two times 16 bits; a chunk has at most 64 of them, a lane's each.
  int before = 0, in_before = 0;
  const int most = all ? 0x7fffffff : need;
  for (int i0 = 0; i0 < n; i0 += kChunk) {  // (uniform)
    if (!LDS) {
      fetch(i0);
      __syncthreads();  // (the numbers of the chunk before have been read)
    }
    u64 more[kPer], in[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      more[j] = __builtin_amdgcn_ballot_w64(held[j] > hi);
      in[j] = __builtin_amdgcn_ballot_w64(held[j] >= lo && held[j] <= hi);
      if (lane == 0) c.count[j * kWaves + wave] = __builtin_popcountll(more[j]) << 16 | __builtin_popcountll(in[j]);
    }
    __syncthreads();
    const int own = lane < kPer * kWaves ? c.count[lane] : 0, to = wave_scan(own);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int at = __builtin_amdgcn_readlane(to - own, j * kWaves + wave);
      const u64 below = (1ull << lane) - 1;
      const int m = before + (at >> 16) + __builtin_popcountll(more[j] & below), e = in_before + (at & 0xffff) + __builtin_popcountll(in[j] & below);
      const bool is_in = in[j] >> lane & 1;
      if ((more[j] >> lane & 1) || (is_in && e < most)) out[m + min(e, most)] = i0 + j * THREADS + tid;
    }
    const int total = __builtin_amdgcn_readlane(to, 63);
    before += total >> 16;
    in_before += total & 0xffff;
  }
  const int kept = before + min(in_before, most);
  for (int i = kept + tid; i < keep; i += THREADS) out[i] = -1;
}

// ---------------------------------------------------------------- kernels
template <int D, int THREADS>
__global__ __launch_bounds__(THREADS) void moda_page_select_kernel(SelectParams p) {
  constexpr int kWaves = THREADS / 64;
  __shared__ u64 keys[Choice<THREADS>::kChunk];
  __shared__ __attribute__((aligned(16))) double sums[2 * D];
  __shared__ Choice<THREADS> c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = blockIdx.x / p.Hk, g = blockIdx.x - b * p.Hk, n = pages_filled(p, b);
  choice_start(c);
  Scorer<D> s;
  s.init(p, b, g, n);
  int first = wave * s.kPages;
  Seen seen;
  const bool choice = n > p.keep;  // (uniform; else all pages that there are)
  if (choice && first < n) s.load(p, first);
  if (choice) query_sums<D, THREADS>(p, b, g, sums);
  __syncthreads();
  if (!choice) {
    for (int i = threadIdx.x; i < n; i += THREADS) seen.add(keys[i] = page_at(s.table, i, p.n_pages) < 0 ? 0ull : kStays);
  } else if (first < n) {  // (uniform over a wave)
    s.query(sums);
    while (true) {
      const u64 k = s.key(p, first);
      if (s.stores() && first + s.page() < n) seen.add(keys[first + s.page()] = k);
      first += kWaves * s.kPages;
      if (first >= n) break;
      s.load(p, first);
    }
  }
  seen.flush(c);
  __syncthreads();
  choose<true>(c, keys, n, p.keep, p.pages + (size_t)blockIdx.x * p.keep);
}

template <int D>
__global__ __launch_bounds__(256) void moda_page_score_kernel(SelectParams p, int batches, int chunks) {
  __shared__ __attribute__((aligned(16))) double sums[2 * D];
  const int bg = blockIdx.x / chunks, b = bg / p.Hk, g = bg - b * p.Hk, n = pages_filled(p, b);
  Scorer<D> s;
  int first = ((blockIdx.x - bg * chunks) * 4 + (threadIdx.x >> 6)) * batches * s.kPages;
  const int end = min(n, first + batches * s.kPages);
  s.init(p, b, g, n);
  u64* keys = p.keys + (size_t)bg * p.cols;
  if (first < end) s.load(p, first);
  query_sums<D, 256>(p, b, g, sums);
  __syncthreads();
  if (first >= end) return;
  s.query(sums);
  while (true) {
    const u64 k = s.key(p, first);
    if (s.stores() && first + s.page() < n) keys[first + s.page()] = k;
    first += s.kPages;
    if (first >= end) break;
    s.load(p, first);
  }
}
template <int THREADS>
__global__ __launch_bounds__(THREADS) void moda_page_choose_kernel(SelectParams p) {
  __shared__ Choice<THREADS> c;
  const u64* keys = p.keys + (size_t)blockIdx.x * p.cols;
  const int n = pages_filled(p, blockIdx.x / p.Hk);
  choice_start(c);
  __syncthreads();
  Seen seen;
  for (int i = threadIdx.x; i < n; i += THREADS) seen.add(keys[i]);
  seen.flush(c);
  __syncthreads();
  choose<false>(c, keys, n, p.keep, p.pages + (size_t)blockIdx.x * p.keep);
}

static int columns(const SelectParams& p) { return (int)(((long long)p.T + (1 << p.shift) - 1) >> p.shift); }

// How a choice is made: 0: two kernels, else one, a workgroup of so many threads per (sequence, key/value head).  1024 threads, which fill a compute
// unit / 256, of which several share one / two kernels, us, (sequence, head)s, pages of the longest sequence; where it matters all as long, evenly down to half, down to a tenth:
//   d = 128   8, 60 6.2 / 5.8 / 7.8;   8, 120 7.4 / 6.5 / 7.7;   8, 250 8.9 / 8.9 / 8.0;   8, 500 11.2 / 13.1 / 8.8;   8, 2000 25.4 / - / 10.2;   64, 250 9.0 / 8.9 / 8.2;   64, 2000 28.3 / - / 20.6
//             128, 250 9.1 / 9.2 / 9.5;   128, 500 12.4 / 15.6 / 12.5, 11.2 / 12.9 / 12.3, 11.3 / 13.1 / 11.8;   128, 2000 29.6 / - / 30.8, 28.6 / - / 24.9, 28.1 / - / 21.2
//             256, 250 9.9 / 10.5 / 11.7;   256, 1000 25.6 / 29.8 / 30.2, 22.6 / 28.8 / 25.3, 19.9 / 28.2 / 21.2;   256, 4000 96 / - / 117, 81 / - / 98, 58 / - / 79
//             512, 120 14.4 / 8.9 / 11.8;   512, 1000 47.7 / 43.1 / 52.7, 38.9 / 38.5 / 42.1, 33.9 / 34.5 / 36.1;   512, 2000 99 / - / 116, 81 / - / 98, 59 / - / 70
//             1024, 250 39.5 / 24.0 / 27.8;   1024, 1000 105.7 / 94.9 / 116.8, 85.9 / 81.2 / 97.7, 63.6 / 58.5 / 65.2
//   d = 64    8, 250 7.2 / 6.8 / 7.9;   8, 500 8.9 / 8.9 / 8.5;   128, 500 9.7 / 9.5 / 10.0;   128, 1000 12.5 / 16.4 / 13.5, 11.5 / 13.4 / 13.2, 11.3 / 13.1 / 12.3
//             256, 1000 16.3 / 18.7 / 19.1, 15.6 / 18.1 / 17.0, 12.9 / 16.5 / 16.5;   1024, 1000 55.8 / 45.1 / 52.4, 47.7 / 38.0 / 43.8, 42.3 / 31.8 / 36.4
// Two kernels would be ahead by a tenth to a quarter where the rule does not take them: 65 to 128 of many pages (72, 2000 28.1 / - / 20.9, 27.9 / - / 19.6, 27.9 / - / 18.2;
// 128 unless all are as long, above), and little more than 256, a second round for a few (264, 500 25.0 / 20.2 / 19.0, 22.1 / 19.9 / 17.0, 19.8 / 19.2 / 16.7;
// 264, 2000 67.6 / - / 55.4).
static int threads_of_one(const SelectParams& p, int d) {
  const int cols = columns(p);
  const long long groups = (long long)p.B * p.Hk;
  if ((long long)cols * d <= (groups > 64 ? 32000 : 24000) || (groups > 256 && cols <= Choice<256>::kChunk)) return 256;
  return groups > 64 && cols <= Choice<1024>::kChunk ? 1024 : 0;
}

size_t select_workspace_bytes(const SelectParams& p) { return (size_t)p.B * p.Hk * columns(p) * sizeof(u64); }

hipError_t launch_select(SelectParams p, int d, void* workspace, hipStream_t stream) {
  p.cols = columns(p);
  p.keys = (u64*)workspace;
  const long long groups = (long long)p.B * p.Hk;
  if (!grid_ok(groups, 1024)) return kGridTooLarge;
  const int threads = threads_of_one(p, d);
  if (threads > 0) {
    auto* kernel = d == 128 ? (threads == 256 ? moda_page_select_kernel<128, 256> : moda_page_select_kernel<128, 1024>)
                            : (threads == 256 ? moda_page_select_kernel<64, 256> : moda_page_select_kernel<64, 1024>);
    return launch_kernel(kernel, dim3((unsigned)groups), dim3(threads), stream, p);
  }
  // a wave takes several batches of pages where there are more than 16 waves a compute unit
  const int per_batch = 8 * 256 / d;
  const long long all = groups * ((p.cols + per_batch - 1) / per_batch);
  const int batches = (int)std::min(8ll, std::max(1ll, all / 4096));
  const int chunks = (p.cols + 4 * batches * per_batch - 1) / (4 * batches * per_batch);
  if (!grid_ok(groups * chunks, 256)) return kGridTooLarge;
  const hipError_t e = launch_kernel(d == 128 ? moda_page_score_kernel<128> : moda_page_score_kernel<64>, dim3((unsigned)(groups * chunks)),
                                     dim3(256), stream, p, batches, chunks);
  if (e != hipSuccess) return e;
  // (250 pages of 8 heads, both kernels: 8.8 us with 1024 threads, 7.7 with 256)
  const bool few = p.cols <= Choice<256>::kChunk;
  return launch_kernel(few ? moda_page_choose_kernel<256> : moda_page_choose_kernel<1024>, dim3((unsigned)groups), dim3(few ? 256 : 1024), stream, p);
}

}  // namespace moda
