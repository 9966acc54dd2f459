// The choice of an eviction (moda_evict.hip) for long caches: the rows of a (sequence, head) are dealt out to workgroups of
// kSegRows rows.  What one workgroup finds out step by step takes a launch per step here:
//   begin    largest position of each segment; counters to zero
//   digit    (three times) a histogram of the next digit of the keys that agree with the digits found so far
//   bits     the rows that stay, a bit each; rows that leave below the new length and that stay behind it, per segment
//   movers   the list of the latter, in ascending order
//   index    the i-th of them fills the i-th hole
// Every workgroup reads a digit off the finished histogram by itself; integer sums only, so any order gives one result.
#include "moda_evict.h"
#include "moda_launch.h"

namespace moda {

constexpr int kSegThreads = 256, kSegWaves = kSegThreads / 64, kSegSteps = 8, kSegRows = kSegThreads * kSegSteps;
constexpr int kBins = 2048;  // of a digit: 11, 11 and 10 bits of the key
constexpr int kLastBins = 1024;

struct EvictSegments {
  int n;                      // segments of a (sequence, head)
  unsigned* hist;             // [group][3][kBins]
  int* found;                 // [group][3][2]: digits found so far (as a key), rows that have to come from those that agree
  unsigned short* last_hist;  // [group][segment][kLastBins]: a segment's share of the third histogram
  int *newest, *holes, *movers;  // [group][segment]
  unsigned long long* bits;   // [group][segment][kSegRows / 64]
  int* list;                  // [group][p.n]
};

// What a workgroup works on: its rows are r0 + 64 i, i < kSegSteps.
struct Segment {
  int bg, seg, len, fit, lane, wave, r0;
  __device__ __forceinline__ Segment(const EvictParams& p, const EvictSegments& s) {
    bg = blockIdx.x / s.n;
    seg = blockIdx.x % s.n;
    const int b = bg / p.Hk;
    len = p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
    fit = min(len, p.keep);
    lane = threadIdx.x & 63;
    wave = threadIdx.x >> 6;
    r0 = seg * kSegRows + wave * (64 * kSegSteps) + lane;
  }
  __device__ __forceinline__ bool nothing() const { return len <= fit || seg * kSegRows >= len; }
};

// Sum and maximum over the workgroup.
__device__ __forceinline__ int block_sum(int x, int* part) {
#pragma unroll
  for (int i = 1; i < 64; i *= 2) x += __shfl_xor(x, i);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0;
#pragma unroll
  for (int i = 0; i < kSegWaves; ++i) x += part[i];
  __syncthreads();
  return x;
}
__device__ __forceinline__ int block_max(int x, int* part) {
#pragma unroll
  for (int i = 1; i < 64; i *= 2) x = max(x, __shfl_xor(x, i));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSegWaves; ++i) x = max(x, part[i]);
  __syncthreads();
  return x;
}

// The keys of a thread's rows.
__device__ __forceinline__ void load_keys(const EvictParams& p, const EvictSegments& s, const Segment& g, int* part, unsigned (&keys)[kSegSteps]) {
  long long above = 0x7fffffffLL;
  const bool by_position = p.recent > 0 && p.positions;
  const size_t at = (size_t)g.bg * p.T_alloc;
  float w[kSegSteps];
  int pos[kSegSteps];
#pragma unroll
  for (int i = 0; i < kSegSteps; ++i) {
    const int r = min(g.r0 + i * 64, g.len - 1);
    w[i] = p.w[at + r];
    pos[i] = by_position ? p.positions[at + r] : r;
  }
  if (p.recent > 0) {
    int newest = g.len - 1;
    if (by_position) {
      newest = (int)0x80000000;
      for (int i = threadIdx.x; i * kSegRows < g.len; i += kSegThreads) newest = max(newest, s.newest[g.bg * s.n + i]);
      newest = block_max(newest, part);
    }
    above = (long long)newest - p.recent;
  }
#pragma unroll
  for (int i = 0; i < kSegSteps; ++i) keys[i] = pos[i] > above ? 0xffffffffu : weight_key(w[i]);
}

// Digit `pass` from its finished histogram: what is found so far, and how many rows have to come from those that agree with it.
__device__ __forceinline__ int2 found_with(const EvictParams& p, const EvictSegments& s, const Segment& g, int pass, int* part, int2* out) {
  const int tid = threadIdx.x, per = (pass == 2 ? kLastBins : kBins) / kSegThreads, top = per * kSegThreads - 1;
  const unsigned* hist = s.hist + ((size_t)g.bg * 3 + pass) * kBins;
  int2 f = {0, g.fit};
  if (pass > 0) f = *(const int2*)(s.found + ((size_t)g.bg * 3 + pass - 1) * 2);
  int mine = 0, c[kBins / kSegThreads];
#pragma unroll
  for (int i = 0; i < kBins / kSegThreads; ++i) {  // bins top - per * tid - i: from the heaviest down
    c[i] = i < per ? (int)hist[top - per * tid - i] : 0;
    mine += c[i];
  }
  int sum = mine;
#pragma unroll
  for (int x = 1; x < 64; x *= 2) {
    const int y = __shfl_up(sum, x);
    if (g.lane >= x) sum += y;
  }
  if (g.lane == 63) part[g.wave] = sum;
  __syncthreads();
  for (int i = 0; i < g.wave; ++i) sum += part[i];
  int before = sum - mine;
  if (before < f.y && sum >= f.y) {  // (one thread)
    int digit = top - per * tid;
    bool open = true;
#pragma unroll
    for (int i = 0; i < kBins / kSegThreads; ++i) {
      open = open && before + c[i] < f.y;
      if (open) {
        before += c[i];
        --digit;
      }
    }
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const int2 r = {(int)((unsigned)f.x | (unsigned)digit << shift), f.y - before};
    *out = r;
    if (g.seg == 0) *(int2*)(s.found + ((size_t)g.bg * 3 + pass) * 2) = r;
  }
  __syncthreads();
  return *out;
}

__global__ __launch_bounds__(kSegThreads) void moda_evict_begin_kernel(EvictParams p, EvictSegments s) {
  __shared__ int part[kSegWaves];
  const Segment g(p, s);
  const int first = g.seg * kSegThreads + threadIdx.x, step = s.n * kSegThreads;
  int* index = p.index + (size_t)g.bg * p.n;
  for (int r = first; r < p.n; r += step)
    if (r >= g.fit || g.len <= g.fit) index[r] = r < g.fit ? r : -1;
  for (int i = first; i < 3 * kBins; i += step) s.hist[(size_t)g.bg * 3 * kBins + i] = 0u;
  if (g.nothing() || p.recent == 0 || !p.positions) return;
  int newest = (int)0x80000000;
#pragma unroll
  for (int i = 0; i < kSegSteps; ++i) newest = max(newest, p.positions[(size_t)g.bg * p.T_alloc + min(g.r0 + i * 64, g.len - 1)]);
  newest = block_max(newest, part);
  if (threadIdx.x == 0) s.newest[g.bg * s.n + g.seg] = newest;
}

template <int PASS>
__global__ __launch_bounds__(kSegThreads) void moda_evict_digit_kernel(EvictParams p, EvictSegments s) {
  constexpr int kShift = PASS == 0 ? 21 : PASS == 1 ? 10 : 0, kCount = PASS == 2 ? kLastBins : kBins;
  constexpr unsigned kMask = PASS == 0 ? 0u : ~0u << (PASS == 1 ? 21 : 10);
  __shared__ unsigned hist[kCount];
  __shared__ int part[kSegWaves];
  __shared__ int2 out;
  const Segment g(p, s);
  if (g.nothing()) return;  // (uniform)
  const int tid = threadIdx.x;
  unsigned keys[kSegSteps];
  load_keys(p, s, g, part, keys);
  for (int i = tid; i < kCount; i += kSegThreads) hist[i] = 0u;
  unsigned so_far = 0;
  if (PASS > 0) so_far = (unsigned)found_with(p, s, g, PASS - 1, part, &out).x;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSegSteps; ++i) {
    const bool in = g.r0 + i * 64 < g.len && (keys[i] & kMask) == so_far;
    const unsigned bin = (keys[i] >> kShift) & (kCount - 1);
    // those that share the first lane's digit are counted at once (equal weights, recent rows)
    const unsigned long long all = __ballot(in);
    if (all) {
      const unsigned lead = __builtin_amdgcn_readlane(bin, __builtin_ctzll(all));
      const unsigned long long same = __ballot(in && bin == lead);
      if (in && bin != lead) atomicAdd(&hist[bin], 1u);
      if (g.lane == 0) atomicAdd(&hist[lead], (unsigned)__popcll(same));
    }
  }
  __syncthreads();
  unsigned* to = s.hist + ((size_t)g.bg * 3 + PASS) * kBins;
  for (int i = tid; i < kCount; i += kSegThreads) {
    const unsigned c = hist[i];
    if (c) atomicAdd(&to[i], c);
    if (PASS == 2) s.last_hist[((size_t)g.bg * s.n + g.seg) * kLastBins + i] = (unsigned short)c;
  }
}

// The rows below `fit` of the 64 from `base` on.
__device__ __forceinline__ unsigned long long rows_below(int fit, int base) {
  return fit - base >= 64 ? ~0ull : fit <= base ? 0ull : (1ull << (fit - base)) - 1;
}

__global__ __launch_bounds__(kSegThreads) void moda_evict_bits_kernel(EvictParams p, EvictSegments s) {
  __shared__ int part[kSegWaves];
  __shared__ int2 out;
  const Segment g(p, s);
  if (g.nothing()) return;  // (uniform)
  unsigned keys[kSegSteps];
  load_keys(p, s, g, part, keys);
  const int2 f = found_with(p, s, g, 2, part, &out);
  const unsigned threshold = (unsigned)f.x;
  // rows with just the last key, in the segments and the waves before
  int seen = 0;
  for (int i = threadIdx.x; i < g.seg; i += kSegThreads) seen += s.last_hist[((size_t)g.bg * s.n + i) * kLastBins + (threshold & (kLastBins - 1))];
  seen = block_sum(seen, part);
  unsigned long long tie[kSegSteps], stay[kSegSteps];
  int ties = 0;
#pragma unroll
  for (int i = 0; i < kSegSteps; ++i) {
    const bool in = g.r0 + i * 64 < g.len;
    tie[i] = __ballot(in && keys[i] == threshold);
    stay[i] = __ballot(in && keys[i] > threshold);
    ties += __popcll(tie[i]);
  }
  if (g.lane == 0) part[g.wave] = ties;
  __syncthreads();
  for (int i = 0; i < g.wave; ++i) seen += part[i];
  __syncthreads();
  const unsigned long long below = (1ull << g.lane) - 1;
  int holes = 0, movers = 0;
#pragma unroll
  for (int i = 0; i < kSegSteps; ++i) {
    const int base = g.r0 - g.lane + i * 64;
    if (seen + __popcll(tie[i]) <= f.y) stay[i] |= tie[i];
    else stay[i] |= __ballot(((tie[i] >> g.lane) & 1) && seen + __popcll(tie[i] & below) < f.y);
    seen += __popcll(tie[i]);
    if (g.lane == 0) s.bits[((size_t)g.bg * s.n + g.seg) * (kSegRows / 64) + g.wave * kSegSteps + i] = stay[i];
    const unsigned long long low = rows_below(g.fit, base);
    holes += __popcll(low & ~stay[i]);
    movers += __popcll(stay[i] & ~low);
  }
  holes = block_sum(g.lane == 0 ? holes : 0, part);
  movers = block_sum(g.lane == 0 ? movers : 0, part);
  if (threadIdx.x == 0) {
    s.holes[g.bg * s.n + g.seg] = holes;
    s.movers[g.bg * s.n + g.seg] = movers;
  }
}

// INDEX: holes take what the list holds for them; else the list is written.
template <bool INDEX>
__global__ __launch_bounds__(kSegThreads) void moda_evict_rows_kernel(EvictParams p, EvictSegments s) {
  __shared__ int part[kSegWaves];
  const Segment g(p, s);
  if (g.nothing() || (INDEX ? g.seg * kSegRows >= g.fit : (g.seg + 1) * (long long)kSegRows <= g.fit)) return;  // (uniform)
  const int* counts = INDEX ? s.holes : s.movers;
  int nth = 0;
  for (int i = threadIdx.x; i < g.seg; i += kSegThreads) nth += counts[g.bg * s.n + i];
  nth = block_sum(nth, part);
  unsigned long long stay[kSegSteps], mine[kSegSteps];
  int n = 0;
#pragma unroll
  for (int i = 0; i < kSegSteps; ++i) {
    stay[i] = s.bits[((size_t)g.bg * s.n + g.seg) * (kSegRows / 64) + g.wave * kSegSteps + i];
    const unsigned long long low = rows_below(g.fit, g.r0 - g.lane + i * 64);
    mine[i] = INDEX ? low & ~stay[i] : stay[i] & ~low;
    n += __popcll(mine[i]);
  }
  if (g.lane == 0) part[g.wave] = n;
  __syncthreads();
  for (int i = 0; i < g.wave; ++i) nth += part[i];
  const unsigned long long below = (1ull << g.lane) - 1;
  int* list = s.list + (size_t)g.bg * p.n;
  int* index = p.index + (size_t)g.bg * p.n;
#pragma unroll
  for (int i = 0; i < kSegSteps; ++i) {
    const int r = g.r0 + i * 64, at = nth + __popcll(mine[i] & below);
    const bool hit = (mine[i] >> g.lane) & 1;
    if (INDEX) {
      if (r < g.fit) index[r] = hit ? list[at] : r;
    } else if (hit) {
      list[at] = r;
    }
    nth += __popcll(mine[i]);
  }
}

// ---------------------------------------------------------------- host
static size_t pad16(size_t x) { return (x + 15) / 16 * 16; }

// The arrays in the workspace; returns its size.
static size_t segments(EvictSegments& s, char* ws, long long groups, int T, int n) {
  s.n = (T + kSegRows - 1) / kSegRows;
  size_t at = 0;
  auto take = [&](auto*& ptr, size_t count) {
    ptr = (std::remove_reference_t<decltype(ptr)>)(ws + at);
    at += pad16(count * sizeof(*ptr));
  };
  const size_t segs = (size_t)groups * s.n;
  take(s.hist, (size_t)groups * 3 * kBins);
  take(s.found, (size_t)groups * 6);
  take(s.last_hist, segs * kLastBins);
  take(s.newest, segs);
  take(s.holes, segs);
  take(s.movers, segs);
  take(s.bits, segs * (kSegRows / 64));
  take(s.list, (size_t)groups * n);
  return at;
}

size_t evict_long_workspace_bytes(long long groups, int T, int n) {
  EvictSegments s;
  return segments(s, nullptr, groups, T, n);
}

bool evict_long_grid_ok(long long groups, int T) { return grid_ok(groups * ((T + kSegRows - 1) / kSegRows), kSegThreads); }

hipError_t launch_evict_choose_long(const EvictParams& p, void* workspace, hipStream_t stream) {
  EvictSegments s;
  const long long groups = (long long)p.B * p.Hk;
  segments(s, (char*)workspace, groups, p.T, p.n);
  const dim3 grid((unsigned)(groups * s.n)), block(kSegThreads);
  for (auto* kernel : {moda_evict_begin_kernel, moda_evict_digit_kernel<0>, moda_evict_digit_kernel<1>, moda_evict_digit_kernel<2>,
                       moda_evict_bits_kernel, moda_evict_rows_kernel<false>, moda_evict_rows_kernel<true>}) {
    const hipError_t e = launch_kernel(kernel, grid, block, stream, p, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace moda
