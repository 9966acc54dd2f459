// Eviction from a sequence cache: which rows of a (sequence, key/value head) stay, and their move.
//
// choice : one workgroup per (sequence, head).  A row's rank is a 32-bit key that orders as its weight does (recent rows
//          above everything else); the key of the last row that stays is found digit by digit from histograms, ties
//          are counted in row order.  Kept rows below the new length keep their row; the i-th kept row
//          behind it takes the i-th hole below it.  Result: `index`, the row that every new row comes from.
// move   : rows of K and V, weights and positions from index[r] to r.  In place, a moved row lies behind the new length
//          and a hole below it, so no row is both read and written, in whatever order the workgroups run.
#include <algorithm>

#include "moda_launch.h"

namespace moda {

constexpr int kEvThreads = 1024, kEvWaves = kEvThreads / 64;

// Orders as the float does; -0 as 0, a NaN below everything.
__device__ __forceinline__ unsigned weight_key(float w) {
  const unsigned u = __builtin_bit_cast(unsigned, w + 0.f);
  return w != w ? 0u : u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

__global__ __launch_bounds__(kEvThreads) void moda_evict_choose_kernel(EvictParams p, int* movers_ws) {
  __shared__ unsigned hist[256];
  __shared__ int part[kEvWaves], part2[kEvWaves];
  __shared__ int s_digit, s_need;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int bg = blockIdx.x, b = bg / p.Hk;
  const int len = p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
  const int fit = min(len, p.keep);
  int* index = p.index + (size_t)bg * p.n;
  for (int r = fit + tid; r < p.n; r += kEvThreads) index[r] = -1;
  if (len <= p.keep) {
    for (int r = tid; r < fit; r += kEvThreads) index[r] = r;
    return;
  }
  const float* w = p.w + (size_t)bg * p.T_alloc;
  const int* pos = p.positions ? p.positions + (size_t)bg * p.T_alloc : nullptr;
  long long above = 0x7fffffffLL;  // rows whose position is above this are recent
  if (p.recent > 0) {
    int newest = len - 1;
    if (pos) {
      newest = (int)0x80000000;
      for (int r = tid; r < len; r += kEvThreads) newest = max(newest, pos[r]);
#pragma unroll
      for (int x = 1; x < 64; x *= 2) newest = max(newest, __shfl_xor(newest, x));
      if (lane == 0) part[wave] = newest;
      __syncthreads();
      for (int i = 0; i < kEvWaves; ++i) newest = max(newest, part[i]);
      __syncthreads();
    }
    above = (long long)newest - p.recent;
  }
  auto key_of = [&](int r) { return (long long)(pos ? pos[r] : r) > above ? 0xffffffffu : weight_key(w[r]); };

  // the key of the fit-th row from the top, and how many of the rows with just that key stay
  unsigned threshold = 0;
  int need = fit;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    const unsigned mask = shift == 24 ? 0u : ~0u << (shift + 8);
    for (int r = tid; r < len; r += kEvThreads) {
      const unsigned k = key_of(r);
      if ((k & mask) == threshold) atomicAdd(&hist[(k >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      int left = need, digit = 255;
      while (left > (int)hist[digit]) left -= hist[digit--];
      s_digit = digit;
      s_need = left;
    }
    __syncthreads();
    threshold |= (unsigned)s_digit << shift;
    need = s_need;
    __syncthreads();
  }

  // a wave takes a stretch of rows, 64 at a time
  const int stretch = (len + kEvThreads - 1) / kEvThreads * 64;
  const int r0 = wave * stretch, r1 = min(len, r0 + stretch);
  const unsigned long long below = (1ull << lane) - 1;
  auto before = [&](int* counts) {  // sum over the waves before this one
    int n = 0;
    for (int i = 0; i < wave; ++i) n += counts[i];
    return n;
  };
  int ties = 0;
  for (int base = r0; base < r1; base += 64)
    ties += __popcll(__ballot(base + lane < r1 && key_of(base + lane) == threshold));
  if (lane == 0) part[wave] = ties;
  __syncthreads();
  const int ties_before = before(part);
  __syncthreads();
  auto walk = [&](auto&& f) {  // f(row, stays) for every row of the stretch, all lanes
    int seen = ties_before;
    for (int base = r0; base < r1; base += 64) {
      const int r = base + lane;
      const unsigned k = r < r1 ? key_of(r) : 0u;
      const unsigned long long tie = __ballot(r < r1 && k == threshold);
      const bool is_tie = (tie >> lane) & 1;
      f(r, r < r1 && (is_tie ? seen + __popcll(tie & below) < need : k > threshold));
      seen += __popcll(tie);
    }
  };
  int holes = 0, movers = 0;
  walk([&](int r, bool stays) {
    holes += __popcll(__ballot(r < fit && r < r1 && !stays));
    movers += __popcll(__ballot(r >= fit && stays));
  });
  if (lane == 0) {
    part[wave] = holes;
    part2[wave] = movers;
  }
  __syncthreads();
  int* list = movers_ws + (size_t)bg * p.n;
  int nth = before(part2);
  walk([&](int r, bool stays) {
    const unsigned long long mv = __ballot(r >= fit && stays);
    if ((mv >> lane) & 1) list[nth + __popcll(mv & below)] = r;
    nth += __popcll(mv);
  });
  __syncthreads();
  nth = before(part);
  walk([&](int r, bool stays) {
    const unsigned long long ho = __ballot(r < fit && r < r1 && !stays);
    if (r < fit && r < r1) index[r] = stays ? r : list[nth + __popcll(ho & below)];
    nth += __popcll(ho);
  });
}

// 16 bytes of K and of V per thread; the thread of a row's first 16 bytes moves its weight and position.
__global__ __launch_bounds__(256) void moda_evict_move_kernel(EvictParams p, int per_row, int n_chunks) {
  const int bg = blockIdx.x / n_chunks, b = bg / p.Hk;
  const long long i = (long long)(blockIdx.x % n_chunks) * 256 + threadIdx.x;
  const int r = (int)(i / per_row), c = (int)(i % per_row);
  if (p.lengths_out && i == 0 && bg == b * p.Hk)
    p.lengths_out[b] = min(p.keep, p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T);
  if (r >= p.n) return;
  const int src = p.index[(size_t)bg * p.n + r];
  if (src < 0 || (p.in_place && src == r)) return;
  const size_t from = (size_t)bg * p.T_alloc + src, to = (size_t)bg * p.out_alloc + r;
  const u32x4 k = *(const u32x4*)(p.K + from * p.row_bytes + c * 16), v = *(const u32x4*)(p.V + from * p.row_bytes + c * 16);
  *(u32x4*)(p.K_out + to * p.row_bytes + c * 16) = k;
  *(u32x4*)(p.V_out + to * p.row_bytes + c * 16) = v;
  if (c == 0) {
    p.w_out[to] = p.w[from];
    if (p.positions) p.positions_out[to] = p.positions[from];
  }
}

size_t evict_workspace_bytes(int B, int Hk, int T, int keep) {
  return std::max<size_t>(16, (size_t)B * Hk * std::min(keep, T) * sizeof(int));
}

hipError_t launch_evict(const EvictParams& p, void* workspace, hipStream_t stream) {
  const long long groups = (long long)p.B * p.Hk;
  const int per_row = p.row_bytes / 16;
  const long long chunks = ((long long)p.n * per_row + 255) / 256;
  if (!grid_ok(groups, kEvThreads) || chunks > 0x7fffffff || !grid_ok(groups * chunks, 256)) return kGridTooLarge;
  const hipError_t e = launch_kernel(moda_evict_choose_kernel, dim3((unsigned)groups), dim3(kEvThreads), stream, p, (int*)workspace);
  if (e != hipSuccess) return e;
  return launch_kernel(moda_evict_move_kernel, dim3((unsigned)(groups * chunks)), dim3(256), stream, p, per_row, (int)chunks);
}

}  // namespace moda
