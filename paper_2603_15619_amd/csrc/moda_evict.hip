// Eviction from a sequence cache: which rows of a (sequence, key/value head) stay, and their move.
//
// choice : one workgroup per (sequence, head).  A row's rank is a 32-bit key that orders as its weight does (recent rows
//          above everything else); the key of the last row that stays is found in three digits from histograms, ties
//          are counted in row order.  Kept rows below the new length keep their row; the i-th kept row
//          behind it takes the i-th hole below it.  Result: `index`, the row that every new row comes from.
// move   : rows of K and V, weights and positions from index[r] to r.  In place, a moved row lies behind the new length
//          and a hole below it, so no row is both read and written, in whatever order the workgroups run.
#include <algorithm>

#include "moda_evict.h"
#include "moda_launch.h"

namespace moda {

constexpr int kEvThreads = 1024;  // most threads of the workgroup that chooses

// THREADS: few for few rows, whose barriers and sums over the waves are then shorter.
// Rows of a (sequence, head): wave w takes N times 64 of them, from w * N * 64 on; a row's key stays in a register from its one
// read on.
template <int N, int THREADS>
__global__ __launch_bounds__(THREADS) void moda_evict_choose_kernel(EvictParams p) {
  constexpr int kBins = 2048, kWaves = THREADS / 64, kPer = kBins / THREADS;
  __shared__ unsigned hist[kBins];
  __shared__ int part[kWaves], part2[kWaves];
  __shared__ unsigned s_digit;
  __shared__ int s_need;
  // rows that stay, a bit each; rows that move, in ascending order (half of all at most: as many as there are holes)
  __shared__ unsigned long long bits[kWaves * N];
  __shared__ unsigned short list[THREADS * N / 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int bg = blockIdx.x, b = bg / p.Hk;
  const int len = p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
  const int fit = min(len, p.keep);
  int* index = p.index + (size_t)bg * p.n;
  for (int r = fit + tid; r < p.n; r += THREADS) index[r] = -1;
  if (len <= p.keep) {
    for (int r = tid; r < fit; r += THREADS) index[r] = r;
    return;
  }
  const float* w = p.w + (size_t)bg * p.T_alloc;
  const int* pos = p.positions ? p.positions + (size_t)bg * p.T_alloc : nullptr;
  const int r0 = wave * N * 64 + lane;  // the lane's rows: r0 + 64 i
  unsigned keys[N];
  // bounds-checked loads from one address register; rows past the end read as 0
  const __amdgpu_buffer_rsrc_t w_buf = __builtin_amdgcn_make_buffer_rsrc((void*)w, 0, len * 4, 0x00020000);
  const __amdgpu_buffer_rsrc_t pos_buf = __builtin_amdgcn_make_buffer_rsrc((void*)pos, 0, pos ? len * 4 : 0, 0x00020000);
  auto each = [&](auto&& f) {  // f(i) for every step
#pragma unroll
    for (int i = 0; i < N; ++i) f(i);
  };

  long long above = 0x7fffffffLL;  // rows whose position is above this are recent
  const bool by_position = p.recent > 0 && pos;
  if (p.recent > 0) {
    int newest = len - 1;
    if (pos) {
      newest = (int)0x80000000;
      each([&](int i) {
        const int x = __builtin_amdgcn_raw_buffer_load_b32(pos_buf, r0 * 4, i * 256, 0);
        keys[i] = (unsigned)x;
        if (r0 + i * 64 < len) newest = max(newest, x);
      });
#pragma unroll
      for (int x = 1; x < 64; x *= 2) newest = max(newest, __shfl_xor(newest, x));
      if (lane == 0) part[wave] = newest;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kWaves; ++i) newest = max(newest, part[i]);
      __syncthreads();
    }
    above = (long long)newest - p.recent;
  }
  each([&](int i) {
    const int at = by_position ? (int)keys[i] : r0 + i * 64;
    const unsigned k = weight_key(__builtin_bit_cast(float, (unsigned)__builtin_amdgcn_raw_buffer_load_b32(w_buf, r0 * 4, i * 256, 0)));
    keys[i] = at > above ? 0xffffffffu : k;
  });

  // the key of the fit-th row from the top, and how many of the rows with just that key stay: 11, 11 and 10 bits
  unsigned threshold = 0;
  int need = fit;
  auto digit = [&](int shift) {
    const unsigned mask = shift == 21 ? 0u : ~0u << (shift == 10 ? 21 : 10);
    for (int i = tid; i < kBins; i += THREADS) hist[i] = 0;
    __syncthreads();
    each([&](int i) {
      const unsigned k = keys[i];
      const bool in = r0 + i * 64 < len && (k & mask) == threshold;
      const unsigned bin = (k >> shift) & (kBins - 1);
      // many rows share a digit (equal weights, recent rows): those that share the first lane's are counted at once
      const unsigned long long in_all = __ballot(in);
      if (in_all) {
        const unsigned lead = __builtin_amdgcn_readlane(bin, __builtin_ctzll(in_all));
        const unsigned long long same = __ballot(in && bin == lead);
        if (in && bin != lead) atomicAdd(&hist[bin], 1u);
        if (lane == 0) atomicAdd(&hist[lead], (unsigned)__popcll(same));
      }
    });
    __syncthreads();
    // thread t: kPer bins from kBins - 1 - kPer t down; `sum` = rows in the bins of threads up to this one
    int c[kPer], both = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) both += c[i] = (int)hist[kBins - 1 - kPer * tid - i];
    int sum = both;
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
      const int y = __shfl_up(sum, x);
      if (lane >= x) sum += y;
    }
    if (lane == 63) part[wave] = sum;
    __syncthreads();
    for (int i = 0; i < wave; ++i) sum += part[i];
    int before = sum - both;
    if (before < need && sum >= need) {  // (one thread)
      int i = 0;
#pragma unroll
      for (int x = 0; x < kPer - 1; ++x)
        if (i == x && before + c[x] < need) {
          before += c[x];
          ++i;
        }
      s_digit = kBins - 1 - kPer * tid - i;
      s_need = need - before;
    }
    __syncthreads();
    threshold |= s_digit << shift;
    need = s_need;
  };
  digit(21);
  digit(10);
  digit(0);

  const unsigned long long below = (1ull << lane) - 1;
  auto before = [&](const int* counts) {  // sum over the waves before this one
    int n = 0;
    for (int i = 0; i < wave; ++i) n += counts[i];
    return n;
  };
  int ties = 0;
  each([&](int i) { ties += __popcll(__ballot(r0 + i * 64 < len && keys[i] == threshold)); });
  if (lane == 0) part[wave] = ties;
  __syncthreads();
  const int ties_before = before(part);
  __syncthreads();
  // which rows stay, one word of bits per step (`bits`), and the waves' holes below the new length and rows to move behind it
  int seen = ties_before, holes = 0, movers = 0;
  each([&](int i) {
    const int r = r0 + i * 64, base = r - lane;
    const unsigned k = keys[i];
    const unsigned long long tie = __ballot(r < len && k == threshold);
    unsigned long long stay = __ballot(r < len && k > threshold);
    if (seen + __popcll(tie) <= need) stay |= tie;
    else stay |= __ballot(((tie >> lane) & 1) && seen + __popcll(tie & below) < need);
    seen += __popcll(tie);
    if (lane == 0) bits[wave * N + i] = stay;
    const unsigned long long low = fit - base >= 64 ? ~0ull : fit <= base ? 0ull : (1ull << (fit - base)) - 1;
    holes += __popcll(low & ~stay);
    movers += __popcll(stay & ~low);
  });
  if (lane == 0) {
    part[wave] = holes;
    part2[wave] = movers;
  }
  __syncthreads();
  int nth = before(part2);
#pragma unroll 4
  for (int i = 0; i < N; ++i) {
    const int r = r0 + i * 64, base = r - lane;
    if (base + 64 <= fit) continue;  // (uniform)
    const unsigned long long stay = bits[wave * N + i];
    const unsigned long long mv = fit <= base ? stay : stay & ~((1ull << (fit - base)) - 1);
    if ((mv >> lane) & 1) list[nth + __popcll(mv & below)] = r;
    nth += __popcll(mv);
  }
  __syncthreads();
  nth = before(part);
#pragma unroll 4
  for (int i = 0; i < N; ++i) {
    const int r = r0 + i * 64, base = r - lane;
    if (base >= fit) continue;  // (uniform)
    const unsigned long long stay = bits[wave * N + i], low = fit - base >= 64 ? ~0ull : (1ull << (fit - base)) - 1;
    const unsigned long long hole = low & ~stay;
    if (r < fit) index[r] = ((hole >> lane) & 1) ? list[nth + __popcll(hole & below)] : r;
    nth += __popcll(hole);
  }
}

// Two 16-byte pieces of K and of V per thread, all loaded before any store; the thread of a row's first piece moves its weight and
// position.
constexpr int kMovePieces = 2;
__global__ __launch_bounds__(256) void moda_evict_move_kernel(EvictParams p, int per_row_log2, int n_chunks) {
  const int bg = blockIdx.x / n_chunks, b = bg / p.Hk;
  const long long i0 = (long long)(blockIdx.x % n_chunks) * (256 * kMovePieces) + threadIdx.x;
  if (p.lengths_out && i0 == 0 && bg == b * p.Hk)
    p.lengths_out[b] = min(p.keep, p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T);
  u32x4 k[kMovePieces], v[kMovePieces];
  long long from[kMovePieces], to[kMovePieces];  // rows; from < 0: nothing to move
  const int c = (int)(i0 & ((1 << per_row_log2) - 1));
#pragma unroll
  for (int u = 0; u < kMovePieces; ++u) {
    const long long r = (i0 + u * 256) >> per_row_log2;
    int src = -1;
    if (r < p.n) src = p.index[(size_t)bg * p.n + r];
    if (p.in_place && src == r) src = -1;
    from[u] = src < 0 ? -1 : (long long)bg * p.T_alloc + src;
    to[u] = (long long)bg * p.out_alloc + r;
  }
#pragma unroll
  for (int u = 0; u < kMovePieces; ++u)
    if (from[u] >= 0) {
      k[u] = __builtin_nontemporal_load((const u32x4*)(p.K + from[u] * p.row_bytes) + c);
      v[u] = __builtin_nontemporal_load((const u32x4*)(p.V + from[u] * p.row_bytes) + c);
    }
#pragma unroll
  for (int u = 0; u < kMovePieces; ++u)
    if (from[u] >= 0) {
      __builtin_nontemporal_store(k[u], (u32x4*)(p.K_out + to[u] * p.row_bytes) + c);
      __builtin_nontemporal_store(v[u], (u32x4*)(p.V_out + to[u] * p.row_bytes) + c);
      if (c == 0) {
        p.w_out[to[u]] = p.w[from[u]];
        if (p.positions) p.positions_out[to[u]] = p.positions[from[u]];
      }
    }
}

// Longest cache that one workgroup chooses from.
constexpr int kEvOneWorkgroup = 32 * kEvThreads;

size_t evict_workspace_bytes(int B, int Hk, int T, int keep) {
  return T <= kEvOneWorkgroup ? 16 : evict_long_workspace_bytes((long long)B * Hk, T, std::min(keep, T));
}

hipError_t launch_evict(const EvictParams& p, void* workspace, hipStream_t stream) {
  const long long groups = (long long)p.B * p.Hk;
  const int per_row_log2 = p.row_bytes == 128 ? 3 : p.row_bytes == 256 ? 4 : 5;  // pieces of 16 bytes of a row: 8, 16 or 32
  const long long chunks = (((long long)p.n << per_row_log2) + 256 * kMovePieces - 1) / (256 * kMovePieces);
  if (!grid_ok(groups, kEvThreads) || chunks > 0x7fffffff || !grid_ok(groups * chunks, 256)) return kGridTooLarge;
  hipError_t e;
  if (p.T > kEvOneWorkgroup) {
    if (!evict_long_grid_ok(groups, p.T)) return kGridTooLarge;
    e = launch_evict_choose_long(p, workspace, stream);
  } else {
    // (1024 / 256 threads, 8 heads, half of the rows stay, whole call: T=100 10.6 / 9.0 us, T=500 10.9 / 9.4, T=1090 12.2 / 15.0)
    const int threads = p.T <= 512 ? 256 : kEvThreads;
    auto* choose = p.T <= 512 ? moda_evict_choose_kernel<2, 256> : p.T <= 1024 ? moda_evict_choose_kernel<1, 1024>
                   : p.T <= 2048 ? moda_evict_choose_kernel<2, 1024> : p.T <= 4096 ? moda_evict_choose_kernel<4, 1024>
                   : p.T <= 8192 ? moda_evict_choose_kernel<8, 1024> : p.T <= 16384 ? moda_evict_choose_kernel<16, 1024>
                   : moda_evict_choose_kernel<32, 1024>;
    e = launch_kernel(choose, dim3((unsigned)groups), dim3(threads), stream, p);
  }
  if (e != hipSuccess) return e;
  return launch_kernel(moda_evict_move_kernel, dim3((unsigned)(groups * chunks)), dim3(256), stream, p, per_row_log2, (int)chunks);
}

}  // namespace moda
