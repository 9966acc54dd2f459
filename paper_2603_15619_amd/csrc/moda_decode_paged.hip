// Decoding step over a paged sequence cache: per new token one softmax over the rows of its sequence's pages, or of those that a list
// names, and its depth slots.
//
// The formulas are those of moda_decode_shared.hip: (m, l, unnormalised O) of disjoint sets of rows merge exactly, so the rows are cut into
// slices over workgroups, whose states go to the workspace in fp32, and a second kernel merges them.
// The cut is made on the device, from the lengths themselves: a paged cache's table is as wide as the longest sequence may become, and a
// cut by that bound would leave most workgroups without rows.  Slices are of about one size for all sequences, so that sequences of any lengths
// fill the chip evenly; every workgroup adds up the lengths and finds its slice (find_slice).
// What bounds it: long calls the reads (8 x 65536 ragged rows, 16 heads, d = 128 6.45 TB/s; 32 x 16000 8-bit rows, 64 heads on 8 5.5), short ones the chain of
// three loads (lengths, page numbers, rows), each of about 0.8 us, and a second launch where a sequence has several slices (4 us).
#include <algorithm>

#include "moda_decode_columns.h"
#include "moda_pages.h"

namespace moda {

constexpr int kPgWaves = 4;
// Workgroups that the cut aims at, and the least rows that it gives them: one per compute unit (whole steps of the waves), as many as are
// resident at once, and, where slices are long, several rounds of them: workgroups do not get equal shares of the memory's rate, and
// in one round the slowest decide.
constexpr int kPgFew = 256, kPgOnce = 512, kPgOnceRows = 512, kPgMany = 2048;

// ---------------------------------------------------------------- the cut
// Rows of a sequence: of its cache, or of the places on its lists (whole pages: what a page holds is looked at later).
__device__ __forceinline__ int paged_rows(const PagedParams& p, int b) {
  return p.selected ? p.n_selected << p.shift : filled(p.lengths, b, p.T);
}

struct Slice {
  int b;            // -1: no such slice
  int begin, rows;  // its first row, and all rows of the sequence
  int per;          // rows of its slices
  int first, n;     // the sequence's first slice, and how many it has
};
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }
// (thousands of rows would do 32 bits, a large batch of long sequences not: 16 bits at a time)
__device__ __forceinline__ long long wave_sum_rows(int rows) { return ((long long)wave_sum(rows >> 16) << 16) + wave_sum(rows & 0xffff); }

// Rows of a slice, in whole steps of 1 << least_shift, where all sequences together have `total`.
__device__ __forceinline__ unsigned slice_rows(const PagedParams& p, long long total) {
  auto share = [&](int workgroups) {
    const long long n = total * p.units + workgroups - 1, step = 1ll << p.least_shift;
    return ((n / workgroups + step - 1) >> p.least_shift) << p.least_shift;
  };
  const long long once = max(share(kPgOnce), (long long)kPgOnceRows), many = max(share(kPgMany), (long long)p.good);
  // (2^30 rows: more than a sequence has)
  return (unsigned)min(max(min(share(kPgFew), min(once, many)), 1ll << p.least_shift), 1ll << 30);
}
// Slice s of the n slices, the first of them slice `first`, that sequence b of so many rows has.
__device__ __forceinline__ Slice slice_of(const PagedParams& p, int s, int b, int rows, int first, int n) {
  // (all of the same size)
  const int per = ((((unsigned)rows + n - 1) / (unsigned)n + (1u << p.least_shift) - 1) >> p.least_shift) << p.least_shift;
  return Slice{b, min((s - first) * per, rows), rows, per, first, n};
}

// Slice s of all slices.  Up to kPgLook sequences every wave looks at their lengths, a lane at one of each 64; more of them moda_paged_deal_kernel
// has dealt the slices out.
constexpr int kPgLook = 256;
__device__ __forceinline__ Slice find_slice(const PagedParams& p, int s, int lane) {
  if (p.B <= kPgLook) {  // (uniform)
    constexpr int kChunks = kPgLook / 64;
    int rows[kChunks];
    long long total = 0;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) rows[i] = i * 64 + lane < p.B ? paged_rows(p, i * 64 + lane) : 0;
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
      if (i * 64 < p.B) total += wave_sum_rows(rows[i]);
    const unsigned per = slice_rows(p, total);
    int before = 0;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (i * 64 >= p.B) break;  // (uniform)
      const int n = i * 64 + lane < p.B ? max((int)(((unsigned)rows[i] + per - 1) / per), 1) : 0;
      const int to = before + wave_scan(n);  // of this sequence and those before it
      const unsigned long long behind = __builtin_amdgcn_ballot_w64(to > s);
      if (behind) {  // (uniform)
        const int l = __builtin_ctzll(behind), n_l = __builtin_amdgcn_readlane(n, l);
        return slice_of(p, s, i * 64 + l, __builtin_amdgcn_readlane(rows[i], l), __builtin_amdgcn_readlane(to, l) - n_l, n_l);
      }
      before = __builtin_amdgcn_readlane(to, 63);
    }
    return Slice{-1, 0, 0, 0, 0, 0};
  }
  // the last sequence whose first slice is s or one before it, among [b, end): 64 of them at a time
  int b = 0, end = p.B;
  while (end - b > 1) {  // (uniform)
    const int step = (end - b + 63) / 64, i = b + lane * step;
    const unsigned long long upto = __builtin_amdgcn_ballot_w64(i < end && p.ws_deal[2 * min(i, end - 1)] <= s);
    b += (__builtin_popcountll(upto) - 1) * step;  // (the first of them is)
    end = min(end, b + step);
  }
  const int first = __builtin_amdgcn_readfirstlane(p.ws_deal[2 * b]), n = __builtin_amdgcn_readfirstlane(p.ws_deal[2 * b + 1]);
  if (s >= first + n) return Slice{-1, 0, 0, 0, 0, 0};
  return slice_of(p, s, b, __builtin_amdgcn_readfirstlane(paged_rows(p, b)), first, n);
}

// Many sequences: first slice and number of slices of each, by one workgroup.
constexpr int kDealThreads = 1024;
__global__ __launch_bounds__(kDealThreads) void moda_paged_deal_kernel(PagedParams p) {
  constexpr int kWaves = kDealThreads / 64;
  __shared__ long long sums[kWaves];
  __shared__ int counts[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  long long total = 0;
  for (int b0 = 0; b0 < p.B; b0 += kDealThreads) total += wave_sum_rows(b0 + tid < p.B ? paged_rows(p, b0 + tid) : 0);
  if (lane == 0) sums[wave] = total;
  __syncthreads();
  total = 0;
  for (int w = 0; w < kWaves; ++w) total += sums[w];
  const unsigned per = slice_rows(p, total);
  int before = 0;
  for (int b0 = 0; b0 < p.B; b0 += kDealThreads) {  // (uniform)
    const int b = b0 + tid, n = b < p.B ? max((int)(((unsigned)paged_rows(p, b) + per - 1) / per), 1) : 0, to = wave_scan(n);
    if (lane == 63) counts[wave] = to;
    __syncthreads();
    const int of_wave = counts[lane % kWaves], up_to = row_scan(of_wave);
    const int first = before + __builtin_amdgcn_readlane(up_to - of_wave, wave) + to - n;  // (with all lanes: one of them is read)
    if (b < p.B) {
      p.ws_deal[2 * b] = first;
      p.ws_deal[2 * b + 1] = n;
    }
    before += __builtin_amdgcn_readlane(up_to, kWaves - 1);
    __syncthreads();  // (the counts have been read)
  }
}

// The one slice of sequence b.
__device__ __forceinline__ Slice whole_sequence(const PagedParams& p, int b) {
  const int rows = paged_rows(p, b);
  return Slice{b, 0, rows, rows, b, 1};
}

// ---------------------------------------------------------------- pages
// 64 pages of a sequence's list from page `base` on, one a lane: its number in the pool, and the rows that the sequence has in it.
struct PageList {
  const int* table;
  const int* selected;  // or null
  int len;              // rows of the sequence
  int base, page, at;   // as the table has it, -1: none
  int id, count;
  __device__ __forceinline__ PageList(const PagedParams& p, int b, int g)
      : table(p.table + (size_t)b * p.max_pages), selected(p.selected ? p.selected + ((size_t)b * p.Hk + g) * p.n_selected : nullptr) {}
  // (which does not wait for the length)
  __device__ __forceinline__ void fetch(const PagedParams& p, int from, int lane) {
    base = from;
    page = from + lane;
    if (selected) page = page < p.n_selected ? selected[page] : -1;
    at = (unsigned)page < (unsigned)p.max_pages ? page_at(table, page, p.n_pages) : -1;
  }
  __device__ __forceinline__ void settle(const PagedParams& p) {
    id = max(at, 0);
    count = at < 0 ? 0 : min(max(len - (page << p.shift), 0), 1 << p.shift);
  }
  __device__ __forceinline__ void load(const PagedParams& p, int from, int lane) {
    fetch(p, from, lane);
    settle(p);
  }
};

// ---------------------------------------------------------------- rows on the vector ALUs
// A lane owns CPL channels (16 bytes of a cached row), D / CPL lanes a row; a wave takes kU batches of adjacent rows at a time.
template <int D, int GT, int CPL>
struct RowState {
  static constexpr int LPR = D / CPL, RPS = 64 / LPR, kU = 4;
  uint32_t q[GT][CPL / 2];
  float m[GT], l[GT], o[GT][CPL];
  template <class Query>
  __device__ __forceinline__ void init(Query&& query, int nh, int l16) {
#pragma unroll
    for (int j = 0; j < GT; ++j) {
#pragma unroll
      for (int k = 0; k < CPL / 8; ++k) *(u32x4*)&q[j][k * 4] = *(const u32x4*)(query(min(j, nh - 1)) + l16 * CPL * 2 + k * 16);
      m[j] = -INFINITY;
      l[j] = 0.f;
#pragma unroll
      for (int k = 0; k < CPL; ++k) o[j][k] = 0.f;
    }
  }
  // kU batches: key(u, i) = channels 2 i, 2 i + 1 as packed bf16, value(u, i) = the same of V as two floats; row rg of batch u counts if rg < left[u].
  template <class Key, class Value>
  __device__ __forceinline__ void fold(Key&& key, Value&& value, const int (&left)[kU], int rg, float c2) {
    float sc[GT][kU];
#pragma unroll
    for (int j = 0; j < GT; ++j)
#pragma unroll
      for (int u = 0; u < kU; ++u) sc[j][u] = 0.f;
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
      for (int i = 0; i < CPL / 2; ++i) {
        const uint32_t k = key(u, i);
#pragma unroll
        for (int j = 0; j < GT; ++j) sc[j][u] = dot2_bf16(q[j][i], k, sc[j][u]);
      }
#pragma unroll
    for (int j = 0; j < GT; ++j) {
      float mn = m[j];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        float a = sc[j][u];
        a += dpp_mov<0xB1>(a);
        a += dpp_mov<0x4E>(a);
        if (LPR >= 8) a += dpp_mov<0x141>(a);
        if (LPR >= 16) a += dpp_mov<0x140>(a);
        sc[j][u] = rg < left[u] ? a : -INFINITY;
        mn = fmaxf(mn, sc[j][u]);
      }
      // (mn is -inf only while every score so far was, or was NaN, which stays NaN; with reference 0 the others weigh nothing)
      const float ref = mn == -INFINITY ? 0.f : mn;
      const float al = fast_exp2((m[j] - ref) * c2);
      m[j] = mn;
      l[j] *= al;
#pragma unroll
      for (int k = 0; k < CPL; ++k) o[j][k] *= al;
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        sc[j][u] = fast_exp2((sc[j][u] - ref) * c2);
        l[j] += sc[j][u];
      }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
      for (int i = 0; i < CPL / 2; ++i) {
        const f32x2 v = value(u, i);
#pragma unroll
        for (int j = 0; j < GT; ++j) {
          o[j][2 * i] += sc[j][u] * v[0];
          o[j][2 * i + 1] += sc[j][u] * v[1];
        }
      }
  }
};

// A batch of rows in flight: 16 bytes of K and of V per lane, and the scales of 8-bit rows.
template <int kU, bool MX>
struct RowBatch {
  u32x4 k[kU], v[kU];
  unsigned ks[MX ? kU : 1], vs[MX ? kU : 1];
  int left[kU];
};

template <int D, int GT, bool MX>
__global__ __launch_bounds__(kPgWaves * 64, 2) void moda_paged_slices_kernel(PagedParams p) {
  constexpr int CPL = MX ? 16 : 8, LPR = D / CPL, RPS = 64 / LPR, RB = D * 2, CB = MX ? D : RB, SB = D / kBlock;
  using State = RowState<D, GT, CPL>;
  constexpr int kU = State::kU, STEP = kPgWaves * kU * RPS;
  __shared__ __attribute__((aligned(16))) float red[kPgWaves * GT * (D + 2)];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane % LPR, rg = lane / LPR;
  const float c2 = p.scale_log2;
  const int unit = blockIdx.x % p.units, s = blockIdx.x / p.units;
  const Slice x = p.single ? whole_sequence(p, s) : find_slice(p, s, lane);
  if (x.b < 0) return;  // (uniform)
  const int b = x.b, G = p.Hq / p.Hk, g = unit % p.Hk, gc = unit / p.Hk;
  const int nh = min(GT, G - gc * GT);
  const size_t bh = (size_t)b * p.Hq + g * G + gc * GT;
  if (unit == 0 && s == x.first && tid == 0 && !p.single && p.B <= kPgLook) {
    p.ws_deal[2 * b] = x.first;
    p.ws_deal[2 * b + 1] = x.n;
  }
  State st;
  st.init([&](int j) { return (const char*)p.Q + (bh + j) * RB; }, nh, l16);
  const int end = min(x.rows, x.begin + x.per);
  if (x.begin < end) {  // (uniform)
    PageList list(p, b, g);
    list.len = filled(p.lengths, b, p.T);
    list.load(p, x.begin >> p.shift, lane);
    using Batch = RowBatch<kU, MX>;
    auto issue = [&](int row, Batch& r) {
      if (((row + kU * RPS - 1) >> p.shift) - list.base >= 64) list.load(p, row >> p.shift, lane);  // (uniform)
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int at = row + u * RPS, i = (at >> p.shift) - list.base, slot = at & ((1 << p.shift) - 1);
        const int id = __builtin_amdgcn_readlane(list.id, i), count = __builtin_amdgcn_readlane(list.count, i);
        const size_t row0 = ((size_t)id * p.Hk + g) << p.shift;
        const __amdgpu_buffer_rsrc_t kb = rows_buffer(p.K + row0 * CB, count * CB), vb = rows_buffer(p.V + row0 * CB, count * CB);
        r.k[u] = __builtin_amdgcn_raw_buffer_load_b128(kb, (slot + rg) * CB + l16 * 16, 0, 2);
        r.v[u] = __builtin_amdgcn_raw_buffer_load_b128(vb, (slot + rg) * CB + l16 * 16, 0, 2);
        if (MX) {
          const __amdgpu_buffer_rsrc_t ksb = rows_buffer(p.Ks + row0 * SB, count * SB), vsb = rows_buffer(p.Vs + row0 * SB, count * SB);
          r.ks[u] = __builtin_amdgcn_raw_buffer_load_b8(ksb, (slot + rg) * SB + l16 * CPL / kBlock, 0, 0);
          r.vs[u] = __builtin_amdgcn_raw_buffer_load_b8(vsb, (slot + rg) * SB + l16 * CPL / kBlock, 0, 0);
        }
        r.left[u] = count - slot;
      }
    };
    const int row0 = x.begin + wave * kU * RPS;
    Batch next;
    issue(row0, next);
    for (int base = x.begin; base < end; base += STEP) {  // (uniform)
      const Batch r = next;
      if (base + STEP < end) issue(row0 + (base - x.begin) + STEP, next);  // (uniform)
      if constexpr (MX) {
        st.fold([&](int u, int i) { return i % 2 ? codes_bf16<true>(r.k[u][i / 2], scale_of(r.ks[u])) : codes_bf16<false>(r.k[u][i / 2], scale_of(r.ks[u])); },
                [&](int u, int i) { return i % 2 ? codes_f32<true>(r.v[u][i / 2], scale_of(r.vs[u])) : codes_f32<false>(r.v[u][i / 2], scale_of(r.vs[u])); },
                r.left, rg, c2);
      } else {
        st.fold([&](int u, int i) { return r.k[u][i]; }, [&](int u, int i) { return (f32x2){bf16_lo(r.v[u][i]), bf16_hi(r.v[u][i])}; }, r.left, rg, c2);
      }
    }
  }
  if (p.depth_count > 0 && s == x.first + x.n - 1) {  // (uniform) the slots go with the sequence's last slice
    const size_t at = ((size_t)b * p.Hk + g) * p.depth_alloc * RB;
    const __amdgpu_buffer_rsrc_t kb = rows_buffer(p.Kd + at, p.depth_count * RB), vb = rows_buffer(p.Vd + at, p.depth_count * RB);
    constexpr int W = CPL / 8;  // 16-byte pieces of a lane's channels
    for (int row = wave * kU * RPS; row < p.depth_count; row += STEP) {
      u32x4 k[kU][W], v[kU][W];
      int left[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
#pragma unroll
        for (int w = 0; w < W; ++w) {
          k[u][w] = __builtin_amdgcn_raw_buffer_load_b128(kb, (row + u * RPS + rg) * RB + l16 * CPL * 2 + w * 16, 0, 0);
          v[u][w] = __builtin_amdgcn_raw_buffer_load_b128(vb, (row + u * RPS + rg) * RB + l16 * CPL * 2 + w * 16, 0, 0);
        }
        left[u] = p.depth_count - row - u * RPS;
      }
      st.fold([&](int u, int i) { return k[u][i / 4][i % 4]; }, [&](int u, int i) { return (f32x2){bf16_lo(v[u][i / 4][i % 4]), bf16_hi(v[u][i / 4][i % 4])}; },
              left, rg, c2);
    }
  }
#pragma unroll
  for (int j = 0; j < GT; ++j) fold_groups<D>(st.m[j], st.l[j], st.o[j], c2, lane, red + (wave * GT + j) * (D + 2));
  __syncthreads();
  const size_t to = (size_t)s * p.Hq + g * G + gc * GT;
  for (int t = tid; t < nh * D; t += kPgWaves * 64) {
    const int j = t / D, ch = t % D;
    float o;
    const f32x2 ml = fold_rows<D, GT, kPgWaves>(red, j, ch, c2, o);
    if (p.single) {  // (uniform)
      const bool none = ml[1] == 0.f;  // nothing seen, or nothing that has weight
      ((__bf16*)p.O)[bh * D + t] = (__bf16)(none ? 0.f : o / ml[1]);
      if (ch == 0) p.LSE[bh + j] = none ? -INFINITY : ml[0] * p.scale + __logf(ml[1]);
    } else {
      p.ws_o[to * D + t] = o;
      if (ch == 0) *(f32x2*)(p.ws_ml + (to + j) * 2) = ml;
    }
  }
}

// ---------------------------------------------------------------- rows on the matrix pipe
// Up to COLS query heads of a group are the columns of S^T = K Q^T and O^T += V^T P^T, a wave folds 32 rows at a time.  32 columns: Columns (moda_decode_columns.h).
// 16 columns, with the 16 x 16 x 32 products: lane l holds column l % 16; S^T of rows 16 t + 4 (l / 16) + j in s[t][j], which packed to bf16 is the
// second operand of the product over rows if that takes the rows in the same order; O^T of channels 16 cb + 4 (l / 16) + j.
// Weights go into that product as bf16, rounded as in Columns, or (SPLIT) as sums of two bf16 numbers, a product each: groups of 3 and 4 heads, to which
// moda_attn_decode gives fp32 weights, are off by O's own rounding alone here too, 0.0017 of their size on N(0,1) data instead of 0.0023.  (Rounded once /
// split, us, sequences down to half of the longest: 64 x 2100 rows of d = 64, 32 heads on 8, 31.5 / 32.0;  32 x 8000 rows of d = 128, 32 on 8, 133.3 / 133.8;
// 32 x 16000 8-bit rows, 32 on 8, 141.0 / 145.7.  More heads, whose weights moda_attn_decode rounds as well: 64 on 8, down to a tenth, 107.1 / 110.7, 256 on 8,
// 32 columns, 167.8 / 176.4; there it is not done.)

// Weights (0 or more) as sums of two bf16 numbers, off by 2^-15 of themselves: the largest one below x, and the rest, rounded.  Both are above 0 where x is
// (2^-102 or more), so that an infinite value stays one and does not become NaN.
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8& high, bf16x8& rest) {
  u32x4 h;
  float r[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned a = __builtin_elementwise_sub_sat(__builtin_bit_cast(unsigned, x[2 * i]), 1u);
    const unsigned b = __builtin_elementwise_sub_sat(__builtin_bit_cast(unsigned, x[2 * i + 1]), 1u);
    h[i] = __builtin_amdgcn_perm(b, a, 0x07060302);  // the upper halves
    r[2 * i] = x[2 * i] - bf16_hi(a);
    r[2 * i + 1] = x[2 * i + 1] - bf16_hi(b);
  }
  high = __builtin_bit_cast(bf16x8, h);
  rest = pack8(r);
}

template <int D, bool SPLIT>
struct Columns16 {
  using Tl = Tile<D>;
  static constexpr int kSteps = D / 32, kBlocks = D / 16;
  bf16x8 q[kSteps];
  f32x4 o[kBlocks];
  float m, l;
  int row, tr;  // this lane's place in a tile: chunk l / 16 of row l % 16; its part of a transposing read
  __device__ __forceinline__ void init(const char* q_row, int lane) {
    const int g = lane >> 4, i = lane & 15;
#pragma unroll
    for (int st = 0; st < kSteps; ++st) q[st] = *(const bf16x8*)(q_row + st * 64 + g * 16);
#pragma unroll
    for (int cb = 0; cb < kBlocks; ++cb) o[cb] = (f32x4){0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = 0.f;
    row = Tl::off(i, g);
    tr = Tl::off(g * 4 + (i >> 2), (i & 3) >> 1) + (i & 1) * 8;
  }
  // What the four lanes of a column hold, put together.
  template <class F>
  __device__ __forceinline__ static float over_column(float x, F&& f) {
    const int i = __builtin_bit_cast(int, x);
    auto r = __builtin_amdgcn_permlane16_swap(i, i, false, false);
    const int y = __builtin_bit_cast(int, f(__builtin_bit_cast(float, (int)r[0]), __builtin_bit_cast(float, (int)r[1])));
    auto h = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    return f(__builtin_bit_cast(float, (int)h[0]), __builtin_bit_cast(float, (int)h[1]));
  }
  // 32 rows: K from LDS address `k`, V from `v`; `lower` of the first 16 and `upper` of the others count.
  __device__ __forceinline__ void fold(unsigned k, unsigned v, int lane, int lower, int upper, float c2) {
    f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      const unsigned x = (unsigned)xor_here((int)(row + k), st << 6);
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8 __attribute__((address_space(3)))*)(size_t)(x + t * 16 * Tl::kRowBytes), q[st], s[t],
                                                       0, 0, 0);
    }
    if (min(lower, upper) < 16) {  // (uniform)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if ((lane >> 4) * 4 + j >= (t == 0 ? lower : upper)) s[t][j] = -INFINITY;
    }
    float bm = s[0][0];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) bm = fmaxf(bm, s[t][j]);
    bm = over_column(bm, [](float a, float b) { return fmaxf(a, b); });
    // (the reference as in Columns: raised when the maximum exceeds it by more than 8 powers of two)
    const bool raise = bm > m + 8.0f / c2 || m == -INFINITY;
    if (__builtin_amdgcn_ballot_w64(raise) != 0) {  // (uniform)
      const float mn = raise ? bm : m;
      const float al = mn == m ? 1.f : fast_exp2((m - mn) * c2);
      m = mn;
      l *= al;
#pragma unroll
      for (int cb = 0; cb < kBlocks; ++cb)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[cb][j] *= al;
    }
    const float mc = m == -INFINITY ? 0.f : m * c2;
    float pv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      pv[i] = fast_exp2(s[i >> 2][i & 3] * c2 - mc);
      l += pv[i];
    }
    bf16x8 pb, rest;
    if constexpr (SPLIT) split8(pv, pb, rest);
    else pb = pack8(pv);
#pragma unroll
    for (int cb = 0; cb < kBlocks; ++cb) {
      const unsigned x = (unsigned)xor_here((int)(tr + v), cb << 5);
      const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(size_t)x);
      const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(size_t)(x + 16 * Tl::kRowBytes));
      const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
      o[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pb, o[cb], 0, 0, 0);
      if constexpr (SPLIT) o[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, rest, o[cb], 0, 0, 0);
    }
  }
  // The states of the workgroup's waves folded, the first n columns to put(column, piece of four channels, sums, (reference, normaliser)).  LDS: piece c of
  // column q at 16 c + (q ^ c % 16), in units of 16 bytes, of the wave's part.
  template <class Put>
  __device__ __forceinline__ void finish(unsigned char* smem, float (*stat)[32][2], float c2, int lane, int wave, int n, Put&& put) const {
    constexpr int kPieces = D / 4, kPart = 16 * D * 4;
    const int i16 = lane & 15, g = lane >> 4;
    const float l_all = over_column(l, [](float a, float b) { return a + b; });
    __syncthreads();  // (the tiles are not read any more)
#pragma unroll
    for (int cb = 0; cb < kBlocks; ++cb) {
      const int piece = cb * 4 + g;
      *(f32x4*)(smem + wave * kPart + (piece * 16 + (i16 ^ (piece & 15))) * 16) = o[cb];
    }
    if (g == 0) {
      stat[wave][i16][0] = m;
      stat[wave][i16][1] = l_all;
    }
    __syncthreads();
#pragma unroll
    for (int i = threadIdx.x; i < 16 * kPieces; i += kShWaves * 64) {
      const int q = i / kPieces, piece = i % kPieces;
      if (q >= n) continue;
      float mm = -INFINITY, ll = 0.f;
      f32x4 oo = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kShWaves; ++w) mm = fmaxf(mm, stat[w][q][0]);
#pragma unroll
      for (int w = 0; w < kShWaves; ++w) {
        const float f = stat[w][q][0] == -INFINITY ? 0.f : fast_exp2((stat[w][q][0] - mm) * c2);
        ll += f * stat[w][q][1];
        const f32x4 x = *(const f32x4*)(smem + w * kPart + (piece * 16 + (q ^ (piece & 15))) * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) oo[j] += f * x[j];
      }
      put(q, piece, oo, (f32x2){mm, ll});
    }
  }
};
template <int D>
struct Columns32 : Columns<D> {
  FragAddr<D> fa;
  __device__ __forceinline__ void init(const char* q_row, int lane) {
    Columns<D>::init(q_row, lane >> 5);
    fa.init(lane);
  }
  __device__ __forceinline__ void fold(unsigned k, unsigned v, int lane, int lower, int upper, float c2) {
    Columns<D>::template fold<1, true>(k, v, fa, lane, lower, c2, nullptr, 0, 0, upper);
  }
  template <class Put>
  __device__ __forceinline__ void finish(unsigned char* smem, float (*stat)[32][2], float c2, int, int, int n, Put&& put) const {
    fold_waves<D, 1>(*this, smem, stat, c2, n, nullptr, nullptr, put);
  }
};
template <int D, int COLS, bool SPLIT>
using ColumnsOf = std::conditional_t<COLS == 16, Columns16<D, SPLIT>, Columns32<D>>;

__device__ __forceinline__ void lds_store(unsigned at, const u32x4& x) { *(u32x4 __attribute__((address_space(3)))*)(size_t)at = x; }

// A block of 32 rows in flight: pieces of 1 KB of K and of V, and the scales of 8-bit rows.
template <int D, bool MX>
struct PageBlock {
  static constexpr int kInst = 32 * (MX ? D : 2 * D) / 1024;
  u32x4 k[kInst], v[kInst];
  unsigned ks[MX ? kInst : 1], vs[MX ? kInst : 1];
  int left[2];  // rows of the first and the other 16 that count
};

// bf16 rows: the chunk that a lane fetches of piece q is the one whose place in the tile it fills: offset g_off ^ piece_xor(q) in the rows.
template <int D>
__device__ __forceinline__ int fetch_offset(int lane) {
  const int row = lane / Tile<D>::kChunks;
  return row * D * 2 + ((lane % Tile<D>::kChunks ^ Tile<D>::swz(row)) << 4);
}
template <int D>
__device__ constexpr int fetch_xor(int q) {
  return D == 128 ? (q & 3) << 4 : (q & 1) * 32;
}

// Every wave by itself: rows [first, first + n) of the list (first, and n unless the sequence ends, multiples of 32), 32 at a time through its two
// LDS tiles at `lds`, kPF blocks in flight in registers.  8-bit rows become bf16 on the way to LDS, exactly: 64 conversions per lane and block
// (d = 128) beside 16 matrix instructions.
template <int D, bool MX, int kPF, class C>
__device__ __forceinline__ void read_pages(C& c, const PagedParams& p, PageList& list, int g, int first, int n, unsigned lds, float c2) {
  using Tl = Tile<D>;
  using Block = PageBlock<D, MX>;
  constexpr int CB = MX ? D : 2 * D, SB = D / kBlock, kInst = Block::kInst, kRows = 32 / kInst, kHalf = 32 * Tl::kRowBytes;
  constexpr int LPR = 64 / kRows;  // lanes of a row
  const int lane = threadIdx.x & 63, jr = lane / LPR, pc = lane % LPR;
  // (8 bits: a lane's two chunks of bf16 go to their places, which differ in one bit)
  const int g_off = MX ? jr * CB + pc * 16 : fetch_offset<D>(lane);
  const int s_off = jr * SB + pc / 2;
  const unsigned to = MX ? lds + jr * Tl::kRowBytes + (((2 * pc) ^ Tl::swz(jr)) << 4) : lds + lane * 16;
  const int n_blocks = (n + 31) / 32;
  auto issue = [&](int blk, Block& r) {
    const int row = first + blk * 32;
    if (blk < n_blocks && ((row + 31) >> p.shift) - list.base >= 64) list.load(p, row >> p.shift, lane);  // (uniform)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = row + h * 16, i = min((at >> p.shift) - list.base, 63), slot = at & ((1 << p.shift) - 1);
      const int id = __builtin_amdgcn_readlane(list.id, i), count = blk < n_blocks ? __builtin_amdgcn_readlane(list.count, i) : 0;
      const size_t row0 = ((size_t)id * p.Hk + g) << p.shift;
      const __amdgpu_buffer_rsrc_t kb = rows_buffer(p.K + row0 * CB, count * CB), vb = rows_buffer(p.V + row0 * CB, count * CB);
      r.left[h] = count - slot;
#pragma unroll
      for (int q = h * kInst / 2; q < (h + 1) * kInst / 2; ++q) {
        const int at_row = slot + q * kRows - h * 16;
        const int v_off = MX ? g_off : xor_here(g_off, fetch_xor<D>(q));
        r.k[q] = __builtin_amdgcn_raw_buffer_load_b128(kb, v_off, at_row * CB, 2);
        r.v[q] = __builtin_amdgcn_raw_buffer_load_b128(vb, v_off, at_row * CB, 2);
      }
      if (MX) {
        const __amdgpu_buffer_rsrc_t ksb = rows_buffer(p.Ks + row0 * SB, count * SB), vsb = rows_buffer(p.Vs + row0 * SB, count * SB);
#pragma unroll
        for (int q = h * kInst / 2; q < (h + 1) * kInst / 2; ++q) {
          const int at_row = slot + q * kRows - h * 16;
          r.ks[q] = __builtin_amdgcn_raw_buffer_load_b8(ksb, s_off, at_row * SB, 0);
          r.vs[q] = __builtin_amdgcn_raw_buffer_load_b8(vsb, s_off, at_row * SB, 0);
        }
      }
    }
  };
  auto stage = [&](const u32x4 (&x)[kInst], const unsigned (&s)[MX ? kInst : 1], int tile) {
#pragma unroll
    for (int q = 0; q < kInst; ++q) {
      if (MX) {
        const float sc = scale_of(s[q]);
        const unsigned at = (unsigned)xor_here((int)(to + tile), D == 128 ? (q & 1) * 32 : 0) + q * kRows * Tl::kRowBytes;
        lds_store(at, (u32x4){codes_bf16<false>(x[q][0], sc), codes_bf16<true>(x[q][0], sc), codes_bf16<false>(x[q][1], sc), codes_bf16<true>(x[q][1], sc)});
        lds_store(at ^ 16, (u32x4){codes_bf16<false>(x[q][2], sc), codes_bf16<true>(x[q][2], sc), codes_bf16<false>(x[q][3], sc), codes_bf16<true>(x[q][3], sc)});
      } else {
        lds_store(to + tile + q * 1024, x[q]);
      }
    }
  };
  Block buf[kPF];
#pragma unroll
  for (int i = 0; i < kPF; ++i) issue(i, buf[i]);
  for (int blk0 = 0; blk0 < n_blocks; blk0 += kPF) {
#pragma unroll
    for (int i = 0; i < kPF; ++i) {
      const int blk = blk0 + i, lower = buf[i].left[0], upper = buf[i].left[1];
      // (a wave's LDS operations execute in order: these writes follow the reads of the block before)
      stage(buf[i].k, buf[i].ks, 0);
      stage(buf[i].v, buf[i].vs, kHalf);
      issue(blk + kPF, buf[i]);
      if (max(lower, upper) > 0)  // (uniform)
        c.fold(lds, lds + kHalf, lane, lower, upper, c2);
    }
  }
}

// The same for n rows of bf16 that lie together (slots).
template <int D, class C>
__device__ __forceinline__ void read_together(C& c, const char* K, const char* V, int n, unsigned lds, float c2) {
  constexpr int RB = D * 2, kInst = 32 * RB / 1024, kRows = 32 / kInst, kHalf = 32 * RB;
  const int lane = threadIdx.x & 63, g_off = fetch_offset<D>(lane);
  const __amdgpu_buffer_rsrc_t kb = rows_buffer(K, n * RB), vb = rows_buffer(V, n * RB);
  for (int row = 0; row < n; row += 32) {
    u32x4 k[kInst], v[kInst];
#pragma unroll
    for (int q = 0; q < kInst; ++q) {
      const int v_off = xor_here(g_off, fetch_xor<D>(q));
      k[q] = __builtin_amdgcn_raw_buffer_load_b128(kb, v_off, (row + q * kRows) * RB, 0);
      v[q] = __builtin_amdgcn_raw_buffer_load_b128(vb, v_off, (row + q * kRows) * RB, 0);
    }
#pragma unroll
    for (int q = 0; q < kInst; ++q) {
      lds_store(lds + q * 1024 + lane * 16, k[q]);
      lds_store(lds + kHalf + q * 1024 + lane * 16, v[q]);
    }
    c.fold(lds, lds + kHalf, lane, n - row, n - row - 16, c2);
  }
}

template <int D, bool MX, int COLS, bool SPLIT>
__global__ __launch_bounds__(kShWaves * 64, 2) void moda_paged_matrix_kernel(PagedParams p) {
  constexpr int RB = D * 2, kPF = D == 128 && !MX ? 1 : 2;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kShWaves * 2 * 32 * RB];
  __shared__ float stat[kShWaves][32][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned lds = (unsigned)(size_t)(lds_ptr)smem + wave * 2 * 32 * RB;
  const float c2 = p.scale_log2;
  const int unit = blockIdx.x % p.units, s = blockIdx.x / p.units;
  const int G = p.Hq / p.Hk, g = unit % p.Hk, gc = unit / p.Hk;
  PageList list(p, p.single ? s : 0, g);
  // (uniform) the first page numbers come together with the length, the slots are through before them (128 heads of 250 rows 8.6 -> 8.1 us, of 6000 rows
  // 68.7 -> 67.2, eight queries each; on the vector ALUs neither changed anything)
  if (p.single) list.fetch(p, 0, lane);
  const Slice x = p.single ? whole_sequence(p, s) : find_slice(p, s, lane);
  if (x.b < 0) return;  // (uniform)
  const int b = x.b;
  const int nh = min(COLS, G - gc * COLS);
  const size_t bh = (size_t)b * p.Hq + g * G + gc * COLS;
  if (unit == 0 && s == x.first && tid == 0 && !p.single && p.B <= kPgLook) {
    p.ws_deal[2 * b] = x.first;
    p.ws_deal[2 * b + 1] = x.n;
  }
  ColumnsOf<D, COLS, SPLIT> c;
  c.init((const char*)p.Q + (bh + min(lane % COLS, nh - 1)) * RB, lane);  // (a column past the last repeats it and is not stored)
  // a wave's part of n rows: a quarter, in whole blocks of 32
  auto part = [&](int n, int& first) {
    const int q = ((n + kShWaves - 1) / kShWaves + 31) / 32 * 32;
    first = min(wave * q, n);
    return min(q, n - first);
  };
  int first;
  const int n = part(max(min(x.rows - x.begin, x.per), 0), first);
  if (!p.single) {  // (uniform)
    list = PageList(p, b, g);
    list.fetch(p, (x.begin + first) >> p.shift, lane);
  }
  if (p.depth_count > 0 && s == x.first + x.n - 1) {  // (uniform) the slots go with the sequence's last slice, first
    int slot;
    const int n_slots = part(p.depth_count, slot);
    const size_t at = (((size_t)b * p.Hk + g) * p.depth_alloc + slot) * RB;
    read_together<D>(c, p.Kd + at, p.Vd + at, n_slots, lds, c2);
  }
  if (n > 0) {  // (uniform)
    list.len = filled(p.lengths, b, p.T);
    list.settle(p);
    read_pages<D, MX, kPF>(c, p, list, g, x.begin + first, n, lds, c2);
  }
  const size_t to = (size_t)s * p.Hq + g * G + gc * COLS;
  c.finish(smem, stat, c2, lane, wave, nh, [&](int j, int piece, const f32x4& o, const f32x2& ml) {
    if (p.single) {  // (uniform)
      const bool none = ml[1] == 0.f;  // nothing seen, or nothing that has weight
      const float inv = none ? 0.f : 1.f / ml[1];
      *(u32x2*)((__bf16*)p.O + (bh + j) * D + piece * 4) =
          none ? (u32x2){0u, 0u} : (u32x2){pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
      if (piece == 0) p.LSE[bh + j] = none ? -INFINITY : ml[0] * p.scale + __logf(ml[1]);
    } else {
      *(f32x4*)(p.ws_o + (to + j) * D + piece * 4) = o;
      if (piece == 0) *(f32x2*)(p.ws_ml + (to + j) * 2) = ml;
    }
  });
}

// ---------------------------------------------------------------- outputs
// `by` slices of a head at a time, D / 4 threads each (four channels a thread), 1024 / D such teams in a workgroup.
template <int D>
__global__ __launch_bounds__(256) void moda_paged_finish_kernel(PagedParams p, int by) {
  constexpr int kTeam = D / 4, kTeams = 256 / kTeam;
  __shared__ __attribute__((aligned(16))) float red[kTeams][D + 4];
  const float c2 = p.scale_log2;
  const int tid = threadIdx.x;
  // (a state whose scores are all -inf is empty: reference -inf, weight zero)
  auto factor = [&](float m, float ref) { return m == -INFINITY ? 0.f : fast_exp2((m - ref) * c2); };
  const int team = tid / kTeam, ch = tid % kTeam * 4, part = team % by;
  const long long bh = (long long)blockIdx.x * (kTeams / by) + team / by, heads = (long long)p.B * p.Hq;
  const int row = (int)min(bh, heads - 1), b = row / p.Hq, h = row % p.Hq;
  const int first = p.ws_deal[2 * b], n = p.ws_deal[2 * b + 1];
  float mm = -INFINITY, ll = 0.f;
  f32x4 oo = {0.f, 0.f, 0.f, 0.f};
  constexpr int kU = 4;
  for (int s0 = part; s0 < n; s0 += kU * by) {
    f32x2 st[kU];
    f32x4 o[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const size_t i = (size_t)(first + min(s0 + u * by, n - 1)) * p.Hq + h;
      st[u] = *(const f32x2*)(p.ws_ml + i * 2);
      o[u] = *(const f32x4*)(p.ws_o + i * D + ch);
    }
    float mn = mm;
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (s0 + u * by < n) mn = fmaxf(mn, st[u][0]);
    const float al = factor(mm, mn);
    mm = mn;
    ll *= al;
#pragma unroll
    for (int j = 0; j < 4; ++j) oo[j] *= al;
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (s0 + u * by < n) {
        const float f = factor(st[u][0], mm);
        ll += f * st[u][1];
#pragma unroll
        for (int j = 0; j < 4; ++j) oo[j] += f * o[u][j];
      }
  }
  if (by > 1) {  // (uniform)
    *(f32x4*)&red[team][ch] = oo;
    if (ch == 0) *(f32x2*)&red[team][D] = (f32x2){mm, ll};
    __syncthreads();
    if (part > 0) return;
    const float m0 = mm;
    for (int k = 1; k < by; ++k) mm = fmaxf(mm, red[team + k][D]);
    const float f0 = factor(m0, mm);
    ll *= f0;
#pragma unroll
    for (int j = 0; j < 4; ++j) oo[j] *= f0;
    for (int k = 1; k < by; ++k) {
      const float f = factor(red[team + k][D], mm);
      ll += f * red[team + k][D + 1];
      const f32x4 x = *(const f32x4*)&red[team + k][ch];
#pragma unroll
      for (int j = 0; j < 4; ++j) oo[j] += f * x[j];
    }
  }
  if (bh >= heads) return;
  const bool none = ll == 0.f;  // nothing seen, or nothing that has weight
  const float inv = none ? 0.f : 1.f / ll;
  *(u32x2*)((__bf16*)p.O + bh * D + ch) = none ? (u32x2){0u, 0u} : (u32x2){pack_bf16(oo[0] * inv, oo[1] * inv), pack_bf16(oo[2] * inv, oo[3] * inv)};
  if (ch == 0) p.LSE[bh] = none ? -INFINITY : mm * p.scale + __logf(ll);
}

// ---------------------------------------------------------------- host side
// Rows that a sequence may have: the lengths themselves are on the device.
static long long rows_bound(const PagedParams& p) { return p.selected ? (long long)p.n_selected << p.shift : p.T; }

// Sequences of one slice each need no second kernel: where they are short, and longer ones where they fill half the chip or all of it anyway.  Two
// kernels / one, us, (batch x key/value heads), rows of the longest sequence: all as long, evenly down to half of it, down to a tenth of it (under 64 groups alike)
//   bf16, d = 128, 1 head   8, 100 7.8 / 4.6;   8, 414 8.2 / 7.4;   8, 515 8.4 / 8.7;   64, 625 9.2 / 9.3, 9.7 / 9.3, 8.9 / 9.3
//                    128, 625 12.0 / 11.7, 11.9 / 10.9, 10.7 / 9.3;   128, 781 13.9 / 14.6, 13.3 / 13.7, 11.1 / 11.4;   192, 937 19.5 / 17.9, 18.1 / 17.0, 16.0 / 16.1
//                    256, 1250 29.1 / 25.9, 24.7 / 23.6, 19.4 / 22.0;   256, 1562 34.7 / 31.9, 28.9 / 28.9, 25.4 / 27.2;   512, 1250 53.7 / 49.1, 42.3 / 41.3, 33.1 / 34.1
//   8 heads          8, 625 9.9 / 9.0;   8, 781 9.8 / 10.8;   128, 937 16.3 / 15.1, 17.1 / 14.0, 13.7 / 13.0;   128, 1562 23.1 / 22.1, 21.7 / 20.4, 19.1 / 19.7
//                    256, 1562 38.1 / 32.3, 36.9 / 26.8, 27.0 / 22.7;   512, 1250 56.6 / 50.2, 51.5 / 41.8, 40.3 / 35.2
//   8 bits, 1 head   8, 625 9.1 / 7.9;   8, 781 9.1 / 9.7;   128, 937 12.8 / 12.1, 13.1 / 11.7, 11.1 / 11.5;   256, 1562 22.6 / 21.3, 20.2 / 19.5, 18.0 / 18.2
//   8 heads          8, 625 11.2 / 10.4;   8, 781 11.1 / 12.4;   128, 1250 18.0 / 15.8, 17.5 / 15.7, 17.1 / 15.6;   256, 1562 27.4 / 20.8, 27.3 / 20.0, 24.4 / 19.6
//   bf16, d = 64     1 head   8, 828 8.3 / 7.5;   8, 1031 8.4 / 8.8;   128, 1250 13.0 / 12.1, 12.3 / 10.8, 10.9 / 9.5;   128, 1562 13.7 / 15.0, 13.1 / 14.0, 11.5 / 11.4
//                    8 heads   8, 828 9.6 / 9.1;   8, 1031 9.6 / 10.5;   256, 2500 30.3 / 25.8, 27.0 / 22.3, 22.5 / 19.3
// The limits are those of the form that crosses first, one head in bf16 (8-bit rows on the vector ALUs have their own below 256 groups).  From 256 groups on raggedness
// decides: at the limit such sequences gain a ninth if all are as long and lose an eighth if they go down to a tenth.  Beyond the limits some forms
// still gain, by up to 27 % (8 heads, 8 bits, 256 x 1562 rows; 192 groups of 8 heads and 1562 rows 33.6 / 25.0, 29.5 / 22.6, 22.0 / 21.2): the rule does not tell
// them apart.
// Lists are as long as each other, and so are the workgroups' times: there one kernel does for any length, where the groups are about a multiple of the
// compute units.  The same for rows that lists name:
//   bf16, d = 128, 8 heads   256, 2812 62.8 / 56.4;   448, 2812 108.4 / 98.1;   512, 11250 467 / 438;   640, 2812 152.3 / 144.5;   but 288, 2812 76.3 / 83.1;   576, 11250 526 / 540
//   8 bits, d = 128, 8 heads   512, 2812 75.2 / 63.4;   1 head   512, 2812 65.3 / 60.5;   640, 2812 80.5 / 80.6;   768, 5625 182.1 / 177.1;   but 320, 5625 83.0 / 86.5
// (Sequences of their own lengths, down to a tenth of the longest: 512, 2812 of bf16 77.4 / 75.2 and, one head, 67.8 / 74.1; 8 bits 51.8 / 45.7 and 40.4 / 43.4.
// 16 waves for one short sequence: 8 x 400 rows of d = 128 7.4 -> 6.9, 8 x 100 4.3 -> 5.5: not built.)
static bool in_one(const PagedParams& p, int d, bool mx) {
  const long long channels = rows_bound(p) * d, groups = (long long)p.B * p.units;
  const long long alone = mx && p.heads_per <= 2 ? 80000 : 53000, units = 256, filled_units = (groups + units - 1) / units * units;
  if (p.selected && groups >= units && groups * 6 >= filled_units * 5) return true;
  return channels <= (groups >= units ? 160000 : groups * 2 >= units ? alone * 3 / 2 : alone);
}

// Slices of all sequences together that find_slice makes of at most so many rows: one of every sequence and as many as have its size.
static int most_slices(const PagedParams& p, long long rows) {
  auto of = [&](long long workgroups, long long least) { return std::min(workgroups / p.units, rows / least); };
  return p.B + (int)std::max(of(kPgFew, 1ll << p.least_shift), std::max(of(kPgOnce, kPgOnceRows), of(kPgMany, p.good)));
}

static void plan(PagedParams& p, int d, bool mx) {
  const int G = p.Hq / p.Hk;
  p.heads_per = G <= 2 ? G : G <= 16 ? 16 : 32;
  p.units = p.Hk * ((G + p.heads_per - 1) / p.heads_per);
  const int least = G <= 2 ? kPgWaves * 4 * 64 * (mx ? 16 : 8) / d : kShWaves * 32;  // what the waves take at a time: 64 to 256
  p.least_shift = __builtin_ctz(least);
  // Rows of a slice in several rounds (us, rows / heads per group; 512 workgroups / 2048 of 512 rows or more / 2048 of 2048 or more; all sequences as long, down
  // to half of the longest, down to a tenth):
  //   vector ALUs    8 x 65536 rows, 16 heads, d = 128: 631 / 633 / 633, 573 / 520 / 519, 444 / 399 / 400;  4 x 16000, 16 heads 84.6 / 85.5 / 84.5, 75.1 / 70.0 / 75.0,
  //   54.3 / 53.7 / 54.0;  32 x 4000 8-bit, 8 heads 48.3 / 49.3 / 48.7, 42.5 / 40.5 / 42.8, 33.2 / 31.0 / 33.4
  //   matrix pipe, 2048 workgroups of 512 / 1024 / 2048 / 4096 rows or more, sequences down to a tenth of the longest: 32 x 16000 8-bit, 64 heads on 8, d = 128
  //   116.5 / 116.1 / 108.7 / 116.0;  32 x 8000 bf16 103.9 / 101.4 / 107.0 / 100.2;  4 x 30000 bf16, 64 on 4 40.9 / 33.0 / 32.9 / 32.9;  16 x 8000 bf16, d = 64
  //   31.5 / 32.6 / 34.1 / 34.0;  512 workgroups of any size 32 x 16000 8-bit, down to 0.7 of the longest: 179 against 162 / 162 / 165 / 157
  p.good = G <= 2 ? 512 : 2048;
  p.n_slices = most_slices(p, 1ll << 40);
}

size_t decode_paged_workspace_bytes(const PagedParams& dims, int d, bool mx) {
  PagedParams p = dims;
  plan(p, d, mx);
  return ((size_t)p.n_slices * p.Hq * (d + 2) + 2 * (size_t)p.B) * sizeof(float);
}

template <int D, bool MX>
static hipError_t launch_d(const PagedParams& p, hipStream_t stream) {
  const long long rows = rows_bound(p), blocks = (long long)p.units * (p.single ? p.B : most_slices(p, p.B * rows)), heads = (long long)p.B * p.Hq;
  constexpr int teams = 1024 / D;
  int by = 1;  // teams that share a head's slices, so that each folds about four of them at a time
  while (by < teams && (long long)by * 4 * p.B < p.n_slices) by *= 2;
  const long long finish_blocks = (heads + teams / by - 1) / (teams / by);
  if (!grid_ok(blocks, kPgWaves * 64) || !grid_ok(finish_blocks, 256)) return kGridTooLarge;
  auto* kernel = p.heads_per == 1 ? moda_paged_slices_kernel<D, 1, MX> : p.heads_per == 2 ? moda_paged_slices_kernel<D, 2, MX>
                 : p.Hq / p.Hk <= 4 ? moda_paged_matrix_kernel<D, MX, 16, true>
                 : p.heads_per == 16 ? moda_paged_matrix_kernel<D, MX, 16, false> : moda_paged_matrix_kernel<D, MX, 32, false>;
  hipError_t e = hipSuccess;
  if (!p.single && p.B > kPgLook) e = launch_kernel(moda_paged_deal_kernel, dim3(1), dim3(kDealThreads), stream, p);
  if (e != hipSuccess) return e;
  e = launch_kernel(kernel, dim3((unsigned)blocks), dim3(kPgWaves * 64), stream, p);
  if (e != hipSuccess || p.single) return e;
  return launch_kernel(moda_paged_finish_kernel<D>, dim3((unsigned)finish_blocks), dim3(256), stream, p, by);
}

hipError_t launch_decode_paged(PagedParams p, int d, bool mx, void* workspace, hipStream_t stream) {
  plan(p, d, mx);
  p.single = in_one(p, d, mx);
  p.ws_o = (float*)workspace;
  p.ws_ml = p.ws_o + (size_t)p.n_slices * p.Hq * d;
  p.ws_deal = (int*)(p.ws_ml + (size_t)p.n_slices * p.Hq * 2);
  if (d == 128) return mx ? launch_d<128, true>(p, stream) : launch_d<128, false>(p, stream);
  return mx ? launch_d<64, true>(p, stream) : launch_d<64, false>(p, stream);
}

}  // namespace moda
