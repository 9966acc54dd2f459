// Decoding step of a batch whose sequences share prefixes and differ in length, with the attention weight of every row of
// the own caches added to an accumulator where the caller keeps one.
//
// With the logits x_c = scale <q, k_c> of a token's prefix rows, own rows and slots,
//     m = max x,  l = sum exp(x_c - m),  O = (1/l) sum exp(x_c - m) v_c,  LSE = m + ln l,
//     weights_out[j] = weights_in[j] + sum over the heads of a group of exp(x_j - LSE).
// (m, l, unnormalised O) of disjoint sets of rows merge exactly, so the rows are cut into slices over workgroups, whose
// states go to the workspace in fp32, and a second kernel merges them.  Where weights are asked for, the own rows' logits go
// there too (4 bytes per row and head, where a row of K and V is 4 d bytes), since no slice knows the LSE.
//
// One launch takes all slices:
//   prefixes   all queries that share a prefix (sequences x heads of a group) read its rows together.  Up to 4 of them on the vector
//              ALUs (read_rows), else they are the columns of matrix products S^T = K Q^T, O^T += V^T P^T: up to 32
//              (read_by_wave) every wave reads its own part of the slice; more (read_by_workgroup), 2 or 4 waves of 32 columns
//              share the K and V tiles of the slice in LDS.
//   own rows   up to 2 heads per group on the vector ALUs (read_rows), where all caches are short up to 8 (own_kind), else the heads
//              are the columns of read_by_wave.
// What bounds it: long calls the reads (32 sequences behind 32768 rows 5.6 TB/s; 8 x 65536 own rows with weights 5.7), 512 queries per
// prefix row the vector ALUs (exponentials; 720 TFLOP/s at 65536 rows, d = 128), short ones two launches of about 4 us.
#include <algorithm>

#include "moda_decode_columns.h"
#include "moda_launch.h"

namespace moda {

// The states in the workspace: O, [state][d], and (reference, normaliser), [state][2].  A slice's states of all its heads are
// adjacent, so that a workgroup writes whole cache lines: prefixes [n_prefixes, Hk, slice, sequence, head of the group], behind
// them own rows [B, Hk, slice, head of the group].
struct HeadStates {  // of one (sequence, query head): prefix slices at first + s * step, the others at own + s * own_step
  size_t first, own;
  int step, own_step;
  __device__ __forceinline__ HeadStates(const SharedParams& p, int b, int g, int j) {
    const int per = p.B / p.Np, G = p.Hq / p.Hk;
    step = per * G;
    own_step = G;
    first = ((size_t)(b / per * p.Hk + g) * p.n_prefix) * step + b % per * G + j;
    own = (size_t)p.B * p.Hq * p.n_prefix + ((size_t)(b * p.Hk + g) * p.n_own) * G + j;
  }
  __device__ __forceinline__ size_t operator()(const SharedParams& p, int s) const {
    return s < p.n_prefix ? first + (size_t)s * step : own + (size_t)(s - p.n_prefix) * own_step;
  }
};

// ---------------------------------------------------------------- rows on the vector ALUs
// A lane owns 8 channels, d/8 lanes a row; a wave takes kU batches of 64 / (d/8) rows at a time, the next ones in
// flight, and raises its reference once for them.  query(j) = the address of query j of GT (from nh on the last one repeats and is
// not stored), `scores` = the first one's logits of the first run, or null.  The waves' states go to red[wave][query][D + 2].
template <int D, int GT, int WAVES, class Query>
__device__ __forceinline__ void walk_rows(const Rows& x, Query&& query, int nh, float c2, float* scores, size_t score_step, float* red) {
  constexpr int LPR = D / 8, RPS = 64 / LPR, RB = D * 2, kU = 4, STEP = WAVES * kU * RPS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, rg = lane / LPR, l16 = lane % LPR;
  u32x4 q[GT];
  float m[GT], l[GT], o[GT][8];
#pragma unroll
  for (int j = 0; j < GT; ++j) {
    q[j] = *(const u32x4*)(query(min(j, nh - 1)) + l16 * 16);
    m[j] = -INFINITY;
    l[j] = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) o[j][k] = 0.f;
  }
  const int row0 = wave * kU * RPS + rg, n = x.n + x.n2;
  if (n > 0) {  // (uniform)
    auto load = [&](const char* first, const char* second, int r) {
      r = min(r, n - 1);
      const char* at = r < x.n ? first + (size_t)r * RB : second + (size_t)(r - x.n) * RB;
      return __builtin_nontemporal_load((const u32x4*)(at + l16 * 16));
    };
    u32x4 kn[kU], vn[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      kn[u] = load(x.K, x.K2, row0 + u * RPS);
      vn[u] = load(x.V, x.V2, row0 + u * RPS);
    }
    for (int base = 0; base < n; base += STEP) {  // (uniform)
      const int r = row0 + base;
      u32x4 kv[kU], vv[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        kv[u] = kn[u];
        vv[u] = vn[u];
      }
      if (base + STEP < n) {  // (uniform)
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          kn[u] = load(x.K, x.K2, r + STEP + u * RPS);
          vn[u] = load(x.V, x.V2, r + STEP + u * RPS);
        }
      } else {  // rows past the end repeat the last one with weight zero, which an infinite value would turn into NaN
#pragma unroll
        for (int u = 0; u < kU; ++u)
          if (r + u * RPS >= n) vv[u] = (u32x4){0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int j = 0; j < GT; ++j) {
        float sc[kU], mn = m[j];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          float a = 0.f;
#pragma unroll
          for (int k = 0; k < 4; ++k) a = dot2_bf16(q[j][k], kv[u][k], a);
          sc[u] = group_sum<LPR>(a);
        }
        if (scores) {  // lane u of a row's lanes stores the logit of batch u
          float a = sc[0];
#pragma unroll
          for (int u = 1; u < kU; ++u) a = l16 == u ? sc[u] : a;
          const int at = r + l16 * RPS;
          if (l16 < kU && at < x.n && j < nh) scores[(size_t)j * score_step + at] = a;
        }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          if (r + u * RPS >= n) sc[u] = -INFINITY;
          mn = fmaxf(mn, sc[u]);
        }
        // (mn is -inf only while every score so far was, or was NaN, which stays NaN; with reference 0 the others weigh nothing)
        const float ref = mn == -INFINITY ? 0.f : mn;
        const float al = fast_exp2((m[j] - ref) * c2);
        m[j] = mn;
        l[j] *= al;
#pragma unroll
        for (int k = 0; k < 8; ++k) o[j][k] *= al;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const float pw = fast_exp2((sc[u] - ref) * c2);
          l[j] += pw;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            o[j][2 * k] += pw * bf16_lo(vv[u][k]);
            o[j][2 * k + 1] += pw * bf16_hi(vv[u][k]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < GT; ++j) fold_groups<D>(m[j], l[j], o[j], c2, lane, red + (wave * GT + j) * (D + 2));
  __syncthreads();
}

// The queries' states of walk_rows, waves folded, to o_out, ml_out.
template <int D, int GT, class Query>
__device__ __forceinline__ void read_rows(const Rows& x, Query&& query, int nh, float c2, float* o_out, float* ml_out, float* scores,
                                          size_t score_step, float* red) {
  walk_rows<D, GT, kShWaves>(x, query, nh, c2, scores, score_step, red);
  for (int t = threadIdx.x; t < nh * D; t += kShWaves * 64) {
    const int j = t / D, ch = t % D;
    float o;
    const f32x2 ml = fold_rows<D, GT, kShWaves>(red, j, ch, c2, o);
    o_out[t] = o;
    if (ch == 0) *(f32x2*)(ml_out + j * 2) = ml;
  }
}

// ---------------------------------------------------------------- short contexts: one kernel
// No prefix, up to 4 heads per group, and as few rows as eight waves read in a few steps: a workgroup has all rows of a (batch,
// key/value head) and finishes outputs and weights by itself; the logits stay in LDS.
constexpr int kOneWaves = 8, kOneRows = 512;
template <int D, int GT>
__global__ __launch_bounds__(kOneWaves * 64, 2) void moda_shared_one_kernel(SharedParams p) {
  constexpr int RB = D * 2;
  __shared__ __attribute__((aligned(16))) float red[kOneWaves * GT * (D + 2)];
  __shared__ float scores[GT][kOneRows], lse2[GT];
  const int tid = threadIdx.x, G = p.Hq / p.Hk, b = blockIdx.x / p.Hk, g = blockIdx.x - b * p.Hk;
  const float c2 = p.scale_log2;
  const size_t at = (size_t)blockIdx.x * p.T_alloc * RB, slot_at = (size_t)blockIdx.x * p.depth_alloc * RB;
  const int len = filled(p.lengths, b, p.T);
  const Rows x = {(const char*)p.Ks + at, (const char*)p.Vs + at, len, (const char*)p.Kd + slot_at, (const char*)p.Vd + slot_at, p.depth_count};
  static_assert(kOneRows <= kOneWaves * 64, "a thread per row");
  float w = 0.f;
  if (p.w_in && tid < len) w = p.w_in[(size_t)blockIdx.x * p.T_alloc + tid];
  const size_t bh = (size_t)b * p.Hq + g * G;
  walk_rows<D, GT, kOneWaves>(x, [&](int j) { return (const char*)p.Q + (bh + j) * RB; }, G, c2, p.w_out ? &scores[0][0] : nullptr, kOneRows, red);
  for (int t = tid; t < G * D; t += kOneWaves * 64) {
    const int j = t / D, ch = t % D;
    float o;
    const f32x2 ml = fold_rows<D, GT, kOneWaves>(red, j, ch, c2, o);
    const bool none = ml[1] == 0.f;  // nothing seen, or nothing that has weight
    ((__bf16*)p.O)[(bh + j) * D + ch] = (__bf16)(none ? 0.f : o / ml[1]);
    if (ch == 0) {
      p.LSE[bh + j] = none ? -INFINITY : ml[0] * p.scale + __logf(ml[1]);
      lse2[j] = none ? INFINITY : ml[0] * c2 + __log2f(ml[1]);
    }
  }
  if (!p.w_out) return;  // (uniform)
  __syncthreads();
  if (tid < len) {
    for (int j = 0; j < G; ++j) w += fast_exp2(__builtin_fmaf(scores[j][tid], c2, -lse2[j]));
    p.w_out[(size_t)blockIdx.x * p.T_alloc + tid] = w;
  }
}

// ---------------------------------------------------------------- rows on the matrix pipe
// The workgroup together: tiles of kRows rows in a ring of kStages stages, all but one of them in flight while one is folded; a wave
// folds all rows of a tile (KW = 1) or 32 of its 64 (KW = 2: waves 2 and 3 hold the columns of waves 0 and 1).
constexpr int ring_bytes(int d) { return d * 512; }
template <int D, int KW>
struct Ring {
  static constexpr int kRows = D == 128 && KW == 1 ? 32 : 64;
  static constexpr int kTile = kRows * D * 2, kStages = ring_bytes(D) / (2 * kTile);
};
template <int D, int KW>
__device__ __forceinline__ void read_by_workgroup(Columns<D>& c, bool idle, const char* K, const char* V, int n, unsigned lds, float c2) {
  using Tl = Tile<D>;
  using R = Ring<D, KW>;
  constexpr int RB = D * 2, kInst = R::kTile / 1024 / kShWaves;  // copies of 1 KB of a wave, of K and of V
  static_assert(kInst == 2 || kInst == 4, "piece_xor(wave * kInst + i) = piece_xor(wave * kInst) ^ piece_xor(i)");
  using Loader = TileLoader<D, kShWaves>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  FragAddr<D> fa;
  fa.init(lane);
  const int j = lane / Tl::kChunks;
  const int g_off = (j * RB + (((lane % Tl::kChunks) ^ Tl::swz(j)) << 4)) ^ Loader::piece_xor(wave * kInst);
  const i32x4 k_buf = make_tile_buffer(K, (unsigned)n * RB), v_buf = make_tile_buffer(V, (unsigned)n * RB);
  // (tiles past the end are asked for as well: they fetch nothing, and the number of copies in flight stays the same)
  auto issue = [&](int i, int stage) {
    const unsigned at = lds + stage * 2 * R::kTile + wave * kInst * 1024;
#pragma unroll
    for (int q = 0; q < kInst; ++q)
      tile_copy16(k_buf, xor_here(g_off, Loader::piece_xor(q)), i * R::kTile + (wave * kInst + q) * 1024, at + q * 1024);
#pragma unroll
    for (int q = 0; q < kInst; ++q)
      tile_copy16(v_buf, xor_here(g_off, Loader::piece_xor(q)), i * R::kTile + (wave * kInst + q) * 1024, at + R::kTile + q * 1024);
  };
  const int n_tiles = (n + R::kRows - 1) / R::kRows;
#pragma unroll
  for (int i = 0; i < R::kStages - 1; ++i) issue(i, i);
  int stage = 0;
  for (int i = 0; i < n_tiles; ++i) {
    wait_own_copies<(R::kStages - 2) * 2 * kInst>();
    __syncthreads();  // the tile is there, and everybody is done with the one before it, whose stage is free
    issue(i + R::kStages - 1, stage == 0 ? R::kStages - 1 : stage - 1);
    const unsigned k = lds + stage * 2 * R::kTile;
    stage = stage == R::kStages - 1 ? 0 : stage + 1;
    const int left = n - i * R::kRows;
    if (idle) continue;
    if constexpr (KW == 1) {
      c.template fold<R::kRows / 32>(k, k + R::kTile, fa, lane, left, c2);
    } else {
      const int half = wave >> 1;
      if (left > half * 32) c.template fold<1>(k + half * 32 * RB, k + half * 32 * RB + R::kTile, fa, lane, left - half * 32, c2);
    }
  }
  wait_own_copies<0>();  // (the ring is about to be used for something else)
}

// ---------------------------------------------------------------- all slices
// PREFIX: how prefixes are read (0: none, 1: by wave, 2 / 4: by workgroup, so many waves of columns, 3: vector ALUs).  OWN: heads per
// workgroup on the vector ALUs (1, 2, 4), or 0: by wave on the matrix pipe.
template <int D, int PREFIX, int OWN>
constexpr int slices_lds() {
  // the ring; or 32 rows of K and V of each wave, where their states go afterwards; or the waves' states of OWN heads
  return PREFIX == 2 || PREFIX == 4 ? ring_bytes(D) : PREFIX == 1 || OWN == 0 ? kShWaves * 2 * 32 * D * 2
         : kShWaves * (PREFIX == 3 ? 4 : OWN) * (D + 2) * 4;
}
// (Three waves per SIMD at d = 64 with prefixes read by workgroups, of which two are resident first: own rows take the
// third place at once.  512 queries behind 16384 rows 44.8 -> 42.5 us, own rows of 64 x 500, 64 heads on 8, 18.6 -> 16.8; without such
// prefixes two are ahead, 33.5 / 36.0 us for 16 x 3100 rows.)
constexpr int waves_per_simd(int d, int prefix) { return d == 64 && (prefix == 2 || prefix == 4) ? 3 : 2; }
template <int D, int PREFIX, int OWN>
__global__ __launch_bounds__(kShWaves * 64, waves_per_simd(D, PREFIX)) void moda_shared_slices_kernel(SharedParams p) {
  constexpr int RB = D * 2;
  constexpr bool kMatrix = (PREFIX > 0 && PREFIX != 3) || OWN == 0;
  constexpr int kAhead = D == 64 && waves_per_simd(D, PREFIX) == 2 ? 2 : 1;  // blocks in flight of a wave that reads by itself: registers
  __shared__ __attribute__((aligned(1024))) unsigned char smem[slices_lds<D, PREFIX, OWN>()];
  __shared__ float stat[kMatrix ? kShWaves : 1][32][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, hi = lane >> 5;
  const unsigned lds = (unsigned)(size_t)(lds_ptr)smem;
  const int G = p.Hq / p.Hk;
  const float c2 = p.scale_log2;
  int id = blockIdx.x;
  // a wave's part of the rows of a run: a quarter, in whole blocks of 32
  auto part = [&](int& n, const char*& K, const char*& V) {
    const int q = ((n + kShWaves - 1) / kShWaves + 31) / 32 * 32, first = min(wave * q, n);
    n = min(q, n - first);
    K += (size_t)first * RB;
    V += (size_t)first * RB;
    return first;
  };
  if (PREFIX > 0 && id < p.prefix_blocks) {  // (they last longest: they come first)
    const int per = p.B / p.Np, M = per * G;  // queries of a prefix and key/value head
    constexpr int CW = PREFIX > 0 && PREFIX != 3 ? PREFIX : 1, kCols = CW * 32;
    // column chunks of the same rows are neighbours on a die (ids equal mod 8), whose L2 then serves all but the first
    const int n_cc = (M + kCols - 1) / kCols;
    const int u = id / (8 * n_cc) * 8 + id % 8, cc = id / 8 % n_cc;
    const int slice = u % p.n_prefix, xg = u / p.n_prefix;
    if (xg >= p.Np * p.Hk) return;  // (padding of the grid; uniform)
    const int x = xg / p.Hk, g = xg - x * p.Hk;
    const int plen = filled(p.prefix_lengths, x, p.P);
    // column -> (sequence of the prefix, head of the group); a column past the last repeats it and is not stored
    auto head_of = [&](int col) { return (size_t)(x * per + col / G) * p.Hq + g * G + col % G; };
    const int begin = slice * p.prefix_per, n = max(0, min(plen - begin, p.prefix_per));
    const size_t at = ((size_t)xg * p.P_alloc + begin) * RB;
    Rows x_rows = {(const char*)p.Kp + at, (const char*)p.Vp + at, n, nullptr, nullptr, 0};
    const size_t to = ((size_t)xg * p.n_prefix + slice) * M + cc * kCols;
    if constexpr (PREFIX == 3) {
      read_rows<D, 4>(x_rows, [&](int j) { return (const char*)p.Q + head_of(j) * RB; }, M, c2, p.ws_o + to * D, p.ws_ml + to * 2,
                      nullptr, 0, (float*)smem);
      return;
    }
    const int col0 = cc * kCols + (wave % CW) * 32;
    Columns<D> c;
    c.init((const char*)p.Q + head_of(min(col0 + l32, M - 1)) * RB, hi);
    if constexpr (PREFIX == 1) {
      part(x_rows.n, x_rows.K, x_rows.V);
      read_by_wave<D, kAhead>(c, x_rows, lds + wave * 2 * 32 * RB, c2);
    } else {
      read_by_workgroup<D, kShWaves / CW>(c, col0 >= M, x_rows.K, x_rows.V, n, lds, c2);
    }
    fold_waves<D, CW>(c, smem, stat, c2, min(kCols, M - cc * kCols), p.ws_o + to * D, p.ws_ml + to * 2);
    return;
  }
  if (PREFIX > 0) id -= p.prefix_blocks;
  // own rows; the slots go with the last slice
  constexpr int kHeads = OWN > 0 ? OWN : 32;  // of a workgroup
  const int slice = id % p.n_own, n_gc = (G + kHeads - 1) / kHeads;
  id /= p.n_own;
  const int gc = id % n_gc, bg = id / n_gc, b = bg / p.Hk, g = bg - b * p.Hk;
  const int h0 = g * G + gc * kHeads, nh = min(kHeads, G - gc * kHeads);
  const int begin = slice * p.own_per;
  const size_t at = ((size_t)bg * p.T_alloc + begin) * RB, slot_at = (size_t)bg * p.depth_alloc * RB;
  Rows x = {(const char*)p.Ks + at, (const char*)p.Vs + at, max(0, min(filled(p.lengths, b, p.T) - begin, p.own_per)),
            (const char*)p.Kd + slot_at, (const char*)p.Vd + slot_at, slice == p.n_own - 1 ? p.depth_count : 0};
  const size_t bh = (size_t)b * p.Hq + h0;
  const size_t to = (size_t)p.B * p.Hq * p.n_prefix + ((size_t)bg * p.n_own + slice) * G + gc * kHeads;
  if constexpr (OWN > 0) {
    read_rows<D, OWN>(x, [&](int j) { return (const char*)p.Q + (bh + j) * RB; }, nh, c2, p.ws_o + to * D, p.ws_ml + to * 2,
                      p.w_out ? p.scores + bh * p.score_step + begin : nullptr, p.score_step, (float*)smem);
  } else {
    Columns<D> c;
    const int j = min(l32, nh - 1);
    c.init((const char*)p.Q + (bh + j) * RB, hi);
    const int first = part(x.n, x.K, x.V);
    part(x.n2, x.K2, x.V2);
    read_by_wave<D, kAhead>(c, x, lds + wave * 2 * 32 * RB, c2, p.w_out ? p.scores + bh * p.score_step + begin + first : nullptr, p.score_step, nh);
    fold_waves<D, 1>(c, smem, stat, c2, nh, p.ws_o + to * D, p.ws_ml + to * 2);
  }
}

// ---------------------------------------------------------------- outputs
// Workgroups [0, merge_blocks): O and LSE.  `by` slices of a head at a time, D / 4 threads each (four channels a thread), 1024 / D
// such teams in a workgroup.  The others: weights_out of 1024 rows of one (batch, key/value head); each finds the LSE of
// the group's heads from the slices' references and normalisers (8 bytes a state).
constexpr int kFinishRows = 1024;
template <int D>
__global__ __launch_bounds__(256) void moda_shared_finish_kernel(SharedParams p, int by, int merge_blocks, int n_chunks) {
  constexpr int kTeam = D / 4, kTeams = 256 / kTeam;
  __shared__ __attribute__((aligned(16))) float red[kTeams][D + 4];
  const float c2 = p.scale_log2;
  const int tid = threadIdx.x;
  // (a state whose scores are all -inf is empty: reference -inf, weight zero)
  auto factor = [&](float m, float ref) { return m == -INFINITY ? 0.f : fast_exp2((m - ref) * c2); };
  if ((int)blockIdx.x < merge_blocks) {
    const int team = tid / kTeam, ch = tid % kTeam * 4, part = team % by;
    const long long bh = (long long)blockIdx.x * (kTeams / by) + team / by, heads = (long long)p.B * p.Hq;
    float mm = -INFINITY, ll = 0.f;
    f32x4 oo = {0.f, 0.f, 0.f, 0.f};
    const int row = (int)min(bh, heads - 1), b = row / p.Hq, h = row % p.Hq, G = p.Hq / p.Hk;
    const HeadStates at(p, b, h / G, h % G);
    constexpr int kU = 4;
    for (int s0 = part; s0 < p.n_slices; s0 += kU * by) {
      f32x2 st[kU];
      f32x4 o[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const size_t i = at(p, min(s0 + u * by, p.n_slices - 1));
        st[u] = *(const f32x2*)(p.ws_ml + i * 2);
        o[u] = *(const f32x4*)(p.ws_o + i * D + ch);
      }
      float mn = mm;
#pragma unroll
      for (int u = 0; u < kU; ++u)
        if (s0 + u * by < p.n_slices) mn = fmaxf(mn, st[u][0]);
      const float al = factor(mm, mn);
      mm = mn;
      ll *= al;
#pragma unroll
      for (int j = 0; j < 4; ++j) oo[j] *= al;
#pragma unroll
      for (int u = 0; u < kU; ++u)
        if (s0 + u * by < p.n_slices) {
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
    return;
  }
  const int id = blockIdx.x - merge_blocks, bg = id / n_chunks, j0 = id % n_chunks * kFinishRows;
  const int b = bg / p.Hk, g = bg - b * p.Hk, G = p.Hq / p.Hk;
  const int len = filled(p.lengths, b, p.T);
  if (j0 >= len) return;
  // four rows a thread, eight heads at a time: their logits are asked for before the LSE is known
  const int j = j0 + tid * 4;
  const size_t row = (size_t)bg * p.T_alloc + j;
  const bool whole = p.T_alloc % 4 == 0 && j + 4 <= len;  // (16-byte aligned then)
  f32x4 w = {0.f, 0.f, 0.f, 0.f};
  if (p.w_in) {
    if (whole) {
      w = *(const f32x4*)(p.w_in + row);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (j + i < len) w[i] = p.w_in[row + i];
    }
  }
  float* lse2 = &red[0][0];  // LSE * log2(e) of eight heads; +inf where nothing has weight
  const int at_row = min(j, (int)p.score_step - 4);  // (what lies behind the sequence is not stored)
  const float* sc = p.scores + ((size_t)b * p.Hq + g * G) * p.score_step + at_row;
  for (int h0 = 0; h0 < G; h0 += 8) {
    f32x4 s[8];
#pragma unroll
    for (int h = 0; h < 8; ++h) s[h] = *(const f32x4*)(sc + (size_t)min(h0 + h, G - 1) * p.score_step);
    __syncthreads();
    {  // 32 lanes per head
      const int h = tid >> 5;
      const HeadStates at(p, b, g, min(h0 + h, G - 1));
      float m = -INFINITY, l = 0.f;
      for (int i = tid & 31; i < p.n_slices; i += 32) {
        const f32x2 x = *(const f32x2*)(p.ws_ml + at(p, i) * 2);
        const float mn = fmaxf(m, x[0]);
        l = l * factor(m, mn) + factor(x[0], mn) * x[1];
        m = mn;
      }
#pragma unroll
      for (int x = 1; x < 32; x *= 2) {
        const float m2 = __shfl_xor(m, x), l2 = __shfl_xor(l, x), mn = fmaxf(m, m2);
        l = l * factor(m, mn) + l2 * factor(m2, mn);
        m = mn;
      }
      if ((tid & 31) == 0) lse2[h] = h0 + h >= G || l == 0.f ? INFINITY : m * c2 + __log2f(l);
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      if (h0 + h >= G) break;  // (uniform)
      const float z = lse2[h];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] += fast_exp2(__builtin_fmaf(s[h][i], c2, -z));
    }
  }
  if (whole) {
    *(f32x4*)(p.w_out + row) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (j + i < len) p.w_out[row + i] = w[i];
  }
}

// ---------------------------------------------------------------- the cut into slices
// How own rows are read: 0 on the matrix pipe, else heads per workgroup on the vector ALUs.  A workgroup of the latter is through in
// half the time, one of the former does less per row: from 3 heads on by the rows of all caches (vector ALUs / matrix pipe, us, with
// weights, 4 heads a group, (batch x key/value heads), rows):
//   d=64   8, 600 8.4 / 10.1;   8, 5000 10.5 / 12.5;   32, 1200 10.1 / 12.0;   32, 2500 12.9 / 13.1;   8, 12000 14.0 / 13.8;   128, 5000 37.8 / 36.0
//   d=128  8, 600 8.6 / 11.9;   8, 5000 12.6 / 14.7;   32, 1200 11.9 / 14.5;   32, 2500 18.1 / 15.9;   8, 12000 20.3 / 16.8;   512, 2500 127 / 120
//   8 heads, in two workgroups:  d=64 8, 1200 8.9 / 10.4;   8, 2500 10.4 / 11.0;   8, 5000 13.3 / 12.6;   d=128 8, 1200 10.9 / 12.4;   8, 5000 19.0 / 14.8
// (One limit for both head dimensions: d = 64 would go on a little longer, 32 x 2500 rows are 0.2 us behind.)
static int own_kind(const SharedParams& p) {
  const int G = p.Hq / p.Hk;
  if (G <= 2) return G;
  return G <= 8 && (long long)p.B * p.Hk * p.T < (G <= 4 ? 65536 : 24576) ? 4 : 0;
}

// Slices of a run of `rows` rows that `units` workgroups read each.  Long runs: `many` workgroups in all, which the chip holds at
// once, as long as a slice has `good` rows; a second round of workgroups costs a workgroup's chain of latencies again, about
// 5 us.  Runs that leave units without work: one workgroup per unit down to `least` rows, what the waves take at a time.
static long long slices_wanted(int rows, long long units, int many, int good, int least) {
  auto most = [&](int size) { return ((long long)rows + size - 1) / size; };
  const long long want = std::max(std::min(256 / units, most(least)), std::min(many / units, most(good)));
  return std::max(std::max(want, 1ll), ((long long)rows >> 22) + 1);  // (a slice is addressed with 32-bit byte offsets)
}
static void cut(int rows, long long units, int many, int good, int least, int& n, int& per) {
  const long long want = slices_wanted(rows, units, many, good, least);
  per = (int)((rows + want - 1) / want + least - 1) / least * least;
  n = per > 0 ? (rows + per - 1) / per : 0;
}

// How the rows of prefixes and of own caches are cut.
struct Cut {
  long long units;
  int many, good, least;
};
struct Plan {
  int kind, own_heads;  // SharedParams::prefix_kind, own_kind
  long long xg, cc;  // prefixes x key/value heads, column chunks of each
  Cut prefix, own;
  Plan(const SharedParams& p, int d) {
    const int G = p.Hq / p.Hk, rows_at_once = kShWaves * 4 * 512 / d;  // (of read_rows)
    const long long M = (long long)p.B / p.Np * G, groups = (long long)p.B * p.Hk;
    kind = p.P == 0 ? 0 : M <= 4 ? 3 : M <= 32 ? 1 : M <= 64 ? 2 : 4;
    xg = (long long)p.Np * p.Hk;
    cc = kind == 2 || kind == 4 ? (M + kind * 32 - 1) / (kind * 32) : 1;
    // By wave 256 workgroups: as many again come with the own rows (32 columns behind 32768 rows, 16 heads: 256 84.8 us, 768 93.8; 64
    // heads of 2000 rows 19.5 / 25.8).  By workgroup 512, or 384 where own rows, a quarter of what the tiles walk or more, fill
    // the rest (512 / 384: 512 columns behind 16384 rows, 64 x 500 own ones 51.1 / 48.3 us, 64 x 300 of d = 128 74.9 / 69.6; 128 behind
    // 8192, 128 x 100 of d = 128 52.4 / 45.3; with one own row 512 behind 65536 110 / 124).
    if (kind == 3) prefix = {xg, 512, 256, rows_at_once};
    else if (kind <= 1) prefix = {xg, 256, 512, 128};
    else prefix = {xg * cc, 4 * groups * p.T >= xg * cc * p.P ? 384 : 512, 256, 64};
    // Beside prefixes, whose workgroups last longer, more of the long own caches' (16 x 2000 rows behind 16000, 16 heads of d = 128, 512 /
    // 1024: 63.5 / 57.1 us; without a prefix 16 x 2000 38.5 / 39.4).
    own_heads = own_kind(p);
    own = own_cut(groups, G, own_heads, p.P > 0, rows_at_once);
  }
  static Cut own_cut(long long groups, int G, int heads, bool prefix, int rows_at_once) {
    if (heads == 0) return {groups * ((G + 31) / 32), 512, 512, 128};
    const long long units = groups * ((G + heads - 1) / heads);
    return prefix ? Cut{units, 1024, 512, rows_at_once} : Cut{units, 512, 256, rows_at_once};
  }
};

static void plan(SharedParams& p, int d) {
  const Plan l(p, d);
  p.prefix_kind = l.kind;
  p.n_prefix = p.prefix_per = p.prefix_blocks = 0;
  if (p.P > 0) {
    cut(p.P, l.prefix.units, l.prefix.many, l.prefix.good, l.prefix.least, p.n_prefix, p.prefix_per);
    const long long blocks = (l.xg * p.n_prefix + 7) / 8 * 8 * l.cc;
    p.prefix_blocks = blocks > 0x7fffffff ? 0x7fffffff : (int)blocks;  // (too many: the launch is refused)
  }
  cut(p.T, l.own.units, l.own.many, l.own.good, l.own.least, p.n_own, p.own_per);
  if (p.depth_count > 0) p.n_own = std::max(p.n_own, 1);
  p.n_slices = p.n_prefix + p.n_own;
  p.score_step = ((size_t)p.T + 31) / 32 * 32;
}

// Calls that take one kernel: no prefix, up to 4 heads per group, and few steps of rows (128 at d = 128, 256 at d = 64), more of them
// where the workgroups fill half the chip anyway.  Two kernels / one, us, (batch x key/value heads), rows, with weights:
//   1 head   d=64 16, 20 7.1 / 4.7;   64, 500 7.2 / 5.4;   512, 500 13.8 / 9.8;   d=128 16, 250 7.8 / 6.7;   16, 500 7.2 / 7.6;   512, 500 23.0 / 18.5
//   2 heads  d=64 8, 500 7.5 / 6.5;   d=128 8, 120 7.3 / 4.9;   8, 250 8.1 / 7.5;   8, 500 7.5 / 8.9;   256, 500 14.7 / 10.5
//   4 heads  d=64 8, 250 9.6 / 8.5;   8, 500 8.5 / 8.7;   d=128 8, 120 8.5 / 6.3;   8, 240 9.8 / 8.8;   8, 500 8.8 / 12.7;   256, 500 19.7 / 14.2
// (The limits in steps are the same for both head dimensions; where they end the one kernel may be a little behind: 1 head d=128 16 x 500, 4
// heads d=64 8 x 500.)
static bool in_one(const SharedParams& p, int d) {
  const int G = p.Hq / p.Hk, step = kOneWaves * 4 * 512 / d;
  if (p.P > 0 || p.T > kOneRows || G > 4) return false;
  const long long steps = ((long long)p.T + p.depth_count + step - 1) / step;
  return steps <= (G == 1 || (long long)p.B * p.Hk >= 128 ? 4 : 2);
}

static size_t state_count(const SharedParams& p) { return ((size_t)p.B * p.Hq * p.n_slices + 1) / 2 * 2; }  // (even: 16-byte pieces)

// What every shorter own cache and prefix takes at most: cuts have no more slices than are wanted, and those never get fewer.
size_t decode_shared_workspace_bytes(const SharedParams& dims, int d, bool with_weights) {
  SharedParams p = dims;
  plan(p, d);
  const Plan l(p, d);
  long long own = 0;  // (whichever way they are read, with a prefix and without)
  for (int heads : {0, l.own_heads > 0 ? l.own_heads : 4})
    for (bool prefix : {false, true}) {
      const Cut c = Plan::own_cut((long long)p.B * p.Hk, p.Hq / p.Hk, heads, prefix, kShWaves * 4 * 512 / d);
      if (p.T > 0) own = std::max(own, slices_wanted(p.T, c.units, c.many, c.good, c.least));
    }
  p.n_slices = (int)(std::max(own, 1ll) + (p.P > 0 ? slices_wanted(p.P, l.prefix.units, std::max(l.prefix.many, l.kind > 1 ? 512 : 0), l.prefix.good, l.prefix.least) : 0));
  return (state_count(p) * (d + 2) + (with_weights ? (size_t)p.B * p.Hq * p.score_step : 0)) * sizeof(float);
}

template <int D, int PREFIX>
static void (*slices_kernel(int own))(SharedParams) {
  return own == 4 ? moda_shared_slices_kernel<D, PREFIX, 4> : own == 2 ? moda_shared_slices_kernel<D, PREFIX, 2>
         : own == 1 ? moda_shared_slices_kernel<D, PREFIX, 1> : moda_shared_slices_kernel<D, PREFIX, 0>;
}

template <int D>
static hipError_t launch_d(const SharedParams& p, hipStream_t stream) {
  const int G = p.Hq / p.Hk, own = own_kind(p);
  if (in_one(p, D)) {
    const long long groups = (long long)p.B * p.Hk;
    if (!grid_ok(groups, kOneWaves * 64)) return kGridTooLarge;
    return launch_kernel(G >= 3 ? moda_shared_one_kernel<D, 4> : G == 2 ? moda_shared_one_kernel<D, 2> : moda_shared_one_kernel<D, 1>,
                         dim3((unsigned)groups), dim3(kOneWaves * 64), stream, p);
  }
  const int heads_per = own > 0 ? own : 32;
  const long long blocks = p.prefix_blocks + (long long)p.B * p.Hk * ((G + heads_per - 1) / heads_per) * p.n_own;
  // teams of a workgroup that share a head's slices, so that each folds four or fewer of them at a time
  const int teams = 1024 / D;
  int by = 1;
  while (by < teams && by * 4 < p.n_slices) by *= 2;
  const long long heads = (long long)p.B * p.Hq, merge_blocks = (heads + teams / by - 1) / (teams / by);
  const int chunks = p.w_out ? (p.T + kFinishRows - 1) / kFinishRows : 0;
  const long long finish_blocks = merge_blocks + (long long)p.B * p.Hk * chunks;
  if ((blocks > 0 && !grid_ok(blocks, kShWaves * 64)) || !grid_ok(finish_blocks, 256)) return kGridTooLarge;
  if (blocks > 0) {
    auto* kernel = p.prefix_kind == 0 ? slices_kernel<D, 0>(own) : p.prefix_kind == 1 ? slices_kernel<D, 1>(own)
                   : p.prefix_kind == 2 ? slices_kernel<D, 2>(own) : p.prefix_kind == 3 ? slices_kernel<D, 3>(own) : slices_kernel<D, 4>(own);
    const hipError_t e = launch_kernel(kernel, dim3((unsigned)blocks), dim3(kShWaves * 64), stream, p);
    if (e != hipSuccess) return e;
  }
  return launch_kernel(moda_shared_finish_kernel<D>, dim3((unsigned)finish_blocks), dim3(256), stream, p, by, (int)merge_blocks, chunks);
}

hipError_t launch_decode_shared(SharedParams p, int d, void* workspace, hipStream_t stream) {
  plan(p, d);
  p.ws_o = (float*)workspace;
  p.ws_ml = p.ws_o + state_count(p) * d;
  p.scores = p.ws_ml + state_count(p) * 2;
  return d == 128 ? launch_d<128>(p, stream) : launch_d<64>(p, stream);
}

}  // namespace moda
