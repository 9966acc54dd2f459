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
//   prefixes   all queries that share a prefix (sequences x heads of a group) are the columns of matrix products
//              S^T = K Q^T, O^T += V^T P^T.  Up to 32 columns (read_by_wave): every wave reads its own part of the slice.
//              More (read_by_workgroup): 2 or 4 waves of 32 columns share the K and V tiles of a slice in LDS.
//   own rows   up to 4 heads per group on the vector ALUs (read_rows), more as the columns of read_by_wave.
#include <algorithm>

#include "moda_decode_fold.h"
#include "moda_launch.h"
#include "moda_tile.h"

namespace moda {

constexpr int kShWaves = 4;

// Floats of a slice's state of one head: channels, reference, normaliser, two unused (so that states are aligned).
constexpr int state_floats(int d) { return d + 4; }

__device__ __forceinline__ int filled(const int* lengths, int i, int most) {
  return lengths ? min(max(lengths[i], 0), most) : most;
}

// ---------------------------------------------------------------- rows on the vector ALUs
// A lane owns 8 channels, d/8 lanes a row; a wave takes kU batches of 64 / (d/8) rows at a time, the next ones in
// flight, and raises its reference once for them.  `q` = GT query rows (heads from nh on repeat the last one and are not
// stored), `dst` = the first head's state of this slice, `scores` = the first head's logits of these rows, or null.
template <int D, int GT>
__device__ __forceinline__ void read_rows(const char* K, const char* V, int n, const char* q_rows, int nh, float c2, float* dst,
                                          size_t dst_step, float* scores, size_t score_step, float* red) {
  constexpr int LPR = D / 8, RPS = 64 / LPR, RB = D * 2, kU = 4, STEP = kShWaves * kU * RPS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, rg = lane / LPR, l16 = lane % LPR;
  u32x4 q[GT];
  float m[GT], l[GT], o[GT][8];
#pragma unroll
  for (int j = 0; j < GT; ++j) {
    q[j] = *(const u32x4*)(q_rows + (size_t)min(j, nh - 1) * RB + l16 * 16);
    m[j] = -INFINITY;
    l[j] = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) o[j][k] = 0.f;
  }
  const int row0 = wave * kU * RPS + rg;
  if (n > 0) {  // (uniform)
    auto load = [&](const char* base, int r) {
      return __builtin_nontemporal_load((const u32x4*)(base + (size_t)min(r, n - 1) * RB + l16 * 16));
    };
    u32x4 kn[kU], vn[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      kn[u] = load(K, row0 + u * RPS);
      vn[u] = load(V, row0 + u * RPS);
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
          kn[u] = load(K, r + STEP + u * RPS);
          vn[u] = load(V, r + STEP + u * RPS);
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
          if (l16 < kU && at < n && j < nh) scores[(size_t)j * score_step + at] = a;
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
  for (int t = tid; t < GT * D; t += kShWaves * 64) {
    const int j = t / D, ch = t % D;
    if (j >= nh) continue;
    float mm = -INFINITY, ll = 0.f, oo = 0.f;
#pragma unroll
    for (int w = 0; w < kShWaves; ++w) mm = fmaxf(mm, red[(w * GT + j) * (D + 2) + D]);
#pragma unroll
    for (int w = 0; w < kShWaves; ++w) {
      const float* x = red + (w * GT + j) * (D + 2);
      const float f = x[D] == -INFINITY ? 0.f : fast_exp2((x[D] - mm) * c2);
      ll += f * x[D + 1];
      oo += f * x[ch];
    }
    float* to = dst + j * dst_step;
    to[ch] = oo;
    if (ch == 0) {
      to[D] = mm;
      to[D + 1] = ll;
    }
  }
}

// ---------------------------------------------------------------- rows on the matrix pipe
// A wave's 32 columns: lanes l and l + 32 hold query l, its running reference and (each its half of) its normaliser.
template <int D>
struct Columns {
  using Tl = Tile<D>;
  bf16x8 q[Tl::kDSteps];
  f32x16 o[Tl::kDBlocks];  // O^T: [channel block], registers = channels 8 i + 4 hi + j
  float m, l;
  __device__ __forceinline__ void init(const char* q_row, int hi) {
#pragma unroll
    for (int st = 0; st < Tl::kDSteps; ++st) q[st] = *(const bf16x8*)(q_row + st * 32 + hi * 16);
#pragma unroll
    for (int cb = 0; cb < Tl::kDBlocks; ++cb)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[cb][i] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }
  // NB blocks of 32 rows: K rows from LDS address `k`, V rows from `v` (layout of Tile<D>); `left` = rows that count.
  // The logits of the lane's column (before the scale) go to scores[row], if not null.
  template <int NB>
  __device__ __forceinline__ void fold(unsigned k, unsigned v, const FragAddr<D>& fa, int hi, int left, float c2, float* scores) {
    f32x16 s[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
    for (int st = 0; st < Tl::kDSteps; ++st) {
      const unsigned xk = (unsigned)xor_here((int)(fa.row + k), st << 5);
#pragma unroll
      for (int b = 0; b < NB; ++b) s[b] = mfma_bf16(FragAddr<D>::row_frag(xk, b, 0), q[st], s[b]);
    }
    if (scores) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = b * 32 + i * 8 + hi * 4;
          if (row + 4 <= left) {
            *(f32x4*)(scores + row) = (f32x4){s[b][4 * i], s[b][4 * i + 1], s[b][4 * i + 2], s[b][4 * i + 3]};
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (row + j < left) scores[row + j] = s[b][4 * i + j];
          }
        }
    }
    if (left < NB * 32) {  // (uniform)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (b * 32 + (i >> 2) * 8 + hi * 4 + (i & 3) >= left) s[b][i] = -INFINITY;
    }
    float bm = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) bm = fmaxf(bm, s[b][i]);
    bm = pair_max(bm);
    // The reference is raised only when the blocks' maximum exceeds it by more than 8 powers of two: weights stay below
    // 2^8, which fp32 sums and bf16 weights hold, and any reference gives the same quotient.  While all scores are
    // -inf it stays there, with an empty state.
    const bool raise = bm > m + 8.0f / c2 || m == -INFINITY;
    if (__builtin_amdgcn_ballot_w64(raise) != 0) {  // (uniform)
      const float mn = raise ? bm : m;
      const float al = mn == m ? 1.f : fast_exp2((m - mn) * c2);
      m = mn;
      l *= al;
#pragma unroll
      for (int cb = 0; cb < Tl::kDBlocks; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[cb][i] *= al;
    }
    const float mc = m == -INFINITY ? 0.f : m * c2;
    const unsigned vt = fa.tr + v, vt8 = fa.tr8 + v;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        float pv[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          pv[i] = fast_exp2(s[b][hf * 8 + i] * c2 - mc);
          l += pv[i];
        }
        // weights as bf16 for the matrix pipe: off by 2^-8 of themselves at most, the normaliser is summed before
        const bf16x8 pb = pack8(pv);
#pragma unroll
        for (int cb = 0; cb < Tl::kDBlocks; ++cb)
          o[cb] = mfma_bf16(FragAddr<D>::tr_frag((unsigned)xor_here((int)vt, cb << 6), (unsigned)xor_here((int)vt8, cb << 6),
                                                 b * 2 + hf, 0),
                            pb, o[cb]);
      }
  }
};

// The states of a workgroup's waves, those with the same columns (wave % CW) folded, to column -> dst(column) (null: a column
// past the last query).  LDS: a wave's O^T as 16-byte pieces of four channels, piece c of column q at 32 c + (q ^ c % 32) of
// the wave's part, so that both the writes (32 columns of a piece) and the reads (the pieces of a column, which make
// whole rows in memory) touch every bank alike.
template <int D, int CW, class Dst>
__device__ __forceinline__ void fold_waves(const Columns<D>& c, unsigned char* smem, float (*stat)[32][2], float c2, Dst&& dst) {
  constexpr int KW = kShWaves / CW, kPieces = D / 4, kPart = 32 * D * 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, hi = lane >> 5;
  const float l_all = pair_sum(c.l);
  __syncthreads();  // (the tiles are not read any more)
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int piece = cb * 8 + i * 2 + hi;
      *(f32x4*)(smem + wave * kPart + (piece * 32 + (l32 ^ (piece & 31))) * 16) =
          (f32x4){c.o[cb][4 * i], c.o[cb][4 * i + 1], c.o[cb][4 * i + 2], c.o[cb][4 * i + 3]};
    }
  if (hi == 0) {
    stat[wave][l32][0] = c.m;
    stat[wave][l32][1] = l_all;
  }
  __syncthreads();
#pragma unroll
  for (int i = tid; i < CW * 32 * kPieces; i += kShWaves * 64) {
    const int col = i / kPieces, piece = i % kPieces, cw = col / 32, q = col % 32;
    float* to = dst(col);
    if (!to) continue;
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KW; ++k) m = fmaxf(m, stat[k * CW + cw][q][0]);
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      const int w = k * CW + cw;
      // (a lone wave's state as it is: its reference may be NaN, which the maximum leaves out)
      const float f = KW == 1 ? 1.f : stat[w][q][0] == -INFINITY ? 0.f : fast_exp2((stat[w][q][0] - m) * c2);
      l += f * stat[w][q][1];
      const f32x4 x = *(const f32x4*)(smem + w * kPart + (piece * 32 + (q ^ (piece & 31))) * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += f * x[j];
    }
    *(f32x4*)(to + piece * 4) = o;
    if (piece == 0) *(f32x2*)(to + D) = (f32x2){m, l};
  }
}

// Every wave by itself: n rows at K and V (its part of the slice), 32 at a time through its two LDS tiles at `lds`; the next
// block(s) are in flight in registers.  Rows past the end read as zeros (bounds-checked buffers) and fetch nothing.
constexpr int waves_ahead(int d) { return d == 64 ? 2 : 1; }  // (d = 128: registers for one)
template <int D>
__device__ __forceinline__ void read_by_wave(Columns<D>& c, const char* K, const char* V, int n, unsigned lds, float c2, float* scores) {
  using Tl = Tile<D>;
  constexpr int RB = D * 2, kInst = 32 * RB / 1024, kHalf = 32 * RB, kPF = waves_ahead(D);
  const int lane = threadIdx.x & 63, hi = lane >> 5;
  FragAddr<D> fa;
  fa.init(lane);
  const __amdgpu_buffer_rsrc_t k_buf = __builtin_amdgcn_make_buffer_rsrc((void*)K, 0, n * RB, 0x00020000);
  const __amdgpu_buffer_rsrc_t v_buf = __builtin_amdgcn_make_buffer_rsrc((void*)V, 0, n * RB, 0x00020000);
  const int jr = lane / Tl::kChunks, pc = lane % Tl::kChunks;
  const int g_off = jr * RB + ((pc ^ Tl::swz(jr)) << 4);
  auto piece_xor = [](int q) { return (D == 128 ? (q & 3) : ((q & 1) << 1)) << 4; };
  struct Block {
    u32x4 k[kInst], v[kInst];
  };
  auto issue = [&](int blk, Block& r) {
    const int soff = blk * kHalf;
#pragma unroll
    for (int q = 0; q < kInst; ++q)
      r.k[q] = __builtin_amdgcn_raw_buffer_load_b128(k_buf, xor_here(g_off, piece_xor(q)), soff + q * 1024, 2);
#pragma unroll
    for (int q = 0; q < kInst; ++q)
      r.v[q] = __builtin_amdgcn_raw_buffer_load_b128(v_buf, xor_here(g_off, piece_xor(q)), soff + q * 1024, 2);
  };
  const int n_blocks = (n + 31) / 32;
  Block buf[kPF];
#pragma unroll
  for (int i = 0; i < kPF; ++i) issue(i, buf[i]);
  for (int blk0 = 0; blk0 < n_blocks; blk0 += kPF) {
#pragma unroll
    for (int i = 0; i < kPF; ++i) {
      const int blk = blk0 + i;
      // (a wave's LDS operations execute in order: these writes follow the reads of the block before)
#pragma unroll
      for (int q = 0; q < kInst; ++q)
        *(u32x4 __attribute__((address_space(3)))*)(size_t)(lds + q * 1024 + lane * 16) = buf[i].k[q];
#pragma unroll
      for (int q = 0; q < kInst; ++q)
        *(u32x4 __attribute__((address_space(3)))*)(size_t)(lds + kHalf + q * 1024 + lane * 16) = buf[i].v[q];
      issue(blk + kPF, buf[i]);
      if (blk < n_blocks) c.template fold<1>(lds, lds + kHalf, fa, hi, n - blk * 32, c2, scores ? scores + blk * 32 : nullptr);
    }
  }
}

// The workgroup together: KW x 32 (or 64, KW = 1) rows at a time in a ring of two stages; a wave folds all of them (KW = 1) or its
// 32 of them (KW = 2: waves 2 and 3 hold the columns of waves 0 and 1).
template <int D, int KW>
__device__ __forceinline__ void read_by_workgroup(Columns<D>& c, bool idle, const char* K, const char* V, int n, unsigned lds, float c2) {
  using Tl = Tile<D>;
  constexpr int RB = D * 2, kStage = 2 * Tl::kBytes;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hi = lane >> 5;
  FragAddr<D> fa;
  fa.init(lane);
  TileLoader<D, kShWaves> loader;
  loader.init(wave, lane);
  const i32x4 k_buf = make_tile_buffer(K, (unsigned)n * RB), v_buf = make_tile_buffer(V, (unsigned)n * RB);
  auto issue = [&](int i) {
    const unsigned at = lds + (i & 1) * kStage;
    loader.issue(k_buf, i * 64, at);
    loader.issue(v_buf, i * 64, at + Tl::kBytes);
  };
  const int n_tiles = (n + 63) / 64;
  if (n_tiles > 0) issue(0);
  for (int i = 0; i < n_tiles; ++i) {
    wait_copies();
    __syncthreads();  // the tile is there, and everybody is done with the other stage
    if (i + 1 < n_tiles) issue(i + 1);
    const unsigned k = lds + (i & 1) * kStage;
    const int left = n - i * 64;
    if (idle) continue;
    if (KW == 1) {
      c.template fold<2>(k, k + Tl::kBytes, fa, hi, left, c2, nullptr);
    } else {
      const int half = wave >> 1;
      if (left > half * 32) c.template fold<1>(k + half * 32 * RB, k + half * 32 * RB + Tl::kBytes, fa, hi, left - half * 32, c2, nullptr);
    }
  }
}

// ---------------------------------------------------------------- all slices
// PREFIX: how prefixes are read (0: none, 1: by wave, 2 / 4: by workgroup, so many waves of columns).  OWN: heads per
// workgroup on the vector ALUs (1, 2, 4), or 0: by wave on the matrix pipe.
template <int D, int PREFIX, int OWN>
constexpr int slices_lds() {
  return PREFIX > 0 || OWN == 0 ? 2 * 2 * 64 * D * 2 : kShWaves * OWN * (D + 2) * 4;
}
template <int D, int PREFIX, int OWN>
__global__ __launch_bounds__(kShWaves * 64, 2) void moda_shared_slices_kernel(SharedParams p) {
  constexpr int RB = D * 2;
  constexpr bool kMatrix = PREFIX > 0 || OWN == 0;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[slices_lds<D, PREFIX, OWN>()];
  __shared__ float stat[kMatrix ? kShWaves : 1][32][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, hi = lane >> 5;
  const unsigned lds = (unsigned)(size_t)(lds_ptr)smem;
  const int G = p.Hq / p.Hk;
  const float c2 = p.scale_log2;
  const size_t state = (size_t)p.n_slices * state_floats(D);  // of one head
  int id = blockIdx.x;
  // a wave's part of the n rows of a slice: a quarter, in whole blocks of 32
  auto part = [&](int n, int& first) {
    const int q = ((n + kShWaves - 1) / kShWaves + 31) / 32 * 32;
    first = min(wave * q, n);
    return min(q, n - first);
  };
  if (PREFIX > 0 && id < p.prefix_blocks) {
    const int per = p.B / p.Np, M = per * G;  // queries of a prefix and key/value head
    constexpr int CW = PREFIX > 0 ? PREFIX : 1, kCols = CW * 32;
    // column chunks of the same rows are neighbours on a die (ids equal mod 8), whose L2 then serves all but the first
    const int n_cc = (M + kCols - 1) / kCols;
    const int u = id / (8 * n_cc) * 8 + id % 8, cc = id / 8 % n_cc;
    const int slice = u % p.n_prefix, xg = u / p.n_prefix;
    if (xg >= p.Np * p.Hk) return;  // (padding of the grid; uniform)
    const int x = xg / p.Hk, g = xg - x * p.Hk;
    const int plen = filled(p.prefix_lengths, x, p.P);
    // column -> (sequence of the prefix, head of the group); a column past the last repeats it and is not stored
    auto head_of = [&](int col) { return (size_t)(x * per + col / G) * p.Hq + g * G + col % G; };
    const int col0 = cc * kCols + (wave % CW) * 32;
    Columns<D> c;
    c.init((const char*)p.Q + head_of(min(col0 + l32, M - 1)) * RB, hi);
    const int begin = slice * p.prefix_per, n = max(0, min(plen - begin, p.prefix_per));
    const size_t at = ((size_t)xg * p.P_alloc + begin) * RB;
    const char *K = (const char*)p.Kp + at, *V = (const char*)p.Vp + at;
    if constexpr (PREFIX == 1) {
      int first;
      const int mine = part(n, first);
      read_by_wave<D>(c, K + (size_t)first * RB, V + (size_t)first * RB, mine, lds + wave * 2 * 32 * RB, c2, nullptr);
    } else {
      read_by_workgroup<D, kShWaves / CW>(c, col0 >= M, K, V, n, lds, c2);
    }
    fold_waves<D, CW>(c, smem, stat, c2, [&](int col) {
      col += cc * kCols;
      return col < M ? p.ws + head_of(col) * state + (size_t)slice * state_floats(D) : nullptr;
    });
    return;
  }
  if (PREFIX > 0) id -= p.prefix_blocks;
  // own rows: slices, then the depth slots
  const int n_own = p.n_slices - p.n_prefix;
  constexpr int kHeads = OWN > 0 ? OWN : 32;  // of a workgroup
  const int slice = id % n_own, n_gc = (G + kHeads - 1) / kHeads;
  id /= n_own;
  const int gc = id % n_gc, bg = id / n_gc, b = bg / p.Hk, g = bg - b * p.Hk;
  const int h0 = g * G + gc * kHeads, nh = min(kHeads, G - gc * kHeads);
  const bool depth = slice == p.n_own;
  const int begin = depth ? 0 : slice * p.own_per;
  const int n = depth ? p.depth_count : max(0, min(filled(p.lengths, b, p.T) - begin, p.own_per));
  const size_t at = ((size_t)bg * (depth ? p.depth_alloc : p.T_alloc) + begin) * RB;
  const char *K = (const char*)(depth ? p.Kd : p.Ks) + at, *V = (const char*)(depth ? p.Vd : p.Vs) + at;
  const size_t bh = (size_t)b * p.Hq + h0;
  float* dst = p.ws + bh * state + (size_t)(p.n_prefix + slice) * state_floats(D);
  const bool keep = p.w_out && !depth;
  if constexpr (OWN > 0) {
    read_rows<D, OWN>(K, V, n, (const char*)p.Q + bh * RB, nh, c2, dst, state, keep ? p.scores + bh * p.score_step + begin : nullptr,
                      p.score_step, (float*)smem);
  } else {
    Columns<D> c;
    const int j = min(l32, nh - 1);
    c.init((const char*)p.Q + (bh + j) * RB, hi);
    int first;
    const int mine = part(n, first);
    read_by_wave<D>(c, K + (size_t)first * RB, V + (size_t)first * RB, mine, lds + wave * 2 * 32 * RB, c2,
                    keep && l32 < nh ? p.scores + (bh + j) * p.score_step + begin + first : nullptr);
    fold_waves<D, 1>(c, smem, stat, c2, [&](int col) { return col < nh ? dst + col * state : nullptr; });
  }
}

// ---------------------------------------------------------------- outputs
// Workgroups [0, merge_blocks): O and LSE.  `by` slices of a head at a time, D / 4 threads each (four channels a thread), 1024 / D
// such teams in a workgroup.  The others: weights_out of 1024 rows of one (batch, key/value head); each finds the LSE of
// the group's heads from the slices' references and normalisers (8 bytes of a state).
constexpr int kFinishRows = 1024, kFinishHeads = 64;
template <int D>
__global__ __launch_bounds__(256) void moda_shared_finish_kernel(SharedParams p, int by, int merge_blocks, int n_chunks) {
  constexpr int kTeam = D / 4, kTeams = 256 / kTeam;
  __shared__ __attribute__((aligned(16))) float red[kTeams][state_floats(D)];
  const float c2 = p.scale_log2;
  const int tid = threadIdx.x;
  // (a state whose scores are all -inf is empty: reference -inf, weight zero)
  auto factor = [&](float m, float ref) { return m == -INFINITY ? 0.f : fast_exp2((m - ref) * c2); };
  if ((int)blockIdx.x < merge_blocks) {
    const int team = tid / kTeam, ch = tid % kTeam * 4, part = team % by;
    const long long bh = (long long)blockIdx.x * (kTeams / by) + team / by, heads = (long long)p.B * p.Hq;
    float mm = -INFINITY, ll = 0.f;
    f32x4 oo = {0.f, 0.f, 0.f, 0.f};
    const float* ws = p.ws + (size_t)min(bh, heads - 1) * p.n_slices * state_floats(D);
    constexpr int kU = 4;
    for (int s0 = part; s0 < p.n_slices; s0 += kU * by) {
      f32x2 st[kU];
      f32x4 o[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const float* x = ws + (size_t)min(s0 + u * by, p.n_slices - 1) * state_floats(D);
        st[u] = *(const f32x2*)(x + D);
        o[u] = *(const f32x4*)(x + ch);
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
  const int b = bg / p.Hk, g = bg - b * p.Hk, G = p.Hq / p.Hk, lane = tid & 63;
  const int len = filled(p.lengths, b, p.T);
  if (j0 >= len) return;
  constexpr int kRows = kFinishRows / 256;
  const size_t row = (size_t)bg * p.T_alloc;
  float w[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int j = min(j0 + i * 256 + tid, len - 1);
    w[i] = p.w_in ? p.w_in[row + j] : 0.f;
  }
  float* lse2 = &red[0][0];  // LSE * log2(e) of kFinishHeads heads; +inf where nothing has weight
  static_assert(kFinishHeads <= kTeams * state_floats(D), "");
  for (int h0 = 0; h0 < G; h0 += kFinishHeads) {
    const int nh = min(kFinishHeads, G - h0);
    __syncthreads();
    for (int h = tid >> 6; h < nh; h += 4) {  // a wave per head
      const float* ws = p.ws + ((size_t)b * p.Hq + g * G + h0 + h) * p.n_slices * state_floats(D) + D;
      float m = -INFINITY, l = 0.f;
      for (int s = lane; s < p.n_slices; s += 64) {
        const f32x2 x = *(const f32x2*)(ws + (size_t)s * state_floats(D));
        const float mn = fmaxf(m, x[0]);
        l = l * factor(m, mn) + factor(x[0], mn) * x[1];
        m = mn;
      }
#pragma unroll
      for (int x = 1; x < 64; x *= 2) {
        const float m2 = __shfl_xor(m, x), l2 = __shfl_xor(l, x), mn = fmaxf(m, m2);
        l = l * factor(m, mn) + l2 * factor(m2, mn);
        m = mn;
      }
      if (lane == 0) lse2[h] = l == 0.f ? INFINITY : m * c2 + __log2f(l);
    }
    __syncthreads();
    const float* sc = p.scores + ((size_t)b * p.Hq + g * G + h0) * p.score_step;
    for (int h = 0; h < nh; ++h) {
      const float z = lse2[h];
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const int j = min(j0 + i * 256 + tid, len - 1);
        w[i] += fast_exp2(__builtin_fmaf(sc[h * p.score_step + j], c2, -z));
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int j = j0 + i * 256 + tid;
    if (j < len) p.w_out[row + j] = w[i];
  }
}

// ---------------------------------------------------------------- the cut into slices
static int own_kind(int G) { return G > 4 ? 0 : G >= 3 ? 4 : G; }

static void plan(SharedParams& p) {
  const int G = p.Hq / p.Hk;
  const long long M = (long long)p.B / p.Np * G;
  auto cut = [](int rows, long long want, int least, int step, int& n, int& per) {
    want = std::max(want, ((long long)rows >> 22) + 1);  // (a slice is addressed with 32-bit byte offsets)
    n = (int)std::min(want, ((long long)rows + least - 1) / least);
    per = n > 0 ? (int)((((long long)rows + n - 1) / n + step - 1) / step * step) : 0;
    n = n > 0 ? (rows + per - 1) / per : 0;
  };
  // prefixes: two workgroups of four waves per compute unit
  p.prefix_kind = p.P == 0 ? 0 : M <= 32 ? 1 : M <= 64 ? 2 : 4;
  p.n_prefix = p.prefix_per = 0;
  long long blocks = 0;
  if (p.P > 0) {
    const long long xg = (long long)p.Np * p.Hk, cc = (M + p.prefix_kind * 32 - 1) / (p.prefix_kind * 32);
    if (p.prefix_kind == 1) cut(p.P, std::max(1ll, 768 / xg), 128, 128, p.n_prefix, p.prefix_per);
    else cut(p.P, std::max(1ll, 512 / (xg * cc)), 256, 64, p.n_prefix, p.prefix_per);
    blocks = (xg * p.n_prefix + 7) / 8 * 8 * cc;
  }
  p.prefix_blocks = blocks > 0x7fffffff ? 0x7fffffff : (int)blocks;  // (too many: the launch is refused)
  const long long groups = (long long)p.B * p.Hk;
  if (own_kind(G) > 0) cut(p.T, std::max(1ll, 2048 / groups), 256, 64, p.n_own, p.own_per);
  else cut(p.T, std::max(1ll, 768 / (groups * ((G + 31) / 32))), 128, 128, p.n_own, p.own_per);
  p.n_slices = p.n_prefix + p.n_own + (p.depth_count > 0 ? 1 : 0);
  p.score_step = ((size_t)p.T + 31) / 32 * 32;
}

static size_t state_bytes(const SharedParams& p, int d) {
  return ((size_t)p.B * p.Hq * p.n_slices * state_floats(d) * sizeof(float) + 15) / 16 * 16;
}

size_t decode_shared_workspace_bytes(const SharedParams& dims, int d, bool with_weights) {
  SharedParams p = dims;
  plan(p);
  const size_t bytes = state_bytes(p, d) + (with_weights ? (size_t)p.B * p.Hq * p.score_step * sizeof(float) : 0);
  return std::max<size_t>(bytes, 16);
}

template <int D, int PREFIX>
static void (*slices_kernel(int own))(SharedParams) {
  return own == 4 ? moda_shared_slices_kernel<D, PREFIX, 4> : own == 2 ? moda_shared_slices_kernel<D, PREFIX, 2>
         : own == 1 ? moda_shared_slices_kernel<D, PREFIX, 1> : moda_shared_slices_kernel<D, PREFIX, 0>;
}

template <int D>
static hipError_t launch_d(const SharedParams& p, hipStream_t stream) {
  const int G = p.Hq / p.Hk, own = own_kind(G), n_own = p.n_slices - p.n_prefix;
  const int heads_per = own > 0 ? own : 32;
  const long long blocks = p.prefix_blocks + (long long)p.B * p.Hk * ((G + heads_per - 1) / heads_per) * n_own;
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
                   : p.prefix_kind == 2 ? slices_kernel<D, 2>(own) : slices_kernel<D, 4>(own);
    const hipError_t e = launch_kernel(kernel, dim3((unsigned)blocks), dim3(kShWaves * 64), stream, p);
    if (e != hipSuccess) return e;
  }
  return launch_kernel(moda_shared_finish_kernel<D>, dim3((unsigned)finish_blocks), dim3(256), stream, p, by, (int)merge_blocks, chunks);
}

hipError_t launch_decode_shared(SharedParams p, int d, void* workspace, hipStream_t stream) {
  plan(p);
  p.ws = (float*)workspace;
  p.scores = (float*)((char*)workspace + state_bytes(p, d));
  return d == 128 ? launch_d<128>(p, stream) : launch_d<64>(p, stream);
}

}  // namespace moda
