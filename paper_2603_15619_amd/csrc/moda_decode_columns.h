// Softmax states of up to 32 queries as the columns of matrix products, for the decoding kernels: S^T = K Q^T, O^T += V^T P^T, rows of K
// and V from LDS.
#pragma once
#include <type_traits>

#include "moda_decode_fold.h"
#include "moda_tile.h"

namespace moda {

constexpr int kShWaves = 4;  // waves of a workgroup

// Rows of K and V: n of one run, then n2 of another (a slice of an own cache, then the slots).
struct Rows {
  const char *K, *V;
  int n;
  const char *K2, *V2;
  int n2;
};

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
  // NB blocks of 32 rows: K rows from LDS address `k`, V rows from `v` (layout of Tile<D>); `left` = rows that count (HALVES, one block: of
  // its first 16 rows, `upper` those of the others).
  // `scores` (a block of 32 rows only), if not null: column q's logits, before the scale, go to scores[q * step + row], q < n.
  template <int NB, bool HALVES = false>
  __device__ __forceinline__ void fold(unsigned k, unsigned v, const FragAddr<D>& fa, int lane, int left, float c2, float* scores = nullptr,
                                       size_t step = 0, int n = 0, int upper = 0) {
    const int hi = lane >> 5;
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
    if (NB == 1 && scores) {  // (uniform)
      // through the K tile, which has been read: 8 pieces of four rows per column, of which eight lanes store a whole cache line
      // (16 x 3100 rows, 64 heads on 8, d = 64: whole call 33.1 us, 33.7 with 16-byte stores from where the logits are)
      const int l32 = lane & 31;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (l32 < n)
          *(f32x4 __attribute__((address_space(3)))*)(size_t)(k + l32 * 128 + (((i * 2 + hi) ^ (l32 & 7)) << 4)) =
              (f32x4){s[0][4 * i], s[0][4 * i + 1], s[0][4 * i + 2], s[0][4 * i + 3]};
      for (int q = lane >> 3; q < n; q += 8) {
        const int row = (lane & 7) * 4;
        const f32x4 x = *(const f32x4 __attribute__((address_space(3)))*)(size_t)(k + q * 128 + (((lane & 7) ^ (q & 7)) << 4));
        float* to = scores + q * step + row;
        if (row + 4 <= left) {
          *(f32x4*)to = x;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (row + j < left) to[j] = x[j];
        }
      }
    }
    if (HALVES) {
      if (min(left, upper) < 16) {  // (uniform)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (((i >> 2) & 1) * 8 + hi * 4 + (i & 3) >= (i < 8 ? left : upper)) s[0][i] = -INFINITY;
      }
    } else if (left < NB * 32) {  // (uniform)
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
        // weights as bf16, the type of the matrix pipe's operands: off by 2^-8 of themselves at most, and not all one way; the normaliser is
        // summed before.  (Outputs of N(0,1) data are off by 0.0023 of their size for it, 0.0017 with fp32 weights, which is O's own
        // rounding.  A second product for what the rounding leaves would double the matrix work on values.)
        const bf16x8 pb = pack8(pv);
#pragma unroll
        for (int cb = 0; cb < Tl::kDBlocks; ++cb)
          o[cb] = mfma_bf16(FragAddr<D>::tr_frag((unsigned)xor_here((int)vt, cb << 6), (unsigned)xor_here((int)vt8, cb << 6),
                                                 b * 2 + hf, 0),
                            pb, o[cb]);
      }
  }
};

// The states of a workgroup's waves, those with the same columns (wave % CW) folded, of the first n of CW * 32 columns: to adjacent states in memory, or put(column,
// piece of four channels, their sums, (reference, normaliser)).  LDS: a wave's O^T as 16-byte pieces of four channels, piece c of column q at 32 c + (q ^ c % 32) of
// the wave's part, so that both the writes (32 columns of a piece) and the reads (the pieces of a column, which make
// whole rows in memory) touch every bank alike.
struct ToMemory {};
template <int D, int CW, class Put = ToMemory>
__device__ __forceinline__ void fold_waves(const Columns<D>& c, unsigned char* smem, float (*stat)[32][2], float c2, int n, float* o_out,
                                           float* ml_out, Put&& put = {}) {
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
    if (col >= n) continue;
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
    if constexpr (std::is_same_v<Put, ToMemory>) {
      *(f32x4*)(o_out + col * D + piece * 4) = o;
      if (piece == 0) *(f32x2*)(ml_out + col * 2) = (f32x2){m, l};
    } else {
      put(col, piece, o, (f32x2){m, l});
    }
  }
}

// Every wave by itself: the rows x, 32 at a time through its two LDS tiles at `lds`; the next block(s) are in flight in
// registers.  Rows past the end of a run read as zeros (bounds-checked buffers) and fetch nothing.
template <int D, int kPF>
__device__ __forceinline__ void read_by_wave(Columns<D>& c, const Rows& x, unsigned lds, float c2, float* scores = nullptr, size_t step = 0,
                                             int nh = 0) {
  using Tl = Tile<D>;
  constexpr int RB = D * 2, kInst = 32 * RB / 1024, kHalf = 32 * RB;
  const int lane = threadIdx.x & 63;
  FragAddr<D> fa;
  fa.init(lane);
  const int n1 = (x.n + 31) / 32, n_blocks = n1 + (x.n2 + 31) / 32;
  const int jr = lane / Tl::kChunks, pc = lane % Tl::kChunks;
  const int g_off = jr * RB + ((pc ^ Tl::swz(jr)) << 4);
  auto piece_xor = [](int q) { return (D == 128 ? (q & 3) : ((q & 1) << 1)) << 4; };
  struct Block {
    u32x4 k[kInst], v[kInst];
  };
  auto issue = [&](int blk, Block& r) {
    const bool first = blk < n1;  // (uniform)
    const int size = (first ? x.n : x.n2) * RB, soff = (first ? blk : blk - n1) * kHalf;
    const __amdgpu_buffer_rsrc_t k_buf = __builtin_amdgcn_make_buffer_rsrc((void*)(first ? x.K : x.K2), 0, size, 0x00020000);
    const __amdgpu_buffer_rsrc_t v_buf = __builtin_amdgcn_make_buffer_rsrc((void*)(first ? x.V : x.V2), 0, size, 0x00020000);
#pragma unroll
    for (int q = 0; q < kInst; ++q)
      r.k[q] = __builtin_amdgcn_raw_buffer_load_b128(k_buf, xor_here(g_off, piece_xor(q)), soff + q * 1024, 2);
#pragma unroll
    for (int q = 0; q < kInst; ++q)
      r.v[q] = __builtin_amdgcn_raw_buffer_load_b128(v_buf, xor_here(g_off, piece_xor(q)), soff + q * 1024, 2);
  };
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
      if (blk < n_blocks)
        c.template fold<1>(lds, lds + kHalf, fa, lane, blk < n1 ? x.n - blk * 32 : x.n2 - (blk - n1) * 32, c2,
                           scores && blk < n1 ? scores + blk * 32 : nullptr, step, nh);
    }
  }
}

}  // namespace moda
