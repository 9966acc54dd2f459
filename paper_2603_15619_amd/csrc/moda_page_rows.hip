// Rows into the pages of a paged sequence cache, and back.
//
// Append: the last n_b rows of sequence b, positions lengths[b] - n_b on, come from K, V [B, Hk, T, d]; where the pages hold 8 bits they are
// quantised (moda_pages.h).  Per page and head the least and the largest value of every key channel, as stored, are kept on the
// way (`bounds`): over the rows of this call, and what was there unless row 0 of the page is among them.  bf16 orders as its bits do
// once those of negative numbers are turned round, so minima and maxima are taken on pairs of 16-bit integers; a NaN among the
// rows makes both bounds of its channel NaN, so that no choice by bounds overlooks it.
// Bound by HBM: every row is read once and written once.  A wave takes the rows of one (sequence, page, head), four loads of K and of V
// in flight; pages of 32 rows are shared by two waves, longer ones by four, which put their bounds together in LDS.
// Read: the same the other way, a wave per 32 (d = 128) or 64 rows.
#include "moda_pages.h"

namespace moda {

typedef short s16x2 __attribute__((ext_vector_type(2)));

// bf16 pairs as 16-bit integers of the same order, and back (the same steps).
__device__ __forceinline__ s16x2 ordered(uint32_t u) {
  const s16x2 x = __builtin_bit_cast(s16x2, u);
  return x ^ ((x >> 15) & (s16x2){0x7fff, 0x7fff});
}
__device__ __forceinline__ uint32_t unordered(s16x2 x) {
  return __builtin_bit_cast(uint32_t, x ^ ((x >> 15) & (s16x2){0x7fff, 0x7fff}));
}
constexpr short kInfOrdered = 0x7f80;  // above it: NaN; below -kInfOrdered - 1: NaN with the sign bit

// Eight channels of a row: codes, and the scale byte of their block of 32, which the four lanes of a quad hold.
__device__ __forceinline__ u32x2 quantise(const u32x4& x, unsigned& byte) {
  float v[8], nan[8], a = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_lo(x[i]);
    v[2 * i + 1] = bf16_hi(x[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    nan[i] = v[i] - v[i];              // 0, or NaN where x is not finite
    a = fmaxf(a, fabsf(v[i]) + nan[i]);  // (the maximum leaves NaN out)
  }
  a = fmaxf(a, dpp_mov<0xB1>(a));
  a = fmaxf(a, dpp_mov<0x4E>(a));
  // 448 = 1.75 * 2^8: the exponent of a less 8, and one more where its mantissa is above 1.75
  byte = max((int)((__builtin_bit_cast(unsigned, a) + 0x1fffffu) >> 23) - 8, kLeastByte);
  const float inv = scale_of(254 - byte), most = byte == kMostByte ? 240.f : 448.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __builtin_amdgcn_fmed3f(v[i] * inv, -most, most) - nan[i];  // (-0 less 0 stays -0)
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
    r[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], w, true);
  }
  return r;
}

// What the lanes at the same place of a wave's groups of LPR (8 or 16) hold, put together.
template <int LPR, class F>
__device__ __forceinline__ s16x2 over_groups(s16x2 v, F&& f) {
  int x = __builtin_bit_cast(int, v);
  auto put = [&](int a, int b) { return __builtin_bit_cast(int, f(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b))); };
  if (LPR == 8) x = put(x, __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false));  // row_ror:8
  auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = put((int)r[0], (int)r[1]);
  auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return __builtin_bit_cast(s16x2, put((int)h[0], (int)h[1]));
}

// Waves that share a page.
__host__ __device__ constexpr int waves_per_page(int shift) { return shift == 4 ? 1 : shift == 5 ? 2 : 4; }

template <int D, bool MX>
__global__ __launch_bounds__(256) void moda_page_append_kernel(PageRowsParams p, int most_pages) {
  constexpr int LPR = D / 8, RPS = 64 / LPR, RB = D * 2, kU = 4;
  __shared__ s16x2 red[4][2][D / 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane % LPR, rg = lane / LPR;
  const int wpp = waves_per_page(p.shift), part = wave % wpp, R = 1 << p.shift;
  // (sequence, head, page), pages fastest
  const long long unit = (long long)blockIdx.x * (4 / wpp) + wave / wpp, bg = unit / most_pages;
  const int j = (int)(unit - bg * most_pages);
  const int b = (int)(bg / p.Hk), g = (int)(bg - (long long)b * p.Hk);
  int id = -1, s0 = 0, s1 = 0;
  long long src = 0;  // row of K and V that goes to row 0 of the page
  if (b < p.B) {
    const int len = p.lengths ? max(p.lengths[b], 0) : p.T;
    const int n = min(min(p.counts ? max(p.counts[b], 0) : p.T, p.T), len);
    const int first = len - n, page = (first >> p.shift) + j;
    if (n > 0 && page <= (len - 1) >> p.shift) {
      s0 = max(first - page * R, 0);
      s1 = min(len - page * R, R);
      if (page < p.max_pages) id = page_at(p.table + (size_t)b * p.max_pages, page, p.n_pages);
    }
    src = bg * p.T + (long long)page * R - first;
  }
  s16x2 lo[4], hi[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[i] = (s16x2){0x7fff, 0x7fff};
    hi[i] = (s16x2){-0x8000, -0x8000};
  }
  const size_t row0 = ((size_t)(id < 0 ? 0 : id) * p.Hk + g) << p.shift;
  if (id >= 0) {  // (uniform over a wave)
    for (int at = s0 + part * kU * RPS; at < s1; at += wpp * kU * RPS) {
      u32x4 k[kU], v[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const size_t from = (size_t)(src + min(at + u * RPS + rg, s1 - 1)) * RB + l16 * 16;
        // What is written in 8 bits is what attention reads from then on: the new rows pass the caches by, the pages stay in them (batch of prompts,
        // written and read back, 69.2 -> 63.8 us).  Rows in bf16 are read again by the prompt's own attention: there the pages pass by (24.4 -> 19.6).
        k[u] = MX ? __builtin_nontemporal_load((const u32x4*)(p.K + from)) : *(const u32x4*)(p.K + from);
        v[u] = MX ? __builtin_nontemporal_load((const u32x4*)(p.V + from)) : *(const u32x4*)(p.V + from);
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int s = at + u * RPS + rg;
        const size_t to = row0 + s;
        uint32_t stored[4];
        if (MX) {
          unsigned kb, vb;
          const u32x2 kc = quantise(k[u], kb), vc = quantise(v[u], vb);
          const float sc = scale_of(kb);
          stored[0] = codes_bf16<false>(kc[0], sc);
          stored[1] = codes_bf16<true>(kc[0], sc);
          stored[2] = codes_bf16<false>(kc[1], sc);
          stored[3] = codes_bf16<true>(kc[1], sc);
          if (s < s1) {
            *(u32x2*)(p.Kp + to * D + l16 * 8) = kc;
            *(u32x2*)(p.Vp + to * D + l16 * 8) = vc;
            if (l16 % 4 == 0) {
              p.Ks[to * (D / kBlock) + l16 / 4] = (unsigned char)kb;
              p.Vs[to * (D / kBlock) + l16 / 4] = (unsigned char)vb;
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) stored[i] = k[u][i];
          if (s < s1) {
            __builtin_nontemporal_store(k[u], (u32x4*)(p.Kp + to * RB + l16 * 16));
            __builtin_nontemporal_store(v[u], (u32x4*)(p.Vp + to * RB + l16 * 16));
          }
        }
        // (rows past the end repeat the last one)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          lo[i] = __builtin_elementwise_min(lo[i], ordered(stored[i]));
          hi[i] = __builtin_elementwise_max(hi[i], ordered(stored[i]));
        }
      }
    }
  }
  if (!p.bounds) return;  // (uniform)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    auto less = [](s16x2 a, s16x2 b) { return __builtin_elementwise_min(a, b); };
    auto more = [](s16x2 a, s16x2 b) { return __builtin_elementwise_max(a, b); };
    lo[i] = over_groups<LPR>(lo[i], less);
    hi[i] = over_groups<LPR>(hi[i], more);
  }
  if (wpp > 1) {  // (uniform)
    if (lane < LPR)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        red[wave][0][lane * 4 + i] = lo[i];
        red[wave][1][lane * 4 + i] = hi[i];
      }
    __syncthreads();
    for (int w = 1; w < wpp; ++w)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int other = wave / wpp * wpp + (part + w) % wpp;
        lo[i] = __builtin_elementwise_min(lo[i], red[other][0][l16 * 4 + i]);
        hi[i] = __builtin_elementwise_max(hi[i], red[other][1][l16 * 4 + i]);
      }
  }
  if (id < 0 || part > 0 || lane >= LPR) return;
  char* at = p.bounds + ((size_t)id * p.Hk + g) * 2 * RB + l16 * 16;
  u32x4 out[2];
  if (s0 > 0) {
    out[0] = *(const u32x4*)at;
    out[1] = *(const u32x4*)(at + RB);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (s0 > 0) {
      lo[i] = __builtin_elementwise_min(lo[i], ordered(out[0][i]));
      hi[i] = __builtin_elementwise_max(hi[i], ordered(out[1][i]));
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (hi[i][k] > kInfOrdered || lo[i][k] < -kInfOrdered - 1) {  // a NaN
        hi[i][k] = 0x7fff;
        lo[i][k] = -0x8000;
      }
    out[0][i] = unordered(lo[i]);
    out[1][i] = unordered(hi[i]);
  }
  *(u32x4*)at = out[0];
  *(u32x4*)(at + RB) = out[1];
}

template <int D, bool MX>
__global__ __launch_bounds__(256) void moda_page_read_kernel(PageRowsParams p, int chunks) {
  constexpr int LPR = D / 8, RPS = 64 / LPR, RB = D * 2, kU = 8, kRows = kU * RPS;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane % LPR, rg = lane / LPR;
  const long long unit = (long long)blockIdx.x * 4 + wave, bg = unit / chunks;
  const int b = (int)(bg / p.Hk), g = (int)(bg - (long long)b * p.Hk);
  if (b >= p.B) return;
  const long long most = (long long)p.max_pages << p.shift;
  const long long len = p.lengths ? min((long long)max(p.lengths[b], 0), most) : most;
  // rows [pos, end) of the sequence, from a whole load on, so that the rows of a load lie in one page
  const long long pos = (p.first / RPS * RPS) + (unit - bg * chunks) * kRows, end = min(len, (long long)p.first + p.T);
  if (pos >= end) return;
  const int* table = p.table + (size_t)b * p.max_pages;
  u32x4 k[kU], v[kU];
  int id[kU];
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const long long at = pos + u * RPS;
    id[u] = at < end ? page_at(table, __builtin_amdgcn_readfirstlane((int)(at >> p.shift)), p.n_pages) : -1;
  }
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const size_t row = (((size_t)max(id[u], 0) * p.Hk + g) << p.shift) + ((pos + u * RPS) & ((1 << p.shift) - 1)) + rg;
    if (MX) {
      const u32x2 kc = *(const u32x2*)(p.Kp + row * D + l16 * 8), vc = *(const u32x2*)(p.Vp + row * D + l16 * 8);
      const float ks = scale_of(p.Ks[row * (D / kBlock) + l16 / 4]), vs = scale_of(p.Vs[row * (D / kBlock) + l16 / 4]);
      k[u] = (u32x4){codes_bf16<false>(kc[0], ks), codes_bf16<true>(kc[0], ks), codes_bf16<false>(kc[1], ks), codes_bf16<true>(kc[1], ks)};
      v[u] = (u32x4){codes_bf16<false>(vc[0], vs), codes_bf16<true>(vc[0], vs), codes_bf16<false>(vc[1], vs), codes_bf16<true>(vc[1], vs)};
    } else {
      k[u] = __builtin_nontemporal_load((const u32x4*)(p.Kp + row * RB + l16 * 16));
      v[u] = __builtin_nontemporal_load((const u32x4*)(p.Vp + row * RB + l16 * 16));
    }
  }
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const long long at = pos + u * RPS + rg;
    if (id[u] >= 0 && at >= p.first && at < end) {
      const size_t to = (size_t)(bg * p.T + at - p.first) * RB + l16 * 16;
      // (past the caches, as the loads: 4 x 16384 rows 89.0 -> 83.2 us)
      __builtin_nontemporal_store(k[u], (u32x4*)(p.K_out + to));
      __builtin_nontemporal_store(v[u], (u32x4*)(p.V_out + to));
    }
  }
}

hipError_t launch_page_append(const PageRowsParams& p, int d, bool mx, hipStream_t stream) {
  const int R = 1 << p.shift, per = 4 / waves_per_page(p.shift);
  const long long most_pages = ((long long)p.T + R - 2) / R + 1;  // that T rows can touch
  if (most_pages > 0x7fffffff) return kGridTooLarge;
  const long long blocks = ((long long)p.B * p.Hk * most_pages + per - 1) / per;
  if (!grid_ok(blocks, 256)) return kGridTooLarge;
  auto* kernel = d == 128 ? (mx ? moda_page_append_kernel<128, true> : moda_page_append_kernel<128, false>)
                          : (mx ? moda_page_append_kernel<64, true> : moda_page_append_kernel<64, false>);
  return launch_kernel(kernel, dim3((unsigned)blocks), dim3(256), stream, p, (int)most_pages);
}

hipError_t launch_page_read(const PageRowsParams& p, int d, bool mx, hipStream_t stream) {
  const int per_load = 512 / d, rows = 8 * per_load;
  const long long from = p.first / per_load * per_load, chunks = ((long long)p.first + p.T - from + rows - 1) / rows;
  if (chunks > 0x7fffffff) return kGridTooLarge;
  const long long blocks = ((long long)p.B * p.Hk * chunks + 3) / 4;
  if (!grid_ok(blocks, 256)) return kGridTooLarge;
  auto* kernel = d == 128 ? (mx ? moda_page_read_kernel<128, true> : moda_page_read_kernel<128, false>)
                          : (mx ? moda_page_read_kernel<64, true> : moda_page_read_kernel<64, false>);
  return launch_kernel(kernel, dim3((unsigned)blocks), dim3(256), stream, p, (int)chunks);
}

}  // namespace moda
