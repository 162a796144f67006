// Generation over a forest of cached segments on gfx950: a paged key/value
// cache, in bf16 or in e4m3 with a power-of-two scale per row and head, and
// attention of new rows through it.
//
//   k_cache_write / k_cache_read  one 16-byte piece (8 elements) a lane; a row's
//                pieces of one head lie in D / 8 neighbouring lanes, which find
//                its largest magnitude with shuffles;
//   k_gen_attn   a workgroup of 4 waves per (work item, key head): a tile of
//                stacked rows (query rows x query heads of the key head)
//                against one split of a segment's keys;
//   k_gen_join   joins the parts of rows that have several.
//
// k_gen_attn keeps everything but the final join in registers.  Products are
// issued with the roles that leave a stacked row in a lane's column: S^T = K Q^T
// and O^T = V^T P^T, bf16 MFMA 16x16x32.  Then
//   - a row's maximum, sum, weights and outputs stay in the lanes of one column
//     (lane % 16 = row; the four lane groups g hold different keys);
//   - two 16-key score tiles are the B operand of the second product as they
//     stand, with slot (g, e) of its 32-deep contraction meaning key 4g + e
//     (e < 4) or 16 + 4g + e - 4, so the weights never leave their lane;
//   - V^T fragments need 8 such keys of one column per lane.  A lane reads the
//     8 rows' D / 16 neighbouring columns (whole rows across the 16 lanes of a
//     group) and transposes them with byte permutes: fragment j holds column
//     (lane % 16) D / 16 + j, and a lane's outputs are D / 4 neighbouring
//     columns of its row;
//   - K fragments are 16-byte reads along d; the contraction order of the first
//     product is free, so the 8-bit cache is read 16 bytes a lane too and Q is
//     read in the matching order.
// No LDS and no barrier in the loop: the keys of the next 32-key step are
// requested as soon as this step's registers are free.  The exponent reference
// of a row moves only when a score exceeds it by 2^8, as the largest weight
// that leaves sums and products far from overflow; most steps then have no
// rescale and no exchange between lanes.  Weights are rounded to bf16 for the
// second product (relative 2^-9 each, as every product of bf16 operands), their
// sum is taken before that in float32.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "gen.hpp"
#include "harts.h"
#include "la_common.hpp"
#include "plan.hpp"

namespace harts {
namespace {

typedef unsigned int u32;
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int GEN_THR = 256;
constexpr float GEN_LOG2E = 1.4426950408889634f;
constexpr float GEN_LN2 = 0.6931471805599453f;
constexpr float GEN_SLACK = 8.f;

// ---------------------------------------------------------------------------
// the cache
// ---------------------------------------------------------------------------

struct CacheView {
  char *k, *v;
  uint8_t *ke, *ve;
  const int32_t *pages, *len;
  int32_t n_pages, n_seg, pitch, H;
};

// Index of (row, head 0) as page * H * 64 + slot of a row table's entry, or -1
// if it names no existing row.
__device__ inline int64_t cache_row(const CacheView& c, int32_t seg, int32_t pos) {
  if (seg < 0 || seg >= c.n_seg) return -1;
  const int32_t n = c.len[seg];
  if (pos < 0) pos += n;
  if (pos < 0 || pos >= n || pos / GEN_PAGE >= c.pitch) return -1;
  const int32_t page = c.pages[static_cast<int64_t>(seg) * c.pitch + pos / GEN_PAGE];
  if (page < 0 || page >= c.n_pages) return -1;
  return static_cast<int64_t>(page) * c.H * GEN_PAGE + pos % GEN_PAGE;
}

// 2^(b - 127) for a biased exponent b in [1, 254]
__device__ inline float exp_scale(u32 b) { return __builtin_bit_cast(float, b << 23); }

// Eight bf16 as e4m3 codes with the scale exponent of the D / 8 lanes that hold
// the row: the smallest e >= -126 with max <= 448 2^e.  448 = 1.75 2^8, so e is
// the maximum's exponent less 8, one more where its significand exceeds 1.75.
// x 2^-e is exact in float32 and at most 448: one rounding, no saturation.
template <int LANES>
__device__ inline u32x2 quantise(const u32x4& x, u32& exponent) {
  u32 top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32 m = (x[i] >> (16 * h)) & 0x7fffu;
      if (m < 0x7f80u && m > top) top = m;
    }
#pragma unroll
  for (int s = 1; s < LANES; s *= 2) {
    const u32 other = __shfl_xor(top, s);
    top = other > top ? other : top;
  }
  const int b = static_cast<int>(top >> 7) - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0);
  exponent = b < 1 ? 1u : static_cast<u32>(b);
  const float inv = exp_scale(254u - exponent);
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32 bits = ((x[i] >> (16 * h)) & 0xffffu) << 16;
      const float y = __builtin_bit_cast(float, bits) * inv;
      f[2 * i + h] = (bits & 0x7f800000u) == 0x7f800000u ? __builtin_nanf("") : y;
    }
  u32x2 out;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
    out[i] = static_cast<u32>(__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], w, true));
  }
  return out;
}

// One lane: 8 elements of (row, head) of k, then of v.
template <int D, bool E4M3>
__global__ __launch_bounds__(GEN_THR) void k_cache_write(CacheView c, const int32_t* __restrict__ rows, int64_t n,
                                                         const u32x4* __restrict__ k_new,
                                                         const u32x4* __restrict__ v_new) {
  constexpr int P = D / 8;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * GEN_THR + threadIdx.x;
  const int64_t rh = i / P;
  const int piece = static_cast<int>(i % P);
  if (rh >= n * c.H) return;
  const int64_t r = rh / c.H;
  const int h = static_cast<int>(rh - r * c.H);
  const u32x4 a = k_new[i], b = v_new[i];
  const int64_t at = cache_row(c, rows[2 * r], rows[2 * r + 1]);
  if (at < 0) return;                                // (the same for all lanes of a row)
  const int64_t slot = at + static_cast<int64_t>(h) * GEN_PAGE;
  if constexpr (E4M3) {
    u32 ea, eb;
    const u32x2 qa = quantise<P>(a, ea), qb = quantise<P>(b, eb);
    reinterpret_cast<u32x2*>(c.k)[slot * P + piece] = qa;
    reinterpret_cast<u32x2*>(c.v)[slot * P + piece] = qb;
    if (piece == 0) {
      c.ke[slot] = static_cast<uint8_t>(ea);
      c.ve[slot] = static_cast<uint8_t>(eb);
    }
  } else {
    reinterpret_cast<u32x4*>(c.k)[slot * P + piece] = a;
    reinterpret_cast<u32x4*>(c.v)[slot * P + piece] = b;
  }
}

// Four e4m3 codes times their row's scale as bf16 (exact).
__device__ inline u32x2 dequantise(u32 w, float scale) {
  const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
  const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
  return u32x2{__builtin_bit_cast(u32, lo), __builtin_bit_cast(u32, hi)};
}

template <int D, bool E4M3>
__global__ __launch_bounds__(GEN_THR) void k_cache_read(CacheView c, const int32_t* __restrict__ rows, int64_t n,
                                                        u32x4* __restrict__ k_out, u32x4* __restrict__ v_out) {
  constexpr int P = D / 8;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * GEN_THR + threadIdx.x;
  const int64_t rh = i / P;
  const int piece = static_cast<int>(i % P);
  if (rh >= n * c.H) return;
  const int64_t r = rh / c.H;
  const int h = static_cast<int>(rh - r * c.H);
  const int64_t at = cache_row(c, rows[2 * r], rows[2 * r + 1]);
  u32x4 a{0, 0, 0, 0}, b{0, 0, 0, 0};
  if (at >= 0) {
    const int64_t slot = at + static_cast<int64_t>(h) * GEN_PAGE;
    if constexpr (E4M3) {
      const u32x2 qa = reinterpret_cast<const u32x2*>(c.k)[slot * P + piece];
      const u32x2 qb = reinterpret_cast<const u32x2*>(c.v)[slot * P + piece];
      const float sa = exp_scale(c.ke[slot]), sb = exp_scale(c.ve[slot]);
      const u32x2 a0 = dequantise(qa[0], sa), a1 = dequantise(qa[1], sa);
      const u32x2 b0 = dequantise(qb[0], sb), b1 = dequantise(qb[1], sb);
      a = u32x4{a0[0], a0[1], a1[0], a1[1]};
      b = u32x4{b0[0], b0[1], b1[0], b1[1]};
    } else {
      a = reinterpret_cast<const u32x4*>(c.k)[slot * P + piece];
      b = reinterpret_cast<const u32x4*>(c.v)[slot * P + piece];
    }
  }
  k_out[i] = a;
  v_out[i] = b;
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------

__device__ inline f32x4 mfma32(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Registers of a 32-key step as they lie in the cache.
template <int D, bool E4M3> struct KvStep;

template <int D> struct KvStep<D, false> {
  static constexpr int ROWB = 2 * D;
  static constexpr int VW = D / 32;              // dwords of a lane's columns of a row
  u32x4 k[2][D / 32];
  u32 v[8][VW];
  // a lane's part of contraction step s of the first product starts at column
  __device__ static inline int k_col(int s, int g) { return 32 * s + 8 * g; }
  __device__ inline void load_k(const char* page, const uint8_t*, int half, int lane) {
    const char* p = page + (32 * half + (lane & 15)) * ROWB + 16 * (lane >> 4);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < D / 32; ++s) k[t][s] = *reinterpret_cast<const u32x4*>(p + t * 16 * ROWB + 64 * s);
  }
  __device__ inline void load_v(const char* page, const uint8_t*, int half, int lane) {
    const char* p = page + (32 * half + 4 * (lane >> 4)) * ROWB + (lane & 15) * (ROWB / 16);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const char* r = p + (e < 4 ? e : 12 + e) * ROWB;
      if constexpr (VW == 4) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(r);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[e][i] = x[i];
      } else {
        const u32x2 x = *reinterpret_cast<const u32x2*>(r);
        v[e][0] = x[0];
        v[e][1] = x[1];
      }
    }
  }
  __device__ inline bf16x8 k_frag(int t, int s) const { return __builtin_bit_cast(bf16x8, k[t][s]); }
  // the lane's columns of its 8 keys as bf16 pairs
  __device__ inline void v_rows(u32 (&w)[8][VW]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int i = 0; i < VW; ++i) w[e][i] = v[e][i];
  }
};

template <int D> struct KvStep<D, true> {
  static constexpr int ROWB = D;
  static constexpr int VW = D / 32;
  u32x4 k[2][D / 64];
  u32 ks[2];
  u32 v[8][D / 64];
  u32 vs[2];
  // (a 16-byte read holds two steps' columns of a lane)
  __device__ static inline int k_col(int s, int g) { return 64 * (s >> 1) + 16 * g + 8 * (s & 1); }
  __device__ inline void load_k(const char* page, const uint8_t* exps, int half, int lane) {
    const int row = 32 * half + (lane & 15);
    const char* p = page + row * ROWB + 16 * (lane >> 4);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < D / 64; ++i) k[t][i] = *reinterpret_cast<const u32x4*>(p + t * 16 * ROWB + 64 * i);
      ks[t] = exps[row + 16 * t];
    }
  }
  __device__ inline void load_v(const char* page, const uint8_t* exps, int half, int lane) {
    const int row = 32 * half + 4 * (lane >> 4);
    const char* p = page + row * ROWB + (lane & 15) * (ROWB / 16);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const char* r = p + (e < 4 ? e : 12 + e) * ROWB;
      if constexpr (D == 128) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(r);
        v[e][0] = x[0];
        v[e][1] = x[1];
      } else {
        v[e][0] = *reinterpret_cast<const u32*>(r);
      }
    }
    vs[0] = *reinterpret_cast<const u32*>(exps + row);
    vs[1] = *reinterpret_cast<const u32*>(exps + row + 16);
  }
  __device__ inline bf16x8 k_frag(int t, int s) const {
    const u32x4& x = k[t][s >> 1];
    const float f = exp_scale(ks[t]);
    const u32x2 a = dequantise(x[2 * (s & 1)], f), b = dequantise(x[2 * (s & 1) + 1], f);
    return __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
  }
  __device__ inline void v_rows(u32 (&w)[8][VW]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float f = exp_scale((vs[e >> 2] >> (8 * (e & 3))) & 0xffu);
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const u32x2 a = dequantise(v[e][i], f);
        w[e][2 * i] = a[0];
        w[e][2 * i + 1] = a[1];
      }
    }
  }
};

// Column j of the lane's 8 rows of pairs as one fragment.
template <int VW>
__device__ inline bf16x8 v_frag(const u32 (&w)[8][VW], int j) {
  u32x4 f;
#pragma unroll
  for (int p = 0; p < 4; ++p)
    f[p] = __builtin_amdgcn_perm(w[2 * p + 1][j >> 1], w[2 * p][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
  return __builtin_bit_cast(bf16x8, f);
}

__device__ inline u32 pack_bf16(float a, float b) {
  const bf16x2 x{static_cast<bf16>(a), static_cast<bf16>(b)};
  return __builtin_bit_cast(u32, x);
}

struct GenArgs {
  CacheView c;
  const int32_t *items, *order, *part_off;
  int32_t Hq;
  float scale;                 // scale * log2(e)
  const bf16* q;
  bf16* o;
  float *lse, *acc, *ml;       // acc [parts][Hq][D], ml [parts][Hq][2]
};

// Floats of one wave's results in LDS: maximum, sum and accumulators of T tiles.
template <int D, int T> constexpr int join_floats() { return (2 * T + T * D / 4) * 64; }

// One work item by waves of T row tiles.  kw: the wave's turn among the KW that
// share the keys of its rows; rt: its place along the rows.
template <int D, bool E4M3, int T>
__device__ inline void gen_item(const GenArgs& A, const int32_t* __restrict__ it, int hk, int wave, int lane,
                                float* __restrict__ lds) {
  typedef KvStep<D, E4M3> Step;
  constexpr int DT = D / 16;                        // 16-column tiles
  const CacheView& c = A.c;
  const int rw = it[GI_WAVES], kws = 4 / rw;
  const int rt = wave % rw, kw = wave / rw;
  const int seg = it[GI_SEG], n_new = it[GI_NEW], group = A.Hq / c.H;
  const int g = lane >> 4, i = lane & 15;

  // rows of this lane's columns
  const int64_t cached = c.len[seg] < 0 ? 0 : c.len[seg];
  const int64_t held = min(cached, static_cast<int64_t>(c.pitch) * GEN_PAGE);
  const int32_t n = static_cast<int32_t>(min(held, static_cast<int64_t>(INT32_MAX - 64)));
  int32_t row[T], head[T], lim[T];
  bool live[T];
  bf16x8 qf[T][D / 32];
  int32_t lo = n, hi = 0;
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int local = 16 * (rt * T + t) + i;
    live[t] = local < it[GI_N];
    const int stacked = it[GI_ROW] + (live[t] ? local : 0);
    const int place = stacked / group;              // among the rows below the segment
    row[t] = A.order[it[GI_FIRST] + place];
    head[t] = hk * group + stacked % group;
    const int64_t own = cached - n_new + place + 1; // rows up to its own
    lim[t] = place < n_new ? static_cast<int32_t>(max(int64_t{0}, min(own, static_cast<int64_t>(n)))) : n;
    if (!live[t]) lim[t] = -1;
    hi = max(hi, lim[t]);
    if (live[t]) lo = min(lo, lim[t]);
    const bf16* qp = A.q + (static_cast<int64_t>(row[t]) * A.Hq + head[t]) * D;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) qf[t][s] = *reinterpret_cast<const bf16x8*>(qp + Step::k_col(s, g));
  }
#pragma unroll
  for (int s = 1; s < 16; s *= 2) {
    hi = max(hi, __shfl_xor(hi, s));
    lo = min(lo, __shfl_xor(lo, s));
  }
  hi = __builtin_amdgcn_readfirstlane(hi);
  lo = __builtin_amdgcn_readfirstlane(lo);
#pragma unroll
  for (int t = 0; t < T; ++t)
    if (!live[t]) lim[t] = INT32_MAX;               // padding rows take part unmasked and are dropped

  // this wave's steps: the item's share of the steps that some row of the
  // workgroup's tile can see would differ between waves; hi of the wave is
  // enough, as rows of a wave see no key past it
  const int32_t steps = (hi + 31) / 32;
  const int32_t per = (((n + 31) / 32) + it[GI_SPLITS] - 1) / it[GI_SPLITS];
  const int64_t from = static_cast<int64_t>(it[GI_SPLIT]) * per;
  const int32_t end = static_cast<int32_t>(min(from + per, static_cast<int64_t>(steps)));

  f32x4 acc[T][DT];
  float ref[T], sum[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    ref[t] = -INFINITY;
    sum[t] = 0.f;
#pragma unroll
    for (int j = 0; j < DT; ++j) acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const int32_t* table = c.pages + static_cast<int64_t>(seg) * c.pitch;
  const auto page_of = [&](int32_t u) {
    const int32_t p = table[u >> 1];
    return p >= 0 && p < c.n_pages ? p : -1;
  };
  const auto base_of = [&](int32_t page) {
    return (static_cast<int64_t>(page < 0 ? 0 : page) * c.H + hk) * GEN_PAGE;
  };
  Step x;
  int64_t u = from + kw;
  int32_t page = -1;
  if (u < end) {
    page = page_of(static_cast<int32_t>(u));
    const int64_t b = base_of(page);
    x.load_k(c.k + b * Step::ROWB, c.ke + b, u & 1, lane);
    x.load_v(c.v + b * Step::ROWB, c.ve + b, u & 1, lane);
  }
  for (; u < end; u += kws) {
    const int32_t key0 = static_cast<int32_t>(u) * 32;
    const bool more = u + kws < end;
    const int32_t next = more ? page_of(static_cast<int32_t>(u + kws)) : page;
    const int64_t nb = base_of(next);
    const int nhalf = more ? static_cast<int>((u + kws) & 1) : static_cast<int>(u & 1);

    f32x4 s[T][2];
#pragma unroll
    for (int t = 0; t < T; ++t) s[t][0] = s[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        const bf16x8 kf = x.k_frag(kt, d);
#pragma unroll
        for (int t = 0; t < T; ++t) s[t][kt] = mfma32(kf, qf[t][d], s[t][kt]);
      }
    x.load_k(c.k + nb * Step::ROWB, c.ke + nb, nhalf, lane);

    const bool edge = key0 + 32 > lo || page < 0;   // some key is hidden from some row
    u32x4 w[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      float y[8], top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[e] = s[t][e >> 2][e & 3] * A.scale;
        if (edge) {
          const int32_t key = key0 + 4 * g + (e < 4 ? e : 12 + e);
          if (key >= lim[t] || key >= n || page < 0) y[e] = -INFINITY;
        }
        top = fmaxf(top, y[e]);
      }
      if (__any(top > ref[t] + GEN_SLACK)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float to = fmaxf(ref[t], top);
        const float f = to == -INFINITY || to == ref[t] ? 1.f : __builtin_amdgcn_exp2f(ref[t] - to);
        ref[t] = to;
        sum[t] *= f;
#pragma unroll
        for (int j = 0; j < DT; ++j) acc[t][j] *= f;
      }
      const float r = ref[t] == -INFINITY ? 0.f : ref[t];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[e] = __builtin_amdgcn_exp2f(y[e] - r);
        sum[t] += y[e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) w[t][e] = pack_bf16(y[2 * e], y[2 * e + 1]);
    }

    u32 vw[8][Step::VW];
    x.v_rows(vw);
    bool apart = false;
    if (edge) {
      // rows that do not exist hold anything: zeros, since a weight of 0 times
      // infinity would not be 0
      bool odd = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool there = page >= 0 && key0 + 4 * g + (e < 4 ? e : 12 + e) < n;
#pragma unroll
        for (int q = 0; q < Step::VW; ++q) {
          vw[e][q] = there ? vw[e][q] : 0u;
          odd |= (vw[e][q] & 0x7f80u) == 0x7f80u || (vw[e][q] & 0x7f800000u) == 0x7f800000u;
        }
      }
      // new rows that are not finite, in a step whose keys some of the rows see
      // and others do not
      apart = lo < min(hi, key0 + 32) && __any(odd);
    }
    if (!apart) {
#pragma unroll
      for (int j = 0; j < DT; ++j) {
        const bf16x8 vf = v_frag(vw, j);
#pragma unroll
        for (int t = 0; t < T; ++t) acc[t][j] = mfma32(vf, __builtin_bit_cast(bf16x8, w[t]), acc[t][j]);
      }
    } else {
      // one column (row) at a time, with the keys that it does not see as zeros
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll 1
        for (int col = 0; col < 16; ++col) {
          const int32_t most = __shfl(lim[t], col);
#pragma unroll
          for (int q = 0; q < Step::VW; ++q) {
            u32 vz[8][1];
#pragma unroll
            for (int e = 0; e < 8; ++e) vz[e][0] = key0 + 4 * g + (e < 4 ? e : 12 + e) < most ? vw[e][q] : 0u;
#pragma unroll
            for (int j = 2 * q; j < 2 * q + 2; ++j) {
              const f32x4 y = mfma32(v_frag(vz, j & 1), __builtin_bit_cast(bf16x8, w[t]), acc[t][j]);
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[t][j][e] = i == col ? y[e] : acc[t][j][e];
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
    }
    x.load_v(c.v + nb * Step::ROWB, c.ve + nb, nhalf, lane);
    page = next;
  }

#pragma unroll
  for (int t = 0; t < T; ++t) {
    sum[t] += __shfl_xor(sum[t], 16);
    sum[t] += __shfl_xor(sum[t], 32);
  }

  // join the waves that shared the keys, half of them into the other half
  for (int step = kws / 2; step >= 1; step /= 2) {
    constexpr int F = join_floats<D, T>();
    if (kw >= step && kw < 2 * step) {
      float* p = lds + static_cast<int64_t>((kw - step) * rw + rt) * F + lane;
#pragma unroll
      for (int t = 0; t < T; ++t) {
        p[64 * (2 * t)] = ref[t];
        p[64 * (2 * t + 1)] = sum[t];
#pragma unroll
        for (int j = 0; j < DT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) p[64 * (2 * T + (t * DT + j) * 4 + e)] = acc[t][j][e];
      }
    }
    __syncthreads();
    if (kw < step) {
      const float* p = lds + static_cast<int64_t>(kw * rw + rt) * F + lane;
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const float r1 = p[64 * (2 * t)], s1 = p[64 * (2 * t + 1)];
        const float to = fmaxf(ref[t], r1);
        const float r = to == -INFINITY ? 0.f : to;
        const float f0 = __builtin_amdgcn_exp2f(ref[t] - r), f1 = __builtin_amdgcn_exp2f(r1 - r);
        ref[t] = to;
        sum[t] = sum[t] * f0 + s1 * f1;
#pragma unroll
        for (int j = 0; j < DT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[t][j][e] = acc[t][j][e] * f0 + p[64 * (2 * T + (t * DT + j) * 4 + e)] * f1;
      }
    }
    if (step > 1) __syncthreads();
  }
  if (kw != 0) return;

#pragma unroll
  for (int t = 0; t < T; ++t) {
    if (!live[t]) continue;
    const int32_t p0 = A.part_off[row[t]], parts = A.part_off[row[t] + 1] - p0;
    const int64_t rh = static_cast<int64_t>(row[t]) * A.Hq + head[t];
    if (parts == 1) {
      const float f = sum[t] == 0.f ? 0.f : 1.f / sum[t];
      u32 out[D / 8];
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < DT; j += 2)
          out[e * (DT / 2) + j / 2] = pack_bf16(acc[t][j][e] * f, acc[t][j + 1][e] * f);
      u32x4* op = reinterpret_cast<u32x4*>(A.o + rh * D + g * (D / 4));
#pragma unroll
      for (int e = 0; e < D / 32; ++e) op[e] = u32x4{out[4 * e], out[4 * e + 1], out[4 * e + 2], out[4 * e + 3]};
      if (A.lse && g == 0)
        A.lse[rh] = sum[t] == 0.f ? -INFINITY : (ref[t] + __builtin_amdgcn_logf(sum[t])) * GEN_LN2;
    } else {
      const int64_t at = (static_cast<int64_t>(p0) + it[GI_PART] + it[GI_SPLIT]) * A.Hq + head[t];
      f32x4* ap = reinterpret_cast<f32x4*>(A.acc + at * D + g * (D / 4));
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < DT; j += 4)
          ap[(e * DT + j) / 4] = f32x4{acc[t][j][e], acc[t][j + 1][e], acc[t][j + 2][e], acc[t][j + 3][e]};
      if (g == 0) {
        A.ml[2 * at] = ref[t];
        A.ml[2 * at + 1] = sum[t];
      }
    }
  }
}

template <int D, bool E4M3>
__global__ __launch_bounds__(GEN_THR, 2) void k_gen_attn(GenArgs A) {
  __shared__ float lds[2 * join_floats<D, 2>()];
  const int item = blockIdx.x / A.c.H, hk = blockIdx.x % A.c.H;
  const int32_t* it = A.items + static_cast<int64_t>(item) * GI_WORDS;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int tiles = it[GI_TILES];
  if (tiles == 1) gen_item<D, E4M3, 1>(A, it, hk, wave, lane, lds);
  else gen_item<D, E4M3, 2>(A, it, hk, wave, lane, lds);
}

// One wave per (row, query head) of several parts: maxima and sums of up to 64
// parts in the lanes, then the accumulators, D / 64 columns a lane.
template <int D>
__global__ __launch_bounds__(GEN_THR) void k_gen_join(GenArgs A, int64_t n) {
  constexpr int W = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t rh = static_cast<int64_t>(blockIdx.x) * (GEN_THR / 64) + (threadIdx.x >> 6);
  if (rh >= n) return;
  const int32_t row = static_cast<int32_t>(rh / A.Hq), head = static_cast<int32_t>(rh % A.Hq);
  const int32_t p0 = A.part_off[row], parts = A.part_off[row + 1] - p0;
  if (parts == 1) return;
  float ref = -INFINITY, sum = 0.f, acc[W];
#pragma unroll
  for (int e = 0; e < W; ++e) acc[e] = 0.f;
  for (int b = 0; b < parts; b += 64) {
    const int m = min(64, parts - b);
    float r1 = -INFINITY, s1 = 0.f;
    if (lane < m) {
      const float* ml = A.ml + 2 * ((static_cast<int64_t>(p0) + b + lane) * A.Hq + head);
      r1 = ml[0];
      s1 = ml[1];
    }
    float to = fmaxf(ref, r1);
#pragma unroll
    for (int s = 1; s < 64; s *= 2) to = fmaxf(to, __shfl_xor(to, s));
    const float r = to == -INFINITY ? 0.f : to;
    const float f0 = __builtin_amdgcn_exp2f(ref - r), f1 = __builtin_amdgcn_exp2f(r1 - r);
    float add = lane < m ? s1 * f1 : 0.f;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) add += __shfl_xor(add, s);
    sum = sum * f0 + add;
    ref = to;
#pragma unroll
    for (int e = 0; e < W; ++e) acc[e] *= f0;
    const float* ap = A.acc + ((static_cast<int64_t>(p0) + b) * A.Hq + head) * D + lane * W;
#pragma unroll 4
    for (int p = 0; p < m; ++p) {
      const float f = __shfl(f1, p);
      const float* x = ap + static_cast<int64_t>(p) * A.Hq * D;
#pragma unroll
      for (int e = 0; e < W; ++e) acc[e] += x[e] * f;
    }
  }
  const float f = sum == 0.f ? 0.f : 1.f / sum;
  bf16* op = A.o + rh * D + lane * W;
#pragma unroll
  for (int e = 0; e < W; ++e) op[e] = static_cast<bf16>(acc[e] * f);
  if (A.lse && lane == 0) A.lse[rh] = sum == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * GEN_LN2;
}

int gen_status(const char* where) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) {
    set_error(std::string(where) + ": " + hipGetErrorString(e));
    return HARTS_EHIP;
  }
  return HARTS_OK;
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int check_cache(const harts_cache* c, const char* where) {
  const auto fail = [&](int code, const char* what) {
    set_error(std::string(where) + ": " + what);
    return code;
  };
  if (!c) return fail(HARTS_EINVAL, "NULL cache");
  if (c->kind != HARTS_BF16 && c->kind != HARTS_E4M3)
    return fail(HARTS_EUNSUPPORTED, "the cache holds HARTS_BF16 or HARTS_E4M3");
  if ((c->d != 64 && c->d != 128) || c->H < 1 || c->H > 65535)
    return fail(HARTS_EUNSUPPORTED, "need d in {64, 128} and 1 <= H <= 65535");
  if (c->n_pages < 1 || c->n_seg < 1 || c->pitch < 1)
    return fail(HARTS_EINVAL, "need at least one page, segment and table column");
  if (!c->k || !c->v || !c->pages || !c->len || !aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->pages, 4) ||
      !aligned(c->len, 4))
    return fail(HARTS_EINVAL, "NULL or misaligned pointer in the cache");
  if (c->kind == HARTS_E4M3 && (!c->k_exp || !c->v_exp || !aligned(c->k_exp, 4) || !aligned(c->v_exp, 4)))
    return fail(HARTS_EINVAL, "NULL or misaligned scale exponents in the cache");
  return HARTS_OK;
}

CacheView view_of(const harts_cache* c) {
  return {static_cast<char*>(c->k), static_cast<char*>(c->v), c->k_exp, c->v_exp, c->pages, c->len,
          c->n_pages, c->n_seg, c->pitch, c->H};
}

// blocks of a launch of one lane per 8 elements, or 0 past a grid's reach
uint32_t piece_blocks(int64_t n, const harts_cache* c) {
  const int64_t b = (n * c->H * (c->d / 8) + GEN_THR - 1) / GEN_THR;
  return b > INT32_MAX ? 0 : static_cast<uint32_t>(b);
}

int check_rows(const harts_cache* c, const int32_t* rows, int64_t n, const void* k, const void* v, const char* where) {
  if (int rc = check_cache(c, where)) return rc;
  if (n < 0) { set_error(std::string(where) + ": negative row count"); return HARTS_EINVAL; }
  if (n == 0) return HARTS_OK;
  if (!rows || !k || !v || !aligned(rows, 4) || !aligned(k, 16) || !aligned(v, 16)) {
    set_error(std::string(where) + ": NULL or misaligned pointer");
    return HARTS_EINVAL;
  }
  if (n > INT32_MAX || piece_blocks(n, c) == 0) {
    set_error(std::string(where) + ": too many rows for one call");
    return HARTS_EUNSUPPORTED;
  }
  return HARTS_OK;
}

}  // namespace
}  // namespace harts

using namespace harts;

extern "C" int harts_cache_write(const harts_cache* cache, const int32_t* rows, int64_t n, const void* k_new,
                                 const void* v_new, void* stream) {
  if (int rc = check_rows(cache, rows, n, k_new, v_new, "harts_cache_write")) return rc;
  if (n == 0) return HARTS_OK;
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(piece_blocks(n, cache)), dim3(GEN_THR), 0, static_cast<hipStream_t>(stream),
                       view_of(cache), rows, n, static_cast<const u32x4*>(k_new), static_cast<const u32x4*>(v_new));
  };
  const bool q = cache->kind == HARTS_E4M3;
  if (cache->d == 128) q ? launch(k_cache_write<128, true>) : launch(k_cache_write<128, false>);
  else q ? launch(k_cache_write<64, true>) : launch(k_cache_write<64, false>);
  return gen_status("k_cache_write");
}

extern "C" int harts_cache_read(const harts_cache* cache, const int32_t* rows, int64_t n, void* k_out, void* v_out,
                                void* stream) {
  if (int rc = check_rows(cache, rows, n, k_out, v_out, "harts_cache_read")) return rc;
  if (n == 0) return HARTS_OK;
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(piece_blocks(n, cache)), dim3(GEN_THR), 0, static_cast<hipStream_t>(stream),
                       view_of(cache), rows, n, static_cast<u32x4*>(k_out), static_cast<u32x4*>(v_out));
  };
  const bool q = cache->kind == HARTS_E4M3;
  if (cache->d == 128) q ? launch(k_cache_read<128, true>) : launch(k_cache_read<128, false>);
  else q ? launch(k_cache_read<64, true>) : launch(k_cache_read<64, false>);
  return gen_status("k_cache_read");
}

extern "C" int harts_gen_attn(const harts_cache* cache, const harts_gen_sizes* sizes, const int32_t* items,
                              const int32_t* order, const int32_t* part_off, int32_t Hq, float scale, const void* q,
                              void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  const char* where = "harts_gen_attn";
  if (int rc = check_cache(cache, where)) return rc;
  if (Hq < cache->H || Hq > 65535 || Hq % cache->H != 0) {
    set_error("harts_gen_attn: query heads have to be a multiple of the cache's heads, at most 65535");
    return HARTS_EUNSUPPORTED;
  }
  if (!sizes || sizes->n_rows < 0 || sizes->n_items < 0 || sizes->n_parts < 0 || sizes->n_join < 0 ||
      sizes->n_rows * Hq > INT32_MAX || sizes->n_items * cache->H > INT32_MAX || sizes->n_parts > INT32_MAX) {
    set_error("harts_gen_attn: NULL or bad sizes");
    return HARTS_EINVAL;
  }
  if (sizes->n_rows == 0) return HARTS_OK;
  size_t need = 0;
  if (int rc = harts_gen_workspace_size(sizes, Hq, cache->d, &need)) return rc;
  if (!items || !order || !part_off || !q || !o || !aligned(items, 4) || !aligned(order, 4) || !aligned(part_off, 4) ||
      !aligned(q, 16) || !aligned(o, 16) || !aligned(lse, 4) || sizes->n_items == 0) {
    set_error("harts_gen_attn: NULL or misaligned pointer, or rows without work items");
    return HARTS_EINVAL;
  }
  if (need > 0 && (!ws || !aligned(ws, 16) || ws_bytes < need)) {
    set_error("harts_gen_attn: NULL, misaligned or small workspace; need " + std::to_string(need) + " bytes");
    return HARTS_EINVAL;
  }
  const size_t span = static_cast<size_t>(sizes->n_rows) * Hq * cache->d * sizeof(bf16);
  const uintptr_t q0 = reinterpret_cast<uintptr_t>(q), o0 = reinterpret_cast<uintptr_t>(o);
  if ((q0 < o0 ? o0 - q0 : q0 - o0) < span) {
    set_error("harts_gen_attn: o overlaps q");
    return HARTS_EINVAL;
  }
  GenArgs A;
  A.c = view_of(cache);
  A.items = items;
  A.order = order;
  A.part_off = part_off;
  A.Hq = Hq;
  A.scale = scale * GEN_LOG2E;
  A.q = static_cast<const bf16*>(q);
  A.o = static_cast<bf16*>(o);
  A.lse = lse;
  A.acc = static_cast<float*>(ws);
  A.ml = need ? A.acc + sizes->n_parts * Hq * cache->d : nullptr;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(sizes->n_items * cache->H)), dim3(GEN_THR), 0, s, A);
  };
  const bool e4m3 = cache->kind == HARTS_E4M3;
  if (cache->d == 128) e4m3 ? launch(k_gen_attn<128, true>) : launch(k_gen_attn<128, false>);
  else e4m3 ? launch(k_gen_attn<64, true>) : launch(k_gen_attn<64, false>);
  if (int rc = gen_status("k_gen_attn")) return rc;
  if (sizes->n_join > 0) {
    const int64_t n = sizes->n_rows * Hq;
    const uint32_t blocks = static_cast<uint32_t>((n + GEN_THR / 64 - 1) / (GEN_THR / 64));
    if (cache->d == 128) hipLaunchKernelGGL(k_gen_join<128>, dim3(blocks), dim3(GEN_THR), 0, s, A, n);
    else hipLaunchKernelGGL(k_gen_join<64>, dim3(blocks), dim3(GEN_THR), 0, s, A, n);
    return gen_status("k_gen_join");
  }
  return HARTS_OK;
}
