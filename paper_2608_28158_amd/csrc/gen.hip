// Generation over a forest of cached segments on gfx950: a paged key/value
// cache, in bf16 or in e4m3 with a power-of-two scale per row and head, and
// attention of new rows through it.
//
//   k_cache_write / k_cache_read  one 16-byte piece (8 elements) a lane; a row's
//                pieces of one head lie in D / 8 neighbouring lanes, which find
//                its largest magnitude with shuffles;
//   k_gen_attn   a workgroup of 4 waves per (work item, key head): a tile of
//                stacked rows (query rows x query heads of the key head)
//                against one split of a segment's keys, in one of two ways;
//   k_gen_join   joins the parts of rows that have several.
//
// Products are issued with the roles that leave a stacked row in a lane's
// column: S^T = K Q^T and O^T = V^T P^T, bf16 MFMA 16x16x32.  A row's maximum,
// sum, weights and outputs then stay in the lanes of one column (lane % 16 =
// row; the four lane groups g hold different keys), and two 16-key score tiles
// are the B operand of the second product as they stand, with slot (g, e) of
// its 32-deep contraction meaning key 4g + e (e < 4) or 16 + 4g + e - 4.
//
// Few rows (gen_few): the item is bound by reading the keys and values, so
// nothing stands between memory and the products.  A wave has 16 rows and every
// second or fourth step of 32 or 64 keys, straight from the cache into registers, with no
// LDS and no barrier in the loop; the next step is requested as soon as this
// one's registers are free, and the waves join through LDS at the end.
//   - V^T fragments need 8 keys of one column per lane.  A lane reads 8 rows'
//     D / 16 neighbouring columns (whole rows across the 16 lanes of a group)
//     and transposes them with byte permutes: fragment j holds column
//     (lane % 16) D / 16 + j, and a lane's outputs are D / 4 neighbouring
//     columns of its row;
//   - K fragments are 16-byte reads along d; the contraction order of the first
//     product is free, so the 8-bit cache is read 16 bytes a lane too and Q is
//     read in the matching order.
// Many rows (gen_many): a wave has 32 rows, the four waves share each step's
// keys through LDS, double-buffered with one barrier a step: bf16 rows are
// loaded straight into it, 8-bit ones on their way through registers, where
// they become bf16 once for all waves.
//
// The exponent reference of a row moves only when a score exceeds it by 2^8, as
// the largest weight that leaves sums and products far from overflow; most
// steps then have no rescale and no exchange between lanes.  Weights are
// rounded to bf16 for the second product (half a step, 2^-8 of each, as any
// bf16 operand); their sum is taken before that in float32.  o is off by 0.0023
// of its norm so, by 0.0017 with float32 weights (its own rounding alone), which
// would take a second product for what bf16 leaves of them.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>
#include <type_traits>

#include "fast_div.hpp"
#include "gen.hpp"
#include "harts_rollout.h"
#include "la_common.hpp"
#include "lds_load.hpp"
#include "plan.hpp"
#include "regions.hpp"

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
  FastDiv by_heads;
};

// Index of (row, head 0) as page * H * 64 + slot of a row table's entry, or -1
// if it names no existing row.
__device__ inline int64_t cache_row(const CacheView& c, int32_t seg, int32_t entry) {
  if (seg < 0 || seg >= c.n_seg) return -1;
  const int32_t n = c.len[seg];
  const int64_t pos = entry < 0 ? static_cast<int64_t>(n) + entry : entry;
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
// x 2^-e is exact in float32 (or so small that its code is 0) and at most 448: one
// rounding.  Only at the largest scale, 2^120, does a code stand for more than
// bf16 holds: 256 and up, the nearest to 248 and more.  Those take 240.
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
  if (__builtin_expect(__any(exponent == 247u), 0)) {
    const float most = exponent == 247u ? 240.f : 448.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = f[e] > most ? most : f[e] < -most ? -most : f[e];
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
template <int D, bool E4M3, bool NT>
__global__ __launch_bounds__(GEN_THR) void k_cache_write(CacheView c, const int32_t* __restrict__ rows, int64_t n,
                                                         const u32x4* __restrict__ k_new,
                                                         const u32x4* __restrict__ v_new) {
  constexpr int P = D / 8;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * GEN_THR + threadIdx.x;
  const int64_t rh = i / P;
  const int piece = static_cast<int>(i % P);
  if (rh >= n * c.H) return;
  const int64_t r = c.by_heads.div(static_cast<u32>(rh));   // (n H < 2^31)
  const int h = static_cast<int>(rh - r * c.H);
  u32x4 a, b;
  if constexpr (!E4M3 && NT) {
    a = __builtin_nontemporal_load(k_new + i);
    b = __builtin_nontemporal_load(v_new + i);
  } else {
    a = k_new[i];
    b = v_new[i];
  }
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

template <int D, bool E4M3, bool NT>
__global__ __launch_bounds__(GEN_THR) void k_cache_read(CacheView c, const int32_t* __restrict__ rows, int64_t n,
                                                        u32x4* __restrict__ k_out, u32x4* __restrict__ v_out) {
  constexpr int P = D / 8;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * GEN_THR + threadIdx.x;
  const int64_t rh = i / P;
  const int piece = static_cast<int>(i % P);
  if (rh >= n * c.H) return;
  const int64_t r = c.by_heads.div(static_cast<u32>(rh));   // (n H < 2^31)
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
  if constexpr (NT) {
    __builtin_nontemporal_store(a, k_out + i);
    __builtin_nontemporal_store(b, v_out + i);
  } else {
    k_out[i] = a;
    v_out[i] = b;
  }
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
  // columns 2q, 2q + 1 of the lane's, of its 8 keys, as bf16 pairs
  __device__ inline void v_pairs(u32 (&w)[8], int q) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = v[e][q];
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
  __device__ inline void v_pairs(u32 (&w)[8], int q) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float f = exp_scale((vs[e >> 2] >> (8 * (e & 3))) & 0xffu);
      const bf16x2 x = (q & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[e][q >> 1], f, true)
                               : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[e][q >> 1], f, false);
      w[e] = __builtin_bit_cast(u32, x);
    }
  }
};

// The first or second column of the lane's 8 pairs as one fragment.
__device__ inline bf16x8 v_frag(const u32 (&w)[8], int second) {
  u32x4 f;
#pragma unroll
  for (int p = 0; p < 4; ++p)
    f[p] = __builtin_amdgcn_perm(w[2 * p + 1], w[2 * p], second ? 0x07060302u : 0x05040100u);
  return __builtin_bit_cast(bf16x8, f);
}

__device__ inline u32 pack_bf16(float a, float b) {
  const bf16x2 x{static_cast<bf16>(a), static_cast<bf16>(b)};
  return __builtin_bit_cast(u32, x);
}

// natural logarithm of sum * 2^ref
__device__ inline float log_sum(float ref, float sum) {
  return sum == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * GEN_LN2;
}

// Tables that the whole wave reads at one address, through the scalar cache: the
// read then waits for none of the requests for keys that are out.
typedef const __attribute__((address_space(4))) int32_t* Scalars;
__device__ inline Scalars scalars(const int32_t* p) { return (Scalars)p; }

struct GenArgs {
  CacheView c;
  const int32_t *items, *order, *part_off;
  int32_t Hq;
  FastDiv by_group, by_Hq;     // query heads of a key head; all
  float scale;                 // |scale| * log2(e)
  u32 sign;                    // 0x80008000 where the scale is negative: q's signs change instead, so
                               // that the largest product is the largest score
  const bf16* q;
  bf16* o;
  float *lse, *acc, *ml;       // acc [parts][Hq][D], ml [parts][Hq][2]
};

__device__ inline bf16x8 q_frag(const GenArgs& A, const bf16* p) {
  return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(p) ^ A.sign);
}

// Place below its segment of a stacked row.
__device__ inline int place_of(const GenArgs& A, int stacked) {
  return static_cast<int>(A.by_group.div(static_cast<u32>(stacked)));
}

// What an item's rows see: rows of the segment that exist (n), all that were
// written or are to come (cached), its own new rows.
struct Reach {
  int64_t cached;
  int32_t n, n_new;
  __device__ inline Reach(const CacheView& c, int32_t seg, int32_t n_new_) : n_new(n_new_) {
    cached = max(scalars(c.len)[seg], 0);
    n = static_cast<int32_t>(min(min(cached, static_cast<int64_t>(c.pitch) * GEN_PAGE),
                                 static_cast<int64_t>(INT32_MAX - GEN_PAGE)));
  }
  // keys that the row at a place below the segment sees
  __device__ inline int32_t of(int32_t place) const {
    const int64_t own = cached - n_new + place + 1;
    return place < n_new ? static_cast<int32_t>(max(int64_t{0}, min(own, static_cast<int64_t>(n)))) : n;
  }
};

// The item's steps [from, to) of T keys, of those up to key `hi`.
template <int T>
__device__ inline void split_steps(Scalars it, int32_t hi, int32_t& from, int32_t& to) {
  const int32_t steps = (hi + T - 1) / T, n = it[GI_SPLITS];
  const FastDiv by(n, static_cast<u32>(it[GI_MUL]), static_cast<u32>(it[GI_SHIFT]));
  const int32_t per = static_cast<int32_t>(by.div(static_cast<u32>(steps + n - 1)));
  from = static_cast<int32_t>(min(static_cast<int64_t>(it[GI_SPLIT]) * per, static_cast<int64_t>(steps)));
  to = min(from + per, steps);
}

// Key of element e of a fragment of 32 keys, for lane group g.
__device__ inline int frag_key(int g, int e) { return 4 * g + (e < 4 ? e : 12 + e); }

// A pair of bf16 without its values that are not finite (exponent all ones);
// `odd` gets a bit if it had one.
__device__ inline u32 finite_pair(u32 w, u32& odd) {
  const u32 t = ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  odd |= t;
  return w & ~((t - (t >> 15)) | t);
}

__device__ inline float over_groups_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float over_groups_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// A row's running reference and sum, with the accumulators of DT tiles.
template <int DT>
struct RowState {
  float ref, sum;
  f32x4 acc[DT];
  __device__ inline void clear() {
    ref = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < DT; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // the reference rises to the rows' maxima
  __device__ inline void raise(float top) {
    const float to = fmaxf(ref, over_groups_max(top));
    const float f = to == ref ? 1.f : __builtin_amdgcn_exp2f(ref - to);
    ref = to;
    sum *= f;
#pragma unroll
    for (int j = 0; j < DT; ++j) acc[j] *= f;
  }
  __device__ inline float zero_point() const { return ref == -INFINITY ? 0.f : ref; }
  // what the accumulators are to be multiplied by; those of a row without weight
  // are set to zeros (they are 0 times an infinity where its keys hold one), out
  // of the way: in line, the selects took a short call 0.17 of 8.3 us
  __device__ inline float inverse() {
    if (__builtin_expect(__any(sum == 0.f), 0)) {
      if (sum == 0.f) clear();
    }
    return sum == 0.f ? 0.f : 1.f / sum;
  }
};

// Values that are not finite, in steps whose keys some rows of a wave see and
// others do not (a weight of 0 times infinity would not be 0): the products of
// such steps leave them out, and afterwards they are added, as they are, to the
// columns [c0, c0 + cols) of the output row (o, or a part's accumulators) that
// the lane has written, if the row sees them.
template <int D, bool E4M3, typename T>
__device__ inline void add_odd(const CacheView& c, Scalars table, int hk, int32_t key0, int32_t keys, int32_t n,
                               int32_t lim, T* out, int c0, int cols) {
  const int32_t page = table[key0 / GEN_PAGE];
  if (page < 0 || page >= c.n_pages) return;
  const int64_t row0 = (static_cast<int64_t>(page) * c.H + hk) * GEN_PAGE + key0 % GEN_PAGE;
#pragma unroll 1
  for (int32_t k = 0; k < keys && key0 + k < min(n, lim); ++k)
#pragma unroll 1
    for (int j = c0; j < c0 + cols; ++j) {
      const int64_t at = (row0 + k) * D + j;
      float x;
      if constexpr (E4M3)      // (codes that a caller wrote itself may stand for more than bf16 holds)
        x = __builtin_bit_cast(float, dequantise(reinterpret_cast<const uint8_t*>(c.v)[at], exp_scale(c.ve[row0 + k]))[0] << 16);
      else x = static_cast<float>(reinterpret_cast<const bf16*>(c.v)[at]);
      if (!(fabsf(x) < INFINITY)) out[j] = static_cast<T>(static_cast<float>(out[j]) + x);
    }
}

constexpr int GEN_JOIN = 9;    // 16-byte pieces that a lane leaves in LDS for a join at D = 128

// Few rows: 16 of them a wave; one, two or four (GI_WAVES) waves along the rows,
// the others share the keys.
template <int D, bool E4M3>
__device__ inline void gen_few(const GenArgs& A, Scalars it, int hk, int wave, int lane,
                               float* __restrict__ lds) {
  typedef KvStep<D, E4M3> Step;
  // keys of a step: 32, or 64 of 64 bytes each, for as many bytes on the way (at
  // D = 128, 64 8-bit keys spill: 64 rows of 2,000 keys, 8 heads 111 us against 63)
  constexpr int NK = E4M3 && D == 64 ? 2 : 1, T = 32 * NK;
  constexpr int DT = D / 16;                        // 16-column tiles
  static_assert(DT + 1 <= GEN_JOIN, "room for a join");
  const CacheView& c = A.c;
  const int rw = it[GI_WAVES], sh = rw >> 1, kws = 4 >> sh;   // (1, 2 or 4)
  const int rt = wave & (rw - 1), kw = wave >> sh;
  const int seg = it[GI_SEG], group = static_cast<int>(A.by_group.d);
  const int g = lane >> 4, i = lane & 15;
  const Reach reach(c, seg, it[GI_NEW]);
  const int32_t n = reach.n;

  const int local = 16 * rt + i;
  const bool live = local < it[GI_N];
  const int stacked = it[GI_ROW] + (live ? local : 0), place = place_of(A, stacked);
  const int32_t row = A.order[it[GI_FIRST] + place], head = hk * group + stacked - place * group;
  const int32_t p0 = A.part_off[row], parts = A.part_off[row + 1] - p0;
  int32_t lim = reach.of(place);
  bf16x8 qf[D / 32];
  const bf16* qp = A.q + (static_cast<int64_t>(row) * A.Hq + head) * D;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) qf[s] = q_frag(A, qp + Step::k_col(s, g));
  // the fewest and the most keys that a row of the wave sees: places grow along
  // it, and what a row sees with its place (own rows one more each, then the
  // descendants', which see all)
  const int first = 16 * rt, last = min(first + 16, it[GI_N]) - 1;
  const int32_t lo = last < first ? n : reach.of(place_of(A, it[GI_ROW] + first));
  const int32_t hi = last < first ? 0 : reach.of(place_of(A, it[GI_ROW] + last));
  if (!live) lim = n;                               // padding rows take part and are dropped

  int32_t from, end;
  split_steps<T>(it, hi, from, end);
  RowState<DT> st;
  st.clear();
  bool odds = false;

  const Scalars table = scalars(c.pages) + static_cast<int64_t>(seg) * c.pitch;
  const auto page_of = [&](int32_t u) {
    const int32_t p = table[u * T / GEN_PAGE];
    return p >= 0 && p < c.n_pages ? p : -1;
  };
  const auto base_of = [&](int32_t page) {
    return (static_cast<int64_t>(page < 0 ? 0 : page) * c.H + hk) * GEN_PAGE;
  };
  Step x[NK];
  const auto load_k = [&](int32_t u, int64_t b) {
#pragma unroll
    for (int h = 0; h < NK; ++h) x[h].load_k(c.k + b * Step::ROWB, c.ke + b, (u * NK + h) & 1, lane);
  };
  const auto load_v = [&](int32_t u, int64_t b) {
#pragma unroll
    for (int h = 0; h < NK; ++h) x[h].load_v(c.v + b * Step::ROWB, c.ve + b, (u * NK + h) & 1, lane);
  };
  int32_t u = from + kw, page = -1;
  if (u < end) {
    page = page_of(u);
    const int64_t b = base_of(page);
    load_k(u, b);
    load_v(u, b);
  }
  for (; u < end; u += kws) {
    const int32_t key0 = u * T, next_u = u + kws;
    const bool more = next_u < end;
    const int32_t next = more ? page_of(next_u) : -1;
    const int64_t nb = base_of(next);

    f32x4 s[2 * NK];
#pragma unroll
    for (int t = 0; t < 2 * NK; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < D / 32; ++d) s[t] = mfma32(x[t / 2].k_frag(t & 1, d), qf[d], s[t]);
    }
    if (more) load_k(next_u, nb);

    const bool edge = key0 + T > lo || page < 0;    // some key is hidden from some row
    float y[8 * NK], top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8 * NK; ++e) {
      y[e] = s[e >> 2][e & 3];
      if (edge && (key0 + 32 * (e / 8) + frag_key(g, e % 8) >= lim || page < 0)) y[e] = -INFINITY;
      top = fmaxf(top, y[e]);
    }
    top *= A.scale;
    if (__any(top > st.ref + GEN_SLACK)) st.raise(top);
    const float r = st.zero_point();
#pragma unroll
    for (int e = 0; e < 8 * NK; ++e) {
      y[e] = __builtin_amdgcn_exp2f(fmaf(y[e], A.scale, -r));
      // (with a scale of 0 too)
      if (edge && (key0 + 32 * (e / 8) + frag_key(g, e % 8) >= lim || page < 0)) y[e] = 0.f;
      st.sum += y[e];
    }
    u32 odd = 0;
#pragma unroll
    for (int h = 0; h < NK; ++h) {
      const float* z = y + 8 * h;
      const bf16x8 w = __builtin_bit_cast(bf16x8, u32x4{pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]),
                                                        pack_bf16(z[4], z[5]), pack_bf16(z[6], z[7])});
#pragma unroll
      for (int q = 0; q < Step::VW; ++q) {
        u32 vw[8];
        x[h].v_pairs(vw, q);
        if (edge) {
          // (rows that do not exist hold anything)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const bool there = page >= 0 && key0 + 32 * h + frag_key(g, e) < n;
            vw[e] = there ? finite_pair(vw[e], odd) : 0u;
          }
        }
        st.acc[2 * q] = mfma32(v_frag(vw, 0), w, st.acc[2 * q]);
        st.acc[2 * q + 1] = mfma32(v_frag(vw, 1), w, st.acc[2 * q + 1]);
      }
    }
    if (edge) odds |= __any(odd != 0);
    if (more) load_v(next_u, nb);
    page = next;
  }
  st.sum = over_groups_sum(st.sum);

  // join the waves that shared the keys, half of them into the other half: 16
  // bytes a lane at a time, as short a code as a once-run one should be
  typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
  for (int step = kws / 2; step >= 1; step /= 2) {
    if (kw >= step && kw < 2 * step) {
      lds_f32x4* p = (lds_f32x4*)lds + ((kw - step) * rw + rt) * (64 * GEN_JOIN) + lane;
#pragma unroll
      for (int j = 0; j < DT; ++j) p[64 * j] = st.acc[j];
      p[64 * DT] = f32x4{st.ref, st.sum, odds ? 1.f : 0.f, 0.f};
    }
    __syncthreads();
    if (kw < step) {
      const lds_f32x4* p = (const lds_f32x4*)lds + (kw * rw + rt) * (64 * GEN_JOIN) + lane;
      const f32x4 head = p[64 * DT];
      const float to = fmaxf(st.ref, head[0]), r = to == -INFINITY ? 0.f : to;
      const float f0 = __builtin_amdgcn_exp2f(st.ref - r), f1 = __builtin_amdgcn_exp2f(head[0] - r);
      st.ref = to;
      st.sum = st.sum * f0 + head[1] * f1;
      odds |= head[2] != 0.f;
#pragma unroll
      for (int j = 0; j < DT; ++j) st.acc[j] = st.acc[j] * f0 + p[64 * j] * f1;
    }
    if (step > 1) __syncthreads();
  }
  if (kw != 0 || !live) return;

  if (parts == 1) {
    const int64_t rh = static_cast<int64_t>(row) * A.Hq + head;
    const float f = st.inverse();
    u32 out[D / 8];
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int j = 0; j < DT; j += 2)
        out[e * (DT / 2) + j / 2] = pack_bf16(st.acc[j][e] * f, st.acc[j + 1][e] * f);
    u32x4* op = reinterpret_cast<u32x4*>(A.o + rh * D + g * (D / 4));
#pragma unroll
    for (int e = 0; e < D / 32; ++e) op[e] = u32x4{out[4 * e], out[4 * e + 1], out[4 * e + 2], out[4 * e + 3]};
    if (A.lse && g == 0) A.lse[rh] = log_sum(st.ref, st.sum);
    if (odds && st.sum != 0.f)
      for (u = max(from, lo / T); u < end; ++u)
        add_odd<D, E4M3>(c, table, hk, u * T, T, n, lim, A.o + rh * D, g * (D / 4), D / 4);
  } else {
    const int64_t at = (static_cast<int64_t>(p0) + it[GI_PART] + it[GI_SPLIT]) * A.Hq + head;
    f32x4* ap = reinterpret_cast<f32x4*>(A.acc + at * D + g * (D / 4));
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int j = 0; j < DT; j += 4)
        ap[(e * DT + j) / 4] = f32x4{st.acc[j][e], st.acc[j + 1][e], st.acc[j + 2][e], st.acc[j + 3][e]};
    if (g == 0) {
      A.ml[2 * at] = st.ref;
      A.ml[2 * at + 1] = st.sum;
    }
    if (odds)
      for (u = max(from, lo / T); u < end; ++u)
        add_odd<D, E4M3>(c, table, hk, u * T, T, n, lim, A.acc + at * D, g * (D / 4), D / 4);
  }
}

// LDS tile of T keys x D bf16, unpadded.  Row r keeps its 16-byte piece p at
// slot p ^ swz(r), chosen for the lanes that the LDS serves together: a 16-byte
// fragment read takes sets of rows r and r ^ 12 at neighbouring pieces, a
// transposed read 8 rows of two neighbouring pieces (both free of conflicts).
template <int D>
struct GenTile {
  static constexpr int PPR = D / 8;
  __device__ static inline int swz(int r) {
    const int hi = (r >> 3) & 1;
    return D == 128 ? (((r & 7) ^ (hi << 2)) << 1) | hi : ((r & 6) ^ (hi << 2)) | hi;
  }
  // Reads by LDS addresses.  A tile starts at a multiple of its row's bytes, so a
  // column's piece goes into the address by exclusive or, and two constants of
  // the lane (and one or two of the step) serve all fragments.
  __device__ static inline u32 rows_lane(int lane) {
    const int i = lane & 15, g = lane >> 4;
    return 2 * D * i + ((g ^ swz(i)) << 4);
  }
  __device__ static inline u32 columns_lane(int lane) {
    const int r = (lane >> 4) * 4 + ((lane & 15) >> 2), c = lane & 3;
    return 2 * D * r + (((c >> 1) ^ swz(r)) << 4) + 8 * (c & 1);
  }
  // lane (g, i): key 16 j + i, columns 32 s + 8 g .. + 7
  __device__ static inline bf16x8 rows(u32 at, int j, int s) {
    typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
    return *(const lds_bf16x8*)((at ^ (s << 6)) + j * 32 * D);
  }
  // lane (g, i): column 16 j + i, keys 32 h + frag_key(g, 0 .. 7)
  __device__ static inline bf16x8 columns(u32 at, int h, int j) {
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    const u32 p = (at ^ (j << 5)) + h * 64 * D;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 32 * D));
    return Frag<bf16>::join(__builtin_bit_cast(bf16x4, lo), __builtin_bit_cast(bf16x4, hi));
  }
};

// Requests of T cached rows of one page half (or page) into a tile.  Thread t
// fills the 16-byte slots t, t + 256, ...: of rows r0, r0 + RPE, ...
template <int D, int T, bool E4M3> struct GenStage;

template <int D, int T> struct GenStage<D, T, false> {
  static constexpr int RPE = GEN_THR / (D / 8), N = T / RPE;
  static_assert(RPE % 16 == 0, "every request starts at a multiple of 16 rows");
  int r0, wave;
  u32 off;
  __device__ inline GenStage(int t, int wave_) : r0(t / (D / 8)), wave(wave_) {
    off = r0 * (2 * D) + 16 * ((t % (D / 8)) ^ GenTile<D>::swz(r0));
  }
  // the first `have` of the rows at src; zeros past those
  __device__ inline void request(const char* src, const uint8_t*, int have, const bf16* tile) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const bf16* dst = tile + (e * GEN_THR + 64 * wave) * 8;
      if (r0 + RPE * e < have) {
        lds_load16(src, off + e * RPE * 2 * D, dst);
      } else {
        typedef __attribute__((address_space(3))) volatile uint64_t lds_u64;
        lds_u64* z = (lds_u64*)(dst + 8 * (threadIdx.x & 63));
        z[0] = 0;
        z[1] = 0;
      }
    }
  }
};

// 8-bit rows land as they are in a buffer of LDS, 16 codes a lane, from where
// the lane that requested them takes them to the tile as bf16: nothing but two
// scale exponents waits in registers while a step computes (with the codes
// there too, 25 registers were spilled: 65k keys, 256 rows, 8 heads 142 us).
template <int D, int T> struct GenStage<D, T, true> {
  static constexpr int LPR = D / 16;         // lanes of a row
  static_assert(T * LPR == GEN_THR, "one request a tile");
  int r, wave, swap, slot0, slot1;
  u32 off, ex;
  __device__ inline GenStage(int t, int wave_) : r(t / LPR), wave(wave_), off(16 * t) {
    // (odd lanes take the second piece first: a write of 16 lanes then fills all
    // banks once, where even pieces alone would take each second one twice)
    const int p = 2 * (t % LPR), x = GenTile<D>::swz(r);
    swap = t & 1;
    slot0 = r * (D / 8) + ((p + swap) ^ x);
    slot1 = r * (D / 8) + ((p + 1 - swap) ^ x);
  }
  __device__ inline void request(const char* src, const uint8_t* exps, int have, const char* raw) {
    ex = 0;                                  // (a row past `have`: its codes are whatever was there)
    if (r < have) {
      lds_load16(src, off, raw + 1024 * wave);
      ex = exps[r];
    }
  }
  // after the wave's requests have landed
  __device__ inline void arrive(const char* raw, bf16* tile) {
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    const u32x4 x = *(const lds_u32x4*)(raw + off);
    const float f = exp_scale(ex);
    u32x4 y[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int second = h ^ swap;
      const u32x2 a = dequantise(second ? x[2] : x[0], f), b = dequantise(second ? x[3] : x[1], f);
      y[h] = ex == 0 ? u32x4{0, 0, 0, 0} : u32x4{a[0], a[1], b[0], b[1]};
    }
    *(lds_u32x4*)(tile + slot0 * 8) = y[0];
    *(lds_u32x4*)(tile + slot1 * 8) = y[1];
  }
};

template <int D> constexpr int gen_step() { return D == 128 ? 32 : 64; }   // keys of a step: 8 KB of a tile

// Many rows: 32 of them a wave, every step's keys through LDS for all four.
template <int D, bool E4M3>
__device__ inline void gen_many(const GenArgs& A, Scalars it, int hk, int wave, int lane,
                                bf16* __restrict__ lds) {
  constexpr int T = gen_step<D>(), NS = D / 32, DT = D / 16, TILE = T * D, ROWB = E4M3 ? D : 2 * D;
  typedef GenTile<D> L;
  const CacheView& c = A.c;
  const int seg = it[GI_SEG], group = static_cast<int>(A.by_group.d), m = it[GI_N];
  const int g = lane >> 4, i = lane & 15;
  const Reach reach(c, seg, it[GI_NEW]);
  const int32_t n = reach.n;
  // (as in gen_few; lo of the tile, so that all waves go over to the masked steps together)
  const int32_t lo = reach.of(place_of(A, it[GI_ROW])), most = reach.of(place_of(A, it[GI_ROW] + m - 1));
  const int32_t hi = 32 * wave < m ? reach.of(place_of(A, it[GI_ROW] + min(32 * wave + 32, m) - 1)) : 0;
  int32_t from, end;
  split_steps<T>(it, most, from, end);

  const Scalars table = scalars(c.pages) + static_cast<int64_t>(seg) * c.pitch;
  GenStage<D, T, E4M3> sk(threadIdx.x, wave), sv(threadIdx.x, wave);
  // the keys and values of step u on their way: bf16 to `tile`, 8-bit to the buffer behind the tiles
  char* raw = reinterpret_cast<char*>(lds + 4 * TILE);
  const auto request = [&](int32_t u, bf16* tile) {
    const int32_t key0 = u * T, p = table[key0 / GEN_PAGE], part = key0 % GEN_PAGE;
    const int have = p >= 0 && p < c.n_pages ? n - key0 : 0;
    const int64_t b = (static_cast<int64_t>(have > 0 ? p : 0) * c.H + hk) * GEN_PAGE + part;
    if constexpr (E4M3) {
      sk.request(c.k + b * ROWB, c.ke + b, have, raw);
      sv.request(c.v + b * ROWB, c.ve + b, have, raw + TILE);
    } else {
      sk.request(c.k + b * ROWB, nullptr, have, tile);
      sv.request(c.v + b * ROWB, nullptr, have, tile + TILE);
    }
  };
  // 8-bit rows of the step requested last, from the buffer to `tile`; the next ones' turn
  const auto arrive = [&](int32_t u, bf16* tile) {
    if constexpr (E4M3) {
      __builtin_amdgcn_s_waitcnt(0x0f70);    // the wave's loads have landed (vmcnt 0)
      asm volatile("" ::: "memory");
      sk.arrive(raw, tile);
      sv.arrive(raw + TILE, tile + TILE);
      __builtin_amdgcn_s_waitcnt(0xc07f);    // and been read (lgkmcnt 0) before others land on them
      asm volatile("" ::: "memory");
      if (u + 1 < end) request(u + 1, nullptr);
    }
  };
  if (from < end) request(from, lds);

  // stacked row of column i of half a (padding rows repeat the last one), and its place
  const auto stacked_of = [&](int a) { return it[GI_ROW] + min(32 * wave + 16 * a + i, m - 1); };
  bf16x8 qf[2][NS];
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    const int r = stacked_of(a), place = place_of(A, r);
    const int64_t row = A.order[it[GI_FIRST] + place], head = hk * group + r - place * group;
    const bf16* qp = A.q + (row * A.Hq + head) * D + 8 * g;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[a][s] = q_frag(A, qp + 32 * s);
  }
  RowState<DT> st[2];
  st[0].clear();
  st[1].clear();
  bool odds = false;
  const u32 klane = L::rows_lane(lane), vlane = L::columns_lane(lane);

  if (from < end) arrive(from, lds);
  // One step; `edge`: some key may be hidden from some row of the tile.
  const auto step = [&](int32_t u, auto edge_) {
    constexpr bool edge = decltype(edge_)::value;
    const int32_t key0 = u * T, buf = (u - from) & 1;
    bf16 *tk = lds + 2 * buf * TILE, *tv = tk + TILE, *next = lds + 2 * (buf ^ 1) * TILE;
    if constexpr (E4M3) {
      __syncthreads();                       // this step's tiles are here, the other pair's readers are done
      if (u + 1 < end) arrive(u + 1, next);
    } else {
      lds_landed();
      if (u + 1 < end) request(u + 1, next);
    }
    const int32_t page = table[key0 / GEN_PAGE];
    if (key0 >= hi || page < 0 || page >= c.n_pages) return;   // (the same for the whole wave)
    typedef __attribute__((address_space(3))) const bf16 lds_bf16;
    const u32 kat = klane + static_cast<u32>(reinterpret_cast<uintptr_t>((lds_bf16*)tk));
    const u32 vat = vlane + static_cast<u32>(reinterpret_cast<uintptr_t>((lds_bf16*)tv));
    f32x4 s[2][T / 16];
#pragma unroll
    for (int j = 0; j < T / 16; ++j) s[0][j] = s[1][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // Fragments are read AHEAD ahead of their products: left alone, the compiler
    // reads each into the same registers and waits for it, the whole LDS latency
    // for every two products (2,000 new rows on 3 prompts of 14k: 407 us, 390 so,
    // with 2 to 4)
    constexpr int NK = NS * (T / 16), NV = DT * (T / 32), AHEAD = 3;
    bf16x8 kf[NK], vf[NV];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) kf[n] = L::rows(kat, n / NS, n % NS);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);           // the SIMD's other waves do their softmax meanwhile
#pragma unroll
    for (int n = 0; n < NK; ++n) {
      if (n + AHEAD < NK) kf[n + AHEAD] = L::rows(kat, (n + AHEAD) / NS, (n + AHEAD) % NS);
      s[0][n / NS] = mfma32(kf[n], qf[0][n % NS], s[0][n / NS]);
      s[1][n / NS] = mfma32(kf[n], qf[1][n % NS], s[1][n / NS]);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) vf[n] = L::columns(vat, n / DT, n % DT);
    __builtin_amdgcn_sched_barrier(0);
    const int32_t lim[2] = {edge ? reach.of(place_of(A, stacked_of(0))) : 0,
                            edge ? reach.of(place_of(A, stacked_of(1))) : 0};
    float top[2];
    bool up = false;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      top[a] = -INFINITY;
#pragma unroll
      for (int j = 0; j < T / 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (edge && key0 + 16 * j + 4 * g + e >= lim[a]) s[a][j][e] = -INFINITY;
          top[a] = fmaxf(top[a], s[a][j][e]);
        }
      top[a] *= A.scale;
      up |= top[a] > st[a].ref + GEN_SLACK;
    }
    if (__any(up)) {
      st[0].raise(top[0]);
      st[1].raise(top[1]);
    }
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      const float r = st[a].zero_point();
#pragma unroll
      for (int j = 0; j < T / 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[a][j][e] = __builtin_amdgcn_exp2f(fmaf(s[a][j][e], A.scale, -r));
          if (edge && key0 + 16 * j + 4 * g + e >= lim[a]) s[a][j][e] = 0.f;   // (with a scale of 0 too)
          st[a].sum += s[a][j][e];
        }
    }
    u32 odd = 0;
    bf16x8 w[T / 32][2];
#pragma unroll
    for (int h = 0; h < T / 32; ++h)
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const f32x4 &x = s[a][2 * h], &y = s[a][2 * h + 1];
        w[h][a] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]),
                                                   pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])});
      }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      if (n + AHEAD < NV) vf[n + AHEAD] = L::columns(vat, (n + AHEAD) / DT, (n + AHEAD) % DT);
      const int j = n % DT;
      if constexpr (edge) {
        u32x4 f = __builtin_bit_cast(u32x4, vf[n]);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = finite_pair(f[e], odd);
        vf[n] = __builtin_bit_cast(bf16x8, f);
      }
      st[0].acc[j] = mfma32(vf[n], w[n / DT][0], st[0].acc[j]);
      st[1].acc[j] = mfma32(vf[n], w[n / DT][1], st[1].acc[j]);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    if constexpr (edge) odds |= __any(odd != 0);
  };
  const int32_t mid = min(end, max(from, lo / T));
  for (int32_t u = from; u < mid; ++u) step(u, std::false_type{});
  for (int32_t u = mid; u < end; ++u) step(u, std::true_type{});

#pragma unroll
  for (int a = 0; a < 2; ++a) {
    st[a].sum = over_groups_sum(st[a].sum);
    if (32 * wave + 16 * a + i >= m) continue;
    const int r = stacked_of(a), place = place_of(A, r);
    const int32_t row = A.order[it[GI_FIRST] + place], head = hk * group + r - place * group;
    const int32_t lim = reach.of(place);
    const int32_t p0 = A.part_off[row], parts = A.part_off[row + 1] - p0;
    if (parts == 1) {
      const int64_t rh = static_cast<int64_t>(row) * A.Hq + head;
      const float f = st[a].inverse();
#pragma unroll
      for (int j = 0; j < DT; ++j) Vec4<bf16>::store(A.o + rh * D + 16 * j + 4 * g, st[a].acc[j] * f);
      if (A.lse && g == 0) A.lse[rh] = log_sum(st[a].ref, st[a].sum);
      if (odds && st[a].sum != 0.f)
        for (int32_t u = mid; u < end; ++u)
          for (int j = 0; j < DT; ++j)
            add_odd<D, E4M3>(c, table, hk, u * T, T, n, lim, A.o + rh * D, 16 * j + 4 * g, 4);
    } else {
      const int64_t at = (static_cast<int64_t>(p0) + it[GI_PART] + it[GI_SPLIT]) * A.Hq + head;
#pragma unroll
      for (int j = 0; j < DT; ++j) *reinterpret_cast<f32x4*>(A.acc + at * D + 16 * j + 4 * g) = st[a].acc[j];
      if (g == 0) {
        A.ml[2 * at] = st[a].ref;
        A.ml[2 * at + 1] = st[a].sum;
      }
      if (odds)
        for (int32_t u = mid; u < end; ++u)
          for (int j = 0; j < DT; ++j)
            add_odd<D, E4M3>(c, table, hk, u * T, T, n, lim, A.acc + at * D, 16 * j + 4 * g, 4);
    }
  }
}

template <int D, bool E4M3>
__global__ __launch_bounds__(GEN_THR, 3) void k_gen_attn(GenArgs A) {
  constexpr int TILE = gen_step<D>() * D * 2;      // bytes
  static_assert(4 * TILE >= 2 * 64 * GEN_JOIN * 16, "a join fits");
  __shared__ __align__(256) char lds[E4M3 ? 5 * TILE : 4 * TILE];   // (rows of 256 bytes, see GenTile)
  const int item = static_cast<int>(A.c.by_heads.div(blockIdx.x)), hk = blockIdx.x - item * A.c.H;
  const Scalars it = scalars(A.items) + static_cast<int64_t>(item) * GI_WORDS;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (it[GI_TILES] == 1) gen_few<D, E4M3>(A, it, hk, wave, lane, reinterpret_cast<float*>(lds));
  else gen_many<D, E4M3>(A, it, hk, wave, lane, reinterpret_cast<bf16*>(lds));
}

// Joins the parts of (row, query head) entries that have several.  D / 4 lanes
// hold a part's accumulators, four columns each; SUBS such groups take an
// entry's parts in turn, each with a reference of its own, and meet in LDS.
// With many parts an entry has the whole workgroup, or their reads, one after
// the other, would set the time (one row of 65k keys, 32 heads, 96 parts: 90 us a
// call with one wave an entry, 63 so).
template <int D, int SUBS>
__global__ __launch_bounds__(GEN_THR) void k_gen_join(GenArgs A, int64_t n) {
  constexpr int LPG = D / 4, ENTRIES = GEN_THR / LPG / SUBS, U = 4;
  const int t = threadIdx.x, c = 4 * (t % LPG), grp = t / LPG, sub = grp % SUBS;
  const int64_t rh = static_cast<int64_t>(blockIdx.x) * ENTRIES + grp / SUBS;
  int32_t p0 = 0, parts = 0, head = 0;
  if (rh < n) {
    const int32_t row = static_cast<int32_t>(A.by_Hq.div(static_cast<u32>(rh)));
    head = static_cast<int32_t>(rh - static_cast<int64_t>(row) * A.Hq);
    p0 = A.part_off[row];
    parts = A.part_off[row + 1] - p0;
  }
  float ref = -INFINITY, sum = 0.f;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  const auto add = [&](float to, float s1, float r1, const f32x4& x) {
    const float r = to == -INFINITY ? 0.f : to;
    const float f = __builtin_amdgcn_exp2f(r1 - r);
    sum += s1 * f;
    acc += x * f;
  };
  const auto rise = [&](float to) {
    const float f = to == ref ? 1.f : __builtin_amdgcn_exp2f(ref - to);
    ref = to;
    sum *= f;
    acc *= f;
  };
  for (int b = sub; b < parts; b += U * SUBS) {
    float r1[U], s1[U];
    f32x4 x[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int p = b + k * SUBS;
      r1[k] = -INFINITY;
      s1[k] = 0.f;
      x[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (p < parts) {
        const int64_t at = (static_cast<int64_t>(p0) + p) * A.Hq + head;
        r1[k] = A.ml[2 * at];
        s1[k] = A.ml[2 * at + 1];
        x[k] = *reinterpret_cast<const f32x4*>(A.acc + at * D + c);
      }
    }
    rise(fmaxf(fmaxf(fmaxf(ref, r1[0]), fmaxf(r1[1], r1[2])), r1[3]));
#pragma unroll
    for (int k = 0; k < U; ++k) add(ref, s1[k], r1[k], x[k]);
  }
  if constexpr (SUBS > 1) {
    __shared__ f32x4 sx[GEN_THR];
    __shared__ float sr[GEN_THR / LPG], ss[GEN_THR / LPG];
    sx[t] = acc;
    if (t % LPG == 0) {
      sr[grp] = ref;
      ss[grp] = sum;
    }
    __syncthreads();
    if (sub != 0) return;
    for (int k = 1; k < SUBS; ++k) {
      rise(fmaxf(ref, sr[grp + k]));
      add(ref, ss[grp + k], sr[grp + k], sx[t + k * LPG]);
    }
  }
  if (parts <= 1) return;
  if (sum == 0.f) acc = f32x4{0.f, 0.f, 0.f, 0.f};   // (as in RowState)
  Vec4<bf16>::store(A.o + rh * D + c, acc * (sum == 0.f ? 0.f : 1.f / sum));
  if (A.lse && c == 0) A.lse[rh] = log_sum(ref, sum);
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
          c->n_pages, c->n_seg, c->pitch, c->H, FastDiv(static_cast<u32>(c->H))};
}

// f(head size, whether 8-bit) of a cache, as constants
template <typename F>
void by_cache(const harts_cache* c, F f) {
  const std::integral_constant<int, 128> d128{};
  const std::integral_constant<int, 64> d64{};
  const bool q = c->kind == HARTS_E4M3;
  if (c->d == 128) q ? f(d128, std::true_type{}) : f(d128, std::false_type{});
  else q ? f(d64, std::true_type{}) : f(d64, std::false_type{});
}

// blocks of a launch of one lane per 8 elements, or 0 past a grid's reach
uint32_t piece_blocks(int64_t n, const harts_cache* c) {
  const int64_t b = (n * c->H * (c->d / 8) + GEN_THR - 1) / GEN_THR;
  return b > INT32_MAX ? 0 : static_cast<uint32_t>(b);
}

// Whether the bf16 side of a call is larger than the chip's L2 caches: it then
// goes around them (30,000 rows x 16 heads of 128: 8-bit read 75 -> 51 us, bf16
// write 84 -> 71; the write that quantises was no faster so, at d = 64 slower).
bool past_l2(int64_t n, const harts_cache* c) { return n * c->H * c->d * 4 > (int64_t{32} << 20); }

// What a cache occupies: keys and values with their scale exponents, and its tables.
struct CacheRegions {
  Region k, v, ke, ve, pages, len;
  explicit CacheRegions(const harts_cache* c) {
    const size_t rows = static_cast<size_t>(c->n_pages) * c->H * GEN_PAGE, held = rows * c->d;
    const bool q = c->kind == HARTS_E4M3;
    k = {c->k, q ? held : 2 * held};
    v = {c->v, k.bytes};
    ke = {c->k_exp, q ? rows : 0};
    ve = {c->v_exp, q ? rows : 0};
    pages = {c->pages, static_cast<size_t>(c->n_seg) * c->pitch * sizeof(int32_t)};
    len = {c->len, static_cast<size_t>(c->n_seg) * sizeof(int32_t)};
  }
};

int check_rows(const harts_cache* c, const int32_t* rows, int64_t n, const void* k, const void* v, const char* where) {
  if (int rc = check_cache(c, where)) return rc;
  if (n < 0) { set_error(std::string(where) + ": negative row count"); return HARTS_EINVAL; }
  if (n == 0) return HARTS_OK;
  if (!rows || !k || !v || !aligned(rows, 4) || !aligned(k, 16) || !aligned(v, 16)) {
    set_error(std::string(where) + ": NULL or misaligned pointer");
    return HARTS_EINVAL;
  }
  if (n > INT32_MAX / c->H || piece_blocks(n, c) == 0) {
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
  const CacheRegions R(cache);
  const size_t span = static_cast<size_t>(n) * cache->H * cache->d * sizeof(bf16);
  const Region kn{k_new, span}, vn{v_new, span}, table{rows, static_cast<size_t>(n) * 2 * sizeof(int32_t)};
  if (overlaps_any(R.k, {kn, vn, table, R.v, R.ke, R.ve, R.pages, R.len}) ||
      overlaps_any(R.v, {kn, vn, table, R.ke, R.ve, R.pages, R.len}) ||
      overlaps_any(R.ke, {kn, vn, table, R.ve, R.pages, R.len}) || overlaps_any(R.ve, {kn, vn, table, R.pages, R.len})) {
    set_error("harts_cache_write: a written part of the cache overlaps another or an input");
    return HARTS_EINVAL;
  }
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(piece_blocks(n, cache)), dim3(GEN_THR), 0, static_cast<hipStream_t>(stream),
                       view_of(cache), rows, n, static_cast<const u32x4*>(k_new), static_cast<const u32x4*>(v_new));
  };
  const auto pick = [&](auto dim, auto kind) {
    constexpr int D = decltype(dim)::value;
    constexpr bool Q = decltype(kind)::value;
    past_l2(n, cache) ? launch(k_cache_write<D, Q, !Q>) : launch(k_cache_write<D, Q, false>);
  };
  by_cache(cache, pick);
  return gen_status("k_cache_write");
}

extern "C" int harts_cache_read(const harts_cache* cache, const int32_t* rows, int64_t n, void* k_out, void* v_out,
                                void* stream) {
  if (int rc = check_rows(cache, rows, n, k_out, v_out, "harts_cache_read")) return rc;
  if (n == 0) return HARTS_OK;
  const CacheRegions R(cache);
  const size_t span = static_cast<size_t>(n) * cache->H * cache->d * sizeof(bf16);
  const Region ko{k_out, span}, vo{v_out, span}, table{rows, static_cast<size_t>(n) * 2 * sizeof(int32_t)};
  if (overlaps_any(ko, {vo, table, R.k, R.v, R.ke, R.ve, R.pages, R.len}) ||
      overlaps_any(vo, {table, R.k, R.v, R.ke, R.ve, R.pages, R.len})) {
    set_error("harts_cache_read: an output overlaps another or an input");
    return HARTS_EINVAL;
  }
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(piece_blocks(n, cache)), dim3(GEN_THR), 0, static_cast<hipStream_t>(stream),
                       view_of(cache), rows, n, static_cast<u32x4*>(k_out), static_cast<u32x4*>(v_out));
  };
  const auto pick = [&](auto dim, auto kind) {
    constexpr int D = decltype(dim)::value;
    constexpr bool Q = decltype(kind)::value;
    past_l2(n, cache) ? launch(k_cache_read<D, Q, true>) : launch(k_cache_read<D, Q, false>);
  };
  by_cache(cache, pick);
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
  const auto out_of = [](int64_t x) { return x < 0 || x > INT32_MAX; };
  if (!sizes || out_of(sizes->n_rows) || out_of(sizes->n_items) || out_of(sizes->n_parts) || sizes->n_join < 0 ||
      sizes->n_rows * Hq > INT32_MAX || sizes->n_items * cache->H > INT32_MAX) {
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
  const CacheRegions R(cache);
  const size_t n_rows = static_cast<size_t>(sizes->n_rows), span = n_rows * Hq * cache->d * sizeof(bf16);
  const Region out{o, span}, sums{lse, n_rows * Hq * sizeof(float)}, parts_of{ws, need}, in{q, span};
  const Region work{items, static_cast<size_t>(sizes->n_items) * GI_WORDS * sizeof(int32_t)};
  const Region places{order, n_rows * sizeof(int32_t)}, offsets{part_off, (n_rows + 1) * sizeof(int32_t)};
  const auto over_an_input = [&](const Region& x) {
    return overlaps_any(x, {in, work, places, offsets, R.k, R.v, R.ke, R.ve, R.pages, R.len});
  };
  if (over_an_input(out) || over_an_input(sums) || over_an_input(parts_of)) {
    set_error("harts_gen_attn: o, lse or the workspace overlaps an input");
    return HARTS_EINVAL;
  }
  if (overlaps_any(out, {sums, parts_of}) || overlap(sums, parts_of)) {
    set_error("harts_gen_attn: o, lse and the workspace overlap");
    return HARTS_EINVAL;
  }
  GenArgs A;
  A.c = view_of(cache);
  A.items = items;
  A.order = order;
  A.part_off = part_off;
  A.Hq = Hq;
  A.by_group = FastDiv(static_cast<u32>(Hq / cache->H));
  A.by_Hq = FastDiv(static_cast<u32>(Hq));
  A.scale = fabsf(scale) * GEN_LOG2E;
  A.sign = scale < 0.f ? 0x80008000u : 0u;
  A.q = static_cast<const bf16*>(q);
  A.o = static_cast<bf16*>(o);
  A.lse = lse;
  A.acc = static_cast<float*>(ws);
  A.ml = need ? A.acc + sizes->n_parts * Hq * cache->d : nullptr;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(sizes->n_items * cache->H)), dim3(GEN_THR), 0, s, A);
  };
  by_cache(cache, [&](auto dim, auto kind) { launch(k_gen_attn<decltype(dim)::value, decltype(kind)::value>); });
  if (int rc = gen_status("k_gen_attn")) return rc;
  if (sizes->n_join > 0) {
    const int64_t n = sizes->n_rows * Hq;
    // groups of an entry by its parts, on average
    const int64_t parts = sizes->n_parts / sizes->n_rows;
    const auto join = [&](auto kernel, int64_t entries) {
      hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>((n + entries - 1) / entries)), dim3(GEN_THR), 0, s, A, n);
    };
    if (cache->d == 128) {
      if (parts >= 32) join(k_gen_join<128, 8>, 1);
      else if (parts >= 8) join(k_gen_join<128, 4>, 2);
      else join(k_gen_join<128, 1>, 8);
    } else {
      if (parts >= 32) join(k_gen_join<64, 16>, 1);
      else if (parts >= 8) join(k_gen_join<64, 4>, 4);
      else join(k_gen_join<64, 1>, 16);
    }
    return gen_status("k_gen_join");
  }
  return HARTS_OK;
}
