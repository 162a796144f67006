// Recurrent steps of linear attention with scalar decay and of KDA, for single
// tokens or a few (gfx950):
//   linear attention  S_t = e^{g_t} S_{t-1} + k_t v_t^T,  o_t = scale S_t^T q_t
//   KDA               D = Diag(e^{g_t}) S_{t-1},
//                     S_t = D + beta_t k_t (v_t - D^T k_t)^T, o_t the same.
//
// A token costs its state read and written once (2 x 4 D^2 bytes per head)
// against 5 to 7 D^2 operations: the call is bound by HBM.  Both recurrences
// keep the state's columns apart, so a wave takes 32 columns of one (sequence,
// head) and holds them in registers for all of the sequence's tokens: lane
// (r, c) = (lane / 8, lane % 8) has rows r D/8 .. r D/8 + D/8 - 1 of columns
// 4c .. 4c + 3.  A request of the wave covers 8 rows x 128 bytes (whole cache
// lines, the D/32 waves of a head side by side), D/8 of them are in flight
// per lane, and q, k and g of a lane's rows are neighbours in memory.  Sums
// over rows are D/8 products in a lane and three exchanges between lanes.
// Everything is float32; o is rounded once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include <string>
#include <type_traits>

#include "fast_div.hpp"
#include "harts_rollout.h"
#include "la_common.hpp"
#include "plan.hpp"
#include "regions.hpp"

namespace harts {
namespace {

constexpr int ST_THR = 256;
constexpr int ST_COLS = 32;   // columns of a wave

struct StepArgs {
  int64_t n_seq, n_rows;
  int32_t H;
  float scale;
  FastDiv by_heads;
  const void *q, *k, *v;
  const float *g, *beta;
  const int32_t* row_off;
  const float* S_in;
  const int32_t* idx_in;
  int64_t n_in;
  float* S_out;
  const int32_t* idx_out;
  int64_t n_out;
  void* o;
};

// A lane's share of one token.
template <typename T, int D, bool KDA>
struct Token {
  static constexpr int NR = D / 8;                 // rows of a lane
  typename Vec4Raw<T>::V k[NR / 4], q[NR / 4], v;
  f32x4 g[KDA ? NR / 4 : 1];
  float g1, beta;
  __device__ inline void load(const StepArgs& A, int64_t row, int h, int col, int r) {
    const int64_t rh = row * A.H + h;
    const T* kp = static_cast<const T*>(A.k) + rh * D + r * NR;
    const T* qp = static_cast<const T*>(A.q) + rh * D + r * NR;
#pragma unroll
    for (int i = 0; i < NR / 4; ++i) {
      k[i] = Vec4Raw<T>::load(kp + 4 * i);
      q[i] = Vec4Raw<T>::load(qp + 4 * i);
    }
    v = Vec4Raw<T>::load(static_cast<const T*>(A.v) + rh * D + col);
    if constexpr (KDA) {
#pragma unroll
      for (int i = 0; i < NR / 4; ++i) g[i] = *reinterpret_cast<const f32x4*>(A.g + rh * D + r * NR + 4 * i);
      beta = A.beta[rh];
    } else {
      g1 = A.g[rh];
    }
  }
};

// Sum over the 8 row groups of a wave (lanes 8, 16 and 32 apart), in every lane,
// by moves between vector registers: a token's chain of dependent steps has two
// of these, and through LDS each exchange takes ten times as long.
__device__ inline float over_rows(float x) {
  typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
  const auto bits = [](float y) { return __builtin_bit_cast(unsigned int, y); };
  const auto val = [](unsigned int y) { return __builtin_bit_cast(float, y); };
  x += val(__builtin_amdgcn_update_dpp(0u, bits(x), 0x128, 0xf, 0xf, true));   // rotate by 8 within 16 lanes
  u32x2 p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(bits(x), bits(x), false, false));
  x = val(p[0]) + val(p[1]);
  p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(bits(x), bits(x), false, false));
  return val(p[0]) + val(p[1]);
}
__device__ inline f32x4 over_rows(const f32x4& x) {
  return f32x4{over_rows(x[0]), over_rows(x[1]), over_rows(x[2]), over_rows(x[3])};
}

template <typename T, int D, bool KDA, bool NT>
__global__ __launch_bounds__(ST_THR) void k_step(StepArgs A) {
  constexpr int NR = D / 8, SLABS = D / ST_COLS;
  const int lane = threadIdx.x & 63;
  const uint32_t unit = blockIdx.x * (ST_THR / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t head = unit / SLABS;              // sequence * H + head
  const int64_t seq = A.by_heads.div(head);
  if (seq >= A.n_seq) return;
  const int h = static_cast<int>(head - seq * A.H);
  const int r = lane >> 3, col = static_cast<int>(unit % SLABS) * ST_COLS + 4 * (lane & 7);

  int64_t src = A.idx_in ? A.idx_in[seq] : seq, dst = A.idx_out ? A.idx_out[seq] : seq;
  if (src < 0 || src >= A.n_in) src = -1;
  if (dst < 0 || dst >= A.n_out) dst = -1;
  int64_t row = seq, end = seq + 1;
  if (A.row_off) {
    row = A.row_off[seq];
    end = A.row_off[seq + 1];
  }
  if (row < 0) row = 0;
  if (end > A.n_rows) end = A.n_rows;

  const int64_t cell = static_cast<int64_t>(r) * NR * D + col;
  f32x4 S[NR];
  if (src >= 0) {
    const float* p = A.S_in + (src * A.H + h) * (D * D) + cell;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const f32x4* x = reinterpret_cast<const f32x4*>(p + i * D);
      S[i] = NT ? __builtin_nontemporal_load(x) : *x;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NR; ++i) S[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  Token<T, D, KDA> x;
  if (row < end) x.load(A, row, h, col, r);

  // an output entry that an earlier sequence names already belongs to that one
  if (A.idx_out && dst >= 0) {
    bool taken = false;
    for (int64_t j = lane; j < seq; j += 64) taken |= A.idx_out[j] == dst;
    if (__any(taken)) {
      for (; row < end; ++row)
        if (r == 0) {
          const float n = __builtin_nanf("");
          Vec4<T>::store(static_cast<T*>(A.o) + (row * A.H + h) * D + col, f32x4{n, n, n, n});
        }
      return;
    }
  }

  for (; row < end; ++row) {
    Token<T, D, KDA> y = x;
    if (row + 1 < end) x.load(A, row + 1, h, col, r);
    f32x4 v = Vec4Raw<T>::widen(y.v), o{0.f, 0.f, 0.f, 0.f};
    if constexpr (KDA) {
      // o = S_t^T q = D^T q + beta (k.q) (v - D^T k): the sums that v waits for
      // and those of o run together
      f32x4 u{0.f, 0.f, 0.f, 0.f};
      float kq = 0.f;
#pragma unroll
      for (int i = 0; i < NR / 4; ++i) {
        const f32x4 k = Vec4Raw<T>::widen(y.k[i]), q = Vec4Raw<T>::widen(y.q[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          S[4 * i + e] *= __expf(y.g[i][e]);   // (16 a lane and token; relative error about |g| 2^-24)
          u += S[4 * i + e] * k[e];
          o += S[4 * i + e] * q[e];
          kq += k[e] * q[e];
        }
      }
      v = (v - over_rows(u)) * y.beta;
      o = over_rows(o) + v * over_rows(kq);
#pragma unroll
      for (int i = 0; i < NR / 4; ++i) {
        const f32x4 k = Vec4Raw<T>::widen(y.k[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) S[4 * i + e] += v * k[e];
      }
    } else {
      const float a = expf(y.g1);
#pragma unroll
      for (int i = 0; i < NR / 4; ++i) {
        const f32x4 k = Vec4Raw<T>::widen(y.k[i]), q = Vec4Raw<T>::widen(y.q[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          S[4 * i + e] = S[4 * i + e] * a + v * k[e];
          o += S[4 * i + e] * q[e];
        }
      }
      o = over_rows(o);
    }
    o *= A.scale;
    if (r == 0) Vec4<T>::store(static_cast<T*>(A.o) + (row * A.H + h) * D + col, o);
  }

  if (dst >= 0) {
    float* p = A.S_out + (dst * A.H + h) * (D * D) + cell;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      f32x4* x = reinterpret_cast<f32x4*>(p + i * D);
      if (NT) __builtin_nontemporal_store(S[i], x);
      else *x = S[i];
    }
  }
}

bool al(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

template <bool KDA>
int step(const char* where, int32_t dtype, int32_t d, const StepArgs& A, void* stream) {
  const auto fail = [&](int code, const char* what) {
    set_error(std::string(where) + ": " + what);
    return code;
  };
  if (dtype != HARTS_BF16 && dtype != HARTS_F32) return fail(HARTS_EUNSUPPORTED, "dtype has to be bf16 or float32");
  if (A.H < 1 || A.H > 65535 || (d != 64 && d != 128))
    return fail(HARTS_EUNSUPPORTED, "need 1 <= H <= 65535 and d in {64, 128}");
  if (A.n_seq < 0 || A.n_rows < 0 || A.n_in < 0 || A.n_out < 0) return fail(HARTS_EINVAL, "negative size");
  if (std::max({A.n_seq, A.n_rows, A.n_in, A.n_out}) > INT32_MAX)
    return fail(HARTS_EUNSUPPORTED, "more than 2^31 - 1 sequences, rows or states");
  if (A.n_seq == 0) return HARTS_OK;
  if (!A.row_off && A.n_rows < A.n_seq) return fail(HARTS_EINVAL, "fewer rows than sequences without row_off");
  if (A.n_rows > 0 && (!A.q || !A.k || !A.v || !A.g || !A.o || (KDA && !A.beta)))
    return fail(HARTS_EINVAL, "NULL pointer");
  if ((A.n_in > 0 && !A.S_in) || (A.n_out > 0 && !A.S_out)) return fail(HARTS_EINVAL, "NULL state pool");
  if (!al(A.q, 16) || !al(A.k, 16) || !al(A.v, 16) || !al(A.o, 16) || !al(A.g, KDA ? 16 : 4) || !al(A.beta, 4) ||
      !al(A.S_in, 16) || !al(A.S_out, 16) || !al(A.row_off, 4) || !al(A.idx_in, 4) || !al(A.idx_out, 4))
    return fail(HARTS_EINVAL, "misaligned pointer");
  const uintptr_t in = reinterpret_cast<uintptr_t>(A.S_in), out = reinterpret_cast<uintptr_t>(A.S_out);
  const size_t state = static_cast<size_t>(A.H) * d * d * sizeof(float);
  const bool same = in == out && A.n_in == A.n_out && A.idx_in == A.idx_out;
  if (!same && A.n_in > 0 && A.n_out > 0 && in < out + A.n_out * state && out < in + A.n_in * state)
    return fail(HARTS_EINVAL, "S_out overlaps S_in (an update in place has one pool and one index)");
  // (the waves of a head read the same q, k and g, and none waits for another)
  const size_t rows = static_cast<size_t>(A.n_rows) * A.H, span = rows * d * (dtype == HARTS_BF16 ? 2 : 4);
  const size_t seqs = static_cast<size_t>(A.n_seq) * sizeof(int32_t);
  const Region o{A.o, span}, S_in{A.S_in, A.n_in * state}, S_out{A.S_out, A.n_out * state};
  const std::initializer_list<Region> inputs = {
      {A.q, span}, {A.k, span}, {A.v, span}, {A.g, rows * (KDA ? d : 1) * sizeof(float)},
      {A.beta, rows * sizeof(float)}, {A.row_off, seqs + sizeof(int32_t)}, {A.idx_in, seqs}, {A.idx_out, seqs}};
  if (overlaps_any(o, inputs)) return fail(HARTS_EINVAL, "o overlaps an input");
  if (overlaps_any(S_out, inputs)) return fail(HARTS_EINVAL, "S_out overlaps an input");
  if (overlaps_any(o, {S_in, S_out})) return fail(HARTS_EINVAL, "o overlaps a state pool");
  const int64_t blocks = (A.n_seq * A.H * (d / ST_COLS) + ST_THR / 64 - 1) / (ST_THR / 64);
  if (A.n_seq * A.H * (d / ST_COLS) > INT32_MAX - ST_THR) return fail(HARTS_EUNSUPPORTED, "too many sequences for one call");
  // States past what the last-level cache holds are not kept in it (512 sequences,
  // 16 heads of 128, two pools of 512 MiB: 214 us, 198 so; 64 sequences 23, 25 so).
  const bool nt = A.n_seq * state > (size_t{128} << 20);
  StepArgs B = A;
  B.by_heads = FastDiv(static_cast<uint32_t>(A.H));
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(ST_THR), 0, static_cast<hipStream_t>(stream), B);
  };
  const auto pick = [&](auto type, auto dim) {
    typedef decltype(type) T;
    constexpr int D = decltype(dim)::value;
    if (nt) launch(k_step<T, D, KDA, true>);
    else launch(k_step<T, D, KDA, false>);
  };
  const std::integral_constant<int, 128> d128{};
  const std::integral_constant<int, 64> d64{};
  if (dtype == HARTS_BF16) d == 128 ? pick(bf16{}, d128) : pick(bf16{}, d64);
  else d == 128 ? pick(float{}, d128) : pick(float{}, d64);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? HARTS_OK : fail(HARTS_EHIP, hipGetErrorString(e));
}

}  // namespace
}  // namespace harts

using namespace harts;

extern "C" int harts_la_step(int32_t dtype, int64_t n_seq, int64_t n_rows, int32_t H, int32_t d, float scale,
                             const void* q, const void* k, const void* v, const float* g, const int32_t* row_off,
                             const float* S_in, const int32_t* idx_in, int64_t n_in, float* S_out,
                             const int32_t* idx_out, int64_t n_out, void* o, void* stream) {
  return step<false>("harts_la_step", dtype, d,
                     {n_seq, n_rows, H, scale, {}, q, k, v, g, nullptr, row_off, S_in, idx_in, n_in, S_out, idx_out, n_out, o},
                     stream);
}

extern "C" int harts_kda_step(int32_t dtype, int64_t n_seq, int64_t n_rows, int32_t H, int32_t d, float scale,
                              const void* q, const void* k, const void* v, const float* g, const float* beta,
                              const int32_t* row_off, const float* S_in, const int32_t* idx_in, int64_t n_in,
                              float* S_out, const int32_t* idx_out, int64_t n_out, void* o, void* stream) {
  return step<true>("harts_kda_step", dtype, d,
                    {n_seq, n_rows, H, scale, {}, q, k, v, g, beta, row_off, S_in, idx_in, n_in, S_out, idx_out, n_out, o},
                    stream);
}
