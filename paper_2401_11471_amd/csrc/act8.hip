// Pack and unpack of 8-bit activation checkpoints, and the activations of a
// feed-forward block with checkpoints beside their forward pass and in place
// of their inputs in the backward pass.
//
// Two to five streams of 1 to 4 bytes an element, a dozen operations each: HBM
// bounds pack, unpack and the silus. A thread takes eight columns (16 bytes of bfloat16), so a
// quad of lanes holds a group and its maximum takes two quad moves. Calls one
// after the other in a graph (a device copy of 4 GiB runs at 4.84 TB/s): 1080000 x
// 512 bf16 pack 300 to 315 us, 5.3 to 5.6 TB/s, unpack 290; gated silu, 67800 x 8192
// bf16, 563 us, 5.9 TB/s; gelu there 490 us, with a checkpoint 572, 4.6 and 4.9 TB/s,
// bound by its vector instructions (0.29 a cycle and SIMD counted, where a kernel at
// the memory's rate has 0.15), from x backward 600 us, 5.5 TB/s; gated silu backward
// from checkpoints, 3136 x 2731 bf16, 17 to 19 us, 4.0 to 4.6 TB/s, partly from the Infinity
// Cache. Eight columns a thread and a thread's rows one after the other: the loads
// of many waves, not of one, cover the latency. A call of one row takes 2.7 us, a
// launch's time.
#include "act8.hpp"

#include <type_traits>

namespace lrcnn {
namespace act8 {
namespace {

// Walk of a kernel over [rows][pitch]: blockIdx.x picks 256 / rpb vectors of
// a row, blockIdx.y a run of rows, rpb rows to a block (a power of two).
struct Walk {
  int64_t rows, cols, pitch;
  int tpr, rpb;  // threads per row, rows per block
};
struct Grid {
  Walk w;
  dim3 grid;
};
Grid walk(int64_t rows, int64_t cols) {
  Grid g;
  g.w.rows = rows, g.w.cols = cols, g.w.pitch = pitch_of(cols);
  const int64_t vecs = g.w.pitch / kVec;
  g.w.tpr = 4;
  while (g.w.tpr < 256 && g.w.tpr < vecs) g.w.tpr *= 2;
  g.w.rpb = 256 / g.w.tpr;
  const int64_t by = (rows + g.w.rpb - 1) / g.w.rpb;
  g.grid = dim3((unsigned)((vecs + g.w.tpr - 1) / g.w.tpr), (unsigned)(by < 65535 ? by : 65535));
  return g;
}
#define FOR_ROWS(w, r, c)                                                               \
  const int64_t c = ((int64_t)blockIdx.x * w.tpr + threadIdx.x % w.tpr) * kVec;         \
  if (c < w.pitch)                                                                      \
    for (int64_t r = (int64_t)blockIdx.y * w.rpb + threadIdx.x / w.tpr; r < w.rows;     \
         r += (int64_t)gridDim.y * w.rpb)

// A matrix whose rows follow each other without a gap and whose width is a
// whole number of groups is one row: the checkpoint has the same bytes. (Up to
// 2^33 columns: the grid's x dimension takes 2^24 blocks.)
template <int N>
void join_rows(int64_t *rows, int64_t *cols, Mat (&m)[N]) {
  if (*cols % kGroup || *cols * *rows > ((int64_t)1 << 33)) return;
  for (const Mat &x : m)
    if (x.p && x.ld != *cols) return;
  *cols *= *rows;
  *rows = 1;
}

template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(Walk w, const T *x, int64_t ldx, Ckpt k) {
  FOR_ROWS(w, r, c) {
    float v[8];
    load8(x + r * ldx + c, w.cols - c).get(v);
    put8(k, r, c, v);
  }
}
template <typename T>
__global__ __launch_bounds__(256) void unpack_kernel(Walk w, Ckpt k, T *y, int64_t ldy) {
  FOR_ROWS(w, r, c) {
    float v[8];
    get8(k, r, c, v);
    store8(y + r * ldy + c, w.cols - c, v);
  }
}

// ------------------------------------------------------------ activations
// 1 / (1 + exp(-x)), exp(-x) = 2^(-x log2 e)
__device__ __forceinline__ float sigmoid(float x) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * x));
}
// f(u) and f'(u). An argument beyond +-100 counts as +-100 in the factors that
// are then 0 or 1 (so that an infinity takes the function's limit); NaN stays.
// gelu: u Phi(u), Phi(-|u|) = exp(-u^2/2) R(|u|), R the Mills ratio over
// sqrt(2 pi), here t P(t) with t = 1 / (1 + 0.3 |u|) and P of degree 7 fitted
// over [0, 14] to 1.5e-7 of R (4.4e-7 as evaluated in float32). The exponential's
// argument is rounded to float32, which adds some u^2 2^-25 of the value (1.4e-6
// at -5, 8e-6 at -13); that of the other two likewise. Below -87, where 1 / (1 +
// exp(-u)) is subnormal, silu is 0. tanh form: u s(2 k (u + 0.044715 u^3)), k =
// sqrt(2 / pi).
template <int KIND>
__device__ __forceinline__ void activate(float u, float &f, float &df) {
  if constexpr (KIND == LRCNN_ACT_RELU) {
    f = u > 0.f || u != u ? u : 0.f;
    df = u > 0.f ? 1.f : u != u ? u : 0.f;
    return;
  }
  const float lo = u < -100.f ? -100.f : u;
  const float x = lo > 100.f ? 100.f : lo;
  if constexpr (KIND == LRCNN_ACT_SILU) {
    const float s = sigmoid(x);
    f = lo * s;
    df = s + x * s * (1.f - s);
  } else if constexpr (KIND == LRCNN_ACT_GELU) {
    const float z = fabsf(x);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, z, 1.f));
    const float e = __builtin_amdgcn_exp2f(-0.72134752f * z * z);
    float p = 0.03567478433251381f;
    p = fmaf(p, t, -0.15720312297344208f);
    p = fmaf(p, t, 0.2063535749912262f);
    p = fmaf(p, t, -0.053683701902627945f);
    p = fmaf(p, t, 0.12856166064739227f);
    p = fmaf(p, t, 0.09991348534822464f);
    p = fmaf(p, t, 0.12075395882129669f);
    p = fmaf(p, t, 0.11962930113077164f);
    const float q = e * (t * p);
    const float phi = x < 0.f ? q : 1.f - q;
    f = lo * phi;
    df = fmaf(x, 0.3989422804f * e, phi);
  } else {
    constexpr float k2 = 1.5957691216f, b = 0.044715f;
    const float x2 = x * x;
    const float s = sigmoid(k2 * x * fmaf(b, x2, 1.f));
    f = lo * s;
    df = s + x * s * (1.f - s) * k2 * fmaf(3.f * b, x2, 1.f);
  }
}

struct ActArgs {
  Walk w;
  Mat a, da, u, v, du, dv;
  Ckpt ku, kv, ka;
};

template <typename T>
__device__ __forceinline__ const T *at(const Mat &m, int64_t r, int64_t c) {
  return (const T *)m.p + r * m.ld + c;
}

template <typename T, int KIND, bool GATED>
__global__ __launch_bounds__(256) void act_fwd_kernel(ActArgs a) {
  FOR_ROWS(a.w, r, c) {
    const int64_t n = a.w.cols - c;
    float u[8], v[8], f[8];
    const Raw8<T> ru = load8(at<T>(a.u, r, c), n);
    if constexpr (GATED) load8(at<T>(a.v, r, c), n).get(v);
    ru.get(u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float df;
      activate<KIND>(u[i], f[i], df);
      if constexpr (GATED) f[i] *= v[i];
    }
    if (a.a.p) store8((T *)at<T>(a.a, r, c), n, f);
    if (a.ku.q) put8(a.ku, r, c, u);
    if constexpr (GATED)
      if (a.kv.q) put8(a.kv, r, c, v);
    if (a.ka.q) put8(a.ka, r, c, f);
  }
}

// du = da f'(u) [v], dv = da f(u); CK: u and v come from their checkpoints
template <typename T, int KIND, bool GATED, bool CK>
__global__ __launch_bounds__(256) void act_bwd_kernel(ActArgs a) {
  FOR_ROWS(a.w, r, c) {
    const int64_t n = a.w.cols - c;
    float d[8], u[8], v[8];
    const Raw8<T> rd = load8(at<T>(a.da, r, c), n);
    if constexpr (CK) {
      get8(a.ku, r, c, u);
      if constexpr (GATED) get8(a.kv, r, c, v);
    } else {
      load8(at<T>(a.u, r, c), n).get(u);
      if constexpr (GATED) load8(at<T>(a.v, r, c), n).get(v);
    }
    rd.get(d);
    float du[8], dv[8], f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float df;
      activate<KIND>(u[i], f[i], df);
      if constexpr (GATED) {
        du[i] = d[i] * df * v[i];
        dv[i] = d[i] * f[i];
        f[i] *= v[i];
      } else {
        du[i] = d[i] * df;
      }
    }
    store8((T *)at<T>(a.du, r, c), n, du);
    if constexpr (GATED) store8((T *)at<T>(a.dv, r, c), n, dv);
    if (a.ka.q) put8(a.ka, r, c, f);
  }
}

template <typename F>
int by_kind(int32_t kind, F &&f) {
  switch (kind) {
    case LRCNN_ACT_RELU: return f(std::integral_constant<int, LRCNN_ACT_RELU>());
    case LRCNN_ACT_GELU: return f(std::integral_constant<int, LRCNN_ACT_GELU>());
    case LRCNN_ACT_GELU_TANH: return f(std::integral_constant<int, LRCNN_ACT_GELU_TANH>());
    case LRCNN_ACT_SILU: return f(std::integral_constant<int, LRCNN_ACT_SILU>());
  }
  return refuse(LRCNN_EINVAL, "unknown activation");
}

}  // namespace
}  // namespace act8
}  // namespace lrcnn

using namespace lrcnn::act8;
#define TRY(x)                         \
  do {                                 \
    const int st_ = (x);               \
    if (st_ != LRCNN_OK) return st_;   \
  } while (0)

extern "C" int lrcnn_act8_bytes(int64_t rows, int64_t cols, size_t *bytes) {
  if (!bytes) return refuse(LRCNN_EINVAL, "null output");
  TRY(take_shape(rows, cols, LRCNN_F32));
  *bytes = ckpt_bytes(rows, cols);
  return LRCNN_OK;
}

extern "C" int lrcnn_act8_pack(int64_t rows, int64_t cols, int32_t dtype, const void *x,
                               int64_t ldx, void *ckpt, void *stream) {
  TRY(take_shape(rows, cols, dtype));
  if (rows == 0) return LRCNN_OK;
  Mat m[1];
  TRY(take("x", x, ldx, cols, dtype == LRCNN_BF16 ? 2 : 4, true, &m[0]));
  TRY(take_ckpt("ckpt", ckpt, true));
  const Ckpt k0 = ckpt_of(ckpt, rows, cols);
  Ckpt k = k0;
  join_rows(&rows, &cols, m);
  k.pitch = pitch_of(cols);
  const Grid g = walk(rows, cols);
  hipStream_t s = (hipStream_t)stream;
  if (dtype == LRCNN_BF16)
    pack_kernel<bf16><<<g.grid, 256, 0, s>>>(g.w, (const bf16 *)m[0].p, m[0].ld, k);
  else
    pack_kernel<float><<<g.grid, 256, 0, s>>>(g.w, (const float *)m[0].p, m[0].ld, k);
  return launched("act8_pack");
}

extern "C" int lrcnn_act8_unpack(int64_t rows, int64_t cols, int32_t dtype, const void *ckpt,
                                 void *y, int64_t ldy, void *stream) {
  TRY(take_shape(rows, cols, dtype));
  if (rows == 0) return LRCNN_OK;
  Mat m[1];
  TRY(take_ckpt("ckpt", ckpt, true));
  TRY(take("y", y, ldy, cols, dtype == LRCNN_BF16 ? 2 : 4, true, &m[0]));
  Ckpt k = ckpt_of(ckpt, rows, cols);
  join_rows(&rows, &cols, m);
  k.pitch = pitch_of(cols);
  const Grid g = walk(rows, cols);
  hipStream_t s = (hipStream_t)stream;
  if (dtype == LRCNN_BF16)
    unpack_kernel<bf16><<<g.grid, 256, 0, s>>>(g.w, k, (bf16 *)m[0].p, m[0].ld);
  else
    unpack_kernel<float><<<g.grid, 256, 0, s>>>(g.w, k, (float *)m[0].p, m[0].ld);
  return launched("act8_unpack");
}

extern "C" int lrcnn_activation_forward(int64_t rows, int64_t cols, int32_t dtype, int32_t kind,
                                        const void *u, int64_t ldu, const void *v, int64_t ldv,
                                        void *a, int64_t lda, void *ckpt_u, void *ckpt_v,
                                        void *ckpt_a, void *stream) {
  TRY(take_shape(rows, cols, dtype));
  const int es = dtype == LRCNN_BF16 ? 2 : 4;
  if (kind < LRCNN_ACT_RELU || kind > LRCNN_ACT_SILU)
    return refuse(LRCNN_EINVAL, "unknown activation");
  if (ckpt_v && !v) return refuse(LRCNN_EINVAL, "ckpt_v without v");
  if (rows == 0) return LRCNN_OK;
  if (!a && !ckpt_u && !ckpt_v && !ckpt_a)
    return refuse(LRCNN_EINVAL, "activation_forward: no output");
  Mat m[3];  // u, v, a
  TRY(take("u", u, ldu, cols, es, true, &m[0]));
  TRY(take("v", v, ldv, cols, es, false, &m[1]));
  TRY(take("a", a, lda, cols, es, false, &m[2]));
  TRY(take_ckpt("ckpt_u", ckpt_u, false));
  TRY(take_ckpt("ckpt_v", ckpt_v, false));
  TRY(take_ckpt("ckpt_a", ckpt_a, false));
  ActArgs g{};
  g.ku = ckpt_of(ckpt_u, rows, cols);
  g.kv = ckpt_of(ckpt_v, rows, cols);
  g.ka = ckpt_of(ckpt_a, rows, cols);
  join_rows(&rows, &cols, m);
  g.ku.pitch = g.kv.pitch = g.ka.pitch = pitch_of(cols);
  g.u = m[0], g.v = m[1], g.a = m[2];
  const Grid wk = walk(rows, cols);
  g.w = wk.w;
  return by_kind(kind, [&](auto K) {
    auto run = [&](auto *t) {
      using T = std::remove_pointer_t<decltype(t)>;
      if (v) act_fwd_kernel<T, K.value, true><<<wk.grid, 256, 0, (hipStream_t)stream>>>(g);
      else act_fwd_kernel<T, K.value, false><<<wk.grid, 256, 0, (hipStream_t)stream>>>(g);
    };
    if (dtype == LRCNN_BF16) run((bf16 *)nullptr);
    else run((float *)nullptr);
    return launched("activation_forward");
  });
}

extern "C" int lrcnn_activation_backward(int64_t rows, int64_t cols, int32_t dtype, int32_t kind,
                                         const void *da, int64_t ldda, const void *u, int64_t ldu,
                                         const void *v, int64_t ldv, const void *ckpt_u,
                                         const void *ckpt_v, void *du, int64_t lddu, void *dv,
                                         int64_t lddv, void *ckpt_a, void *stream) {
  TRY(take_shape(rows, cols, dtype));
  const int es = dtype == LRCNN_BF16 ? 2 : 4;
  if (kind < LRCNN_ACT_RELU || kind > LRCNN_ACT_SILU)
    return refuse(LRCNN_EINVAL, "unknown activation");
  const bool ck = ckpt_u != nullptr, gated = v || ckpt_v;
  if (rows == 0) return LRCNN_OK;
  if ((u != nullptr) == ck || (gated && ((ckpt_v != nullptr) != ck || (v != nullptr) == ck)))
    return refuse(LRCNN_EINVAL, "give u (and v) either full-width or as checkpoints");
  if (gated != (dv != nullptr)) return refuse(LRCNN_EINVAL, "dv goes with v or ckpt_v");
  Mat m[5];  // da, u, v, du, dv
  TRY(take("da", da, ldda, cols, es, true, &m[0]));
  TRY(take("u", u, ldu, cols, es, false, &m[1]));
  TRY(take("v", v, ldv, cols, es, false, &m[2]));
  TRY(take("du", du, lddu, cols, es, true, &m[3]));
  TRY(take("dv", dv, lddv, cols, es, false, &m[4]));
  TRY(take_ckpt("ckpt_u", ckpt_u, false));
  TRY(take_ckpt("ckpt_v", ckpt_v, false));
  TRY(take_ckpt("ckpt_a", ckpt_a, false));
  ActArgs g{};
  g.ku = ckpt_of(ckpt_u, rows, cols);
  g.kv = ckpt_of(ckpt_v, rows, cols);
  g.ka = ckpt_of(ckpt_a, rows, cols);
  join_rows(&rows, &cols, m);
  g.ku.pitch = g.kv.pitch = g.ka.pitch = pitch_of(cols);
  g.da = m[0], g.u = m[1], g.v = m[2], g.du = m[3], g.dv = m[4];
  const Grid wk = walk(rows, cols);
  g.w = wk.w;
  return by_kind(kind, [&](auto K) {
    hipStream_t s = (hipStream_t)stream;
    auto run = [&](auto *t, auto ckc) {
      using T = std::remove_pointer_t<decltype(t)>;
      if (gated) act_bwd_kernel<T, K.value, true, ckc.value><<<wk.grid, 256, 0, s>>>(g);
      else act_bwd_kernel<T, K.value, false, ckc.value><<<wk.grid, 256, 0, s>>>(g);
    };
    auto typed = [&](auto *t) {
      if (ck) run(t, std::true_type());
      else run(t, std::false_type());
    };
    if (dtype == LRCNN_BF16) typed((bf16 *)nullptr);
    else typed((float *)nullptr);
    return launched("activation_backward");
  });
}
