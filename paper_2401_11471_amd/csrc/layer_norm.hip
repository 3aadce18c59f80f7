// Layer norm over the columns of a row, forward and backward.
//
//   forward   t = x [+ residual, rounded to the storage type],
//             xh = (t - mean) rstd, y = gamma xh + beta
//   backward  g = gamma dy, dx = rstd (g - mean(g) - xh mean(g xh)) [+ dres],
//             dgamma = sum over rows of dy xh, dbeta = sum over rows of dy
//
// Both read a row once: it stays in registers (TPR threads of NV vectors of
// eight columns) between its statistics and its result. Widths that fill their
// threads with one vector are bound by HBM: 67800 x 2048 bf16 with residual and
// checkpoint 229 us forward (5.4 TB/s), 190 and 5.5 for the join backward from the
// checkpoint (5.2 TB/s). Others are slower, bf16 forward with the checkpoint in TB/s:
// 1024 columns 4.9, 1100 2.6, 2048 5.1, 2560 3.2, 4096 4.4, 5120 2.9, 8192 3.4; float32
// 4.7 to 5.4 at all of them. One row takes 3.2 us, a launch's time. Statistics and sums are float32: the mean first,
// then the centred sum of squares, so a large mean costs no digits of the
// variance, and for float32 rows the centred sum too, so that it costs none of the
// normalised values.
#include "act8.hpp"

#include <algorithm>
#include <type_traits>

namespace lrcnn {
namespace act8 {
namespace {

constexpr int kMaxNormCols = 16384;
// Backward: blocks that each keep a running dgamma and dbeta of their rows, three
// to a CU, as many as fit with four rows in flight: 67800 x 2048 bf16 from a
// checkpoint with dres 192 us (512 blocks 224, 1024 231, 2048 209; two rows in
// flight and 1024 blocks 190, but float32 30000 x 2048 171 us to 152).
constexpr int kMaxParts = 768;
// Backward, rows of one wave or less: where four rows at a time would be fewer
// blocks than CUs, two (both launches, by four and by two, us: 1183 x 509 float32
// 10.1 and 8.3, 12000 x 33 bf16 11.7 and 10.1, 392 x 512 float32 7.6 and 7.3; by
// one 8.9, 14.6, 7.7; wider rows gain nothing, 1000 x 1024 bf16 10.3 and 10.5).
constexpr int kFewParts = 256;
// Forward: blocks that walk the rows. Rows of one vector a thread take many
// (67800 x 2048 bf16 with residual and checkpoint: 2048 blocks 267 us, 8192
// 234, 16384 230, 65536 235; 512 columns 61.8, 55.5, 55.5, 55.2), wider ones few
// (20000 x 4096 bf16: 2048 blocks 78 us, 16384 93).
constexpr int kFwdBlocks = 8192, kFwdBlocksWide = 2048;

// Sum over a wave, the same in every lane: adds inside rows of 16 lanes, then
// across rows, a fixed tree.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(
                 0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float x) {
  x = dpp_add<0x111>(x);  // row_shr 1, 2, 4, 8: lane 15 of a row has its sum
  x = dpp_add<0x112>(x);
  x = dpp_add<0x114>(x);
  x = dpp_add<0x118>(x);
  const uint32_t u = __float_as_uint(x);
  const float a = __uint_as_float(__builtin_amdgcn_readlane(u, 15));
  const float b = __uint_as_float(__builtin_amdgcn_readlane(u, 31));
  const float c = __uint_as_float(__builtin_amdgcn_readlane(u, 47));
  const float d = __uint_as_float(__builtin_amdgcn_readlane(u, 63));
  return (a + b) + (c + d);
}
// Sum over TPR <= 32 neighbouring lanes, the same in each: swaps inside four
// lanes, of the fours of eight, of the eights of sixteen, of the sixteens.
template <int CTRL>
__device__ __forceinline__ float swap_add(float x) {
  return x + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xf,
                                                                0xf, true));
}
template <int TPR>
__device__ __forceinline__ float lanes_sum(float x) {
  x = swap_add<0xb1>(x);                           // lane ^ 1
  x = swap_add<0x4e>(x);                           // lane ^ 2
  if constexpr (TPR >= 8) x = swap_add<0x141>(x);  // 7 - lane of eight
  if constexpr (TPR >= 16) x = swap_add<0x140>(x); // 15 - lane of sixteen
  if constexpr (TPR >= 32) x += __shfl_xor(x, 16);
  return x;
}
// N sums over the TPR threads of a row, by all threads of the block. `red`
// has two halves, used in turn, so one barrier a call is enough.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&s)[N], float *red, int &turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = TPR < 64 ? lanes_sum<TPR>(s[i]) : wave_sum(s[i]);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64, ALL = (TPR > 256 ? TPR : 256) / 64;  // waves of a row, a block
    float *b = red + turn * ALL * N;
    turn ^= 1;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) b[wave * N + i] = s[i];
    }
    __syncthreads();
    b += wave / W * W * N;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t = b[i];
#pragma unroll
      for (int w = 1; w < W; ++w) t += b[w * N + i];
      s[i] = t;
    }
  }
}

struct FwdArgs {
  int64_t rows;
  int cols, pitch;
  float n, eps;  // n: cols
  Mat x, res, total, y;
  const float *gamma, *beta;
  float *mean, *rstd;
  Ckpt k;
};

// A block's threads are TPR per row and hold R rows at a time.
template <typename T, int TPR, int NV, int R>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void ln_fwd_kernel(FwdArgs a) {
  constexpr int BS = TPR > 256 ? TPR : 256, RB = BS / TPR;
  constexpr int M = std::is_same<T, float>::value ? 2 : 1;  // sums over the centred row
  __shared__ float red[2 * (BS / 64) * M * R];
  int turn = 0;
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float ga[NV][8], be[NV][8];
  int n[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * TPR + t) * kVec;
    n[j] = a.cols - c;
#pragma unroll
    for (int i = 0; i < 8; ++i) ga[j][i] = 1.f, be[j][i] = 0.f;
    if (a.gamma && n[j] > 0) load8(a.gamma + c, n[j]).get(ga[j]);
    if (a.beta && n[j] > 0) load8(a.beta + c, n[j]).get(be[j]);
  }
  for (int64_t r0 = ((int64_t)blockIdx.x * RB) * R; r0 < a.rows;
       r0 += (int64_t)gridDim.x * RB * R) {
    // rows r0 + sub R + q; those past the end read the last row and store nothing
    float v[R][NV][8], s[R];
    int64_t row[R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      row[q] = min(r0 + sub * R + q, a.rows - 1);
      s[q] = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * TPR + t) * kVec;
        if (n[j] > 0) {
          load8((const T *)a.x.p + row[q] * a.x.ld + c, n[j]).get(v[q][j]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[q][j][i] = 0.f;
        }
      }
    }
    if (a.res.p) {
#pragma unroll
      for (int q = 0; q < R; ++q)
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (n[j] > 0) {
            const int c = (j * TPR + t) * kVec;
            float z[8];
            load8((const T *)a.res.p + row[q] * a.res.ld + c, n[j]).get(z);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              // the sum as the residual stream carries it
              T w;
              put(&w, v[q][j][i] + z[i]);
              v[q][j][i] = to_f(w);
            }
            if (a.total.p && r0 + sub * R + q < a.rows)
              store8((T *)a.total.p + row[q] * a.total.ld + c, n[j], v[q][j]);
          }
    }
#pragma unroll
    for (int q = 0; q < R; ++q)
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[q] += v[q][j][i];
    row_sums<TPR, R>(s, red, turn);
    // The sum of large float32 values rounds: the centred ones' own mean, all but
    // exact, corrects it (a constant row's mean becomes its value, its xh zero).
    // bfloat16 ones need none of it: with 16 bits to spare, kMaxNormCols values of
    // one binade sum exactly. (In a graph, us: 1183 x 509 float32 5.5 and 5.7, 4000
    // x 16384 219 and 224, 30000 x 2048 106 both.)
    float mu[R], m[M * R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      mu[q] = s[q] / a.n;
      m[M * q] = m[M * q + M - 1] = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          v[q][j][i] = i < n[j] ? v[q][j][i] - mu[q] : 0.f;
          m[M * q] += v[q][j][i] * v[q][j][i];
          if constexpr (M == 2) m[M * q + 1] += v[q][j][i];
        }
    }
    row_sums<TPR, M * R>(m, red, turn);
#pragma unroll
    for (int q = 0; q < R; ++q) {
      float var = m[M * q] / a.n, off = 0.f;
      if constexpr (M == 2) {
        off = m[M * q + 1] / a.n;
        mu[q] += off;
        var -= off * off;
        var = var < 0.f ? 0.f : var;  // (NaN stays)
      }
      const float rs = rsqrt_rounded(var + a.eps);
      if (r0 + sub * R + q >= a.rows) continue;
      if (t == 0) {
        if (a.mean) a.mean[row[q]] = mu[q];
        if (a.rstd) a.rstd[row[q]] = rs;
      }
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * TPR + t) * kVec;
        if (c >= a.pitch) continue;
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (M == 2) v[q][j][i] = i < n[j] ? v[q][j][i] - off : 0.f;
          v[q][j][i] *= rs;
          o[i] = fmaf(v[q][j][i], ga[j][i], be[j][i]);
        }
        if (n[j] > 0) store8((T *)a.y.p + row[q] * a.y.ld + c, n[j], o);
        if (a.k.q) put8(a.k, row[q], c, v[q][j]);
      }
    }
  }
}

struct BwdArgs {
  int64_t rows;
  int cols, pitch;
  float inv;
  Mat dy, x, dres, dx;
  const float *mean, *rstd, *gamma;
  float *part;  // [gridDim.x][2][cols], or null
  Ckpt k;
};

// CK: xh comes from its checkpoint, else from x, mean and rstd
template <typename T, bool CK, int TPR, int NV, int R>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void ln_bwd_kernel(BwdArgs a) {
  constexpr int BS = TPR > 256 ? TPR : 256, RB = BS / TPR;
  __shared__ float red[2 * (BS / 64) * 2 * R];
  int turn = 0;
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float ga[NV][8], dg[NV][8], db[NV][8];
  int n[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * TPR + t) * kVec;
    n[j] = a.cols - c;
#pragma unroll
    for (int i = 0; i < 8; ++i) ga[j][i] = 1.f, dg[j][i] = db[j][i] = 0.f;
    if (a.gamma && n[j] > 0) load8(a.gamma + c, n[j]).get(ga[j]);
  }
  for (int64_t r0 = ((int64_t)blockIdx.x * RB) * R; r0 < a.rows;
       r0 += (int64_t)gridDim.x * RB * R) {
    Raw8<T> rd[R][NV], rx[R][NV];
    uint2 rq[R][NV];
    uint32_t re[R][NV];
    float rs[R], mu[R], s[2 * R];
    int64_t row[R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      row[q] = min(r0 + sub * R + q, a.rows - 1);
      rs[q] = a.rstd[row[q]];
      if constexpr (!CK) mu[q] = a.mean[row[q]];
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * TPR + t) * kVec;
        if (n[j] <= 0) continue;
        rd[q][j] = load8((const T *)a.dy.p + row[q] * a.dy.ld + c, n[j]);
        if constexpr (CK) {
          rq[q][j] = *(const uint2 *)(a.k.q + row[q] * a.k.pitch + c);
          re[q][j] = a.k.e[row[q] * (a.k.pitch / kGroup) + c / kGroup];
        } else {
          rx[q][j] = load8((const T *)a.x.p + row[q] * a.x.ld + c, n[j]);
        }
      }
    }
    auto xhat = [&](int q, int j, float (&h)[8]) {
      if constexpr (CK) {
        decode8(rq[q][j], re[q][j], h);
      } else {
        rx[q][j].get(h);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = i < n[j] ? (h[i] - mu[q]) * rs[q] : 0.f;
      }
    };
#pragma unroll
    for (int q = 0; q < R; ++q) {
      s[2 * q] = s[2 * q + 1] = 0.f;
      const bool in = r0 + sub * R + q < a.rows;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (n[j] <= 0) continue;
        float d[8], h[8];
        rd[q][j].get(d);
        xhat(q, j, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float g = d[i] * ga[j][i];
          s[2 * q] += g;
          s[2 * q + 1] += g * h[i];
          if (in) {
            dg[j][i] += d[i] * h[i];
            db[j][i] += d[i];
          }
        }
      }
    }
    row_sums<TPR, 2 * R>(s, red, turn);
#pragma unroll
    for (int q = 0; q < R; ++q) {
      if (r0 + sub * R + q >= a.rows) continue;
      const float m1 = s[2 * q] * a.inv, m2 = s[2 * q + 1] * a.inv;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * TPR + t) * kVec;
        if (n[j] <= 0) continue;
        float d[8], h[8], o[8];
        rd[q][j].get(d);
        xhat(q, j, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = rs[q] * (d[i] * ga[j][i] - m1 - h[i] * m2);
        if (a.dres.p) {
          float z[8];
          load8((const T *)a.dres.p + row[q] * a.dres.ld + c, n[j]).get(z);
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] += z[i];
        }
        store8((T *)a.dx.p + row[q] * a.dx.ld + c, n[j], o);
      }
    }
  }
  if (!a.part) return;
  // a block's rows joined in the order of its row slots
  float *pg = a.part + (int64_t)blockIdx.x * 2 * a.cols;
  if constexpr (RB == 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (n[j] > 0) {
        const int c = (j * TPR + t) * kVec;
        store8(pg + c, n[j], dg[j]);
        store8(pg + a.cols + c, n[j], db[j]);
      }
  } else {
    __shared__ float join[RB][TPR][16];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) join[sub][t][i] = dg[j][i], join[sub][t][8 + i] = db[j][i];
      __syncthreads();
      if (sub == 0 && n[j] > 0) {
        const int c = (j * TPR + t) * kVec;
        float g[8], b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          g[i] = join[0][t][i], b[i] = join[0][t][8 + i];
#pragma unroll
          for (int w = 1; w < RB; ++w) g[i] += join[w][t][i], b[i] += join[w][t][8 + i];
        }
        store8(pg + c, n[j], g);
        store8(pg + a.cols + c, n[j], b);
      }
    }
  }
}

// dgamma, dbeta = [their value +] the sum over the blocks' parts in a fixed
// order: 16 groups of 16 threads take the parts p = g, g + 16, ... of 16
// columns, then the groups' sums are added in order.
__global__ __launch_bounds__(256) void ln_join_kernel(const float *part, int parts, int cols,
                                                      float *dgamma, float *dbeta,
                                                      int accumulate) {
  __shared__ float red[16][17];
  const int g = threadIdx.x >> 4, e = threadIdx.x & 15;
  const int i = blockIdx.x * 16 + e;
  float s = 0.f;
  if (i < 2 * cols) {
#pragma unroll 8
    for (int p = g; p < parts; p += 16) s += part[(int64_t)p * 2 * cols + i];
  }
  red[g][e] = s;
  __syncthreads();
  if (g == 0 && i < 2 * cols) {
#pragma unroll
    for (int k = 1; k < 16; ++k) s += red[k][e];
    float *out = i < cols ? dgamma : dbeta;
    const int c = i < cols ? i : i - cols;
    if (out) out[c] = accumulate ? out[c] + s : s;
  }
}

// Threads and vectors of a row: four to sixty-four lanes up to 512 columns, so
// that narrow rows share a wave, two waves up to 1024, four up to 8192, eight
// beyond. (1000000 rows bf16 forward, one wave a row and as here, us: 17 columns
// 238 and 25, 64 columns 228 and 46; 500000 x 200 164 and 87.)
template <typename F>
void by_width(int cols, F &&f) {
  using std::integral_constant;
  auto go = [&](auto tpr, auto nv) { f(tpr, nv); };
#define W(t, v) go(integral_constant<int, t>(), integral_constant<int, v>())
  if (cols <= 32) W(4, 1);
  else if (cols <= 64) W(8, 1);
  else if (cols <= 128) W(16, 1);
  else if (cols <= 256) W(32, 1);
  else if (cols <= 512) W(64, 1);
  else if (cols <= 1024) W(128, 1);
  else if (cols <= 2048) W(256, 1);
  else if (cols <= 4096) W(256, 2);
  else if (cols <= 8192) W(256, 4);
  else W(512, 4);
#undef W
}

int parts_of(int64_t rows) { return (int)std::min<int64_t>(std::max<int64_t>(rows, 1), kMaxParts); }

int norm_shape(int64_t rows, int64_t cols, int32_t dtype) {
  const int st = take_shape(rows, cols, dtype);
  if (st != LRCNN_OK) return st;
  if (cols > kMaxNormCols)
    return refuse(LRCNN_ESHAPE, "layer norm takes at most ", kMaxNormCols, " columns");
  return LRCNN_OK;
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

extern "C" int lrcnn_layer_norm_forward(int64_t rows, int64_t cols, int32_t dtype, const void *x,
                                        int64_t ldx, const void *residual, int64_t ldr,
                                        const float *gamma, const float *beta, float eps,
                                        void *total, int64_t ldt, void *y, int64_t ldy,
                                        float *mean, float *rstd, void *ckpt, void *stream) {
  TRY(norm_shape(rows, cols, dtype));
  if (!(eps >= 0.f) || !(eps < INFINITY))
    return refuse(LRCNN_EINVAL, "eps must be finite and not negative");
  if (total && !residual) return refuse(LRCNN_EINVAL, "total goes with residual");
  if (rows == 0) return LRCNN_OK;
  const int es = dtype == LRCNN_BF16 ? 2 : 4;
  FwdArgs a{};
  TRY(take("x", x, ldx, cols, es, true, &a.x));
  TRY(take("residual", residual, ldr, cols, es, false, &a.res));
  TRY(take("total", total, ldt, cols, es, false, &a.total));
  TRY(take("y", y, ldy, cols, es, true, &a.y));
  TRY(take_f32("gamma", gamma, false));
  TRY(take_f32("beta", beta, false));
  TRY(take_f32("mean", mean, false));
  TRY(take_f32("rstd", rstd, false));
  TRY(take_ckpt("ckpt", ckpt, false));
  a.rows = rows, a.cols = (int)cols, a.pitch = (int)pitch_of(cols);
  a.n = (float)cols, a.eps = eps;
  a.gamma = gamma, a.beta = beta, a.mean = mean, a.rstd = rstd;
  a.k = ckpt_of(ckpt, rows, cols);
  by_width((int)cols, [&](auto tpr, auto nv) {
    constexpr int TPR = tpr.value, NV = nv.value, BS = TPR > 256 ? TPR : 256;
    constexpr int R = NV == 1 ? 2 : 1;
    const int64_t per = (int64_t)(BS / TPR) * R;
    const int64_t most = (NV == 1 ? kFwdBlocks : kFwdBlocksWide) * 256 / BS;
    const unsigned g = (unsigned)std::min<int64_t>((rows + per - 1) / per, most);
    if (dtype == LRCNN_BF16)
      ln_fwd_kernel<bf16, TPR, NV, R><<<g, BS, 0, (hipStream_t)stream>>>(a);
    else
      ln_fwd_kernel<float, TPR, NV, R><<<g, BS, 0, (hipStream_t)stream>>>(a);
  });
  return launched("layer_norm_forward");
}

extern "C" int lrcnn_layer_norm_workspace_bytes(int64_t rows, int64_t cols, size_t *bytes) {
  if (!bytes) return refuse(LRCNN_EINVAL, "null output");
  TRY(norm_shape(rows, cols, LRCNN_F32));
  *bytes = a256((size_t)parts_of(rows) * 2 * (size_t)cols * 4);
  return LRCNN_OK;
}

extern "C" int lrcnn_layer_norm_backward(int64_t rows, int64_t cols, int32_t dtype,
                                         const void *dy, int64_t lddy, const void *x, int64_t ldx,
                                         const float *mean, const void *ckpt, const float *rstd,
                                         const float *gamma, const void *dres, int64_t lddr,
                                         void *dx, int64_t lddx, float *dgamma, float *dbeta,
                                         int32_t accumulate, void *workspace, size_t ws_bytes,
                                         void *stream) {
  TRY(norm_shape(rows, cols, dtype));
  const int es = dtype == LRCNN_BF16 ? 2 : 4;
  BwdArgs a{};
  TRY(take_f32("dgamma", dgamma, false));
  TRY(take_f32("dbeta", dbeta, false));
  const bool grads = dgamma || dbeta;
  if (rows) {
    if ((x != nullptr) == (ckpt != nullptr) || (x != nullptr) != (mean != nullptr))
      return refuse(LRCNN_EINVAL, "give x with mean, or ckpt");
    TRY(take("dy", dy, lddy, cols, es, true, &a.dy));
    TRY(take("x", x, ldx, cols, es, false, &a.x));
    TRY(take("dres", dres, lddr, cols, es, false, &a.dres));
    TRY(take("dx", dx, lddx, cols, es, true, &a.dx));
    TRY(take_f32("mean", mean, false));
    TRY(take_f32("rstd", rstd, true));
    TRY(take_f32("gamma", gamma, false));
    TRY(take_ckpt("ckpt", ckpt, false));
  }
  const size_t need = a256((size_t)parts_of(rows) * 2 * (size_t)cols * 4);
  if (grads && (!workspace || ((uintptr_t)workspace & 15)))
    return refuse(LRCNN_EINVAL, "workspace null or misaligned");
  if (grads && ws_bytes < need)
    return refuse(LRCNN_EWORKSPACE, "workspace needs ", need, " bytes, got ", ws_bytes);
  hipStream_t s = (hipStream_t)stream;
  int parts = 0;
  if (rows) {
    a.rows = rows, a.cols = (int)cols, a.pitch = (int)pitch_of(cols);
    a.inv = 1.f / (float)cols;
    a.mean = mean, a.rstd = rstd, a.gamma = gamma;
    a.part = grads ? (float *)workspace : nullptr;
    a.k = ckpt_of(ckpt, rows, cols);
    by_width((int)cols, [&](auto tpr, auto nv) {
      constexpr int TPR = tpr.value, NV = nv.value, BS = TPR > 256 ? TPR : 256;
      auto run = [&](auto *tp, auto ck) {
        using T = std::remove_pointer_t<decltype(tp)>;
        auto with = [&](auto r) {  // r rows of a group of threads at a time
          const int64_t per = (int64_t)(BS / TPR) * r.value;
          parts = (int)std::min<int64_t>((rows + per - 1) / per, kMaxParts);
          ln_bwd_kernel<T, ck.value, TPR, NV, r.value><<<parts, BS, 0, s>>>(a);
        };
        if constexpr (TPR <= 64) {
          if (rows <= (int64_t)(BS / TPR) * 4 * kFewParts)
            return with(std::integral_constant<int, 2>());
        }
        with(std::integral_constant<int, NV == 1 ? 4 : 1>());
      };
      if (dtype == LRCNN_BF16) {
        if (ckpt) run((bf16 *)nullptr, std::true_type());
        else run((bf16 *)nullptr, std::false_type());
      } else {
        if (ckpt) run((float *)nullptr, std::true_type());
        else run((float *)nullptr, std::false_type());
      }
    });
  }
  if (grads)
    ln_join_kernel<<<(unsigned)((2 * cols + 15) / 16), 256, 0, s>>>((const float *)workspace, parts,
                                                                    (int)cols, dgamma, dbeta,
                                                                    accumulate != 0);
  return launched("layer_norm_backward");
}
