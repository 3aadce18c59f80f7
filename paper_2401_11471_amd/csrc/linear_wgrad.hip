// Weight and bias gradient of a linear layer whose input is an 8-bit
// checkpoint: with x[m][k] = scale[k] q[m][k] + shift[k] (q: what the
// checkpoint stands for),
//   S[n][k]  = sum over rows m of dy[m][n] q[m][k],
//   db[n]    = sum over rows m of dy[m][n],
//   dW[n][k] = scale[k] S[n][k] + shift[k] db[n].
// So the checkpoint of a norm's normalised rows serves the norm's backward pass
// and the weight gradient of the linear layer behind it.
//
// q is a bfloat16 number, so S is a bfloat16 matrix product that rounds only
// its float32 sums. A float32 dy is cut into three bfloat16 pieces (8 bits
// each of its 24-bit significand, by truncation: exact) and three products are
// summed, all into the same float32 accumulator.
#include "act8.hpp"
#include "kdev.hpp"

#include <algorithm>
#include <type_traits>

namespace lrcnn {
namespace act8 {
namespace {

constexpr int kTile = 128, kStep = 32;  // tile of dW (n and k), rows per step

struct WgArgs {
  int64_t rows;
  int n, k;             // outputs, inputs
  int64_t chunk;        // rows per split
  Mat dy;
  Ckpt q;
  const float *scale, *shift;
  float *dw, *db;
  float *part, *dbpart;  // [splits][n][k], [splits][n]; null with one split
  int accumulate;
};

// hi + mid + lo == v (hi alone where v is not finite)
__device__ __forceinline__ void cut3(float v, float (&p)[3]) {
  p[0] = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
  const float r = (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u ? 0.f : v - p[0];
  p[1] = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
  p[2] = r - p[1];
}

template <typename T>
__global__ __launch_bounds__(256, 2) void wgrad8_kernel(WgArgs a) {
  constexpr int P = std::is_same<T, float>::value ? 3 : 1;
  using M = KM<bf16, kTile>;
  __shared__ __align__(16) bf16 As[2][P][kStep * kTile];
  __shared__ __align__(16) bf16 Bs[2][kStep * kTile];
  __shared__ float dbs[kTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const TileId tl = xcd_tile(false);
  const int n0 = tl.x * kTile, k0 = tl.y * kTile;
  const int64_t m0 = (int64_t)tl.z * a.chunk, m1 = min(a.rows, m0 + a.chunk);
  // dy: rows ar, ar + 16 of a step, columns an .. an + 7; codes: row br,
  // columns bk .. bk + 15
  const int ar = tid >> 4, an = (tid & 15) * 8;
  const int br = tid >> 3, bk = (tid & 7) * 16;
  const int64_t nleft = a.n - (n0 + an);
  const bool kin = k0 + bk < a.q.pitch;
  Raw8<T> ra[2];
  uint4 rb;
  uint32_t re;
  auto gload = [&](int64_t m) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t r = m + ar + 16 * i;
      ra[i] = load8((const T *)a.dy.p + r * a.dy.ld + n0 + an, r < m1 ? nleft : 0);
    }
    const int64_t r = m + br;
    rb = make_uint4(0, 0, 0, 0);
    re = 7;
    if (r < m1 && kin) {
      rb = *(const uint4 *)(a.q.q + r * a.q.pitch + k0 + bk);
      re = a.q.e[r * (a.q.pitch / kGroup) + (k0 + bk) / kGroup];
    }
  };
  float dbv[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dbv[i] = 0.f;
  auto store = [&](int st) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float v[8];
      ra[i].get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) dbv[e] += v[e];
      const int at = M::off(ar + 16 * i, an);
      if constexpr (P == 1) {
        *(uint4 *)&As[st][0][at] = make_uint4(ra[i].w[0], ra[i].w[1], ra[i].w[2], ra[i].w[3]);
      } else {
        float c[8][3];
#pragma unroll
        for (int e = 0; e < 8; ++e) cut3(v[e], c[e]);
#pragma unroll
        for (int p = 0; p < P; ++p)
          *(uint4 *)&As[st][p][at] =
              make_uint4(bf_pair(c[0][p], c[1][p]), bf_pair(c[2][p], c[3][p]),
                         bf_pair(c[4][p], c[5][p]), bf_pair(c[6][p], c[7][p]));
      }
    }
    float q[16];
    const float s = step_of(re);
    decode4(rb.x, s, q), decode4(rb.y, s, q + 4), decode4(rb.z, s, q + 8), decode4(rb.w, s, q + 12);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *(uint4 *)&Bs[st][M::off(br, bk + 8 * h)] =
          make_uint4(bf_pair(q[8 * h], q[8 * h + 1]), bf_pair(q[8 * h + 2], q[8 * h + 3]),
                     bf_pair(q[8 * h + 4], q[8 * h + 5]), bf_pair(q[8 * h + 6], q[8 * h + 7]));
  };
  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  const int wn = (wave & 1) * 64, wk = (wave >> 1) * 64;
  if (m0 < m1) {
    gload(m0);
    store(0);
  }
  __syncthreads();
  int st = 0;
  for (int64_t m = m0; m < m1; m += kStep) {
    const bool more = m + kStep < m1;
    if (more) gload(m + kStep);
    bf16x8 b[2][2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int s = 0; s < 2; ++s) b[j][s] = ld_tr8<kTile, 2>(Bs[st], wk + 32 * j, s, lane);
#pragma unroll
    for (int p = P - 1; p >= 0; --p)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const bf16x8 f = ld_tr8<kTile, 2>(As[st][p], wn + 32 * i, s, lane);
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, b[j][s], acc[i][j], 0, 0, 0);
        }
    if (more) store(st ^ 1);
    __syncthreads();
    st ^= 1;
  }
  // db of the tile's columns: the 16 row slots added in order
  float *slots = (float *)&As[0][0][0];  // [16][128]
#pragma unroll
  for (int e = 0; e < 8; ++e) slots[ar * kTile + an + e] = dbv[e];
  __syncthreads();
  if (tid < kTile) {
    float s = 0.f;
    for (int r = 0; r < 16; ++r) s += slots[r * kTile + tid];
    dbs[tid] = s;
    const int nn = n0 + tid;
    if (tl.y == 0 && nn < a.n) {
      if (a.part) a.dbpart[(int64_t)tl.z * a.n + nn] = s;
      else if (a.db) a.db[nn] = a.accumulate ? a.db[nn] + s : s;
    }
  }
  __syncthreads();
  float *out = a.part ? a.part + (int64_t)tl.z * a.n * a.k : a.dw;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int kk = k0 + wk + 32 * j + (lane & 31);
    if (kk >= a.k) continue;
    const float sc = a.scale && !a.part ? a.scale[kk] : 1.f;
    const float sh = a.shift && !a.part ? a.shift[kk] : 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int nl = wn + 32 * i + acc_row(v, lane);
        if (n0 + nl >= a.n) continue;
        float *d = out + (int64_t)(n0 + nl) * a.k + kk;
        float r = acc[i][j][v];
        if (!a.part) {
          if (a.scale) r *= sc;
          if (a.shift) r = fmaf(sh, dbs[nl], r);
          if (a.accumulate) r += *d;
        }
        *d = r;
      }
  }
}

// dW and db from the splits' sums, added in a fixed order: eight groups of 32
// threads take the splits z = g, g + 8, ... of 32 vectors of V columns, then
// the groups' sums are added in order.
template <int V>
__global__ __launch_bounds__(256) void wgrad8_join_kernel(WgArgs a, int splits) {
  __shared__ float red[8][32][V + 1];
  const int g = threadIdx.x >> 5, e = threadIdx.x & 31;
  const int64_t nk = (int64_t)a.n * a.k, i = ((int64_t)blockIdx.x * 32 + e) * V;
  float s[V], d = 0.f;
  const int n = i < nk ? (int)(i / a.k) : 0, k = (int)(i - (int64_t)n * a.k);
#pragma unroll
  for (int c = 0; c < V; ++c) s[c] = 0.f;
  if (i < nk) {
#pragma unroll 4
    for (int z = g; z < splits; z += 8) {
      const float *p = a.part + z * nk + i;
      if constexpr (V == 4) {
        const float4 q = *(const float4 *)p;
        s[0] += q.x, s[1] += q.y, s[2] += q.z, s[3] += q.w;
      } else {
        s[0] += *p;
      }
      d += a.dbpart[(int64_t)z * a.n + n];
    }
  }
#pragma unroll
  for (int c = 0; c < V; ++c) red[g][e][c] = s[c];
  red[g][e][V] = d;
  __syncthreads();
  if (g || i >= nk) return;
#pragma unroll
  for (int z = 1; z < 8; ++z) {
#pragma unroll
    for (int c = 0; c < V; ++c) s[c] += red[z][e][c];
    d += red[z][e][V];
  }
#pragma unroll
  for (int c = 0; c < V; ++c) {
    if (a.scale) s[c] *= a.scale[k + c];
    if (a.shift) s[c] = fmaf(a.shift[k + c], d, s[c]);
    float *o = a.dw + i + c;
    *o = a.accumulate ? *o + s[c] : s[c];
  }
  if (k == 0 && a.db) a.db[n] = a.accumulate ? a.db[n] + d : d;
}

// Rows per split: two workgroups a CU, at least 256 rows each.
struct Split {
  int splits;
  int64_t chunk;
};
Split split_of(int64_t rows, int64_t n, int64_t k) {
  const int64_t tiles = ((n + kTile - 1) / kTile) * ((k + kTile - 1) / kTile);
  int64_t s = std::max<int64_t>(1, 512 / tiles);
  s = std::min(s, std::max<int64_t>(1, rows / 256));
  Split r;
  r.chunk = ((rows + s - 1) / s + kStep - 1) / kStep * kStep;
  if (r.chunk < kStep) r.chunk = kStep;
  r.splits = (int)std::max<int64_t>(1, (rows + r.chunk - 1) / r.chunk);
  return r;
}
size_t wgrad_ws(int64_t rows, int64_t n, int64_t k) {
  const Split s = split_of(rows, n, k);
  return s.splits == 1 ? 0 : a256((size_t)s.splits * n * k * 4) + a256((size_t)s.splits * n * 4);
}

int wgrad_shape(int64_t rows, int64_t n_in, int64_t n_out, int32_t dtype) {
  int st = take_shape(rows, n_in, dtype);
  if (st == LRCNN_OK) st = take_shape(rows, n_out, dtype);
  if (st == LRCNN_OK) st = take_shape(n_out, n_in, dtype);
  return st;
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

extern "C" int lrcnn_linear_wgrad_workspace_bytes(int64_t rows, int64_t n_in, int64_t n_out,
                                                  int32_t dtype, size_t *bytes) {
  if (!bytes) return lrcnn_fail(LRCNN_EINVAL, "null output");
  TRY(wgrad_shape(rows, n_in, n_out, dtype));
  *bytes = wgrad_ws(rows, n_out, n_in);
  return LRCNN_OK;
}

extern "C" int lrcnn_linear_wgrad(int64_t rows, int64_t n_in, int64_t n_out, int32_t dtype,
                                  const void *dy, int64_t lddy, const void *ckpt,
                                  const float *scale, const float *shift, float *dw, float *db,
                                  int32_t accumulate, void *workspace, size_t ws_bytes,
                                  void *stream) {
  TRY(wgrad_shape(rows, n_in, n_out, dtype));
  WgArgs a{};
  TRY(take("dy", dy, lddy, n_out, dtype == LRCNN_BF16 ? 2 : 4, rows > 0, &a.dy));
  TRY(take_ckpt("ckpt", ckpt, rows > 0));
  TRY(take_f32("scale", scale, false));
  TRY(take_f32("shift", shift, false));
  TRY(take_f32("dw", dw, true));
  TRY(take_f32("db", db, false));
  const Split sp = split_of(rows, n_out, n_in);
  const size_t need = wgrad_ws(rows, n_out, n_in);
  if (need && (!workspace || ((uintptr_t)workspace & 15)))
    return lrcnn_fail(LRCNN_EINVAL, "workspace null or misaligned");
  if (ws_bytes < need)
    return lrcnn_fail(LRCNN_EWORKSPACE, "workspace needs " + std::to_string(need) +
                                            " bytes, got " + std::to_string(ws_bytes));
  a.rows = rows, a.n = (int)n_out, a.k = (int)n_in, a.chunk = sp.chunk;
  a.q = ckpt_of(ckpt, rows, n_in);
  a.q.pitch = pitch_of(n_in);
  a.scale = scale, a.shift = shift, a.dw = dw, a.db = db, a.accumulate = accumulate != 0;
  if (sp.splits > 1) {
    a.part = (float *)workspace;
    a.dbpart = (float *)((char *)workspace + a256((size_t)sp.splits * n_out * n_in * 4));
  }
  const dim3 grid((unsigned)((n_out + kTile - 1) / kTile), (unsigned)((n_in + kTile - 1) / kTile),
                  (unsigned)sp.splits);
  if (grid.y > 65535) return lrcnn_fail(LRCNN_ESHAPE, "too many input features");
  hipStream_t s = (hipStream_t)stream;
  if (dtype == LRCNN_BF16) wgrad8_kernel<bf16><<<grid, 256, 0, s>>>(a);
  else wgrad8_kernel<float><<<grid, 256, 0, s>>>(a);
  if (sp.splits > 1) {
    const int64_t nk = n_out * n_in;
    if (n_in % 4 == 0 && ((uintptr_t)workspace & 15) == 0)
      wgrad8_join_kernel<4><<<(unsigned)((nk / 4 + 31) / 32), 256, 0, s>>>(a, sp.splits);
    else
      wgrad8_join_kernel<1><<<(unsigned)((nk + 31) / 32), 256, 0, s>>>(a, sp.splits);
  }
  return launched("linear_wgrad");
}
