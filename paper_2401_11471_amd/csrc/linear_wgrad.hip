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

constexpr int kStep = 32;  // rows of dy and of the checkpoint per step

struct WgArgs {
  int64_t rows;
  int n, k;             // outputs, inputs
  int64_t chunk;        // rows per split, a multiple of kStep
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
__device__ __forceinline__ uint4 bf_vec(const float *v) {
  return make_uint4(bf_pair(v[0], v[1]), bf_pair(v[2], v[3]), bf_pair(v[4], v[5]),
                    bf_pair(v[6], v[7]));
}

// Tiles run through a panel of eight tiles of n before the next k, so that
// the run of tiles an XCD works on shares rows of both operands in its L2.
__device__ __forceinline__ TileId panel_tile() {
  const int gx = gridDim.x, gy = gridDim.y;
  TileId t = xcd_tile(false);
  const int id = t.x + gx * t.y, panel = id / (8 * gy), r = id - panel * 8 * gy;
  const int w = min(8, gx - 8 * panel);
  t.y = r / w;
  t.x = 8 * panel + (r - t.y * w);
  return t;
}

// A W x W tile of S by four waves of W/2 x W/2. Both operands go through
// registers into k-major LDS tiles (the codes as bfloat16, dy as it is or in
// three pieces), and to the matrix cores by transposing reads. A step's loads
// are issued RS steps before its tile is written to LDS, the tile is written
// one step before it is multiplied, and a unit's fragments (16 rows; one
// piece of dy) are read one unit before their MFMAs.
template <typename T, int W>
__global__ __launch_bounds__(256, W == 256 ? 1 : 2) void wgrad8_kernel(WgArgs a) {
  constexpr int P = std::is_same<T, float>::value ? 3 : 1;  // pieces of dy
  constexpr int ST = P == 1 ? 3 : 2;                         // LDS tiles and load slots
  constexpr int NB = W / 64;                                 // 32 x 32 blocks per wave and side
  constexpr int U = 2 * P;                                   // units per step
  constexpr int LA = W / 8, RA = 256 / LA, NA = kStep / RA;  // dy: lanes, rows, passes
  constexpr int LB = W / 16, RB = 256 / LB, NQ = kStep / RB; // codes
  using M = KM<bf16, W>;
  constexpr int TS = kStep * W;  // elements of an LDS tile
  __shared__ __align__(16) bf16 smem[ST * (P + 1) * TS];
  __shared__ float dbs[W];
  auto As = [&](int st, int p) { return smem + (st * P + p) * TS; };
  auto Bs = [&](int st) { return smem + (ST * P + st) * TS; };
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const TileId tl = panel_tile();
  const int n0 = tl.x * W, k0 = tl.y * W;
  const int64_t m0 = (int64_t)tl.z * a.chunk, m1 = min(a.rows, m0 + a.chunk);
  const int steps = (int)((m1 - m0 + kStep - 1) / kStep);
  // Columns past the matrix are read from its first ones: what they give is
  // never stored. A vector that straddles the last column reads into the
  // next row; only the last row of all has none.
  const int ar = tid / LA, ac = n0 + (tid % LA) * 8;
  const int br = tid / LB, bc = k0 + (tid % LB) * 16;
  const int al = ac < a.n ? ac : 0, bl = bc < a.q.pitch ? bc : 0;
  const int64_t fast = min(m1, a.rows - 1) - kStep;  // steps up to this row read whole vectors
  struct Slot {
    Raw8<T> a[NA];
    uint4 q[NQ];
    uint32_t e[NQ];
  } slot[ST];
  auto gload = [&](Slot &s, int step) {
    const int64_t m = m0 + (int64_t)step * kStep;
    const T *pa = (const T *)a.dy.p + m * a.dy.ld;
    const int8_t *pq = a.q.q + m * a.q.pitch;
    const uint8_t *pe = a.q.e + m * (a.q.pitch / kGroup);
    if (m <= fast) {
#pragma unroll
      for (int i = 0; i < NA; ++i) s.a[i] = load8(pa + (int64_t)(ar + RA * i) * a.dy.ld + al, 8);
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        const int64_t r = br + RB * i;
        s.q[i] = *(const uint4 *)(pq + r * a.q.pitch + bl);
        s.e[i] = pe[r * (a.q.pitch / kGroup) + bl / kGroup];
      }
    } else {
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        const int64_t r = ar + RA * i;
        s.a[i] = load8(pa + r * a.dy.ld + al, m + r < m1 ? a.n - al : 0);
      }
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        const int64_t r = br + RB * i;
        s.q[i] = make_uint4(0, 0, 0, 0);
        s.e[i] = 7;
        if (m + r < m1) {
          s.q[i] = *(const uint4 *)(pq + r * a.q.pitch + bl);
          s.e[i] = pe[r * (a.q.pitch / kGroup) + bl / kGroup];
        }
      }
    }
  };
  auto put_dy = [&](const Slot &s, int st) {
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int at = M::off(ar + RA * i, (tid % LA) * 8);
      if constexpr (P == 1) {
        *(uint4 *)(As(st, 0) + at) =
            make_uint4(s.a[i].w[0], s.a[i].w[1], s.a[i].w[2], s.a[i].w[3]);
      } else {
        float v[8], c[P][8];
        s.a[i].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float t[3];
          cut3(v[e], t);
#pragma unroll
          for (int p = 0; p < P; ++p) c[p][e] = t[p];
        }
#pragma unroll
        for (int p = 0; p < P; ++p) *(uint4 *)(As(st, p) + at) = bf_vec(c[p]);
      }
    }
  };
  auto put_q = [&](const Slot &s, int st) {
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const float step = step_of(s.e[i]);
      const uint32_t w[4] = {s.q[i].x, s.q[i].y, s.q[i].z, s.q[i].w};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[8];
        decode4(w[2 * h], step, v), decode4(w[2 * h + 1], step, v + 4);
        *(uint4 *)(Bs(st) + M::off(br + RB * i, (tid % LB) * 16 + 8 * h)) = bf_vec(v);
      }
    }
  };

  f32x16 acc[NB][NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  const int wn = (wave & 1) * (W / 2), wk = (wave >> 1) * (W / 2);
  // fragments of the unit being multiplied and of the next one; b by slice
  bf16x8 fa[2][NB], fb[2][NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) fa[1][i][e] = fb[1][i][e] = (__bf16)0.f;
  // db: the sums of this wave's fragments of dy, slice 0 or 1 of every step
  // by the side of k it works on (two waves hold the same dy)
  const bool want_db = tl.y == 0 || (a.shift && !a.part);
  float dbv[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) dbv[i] = 0.f;
  auto read = [&](int st, auto u) {
    constexpr int u_ = decltype(u)::value, s = u_ / P, p = u_ % P;
#pragma unroll
    for (int i = 0; i < NB; ++i) fa[u_ & 1][i] = ld_tr8<W, 2>(As(st, p), wn + 32 * i, s, lane);
    if constexpr (p == 0) {
#pragma unroll
      for (int j = 0; j < NB; ++j) fb[s][j] = ld_tr8<W, 2>(Bs(st), wk + 32 * j, s, lane);
    }
  };
  auto mma = [&](auto u) {
    constexpr int u_ = decltype(u)::value, s = u_ / P;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[u_ & 1][i], fb[s][j], acc[i][j],
                                                            0, 0, 0);
    if (want_db && (wave >> 1) == s) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) dbv[i] += (float)fa[u_ & 1][i][e];
    }
  };
  using std::integral_constant;
  // Step t (tile t is in LDS buffer t % ST): units are read one ahead of
  // their MFMAs; the tile of step t + 1 is written; loads of step t + 1 + ST
  // take its slot.
  auto step = [&](auto sc, int t) {
    constexpr int st = decltype(sc)::value, nx = (st + 1) % ST;
    const bool more = t + 1 < steps;
    auto unit = [&](auto u) {
      constexpr int u_ = decltype(u)::value;
      read(st, u);
      mma(integral_constant<int, (u_ + U - 1) % U>());
      if (more) {
        if constexpr (u_ == 0) put_dy(slot[nx], nx);
        if constexpr (u_ == U / 2) {
          put_q(slot[nx], nx);
          if (t + 1 + ST < steps) gload(slot[nx], t + 1 + ST);
        }
      }
    };
    unit(integral_constant<int, 0>());
    unit(integral_constant<int, 1>());
    if constexpr (U == 6) {
      unit(integral_constant<int, 2>());
      unit(integral_constant<int, 3>());
      unit(integral_constant<int, 4>());
      unit(integral_constant<int, 5>());
    }
    __syncthreads();
  };
  if (steps > 0) {
#pragma unroll
    for (int i = 0; i < ST; ++i)
      if (i < steps) gload(slot[i], i);
    put_dy(slot[0], 0);
    put_q(slot[0], 0);
    if (ST < steps) gload(slot[0], ST);
    __syncthreads();
    int t = 0;
    for (; t + ST <= steps; t += ST) {
      step(integral_constant<int, 0>(), t);
      step(integral_constant<int, 1>(), t + 1);
      if constexpr (ST == 3) step(integral_constant<int, 2>(), t + 2);
    }
    if (t < steps) step(integral_constant<int, 0>(), t);
    if (ST == 3 && t + 1 < steps) step(integral_constant<int, 1>(), t + 1);
    mma(integral_constant<int, U - 1>());
  }
  // db of the tile's columns: halves of a fragment, then the two slices
  float *slots = (float *)smem;  // [2][W]
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const float s = dbv[i] + __shfl_xor(dbv[i], 32);
    if (lane < 32) slots[(wave >> 1) * W + wn + 32 * i + lane] = s;
  }
  __syncthreads();
  if (tid < W) {
    const float s = slots[tid] + slots[W + tid];
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
  for (int j = 0; j < NB; ++j) {
    const int kk = k0 + wk + 32 * j + (lane & 31);
    if (kk >= a.k) continue;
    const float sc = a.scale && !a.part ? a.scale[kk] : 1.f;
    const float sh = a.shift && !a.part ? a.shift[kk] : 0.f;
#pragma unroll
    for (int i = 0; i < NB; ++i)
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

// Tile width and rows per split.
struct Split {
  int tile, splits;
  int64_t chunk;
};
Split split_of(int64_t rows, int64_t n, int64_t k) {
  Split r;
  auto tiles = [&](int w) { return ((n + w - 1) / w) * ((k + w - 1) / w); };
  r.tile = n > 128 && k > 128 && tiles(256) * std::max<int64_t>(1, rows / 1024) >= 256 ? 256 : 128;
  int64_t s = std::max<int64_t>(1, (r.tile == 256 ? 256 : 512) / tiles(r.tile));
  s = std::min(s, std::max<int64_t>(1, rows / 256));
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
  const dim3 grid((unsigned)((n_out + sp.tile - 1) / sp.tile),
                  (unsigned)((n_in + sp.tile - 1) / sp.tile), (unsigned)sp.splits);
  if (grid.y > 65535 || (int64_t)grid.x * grid.y * grid.z > INT32_MAX)
    return lrcnn_fail(LRCNN_ESHAPE, "too many features");
  hipStream_t s = (hipStream_t)stream;
  auto run = [&](auto *t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (sp.tile == 256) wgrad8_kernel<T, 256><<<grid, 256, 0, s>>>(a);
    else wgrad8_kernel<T, 128><<<grid, 256, 0, s>>>(a);
  };
  if (dtype == LRCNN_BF16) run((bf16 *)nullptr);
  else run((float *)nullptr);
  if (sp.splits > 1) {
    const int64_t nk = n_out * n_in;
    if (n_in % 4 == 0 && ((uintptr_t)workspace & 15) == 0)
      wgrad8_join_kernel<4><<<(unsigned)((nk / 4 + 31) / 32), 256, 0, s>>>(a, sp.splits);
    else
      wgrad8_join_kernel<1><<<(unsigned)((nk + 31) / 32), 256, 0, s>>>(a, sp.splits);
  }
  return launched("linear_wgrad");
}
