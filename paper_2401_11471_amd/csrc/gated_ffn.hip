// Gated feed-forward block, forward and backward.
//
//   forward   u = x Wu^T + bu, v = x Wv^T + bv, a = f(u) v (one kernel, u and v kept
//             where the caller wants them), z = a W2^T + b2
//   backward  da = dz W2, du = da f'(u) v, dv = da f(u) (one kernel), dx = [du dv] W1
//
// All are products of rows with weights whose depth runs along both operands' rows.
// The weights are the matrix instruction's first operand: a lane then holds
// 16 of 32 neighbouring features of one row, its other half of the wave the other 16,
// so that a checkpoint's group is 16 registers and one exchange between the halves, and
// u and v of the same features are the same registers of two accumulators.
#include "activation.hpp"
#include "kdev.hpp"

#include <algorithm>
#include <type_traits>

namespace lrcnn {
namespace act8 {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int64_t kMaxFeatures = 1 << 24, kMaxFfnRows = 1 << 30;
constexpr int kRow = 128;  // bytes of a tile's row in LDS: 64 bfloat16 or 32 float32 of depth

enum Epi {
  EPI_GATE,  // f(u) v, u and v
  EPI_BACK,  // du and dv from da
  EPI_PLAIN  // + bias
};

struct FfnArgs {
  int rows, depth;
  int feats;   // features of the result; EPI_GATE, EPI_BACK: the hidden ones
  int kind;
  int gx, gy;  // tiles of rows and of features
  FastDiv panel, rest;
  const char *w;  // [feats, EPI_GATE: 2 feats][depth]
  const float *bias;
  Mat x, out, uv;
  Ckpt ku, kv, ka;
};

// ------------------------------------------------------- wave halves
// A 32 x 32 block of the result: register 4 g + e of a lane is feature
// 8 g + 4 (lane >> 5) + e of row lane & 31 -- of the eight quads of features the
// lower half of the wave has the even ones. Exchanged: the lower half has the
// first 16 features of the row in order, the upper half the last 16.
__device__ __forceinline__ void swap_halves(uint32_t &x, uint32_t &y) {
  const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
  x = r[0], y = r[1];
}
// N registers a quad, natural quads <-> 16 in a row (the exchange is its own inverse)
template <int N>
__device__ __forceinline__ void to_runs(uint32_t (&q)[4][N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    swap_halves(q[0][i], q[2][i]);
    swap_halves(q[1][i], q[3][i]);
    const uint32_t t = q[1][i];
    q[1][i] = q[2][i], q[2][i] = t;
  }
}
template <int N>
__device__ __forceinline__ void to_quads(uint32_t (&q)[4][N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t t = q[1][i];
    q[1][i] = q[2][i], q[2][i] = t;
    swap_halves(q[0][i], q[2][i]);
    swap_halves(q[1][i], q[3][i]);
  }
}
// 32 features of row `p` on (`left` of them exist), stored where `in`
__device__ __forceinline__ void store_feats(bf16 *p, int left, bool in, const float (&v)[16]) {
  uint32_t q[4][2];
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    q[g][0] = bf_pair(v[4 * g], v[4 * g + 1]);
    q[g][1] = bf_pair(v[4 * g + 2], v[4 * g + 3]);
  }
  to_runs(q);
  const int h = (threadIdx.x & 32) / 2;
  p += h, left -= h;
  if (!in) return;
  if (left >= 16) {
    *(u32x4_a2 *)p = (u32x4_a2){q[0][0], q[0][1], q[1][0], q[1][1]};
    *(u32x4_a2 *)(p + 8) = (u32x4_a2){q[2][0], q[2][1], q[3][0], q[3][1]};
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < left) p[i] = (bf16)(q[i / 4][i / 2 % 2] >> (16 * (i & 1)));
  }
}
__device__ __forceinline__ void store_feats(float *p, int left, bool in, const float (&v)[16]) {
  uint32_t q[4][4];
#pragma unroll
  for (int i = 0; i < 16; ++i) q[i / 4][i % 4] = __float_as_uint(v[i]);
  to_runs(q);
  const int h = (threadIdx.x & 32) / 2;
  p += h, left -= h;
  if (!in) return;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    if (left >= 4 * g + 4) {
      *(f32x4_a4 *)(p + 4 * g) =
          (f32x4_a4){__uint_as_float(q[g][0]), __uint_as_float(q[g][1]),
                     __uint_as_float(q[g][2]), __uint_as_float(q[g][3])};
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (4 * g + i < left) p[4 * g + i] = __uint_as_float(q[g][i]);
    }
  }
}
// The same features read; zeros behind the last one
__device__ __forceinline__ void load_feats(const bf16 *p, int left, float (&v)[16]) {
  const int h = (threadIdx.x & 32) / 2;
  const Raw8<bf16> a = load8(p + h, left - h), b = load8(p + h + 8, left - h - 8);
  uint32_t q[4][2] = {{a.w[0], a.w[1]}, {a.w[2], a.w[3]}, {b.w[0], b.w[1]}, {b.w[2], b.w[3]}};
  to_quads(q);
#pragma unroll
  for (int i = 0; i < 16; ++i)
    v[i] = __uint_as_float(i & 1 ? q[i / 4][i / 2 % 2] & 0xffff0000u : q[i / 4][i / 2 % 2] << 16);
}
__device__ __forceinline__ void load_feats(const float *p, int left, float (&v)[16]) {
  const int h = (threadIdx.x & 32) / 2;
  float t[2][8];
  load8(p + h, left - h).get(t[0]);
  load8(p + h + 8, left - h - 8).get(t[1]);
  uint32_t q[4][4];
#pragma unroll
  for (int i = 0; i < 16; ++i) q[i / 4][i % 4] = __float_as_uint(t[i / 8][i % 8]);
  to_quads(q);
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(q[i / 4][i % 4]);
}
// A vector over the features (bias), the lane's own quads; zeros without one
__device__ __forceinline__ void load_quads(const float *p, int left, float (&v)[16]) {
  const int h = (threadIdx.x & 32) / 8;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int f = 8 * (i / 4) + h + i % 4;
    v[i] = p && f < left ? p[f] : 0.f;
  }
}
// The checkpoint's group of 32 features of a row: codes and exponent byte, by the
// rules of encode8.
__device__ __forceinline__ void put_feats(const Ckpt &k, int64_t row, int c, bool in,
                                          const float (&v)[16]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  uint32_t o = m;
  swap_halves(m, o);
  m = max(m, o);
  uint32_t E = max((m + 0x10000u) >> 23, 7u), q[4][1];
  if (__builtin_expect(m >= 0x7f7f0000u, 0)) {
    const bool bad = m >= 0x7f800000u;
    E = bad ? 255u : 254u;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      q[g][0] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float s = fminf(fmaxf(v[4 * g + i] * 0x1p-121f, -127.f), 127.f);
        q[g][0] |= (bad ? 0 : __float_as_uint(s + 12582912.f) & 0xffu) << (8 * i);
      }
    }
  } else {
    const float inv = __uint_as_float((260u - E) << 23);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      uint32_t b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(fmaf(v[4 * g + i], inv, 12582912.f));
      q[g][0] = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u) |
                __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
    }
  }
  to_runs(q);
  if (!in) return;
  const int half = threadIdx.x & 32;
  *(u32x4 *)(k.q + row * k.pitch + c + half / 2) = (u32x4){q[0][0], q[1][0], q[2][0], q[3][0]};
  if (!half) k.e[row * (k.pitch / kGroup) + c / kGroup] = (uint8_t)E;
}
__device__ __forceinline__ void get_feats(const Ckpt &k, int64_t row, int c, float (&v)[16]) {
  const u32x4 w = *(const u32x4 *)(k.q + row * k.pitch + c + (threadIdx.x & 32) / 2);
  const float step = step_of(k.e[row * (k.pitch / kGroup) + c / kGroup]);
  uint32_t q[4][1] = {{w.x}, {w.y}, {w.z}, {w.w}};
  to_quads(q);
#pragma unroll
  for (int g = 0; g < 4; ++g) decode4(q[g][0], step, v + 4 * g);
}

// ----------------------------------------------------------- epilogues
// f of the call's kind on 16 values (the same branch for all threads)
__device__ __forceinline__ void activate16(int kind, const float (&u)[16], float (&f)[16],
                                           float (&df)[16]) {
  auto all = [&](auto K) {
#pragma unroll
    for (int i = 0; i < 16; ++i) activate<decltype(K)::value>(u[i], f[i], df[i]);
  };
  using std::integral_constant;
  if (kind == LRCNN_ACT_SILU) all(integral_constant<int, LRCNN_ACT_SILU>());
  else if (kind == LRCNN_ACT_GELU) all(integral_constant<int, LRCNN_ACT_GELU>());
  else if (kind == LRCNN_ACT_GELU_TANH) all(integral_constant<int, LRCNN_ACT_GELU_TANH>());
  else all(integral_constant<int, LRCNN_ACT_RELU>());
}
// Features c .. c + 31 of a row from its accumulators: b0 (EPI_GATE: of u, and b1 of v)
template <typename T, int EPI>
__device__ __forceinline__ void finish(const FfnArgs &a, int row, int c, const float (&bias0)[16],
                                       const float (&bias1)[16], const f32x16 &b0,
                                       const f32x16 &b1) {
  const bool in = row < a.rows;
  const int64_t r = min(row, a.rows - 1);
  const int left = a.feats - c;
  if (left <= 0) return;
  float f[16], df[16], u[16], v[16];
  if constexpr (EPI == EPI_GATE) {
    const int h = (threadIdx.x & 32) / 8;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const bool is = 8 * (i / 4) + h + i % 4 < left;
      u[i] = is ? b0[i] + bias0[i] : 0.f;
      v[i] = is ? b1[i] + bias1[i] : 0.f;
    }
    if (a.uv.p) {
      T *p = (T *)a.uv.p + r * a.uv.ld + c;
      store_feats(p, left, in, u);
      store_feats(p + a.feats, left, in, v);
    }
    if (a.ku.q) put_feats(a.ku, r, c, in, u);
    if (a.kv.q) put_feats(a.kv, r, c, in, v);
    activate16(a.kind, u, f, df);
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] *= v[i];
    store_feats((T *)a.out.p + r * a.out.ld + c, left, in, f);
  } else if constexpr (EPI == EPI_BACK) {
    if (a.uv.p) {
      const T *p = (const T *)a.uv.p + r * a.uv.ld + c;
      load_feats(p, left, u);
      load_feats(p + a.feats, left, v);
    } else {
      get_feats(a.ku, r, c, u);
      get_feats(a.kv, r, c, v);
    }
    activate16(a.kind, u, f, df);
    float du[16], dv[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      du[i] = b0[i] * df[i] * v[i];
      dv[i] = b0[i] * f[i];
      f[i] *= v[i];
    }
    T *p = (T *)a.out.p + r * a.out.ld + c;
    store_feats(p, left, in, du);
    store_feats(p + a.feats, left, in, dv);
    if (a.ka.q) put_feats(a.ka, r, c, in, f);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = b0[i] + bias0[i];
    store_feats((T *)a.out.p + r * a.out.ld + c, left, in, f);
  }
}

// ------------------------------------------------------------- products
// This workgroup's tile: each XCD (workgroups go to the eight in turn) gets one run
// of tiles, eight tiles of rows before the next features, so that the tiles it works on
// share both operands in its L2.
__device__ __forceinline__ void tile_of(const FfnArgs &a, int *x, int *y) {
  const uint32_t total = gridDim.x, w = blockIdx.x;
  const uint32_t q = total >> 3, o = total & 7, c = w & 7, k = w >> 3;
  const uint32_t id = c < o ? c * (q + 1) + k : o * (q + 1) + (c - o) * q + k;
  uint32_t p, r, tx, ty;
  fdiv_qr(id, a.panel, p, r);
  if (8 * p + 8 <= (uint32_t)a.gx) ty = r >> 3, tx = r & 7;
  else fdiv_qr(r, a.rest, ty, tx);
  *x = (int)(8 * p + tx), *y = (int)ty;
}

// A tile of WF FB blocks of 32 features by WR RB of 32 rows. KS waves split the depth
// of each step among them and are summed at the end (1: WF x WR waves of FB x RB blocks each).
// ST: LDS stages.
template <int WF_, int FB_, int WR_, int RB_, int KS_, int ST_>
struct Tile {
  static constexpr int WF = WF_, FB = FB_, WR = WR_, RB = RB_, KS = KS_, ST = ST_;
  static constexpr int F = 32 * WF * FB, R = 32 * WR * RB, THREADS = 64 * WF * WR * KS;
  static constexpr int STAGE = (F + R) * kRow;
  static constexpr int SUMS = KS > 1 ? KS * FB * RB * 64 * 16 * 4 : 0;
  static constexpr int LDS = ST * STAGE > SUMS ? ST * STAGE : SUMS;
};

// One step's products: fragments from an LDS stage. K order: lane half g takes the
// 16-byte vectors 4 g + q of a tile row, q = 0 .. 3, of both operands alike.
template <typename T, int FB, int RB>
__device__ __forceinline__ void products(const char *wt, const char *xt, int q, int lane,
                                         f32x16 (&acc)[FB][RB]) {
  const int g = lane >> 5, r = lane & 31;
  auto at = [&](const char *t, int row) {
    return *(const u32x4 *)(t + row * kRow + swz<8>(row, 4 * g + q) * 16);
  };
  u32x4 fw[FB], fx[RB];
#pragma unroll
  for (int i = 0; i < FB; ++i) fw[i] = at(wt, 32 * i + r);
#pragma unroll
  for (int j = 0; j < RB; ++j) fx[j] = at(xt, 32 * j + r);
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < FB; ++i)
#pragma unroll
      for (int j = 0; j < RB; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fw[i]),
                                                            __builtin_bit_cast(bf16x8, fx[j]),
                                                            acc[i][j], 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < FB; ++i)
#pragma unroll
        for (int j = 0; j < RB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(
              __uint_as_float(fw[i][e]), __uint_as_float(fx[j][e]), acc[i][j], 0, 0, 0);
  }
}

// DMA: rows of both operands at 16-byte steps from aligned bases and a depth of whole
// 16-byte vectors: copied straight into LDS. Else through registers, at the elements'
// alignment.
template <typename T, typename TL, int EPI, bool DMA>
__global__ __launch_bounds__(TL::THREADS) void ffn_kernel(FfnArgs a) {
  constexpr int E = 16 / (int)sizeof(T), BK = kRow / (int)sizeof(T);
  constexpr int FB = TL::FB, RB = TL::RB, ST = TL::ST, KS = TL::KS;
  constexpr int RP = TL::THREADS / 8;               // tile rows of a pass
  constexpr int NF = TL::F / RP, NR = TL::R / RP;   // passes
  static_assert(TL::F % RP == 0 && TL::R % RP == 0 && RP % 16 == 0, "tile rows and threads");
  __shared__ __align__(16) char smem[TL::LDS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int tx, ty;
  tile_of(a, &tx, &ty);
  const int r0 = tx * TL::R, f0 = ty * (EPI == EPI_GATE ? TL::F / 2 : TL::F);
  const int steps = (a.depth + BK - 1) / BK;
  // What this thread brings: rows tid / 8 + RP j, one 16-byte vector each, which goes to
  // slot tid % 8. Rows and features past the end repeat the last one: their results
  // are not stored.
  const int br = tid / 8, vec = (tid & 7) ^ ((br >> 1) & 7);
  const char *gp[NF + NR];
#pragma unroll
  for (int j = 0; j < NF; ++j) {
    const int t = br + RP * j;
    int64_t f;
    if constexpr (EPI == EPI_GATE) {
      // blocks of u and v in turn
      const int h = f0 + t / 64 * 32 + (t & 31);
      f = min(h, a.feats - 1) + ((t >> 5) & 1 ? (int64_t)a.feats : 0);
    } else {
      f = min(f0 + t, a.feats - 1);
    }
    gp[j] = a.w + (f * a.depth + vec * E) * (int64_t)sizeof(T);
  }
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    const int64_t r = min(r0 + br + RP * j, a.rows - 1);
    gp[NF + j] = a.x.p + (r * a.x.ld + vec * E) * (int64_t)sizeof(T);
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
  int kpos = vec * E;  // of the step to load
  f32x16 acc[FB][RB];
#pragma unroll
  for (int i = 0; i < FB; ++i)
#pragma unroll
    for (int j = 0; j < RB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  const int wk = KS > 1 ? wave : 0, wp = KS > 1 ? 0 : wave;
  const int wf = wp % TL::WF, wr = wp / TL::WF;
  auto multiply = [&](int st) {
    const char *wt = smem + st * TL::STAGE + wf * 32 * FB * kRow;
    const char *xt = smem + st * TL::STAGE + (TL::F + wr * 32 * RB) * kRow;
    if constexpr (KS > 1) {
      products<T, FB, RB>(wt, xt, wk, lane, acc);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) products<T, FB, RB>(wt, xt, q, lane, acc);
    }
  };
  if constexpr (DMA) {
    const void *zero = &g_zero16[0];
    auto bring = [&](int st) {
      const bool ok = kpos < a.depth;
#pragma unroll
      for (int j = 0; j < NF + NR; ++j) {
        const int row = j < NF ? RP * j : TL::F + RP * (j - NF);
        load16_lds_a(gp[j], ok, lds0 + st * TL::STAGE + (row + wave * 8) * kRow, zero);
        gp[j] += kRow;
      }
      kpos += BK;
    };
    // Stage of step t + ST - 1: every wave has multiplied step t - 1 from it by the
    // barrier of step t.
    constexpr int LD = NF + NR;
#pragma unroll
    for (int i = 0; i < ST - 1; ++i)
      if (i < steps) bring(i);
    int st = 0;
    for (int t = 0; t < steps; ++t) {
      if (ST > 2 && t + 1 < steps) wait_vmcnt<(ST - 2) * LD>();
      else wait_vmcnt<0>();
      __syncthreads();
      if (t + ST - 1 < steps) bring(st == 0 ? ST - 1 : st - 1);
      multiply(st);
      st = st == ST - 1 ? 0 : st + 1;
    }
  } else {
    u32x4 reg[NF + NR];
    auto fetch = [&]() {
      const int n = a.depth - kpos;
#pragma unroll
      for (int j = 0; j < NF + NR; ++j) {
        if constexpr (sizeof(T) == 2) {
          reg[j] = __builtin_bit_cast(u32x4, load8((const bf16 *)gp[j], n).w);
        } else {
          const float *p = (const float *)gp[j];
          f32x4 v;
          if (n >= 4) {
            v = __builtin_bit_cast(f32x4, *(const f32x4_a4 *)p);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = e < n ? p[e] : 0.f;
          }
          reg[j] = __builtin_bit_cast(u32x4, v);
        }
        gp[j] += kRow;
      }
      kpos += BK;
    };
    auto keep = [&](int st) {
#pragma unroll
      for (int j = 0; j < NF + NR; ++j) {
        const int row = br + (j < NF ? RP * j : TL::F + RP * (j - NF));
        *(u32x4 *)(smem + st * TL::STAGE + row * kRow + (tid & 7) * 16) = reg[j];
      }
    };
    fetch();
    keep(0);
    if (steps > 1) fetch();
    for (int t = 0; t < steps; ++t) {
      __syncthreads();
      if (t + 1 < steps) keep((t + 1) & 1);
      if (t + 2 < steps) fetch();
      multiply(t & 1);
    }
  }
  if constexpr (KS > 1) {
    // the waves' sums joined in order; wave j takes the blocks of rows j
    float *red = (float *)smem;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FB; ++i)
#pragma unroll
      for (int j = 0; j < RB; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          red[(((wk * FB + i) * RB + j) * 16 + v) * 64 + lane] = acc[i][j][v];
    __syncthreads();
    if (wave >= RB) return;
#pragma unroll
    for (int i = 0; i < FB; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) s += red[(((k * FB + i) * RB + wave) * 16 + v) * 64 + lane];
        acc[i][0][v] = s;
      }
  }
  constexpr int STEP = EPI == EPI_GATE ? 2 : 1;
#pragma unroll
  for (int i = 0; i < FB; i += STEP) {
    const int c = f0 + (wf * FB + i) / STEP * 32;
    float bias0[16], bias1[16];
    if constexpr (EPI != EPI_BACK) load_quads(a.bias ? a.bias + c : nullptr, a.feats - c, bias0);
    if constexpr (EPI == EPI_GATE)
      load_quads(a.bias ? a.bias + a.feats + c : nullptr, a.feats - c, bias1);
    if constexpr (KS > 1) {
      finish<T, EPI>(a, r0 + 32 * wave + (lane & 31), c, bias0, bias1, acc[i][0],
                     acc[i + STEP - 1][0]);
    } else {
#pragma unroll
      for (int j = 0; j < RB; ++j)
        finish<T, EPI>(a, r0 + 32 * (wr * RB + j) + (lane & 31), c, bias0, bias1, acc[i][j],
                       acc[i + STEP - 1][j]);
    }
  }
}

// Few rows (up to 16 NC): the weights' bytes bound it. 16 features (of u and of v) a
// workgroup, eight waves that take turns along the depth, 128 bytes of a weight
// row a step, straight into registers.
template <typename T, int NC, int EPI>
__global__ __launch_bounds__(512) void ffn_few_kernel(FfnArgs a) {
  constexpr int E = 16 / (int)sizeof(T), BK = kRow / (int)sizeof(T);
  constexpr int H = EPI == EPI_GATE ? 2 : 1, W = 8, U = 4 / H;
  __shared__ float red[W][H][NC][64][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int f0 = blockIdx.x * 16, g = lane >> 4;
  const int f = min(f0 + (lane & 15), a.feats - 1);
  const T *w[H], *x[NC];
#pragma unroll
  for (int h = 0; h < H; ++h)
    w[h] = (const T *)a.w + (f + (int64_t)h * a.feats) * a.depth + g * 2 * E;
#pragma unroll
  for (int c = 0; c < NC; ++c)
    x[c] = (const T *)a.x.p + (int64_t)min(16 * c + (lane & 15), a.rows - 1) * a.x.ld + g * 2 * E;
  f32x4 acc[H][NC];
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[h][c] = (f32x4){0.f, 0.f, 0.f, 0.f};
  auto load = [&](const T *p, int n, auto whole) -> u32x4 {
    if constexpr (sizeof(T) == 2) {
      if constexpr (decltype(whole)::value) return __builtin_bit_cast(u32x4, *(const u32x4_a2 *)p);
      return __builtin_bit_cast(u32x4, load8((const bf16 *)p, n).w);
    } else {
      if constexpr (decltype(whole)::value) return __builtin_bit_cast(u32x4, *(const f32x4_a4 *)p);
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = e < n ? ((const float *)p)[e] : 0.f;
      return __builtin_bit_cast(u32x4, v);
    }
  };
  // N steps, W apart, from depth k on
  auto some = [&](int k, auto whole, auto many) {
    constexpr int N = decltype(many)::value;
    u32x4 fw[N][H][2], fx[N][NC][2];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int at = k + n * W * BK + q * E, left = a.depth - at - g * 2 * E;
#pragma unroll
        for (int h = 0; h < H; ++h) fw[n][h][q] = load(w[h] + at, left, whole);
#pragma unroll
        for (int c = 0; c < NC; ++c) fx[n][c][q] = load(x[c] + at, left, whole);
      }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            if constexpr (sizeof(T) == 2) {
              acc[h][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  __builtin_bit_cast(bf16x8, fw[n][h][q]), __builtin_bit_cast(bf16x8, fx[n][c][q]),
                  acc[h][c], 0, 0, 0);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                acc[h][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                    __uint_as_float(fw[n][h][q][e]), __uint_as_float(fx[n][c][q][e]), acc[h][c], 0,
                    0, 0);
            }
          }
  };
  int k = wave * BK;
  for (; k + ((U - 1) * W + 1) * BK <= a.depth; k += U * W * BK)
    some(k, std::true_type(), std::integral_constant<int, U>());
  for (; k + BK <= a.depth; k += W * BK)
    some(k, std::true_type(), std::integral_constant<int, 1>());
  if (k < a.depth) some(k, std::false_type(), std::integral_constant<int, 1>());
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int c = 0; c < NC; ++c) *(f32x4 *)red[wave][h][c][lane] = acc[h][c];
  __syncthreads();
  for (int t = threadIdx.x; t < 256 * NC; t += 512) {
    const int ft = t & 15, row = t >> 4, c = row >> 4, l = (ft >> 2) * 16 + (row & 15);
    if (row >= a.rows || f0 + ft >= a.feats) continue;
    float s[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      s[h] = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) s[h] += red[i][h][c][l][ft & 3];
      if (a.bias) s[h] += a.bias[h * a.feats + f0 + ft];
    }
    if constexpr (EPI == EPI_GATE) {
      if (a.uv.p) {
        T *p = (T *)a.uv.p + row * a.uv.ld + f0 + ft;
        put(p, s[0]);
        put(p + a.feats, s[1]);
      }
      float fu = 0.f, df;
      if (a.kind == LRCNN_ACT_SILU) activate<LRCNN_ACT_SILU>(s[0], fu, df);
      else if (a.kind == LRCNN_ACT_GELU) activate<LRCNN_ACT_GELU>(s[0], fu, df);
      else if (a.kind == LRCNN_ACT_GELU_TANH) activate<LRCNN_ACT_GELU_TANH>(s[0], fu, df);
      else activate<LRCNN_ACT_RELU>(s[0], fu, df);
      s[0] = fu * s[1];
    }
    put((T *)a.out.p + row * a.out.ld + f0 + ft, s[0]);
  }
}

// ------------------------------------------------------------- launches
typedef Tile<4, 2, 2, 4, 1, 2> Big;    // 256 features x 256 rows, 8 waves
typedef Tile<2, 2, 2, 2, 1, 2> Mid;    // 128 x 128, 4 waves
typedef Tile<1, 2, 1, 2, 4, 3> Small;  // 64 x 64, 4 waves that split the depth
constexpr int kFewRows = 32;

template <typename T, typename TL, int EPI, bool DMA>
int launch(FfnArgs &a, hipStream_t s) {
  constexpr int F = EPI == EPI_GATE ? TL::F / 2 : TL::F;
  a.gx = (a.rows + TL::R - 1) / TL::R;
  a.gy = (a.feats + F - 1) / F;
  if ((int64_t)a.gx * a.gy > 1 << 22) return refuse(LRCNN_ESHAPE, "gated_ffn: too many tiles");
  a.panel = fast_div(8 * (uint32_t)a.gy);
  a.rest = fast_div((uint32_t)std::max(a.gx & 7, 1));
  ffn_kernel<T, TL, EPI, DMA><<<(unsigned)(a.gx * a.gy), TL::THREADS, 0, s>>>(a);
  return LRCNN_OK;
}

template <typename T, int EPI>
int product(FfnArgs a, hipStream_t s) {
  constexpr int H = EPI == EPI_GATE ? 2 : 1;
  if constexpr (EPI != EPI_BACK) {
    if (a.rows <= kFewRows && !a.ku.q && !a.kv.q) {
      const unsigned g = (unsigned)((a.feats + 15) / 16);
      if (a.rows <= 16) ffn_few_kernel<T, 1, EPI><<<g, 512, 0, s>>>(a);
      else ffn_few_kernel<T, 2, EPI><<<g, 512, 0, s>>>(a);
      return LRCNN_OK;
    }
  }
  constexpr int E = 16 / (int)sizeof(T);
  const bool dma = ((uintptr_t)a.x.p | (uintptr_t)a.w) % 16 == 0 && a.x.ld % E == 0 &&
                   a.depth % E == 0;
  auto tiles = [&](int64_t f, int64_t r) {
    return (((int64_t)a.feats * H + f - 1) / f) * ((a.rows + r - 1) / r);
  };
  if (tiles(Mid::F, Mid::R) < 256)
    return dma ? launch<T, Small, EPI, true>(a, s) : launch<T, Small, EPI, false>(a, s);
  if (!dma) return launch<T, Mid, EPI, false>(a, s);
  if (tiles(Big::F, Big::R) < 256) return launch<T, Mid, EPI, true>(a, s);
  return launch<T, Big, EPI, true>(a, s);
}

template <int EPI>
int run(int32_t dtype, const FfnArgs &a, void *stream) {
  return dtype == LRCNN_BF16 ? product<bf16, EPI>(a, (hipStream_t)stream)
                             : product<float, EPI>(a, (hipStream_t)stream);
}

int ffn_shape(int64_t rows, int64_t n, int64_t hidden, int32_t dtype, int32_t kind) {
  const int st = take_shape(rows, n, dtype);
  if (st != LRCNN_OK) return st;
  if (hidden < 1) return refuse(LRCNN_ESHAPE, "need hidden >= 1");
  if (n > kMaxFeatures || hidden > kMaxFeatures / 2 || rows > kMaxFfnRows)
    return refuse(LRCNN_ESHAPE, "gated_ffn takes at most 2^24 features and 2^30 rows");
  if (kind < LRCNN_ACT_RELU || kind > LRCNN_ACT_SILU)
    return refuse(LRCNN_EINVAL, "unknown activation");
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

extern "C" int lrcnn_gated_ffn_forward(int64_t rows, int64_t n_in, int64_t hidden, int64_t n_out,
                                       int32_t dtype, int32_t kind, const void *x, int64_t ldx,
                                       const void *w1, const float *b1, void *a, int64_t lda,
                                       void *uv, int64_t lduv, void *ckpt_u, void *ckpt_v,
                                       const void *w2, const float *b2, void *z, int64_t ldz,
                                       void *stream) {
  TRY(ffn_shape(rows, n_in, hidden, dtype, kind));
  if (z) TRY(ffn_shape(rows, n_out, hidden, dtype, kind));
  if (rows == 0) return LRCNN_OK;
  const int es = dtype == LRCNN_BF16 ? 2 : 4;
  FfnArgs g{};
  Mat w, w2m, zm;
  TRY(take("x", x, ldx, n_in, es, true, &g.x));
  TRY(take("w1", w1, 0, n_in, es, true, &w));
  TRY(take_f32("b1", b1, false));
  TRY(take("a", a, lda, hidden, es, true, &g.out));
  TRY(take("uv", uv, lduv, 2 * hidden, es, false, &g.uv));
  TRY(take_ckpt("ckpt_u", ckpt_u, false));
  TRY(take_ckpt("ckpt_v", ckpt_v, false));
  if (z) {
    TRY(take("w2", w2, 0, hidden, es, true, &w2m));
    TRY(take_f32("b2", b2, false));
    TRY(take("z", z, ldz, n_out, es, true, &zm));
  }
  g.rows = (int)rows, g.depth = (int)n_in, g.feats = (int)hidden, g.kind = kind;
  g.w = w.p, g.bias = b1;
  g.ku = ckpt_of(ckpt_u, rows, hidden);
  g.kv = ckpt_of(ckpt_v, rows, hidden);
  TRY(run<EPI_GATE>(dtype, g, stream));
  if (z) {
    FfnArgs d{};
    d.rows = (int)rows, d.depth = (int)hidden, d.feats = (int)n_out;
    d.x = g.out, d.w = w2m.p, d.bias = b2, d.out = zm;
    TRY(run<EPI_PLAIN>(dtype, d, stream));
  }
  return launched("gated_ffn_forward");
}

extern "C" int lrcnn_gated_ffn_backward(int64_t rows, int64_t n_in, int64_t hidden, int64_t n_out,
                                        int32_t dtype, int32_t kind, const void *dz, int64_t lddz,
                                        const void *w2t, const void *uv, int64_t lduv,
                                        const void *ckpt_u, const void *ckpt_v, void *duv,
                                        int64_t ldduv, void *ckpt_a, const void *w1t, void *dx,
                                        int64_t lddx, void *stream) {
  TRY(ffn_shape(rows, n_out, hidden, dtype, kind));
  if (dx) TRY(ffn_shape(rows, n_in, hidden, dtype, kind));
  if (rows == 0) return LRCNN_OK;
  if ((ckpt_u != nullptr) != (ckpt_v != nullptr) || (uv != nullptr) == (ckpt_u != nullptr))
    return refuse(LRCNN_EINVAL, "give uv, or ckpt_u and ckpt_v");
  const int es = dtype == LRCNN_BF16 ? 2 : 4;
  FfnArgs g{};
  Mat w, w1m, xm;
  TRY(take("dz", dz, lddz, n_out, es, true, &g.x));
  TRY(take("w2t", w2t, 0, n_out, es, true, &w));
  TRY(take("uv", uv, lduv, 2 * hidden, es, false, &g.uv));
  TRY(take_ckpt("ckpt_u", ckpt_u, false));
  TRY(take_ckpt("ckpt_v", ckpt_v, false));
  TRY(take("duv", duv, ldduv, 2 * hidden, es, true, &g.out));
  TRY(take_ckpt("ckpt_a", ckpt_a, false));
  if (dx) {
    TRY(take("w1t", w1t, 0, 2 * hidden, es, true, &w1m));
    TRY(take("dx", dx, lddx, n_in, es, true, &xm));
  }
  g.rows = (int)rows, g.depth = (int)n_out, g.feats = (int)hidden, g.kind = kind;
  g.w = w.p;
  g.ku = ckpt_of(ckpt_u, rows, hidden);
  g.kv = ckpt_of(ckpt_v, rows, hidden);
  g.ka = ckpt_of(ckpt_a, rows, hidden);
  TRY(run<EPI_BACK>(dtype, g, stream));
  if (dx) {
    FfnArgs d{};
    d.rows = (int)rows, d.depth = (int)(2 * hidden), d.feats = (int)n_in;
    d.x = g.out, d.w = w1m.p, d.out = xm;
    TRY(run<EPI_PLAIN>(dtype, d, stream));
  }
  return launched("gated_ffn_backward");
}
