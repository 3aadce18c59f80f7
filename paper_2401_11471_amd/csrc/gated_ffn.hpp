// Gated feed-forward block, forward and backward.
//
//   forward   u = x Wu^T + bu, v = x Wv^T + bv, a = f(u) v (one kernel, u and v kept
//             where the caller wants them), z = a W2^T + b2
//   backward  da = dz W2, du = da f'(u) v, dv = da f(u) (one kernel), dx = [du dv] W1
//
// All are products of rows with weights whose depth runs along both operands' rows,
// and differ in what becomes of a result. The weights are the matrix instruction's first
// operand: a lane then holds runs of four neighbouring features of one row, and u and v of
// the same features are the same registers of two accumulators.
//
// 67800 x 2048 x 8192 bf16, by the card: forward 3.70 to 3.98 ms for the first kernel with
// both checkpoints (4.55 TFLOP, 1140 to 1230 TFLOP/s; the library's product of its size
// alone 3.25 to 3.29), 1.66 to 1.72 for the second (1320 to 1370 TFLOP/s; 1.58 to 1.63);
// backward 2.53 to 2.66 and 3.36 to 3.52 ms (the library's products 1.57 to 1.61 and 3.12 to
// 3.17). Launch by launch in a trace, whose clocks vary more: up to 4.60 and 2.76 ms for the
// first kernels. The plain products keep the matrix pipes 80% busy at 1.5 to 1.6 GHz,
// the clock that their own power leaves; the first forward kernel 65% at 1.6, the first backward
// one 44% at 1.9: of a tile's 57 and 76 us its results take 20 and 39, which one wave on a
// SIMD doesn't overlap with products. Their vector instructions are 8 and 17 of them.
#pragma once

#include "activation.hpp"
#include "kdev.hpp"

#include <algorithm>
#include <atomic>
#include <type_traits>

namespace lrcnn {
namespace act8 {
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

// Products of one storage type (gated_ffn_bf16.hip, gated_ffn_f32.hip)
void ffn_bf16(Epi epi, const FfnArgs &a, hipStream_t s);
void ffn_f32(Epi epi, const FfnArgs &a, hipStream_t s);
extern std::atomic<int> g_ffn_tile;  // test hook: the variant to take where it can
constexpr int64_t kMaxFeatures = 1 << 24, kMaxFfnRows = 1 << 30;
// Tiles that a grid takes: fewer than 2^32 threads, 256 a tile. Calls have fewer than 2^22
// tiles of 128 x 128, so 64 x 64 ones, which take all operands, always fit.
constexpr int64_t kMostTiles = (1 << 24) - 1, kMostMidTiles = (1 << 22) - 1;

#ifdef LRCNN_FFN_KERNELS
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int kRow = 128;  // bytes of a tile's row in LDS: 64 bfloat16 or 32 float32 of depth

// ------------------------------------------------------------- results
// f(0), f(1), ... f(N - 1), the index a constant
template <int B, int E, typename F>
__device__ __forceinline__ void each(F &&f) {
  if constexpr (B < E) {
    f(std::integral_constant<int, B>());
    each<B + 1, E>(f);
  }
}
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
constexpr int least(int a, int b) { return a < b ? a : b; }
// The wave's LDS accesses before are done as its other lanes see them
__device__ __forceinline__ void wave_meets() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// Results leave the accumulators by strips of 32 rows through a wave's own LDS, float32
// [32][32 FB]: registers 4 g .. 4 g + 3 of a 32 x 32 block are features 8 g + 4 (lane / 32)
// on of row lane % 32. They are read back eight features to a lane, a row's
// lanes next to each other: whole cache lines to memory, a checkpoint's group in a quad of
// lanes, and one copy of the code for all strips (unrolled over the accumulators it
// is fetched anew for every tile: with silu, without checkpoints, 22 us a tile of 256 x 256
// beside its products, so 14). 16-byte slots are swapped by the row, so the lanes of a
// pass take different banks.
template <int FB>
__device__ __forceinline__ lds_char *slot_of(lds_char *l, int row, int slot) {
  return l + (row * 8 * FB + (slot ^ (row & 7))) * 16;
}
template <int FB>
__device__ __forceinline__ void strip_put(lds_char *l, int i, const f32x16 &b) {
  const int row = threadIdx.x & 31, half = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int g = 0; g < 4; ++g)
    *(lds_f32x4 *)slot_of<FB>(l, row, 8 * i + 2 * g + half) =
        (f32x4){b[4 * g], b[4 * g + 1], b[4 * g + 2], b[4 * g + 3]};
}
// Branches that end with different N stay apart, and their accumulators are stored from
// where they are: joined, all are copied to the same registers first.
template <int N>
__device__ __forceinline__ void own_branch() {
  asm volatile("; strip %0" ::"n"(N));
}
template <int FB>
__device__ __forceinline__ void strip_get(lds_char *l, int row, int slot, float (&v)[8]) {
  const f32x4 x = *(lds_f32x4 *)slot_of<FB>(l, row, slot);
  const f32x4 y = *(lds_f32x4 *)slot_of<FB>(l, row, slot + 1);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = x[i], v[4 + i] = y[i];
}
__device__ __forceinline__ uint2 lds_pair(const lds_char *p) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 v = *(__attribute__((address_space(3))) const u32x2 *)p;
  return make_uint2(v.x, v.y);
}
// f(the call's kind, a constant): the same branch for all threads
template <typename F>
__device__ __forceinline__ void with_kind(int kind, F &&f) {
  using std::integral_constant;
  if (kind == LRCNN_ACT_SILU) f(integral_constant<int, LRCNN_ACT_SILU>());
  else if (kind == LRCNN_ACT_GELU) f(integral_constant<int, LRCNN_ACT_GELU>());
  else if (kind == LRCNN_ACT_GELU_TANH) f(integral_constant<int, LRCNN_ACT_GELU_TANH>());
  else f(integral_constant<int, LRCNN_ACT_RELU>());
}
template <int N>
__device__ __forceinline__ void activate_all(int kind, const float (&u)[N], float (&f)[N],
                                             float (&df)[N]) {
  with_kind(kind, [&](auto K) {
#pragma unroll
    for (int i = 0; i < N; ++i) activate<decltype(K)::value, true>(u[i], f[i], df[i]);
  });
}
// A lane's eight features of a strip of FB blocks (EPI_GATE: blocks of u and v in turn)
template <int EPI, int FB>
struct Lanes {
  static constexpr int WIDTH = 32 * FB / (EPI == EPI_GATE ? 2 : 1);  // features of a strip
  static constexpr int PER = WIDTH / 8, ROWS = 64 / PER;             // lanes a row, rows a pass
};
struct Bias {
  float u[8], v[8];
  // of the features c .. c + 7
  template <int EPI>
  __device__ __forceinline__ void load(const FfnArgs &a, int c) {
    const int n = a.feats - c;
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = v[i] = 0.f;
    if (EPI == EPI_BACK || !a.bias || n <= 0) return;
    load8(a.bias + c, n).get(u);
    if (EPI == EPI_GATE) load8(a.bias + a.feats + c, n).get(v);
  }
};
// Rows r0 .. r0 + 31 and features c0 on from their strip. codes(row, u, v): EPI_BACK, u
// and v of this lane's features of a row of the strip; all lanes call it.
template <typename T, int EPI, int FB, typename Codes>
__device__ __forceinline__ void strip_rows(const FfnArgs &a, lds_char *l, int r0, int c0,
                                           const Bias &bias, Codes &&codes) {
  typedef Lanes<EPI, FB> N;
  const int lane = threadIdx.x & 63, k = lane % N::PER, c = c0 + 8 * k, n = a.feats - c;
#pragma unroll 1
  for (int p = 0; p < 32 / N::ROWS; ++p) {
    const int row = p * N::ROWS + lane / N::PER;
    const int64_t r = r0 + row;
    float u[8], v[8], f[8], df[8];
    if constexpr (EPI == EPI_BACK) codes(row, u, v);
    // (the quad of a checkpoint's group goes on or stops as one)
    if (r >= a.rows || n <= (EPI == EPI_PLAIN ? 0 : -(-a.feats & (kGroup - 1)))) continue;
    if constexpr (EPI == EPI_GATE) {
      const int slot = k / 4 * 16 + k % 4 * 2;
      strip_get<FB>(l, row, slot, u);
      strip_get<FB>(l, row, slot + 8, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] += bias.u[i], v[i] += bias.v[i];
      if (n < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i >= n) u[i] = v[i] = 0.f;
      }
      if (a.uv.p) {
        T *q = (T *)a.uv.p + r * a.uv.ld + c;
        store8(q, n, u);
        store8(q + a.feats, n, v);
      }
      if (a.ku.q) put8(a.ku, r, c, u);
      if (a.kv.q) put8(a.kv, r, c, v);
      activate_all(a.kind, u, f, df);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= v[i];
      store8((T *)a.out.p + r * a.out.ld + c, n, f);
    } else if constexpr (EPI == EPI_BACK) {
      float d[8];
      strip_get<FB>(l, row, 2 * k, d);
      activate_all(a.kind, u, f, df);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        df[i] *= d[i] * v[i];
        d[i] *= f[i];
        f[i] *= v[i];
      }
      T *q = (T *)a.out.p + r * a.out.ld + c;
      store8(q, n, df);
      store8(q + a.feats, n, d);
      if (a.ka.q) put8(a.ka, r, c, f);
    } else {
      strip_get<FB>(l, row, 2 * k, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] += bias.u[i];
      store8((T *)a.out.p + r * a.out.ld + c, n, f);
    }
  }
}
// Checkpoints of P rows, `step` rows apart; a rare group's branch is behind all of
// their chains.
template <int P>
__device__ __forceinline__ void put_rows(const Ckpt &k, int64_t r, int step, int c,
                                         const float (&v)[P][8]) {
  uint32_t m[P], E[P];
  uint2 q[P];
  bool top = false;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    m[i] = largest_of(v[i]);
    E[i] = exponent_of(m[i]);
    q[i] = codes_of(v[i], E[i]);
    top |= at_top(m[i]);
  }
  if (__builtin_expect(top, 0)) {
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (at_top(m[i])) q[i] = top_codes_of(v[i], m[i], &E[i]);
  }
#pragma unroll
  for (int i = 0; i < P; ++i) *(uint2 *)(k.q + (r + i * step) * k.pitch + c) = q[i];
  if ((c & (kGroup - 1)) == 0) {
#pragma unroll
    for (int i = 0; i < P; ++i)
      k.e[(r + i * step) * (k.pitch / kGroup) + c / kGroup] = (uint8_t)E[i];
  }
}
// As strip_rows where all of the strip's rows and features are there: its passes side by
// side, without branches between their instructions. The wave has a SIMD for
// itself, and each pass is a chain of dependent ones (67800 x 2048 x 8192 bf16 with
// checkpoints, one pass after another, two and four side by side: forward 4.14, 3.89, 3.85
// ms, backward 2.98, 2.62, 2.62).
template <typename T, int EPI, int FB, int KIND, typename Codes>
__device__ __forceinline__ void strip_whole(const FfnArgs &a, lds_char *l, int r0, int c0,
                                            const Bias &bias, Codes &&codes) {
  typedef Lanes<EPI, FB> N;
  constexpr int P = 32 / N::ROWS;
  const int lane = threadIdx.x & 63, k = lane % N::PER, c = c0 + 8 * k, row = lane / N::PER;
  const int64_t r = r0 + row;
  float u[P][8], v[P][8], f[P][8], df[P][8];
  if constexpr (EPI == EPI_GATE) {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int rj = row + j * N::ROWS, slot = k / 4 * 16 + k % 4 * 2;
      strip_get<FB>(l, rj, slot, u[j]);
      strip_get<FB>(l, rj, slot + 8, v[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[j][i] += bias.u[i], v[j][i] += bias.v[i];
    }
#pragma unroll
    for (int j = 0; j < P; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        activate<KIND, true>(u[j][i], f[j][i], df[j][i]);
        f[j][i] *= v[j][i];
      }
  } else {
    codes(row, u, v);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      float d[8];
      strip_get<FB>(l, row + j * N::ROWS, 2 * k, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        activate<KIND, true>(u[j][i], f[j][i], df[j][i]);
        df[j][i] *= d[i] * v[j][i];
        d[i] *= f[j][i];
        f[j][i] *= v[j][i];
        v[j][i] = d[i];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < P; ++j) {
    T *q = (T *)a.out.p + (r + j * N::ROWS) * a.out.ld + c;
    if constexpr (EPI == EPI_GATE) {
      store8(q, 8, f[j]);
    } else {
      store8(q, 8, df[j]);
      store8(q + a.feats, 8, v[j]);
    }
  }
  if constexpr (EPI == EPI_GATE) {
    if (a.uv.p) {
#pragma unroll
      for (int j = 0; j < P; ++j) {
        T *q = (T *)a.uv.p + (r + j * N::ROWS) * a.uv.ld + c;
        store8(q, 8, u[j]);
        store8(q + a.feats, 8, v[j]);
      }
    }
    if (a.ku.q) put_rows<P>(a.ku, r, N::ROWS, c, u);
    if (a.kv.q) put_rows<P>(a.kv, r, N::ROWS, c, v);
  } else {
    if (a.ka.q) put_rows<P>(a.ka, r, N::ROWS, c, f);
  }
}
// EPI_BACK: u and v of eight features from memory, zeros where there are none
template <typename T>
__device__ __forceinline__ void read_uv(const FfnArgs &a, int64_t r, int c, float (&u)[8],
                                        float (&v)[8]) {
  r = min(r, (int64_t)a.rows - 1);
  if (a.uv.p) {
    const T *q = (const T *)a.uv.p + r * a.uv.ld + c;
    load8(q, a.feats - c).get(u);
    load8(q + a.feats, a.feats - c).get(v);
  } else if (c < a.ku.pitch) {
    get8(a.ku, r, c, u);
    get8(a.kv, r, c, v);
  }
}

// As read_uv, P rows `step` rows apart, all of them and the eight features there
template <typename T, int P>
__device__ __forceinline__ void read_whole(const FfnArgs &a, int64_t r, int step, int c,
                                           float (&u)[P][8], float (&v)[P][8]) {
  if (a.uv.p) {
    Raw8<T> ru[P], rv[P];
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const T *q = (const T *)a.uv.p + (r + j * step) * a.uv.ld + c;
      ru[j] = load8(q, 8);
      rv[j] = load8(q + a.feats, 8);
    }
#pragma unroll
    for (int j = 0; j < P; ++j) ru[j].get(u[j]), rv[j].get(v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      get8(a.ku, r + j * step, c, u[j]);
      get8(a.kv, r + j * step, c, v[j]);
    }
  }
}

// A strip's results, EPI_BACK: with u and v from memory. whole: all of its rows and
// features are there.
template <typename T, int EPI, int FB, bool BESIDE>
__device__ __forceinline__ void strip_out(const FfnArgs &a, lds_char *l, int r0, int c0,
                                          const Bias &bias, bool whole) {
  typedef Lanes<EPI, FB> N;
  const int c = c0 + 8 * (threadIdx.x % 64 % N::PER);
  if constexpr (BESIDE && EPI != EPI_PLAIN) {
    if (whole) {
      with_kind(a.kind, [&](auto K) {
        strip_whole<T, EPI, FB, decltype(K)::value>(
            a, l, r0, c0, bias, [&](int row, auto &u, auto &v) {
              read_whole<T>(a, (int64_t)r0 + row, N::ROWS, c, u, v);
            });
      });
      return;
    }
  }
  strip_rows<T, EPI, FB>(a, l, r0, c0, bias, [&](int row, float (&u)[8], float (&v)[8]) {
    read_uv<T>(a, r0 + row, c, u, v);
  });
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

// Small products: a tile of FB blocks of 32 features by RB of 32 rows. Its four waves
// split the depth of each step, a quarter each, and are summed at the end; so 32 rows by 32
// features are still work for a whole CU. ST: LDS stages.
template <int FB_, int RB_, int ST_>
struct Tile {
  static constexpr int FB = FB_, RB = RB_, ST = ST_, KS = 4;
  static constexpr int F = 32 * FB, R = 32 * RB, THREADS = 64 * KS;
  static constexpr int STAGE = (F + R) * kRow, SUMS = KS * FB * RB * 64 * 16 * 4;
  static constexpr int LDS = ST * STAGE > SUMS ? ST * STAGE : SUMS;
  static_assert(LDS >= RB * 32 * 32 * FB * 4, "a strip for each wave that has rows");
};

// A quarter of a step's products: fragments from an LDS stage. K order: lane half g takes
// the 16-byte vectors 4 g + q of a tile row, q = 0 .. 3, of both operands alike.
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

// 16 bytes a lane from global memory straight into LDS, lane l's to bytes 16 l of the
// wave's address: as load16_lds_a, with the wait state between writing M0 and its
// use by the copy that the GFX9 hazard rules ask for, which assembly has to keep by
// itself. The second form takes a scalar base and a lane's offset from it.
__device__ __forceinline__ void copy16(const void *p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(lds), "v"(p)
               : "memory", "m0");
}
__device__ __forceinline__ void copy16(const char *base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}

// Waits until at most min(k, MOST) steps' copies of LD each are on their way
template <int LD, int MOST>
__device__ __forceinline__ void wait_tiles(int k) {
  if constexpr (MOST > 0) {
    if (k >= MOST) return wait_vmcnt<MOST * LD>();
    wait_tiles<LD, MOST - 1>(k);
  } else {
    wait_vmcnt<0>();
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
  auto multiply = [&](int st) {
    const char *wt = smem + st * TL::STAGE;
    products<T, FB, RB>(wt, wt + TL::F * kRow, wave, lane, acc);
  };
  if constexpr (DMA) {
    const void *zero = &g_zero16[0];
    auto bring = [&](int st) {
      const bool ok = kpos < a.depth;
#pragma unroll
      for (int j = 0; j < NF + NR; ++j) {
        const int row = j < NF ? RP * j : TL::F + RP * (j - NF);
        copy16(ok ? gp[j] : (const char *)zero, lds0 + st * TL::STAGE + (row + wave * 8) * kRow);
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
      wait_tiles<LD, ST - 2>(steps - 1 - t);
      __syncthreads();
      if (t + ST - 1 < steps) bring(st == 0 ? ST - 1 : st - 1);
      multiply(st);
      st = st == ST - 1 ? 0 : st + 1;
    }
  } else {
    typedef std::conditional_t<sizeof(T) == 2, u32x4_a2, u32x4_a4> u32x4_a;
    // (two steps' loads are on their way while a third is multiplied)
    u32x4 reg0[NF + NR], reg1[NF + NR];
    auto fetch = [&](u32x4 (&reg)[NF + NR]) {
      if (kpos - vec * E + BK <= a.depth) {  // (the same for all threads)
#pragma unroll
        for (int j = 0; j < NF + NR; ++j) reg[j] = *(const u32x4_a *)gp[j];
      } else {
        const int n = a.depth - kpos;
#pragma unroll
        for (int j = 0; j < NF + NR; ++j) {
          const T *p = (const T *)gp[j];
          uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (e < n) {
              if constexpr (sizeof(T) == 2) w[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
              else w[e] = __float_as_uint(p[e]);
            }
          reg[j] = (u32x4){w[0], w[1], w[2], w[3]};
        }
      }
#pragma unroll
      for (int j = 0; j < NF + NR; ++j) gp[j] += kRow;
      kpos += BK;
    };
    auto keep = [&](const u32x4 (&reg)[NF + NR], int st) {
#pragma unroll
      for (int j = 0; j < NF + NR; ++j) {
        const int row = br + (j < NF ? RP * j : TL::F + RP * (j - NF));
        *(u32x4 *)(smem + st * TL::STAGE + row * kRow + (tid & 7) * 16) = reg[j];
      }
    };
    fetch(reg0);
    keep(reg0, 0);
    if (steps > 1) fetch(reg1);
    if (steps > 2) fetch(reg0);
    auto step = [&](int t, u32x4 (&next)[NF + NR]) {
      __syncthreads();
      if (t + 1 < steps) keep(next, (t + 1) & 1);
      if (t + 3 < steps) fetch(next);
      multiply(t & 1);
    };
    for (int t = 0; t < steps; t += 2) {
      step(t, reg1);
      if (t + 1 < steps) step(t + 1, reg0);
    }
  }
  Bias bias;
  const int c = f0 + 8 * (lane % Lanes<EPI, FB>::PER);
  bias.load<EPI>(a, c);
  __syncthreads();
  // the waves' sums joined in order; wave j takes the blocks of rows j
  float *red = (float *)smem;
#pragma unroll
  for (int i = 0; i < FB; ++i)
#pragma unroll
    for (int j = 0; j < RB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        red[(((wave * FB + i) * RB + j) * 16 + v) * 64 + lane] = acc[i][j][v];
  __syncthreads();
  if (wave < RB) {
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
  __syncthreads();
  if (wave >= RB) return;
  lds_char *const strip = (lds_char *)smem + wave * 32 * 32 * FB * 4;
  each<0, FB>([&](auto i) { strip_put<FB>(strip, i, acc[i][0]); });
  wave_meets();
  const int rj = r0 + 32 * wave;
  // (64 x 32, EPI_BACK: the registers of passes side by side cost it workgroups of the CU,
  // 3136 x 1024 x 2736 bf16 59 -> 74 us; 64 x 64 59 -> 53)
  constexpr bool BESIDE = !(EPI == EPI_BACK && FB > RB);
  strip_out<T, EPI, FB, BESIDE>(a, strip, rj, f0, bias,
                                rj + 32 <= a.rows && f0 + Lanes<EPI, FB>::WIDTH <= a.feats);
}

// Large products: four waves of FB x RB blocks of 32 x 32, one on each matrix pipe, two by
// two. Of 128 x 128 (FB = RB = 4) a wave reads (128 + 128) rows of fragments for 128 x 128
// products; with half-sized ones, eight waves to a tile, the LDS reads and the copies into it
// would take as long as the products. Tile rows of 128 bytes (64 bfloat16 or 32
// float32 of depth): whole cache lines; with rows of 64 bytes and twice the stages the
// L2's requests bound it. Two stages, of 64 KB with FB = RB = 4.
//
// A step has four slices of 16 bytes. Its order is laid down slot by slot, one block's
// products to a slot, with a share of the LDS reads of later slices' fragments and of the
// copies of a later step. A copy holds the memory pipe of the CU for 16 cycles, so the
// 4 LD of a step are spread over several slices: in one they stall the products. After
// the second slice all of the step's fragments are on their way or read, the waves meet,
// and its stage may be copied over. With two stages the copies of the step two ahead go
// out in three slices and have two to arrive, until the waves meet again before the
// fourth. With more they go out in four, and once a step the waves meet. Past the last
// step zeros are copied, so every step is alike.
// Four neighbouring exponent bytes, of those that there are
__device__ __forceinline__ uint32_t exponents4(const Ckpt &k, int64_t row, int c) {
  typedef uint32_t u32_a1 __attribute__((aligned(1)));
  const uint8_t *p = k.e + row * (k.pitch / kGroup) + c / kGroup;
  const int64_t left = k.pitch - c;
  if (left >= 4 * kGroup) return *(const u32_a1 *)p;
  uint32_t e = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i * kGroup < left) e |= (uint32_t)p[i] << (8 * i);
  return e;
}
template <int FB_, int RB_, int ST_>
struct Wide {
  static constexpr int FB = FB_, RB = RB_, F = 64 * FB, R = 64 * RB, STAGE = (F + R) * kRow;
  static constexpr int ST = ST_;
  // EPI_BACK, 128 features a wave: a strip of 64 features and the codes of u and v, 8 KB
  // for every 32 rows. The first rows' are behind the stages, if there is room.
  static constexpr bool EARLY = ST * STAGE + 4 * 8192 <= 163840;
  static constexpr int PART = 8192 + 8192 * (EARLY ? RB - 1 : RB);
  static constexpr int LDS = FB < 4 ? ST * STAGE : EARLY ? ST * STAGE + 4 * 8192
                             : ST * STAGE > 4 * PART ? ST * STAGE : 4 * PART;
  static_assert(FB < 4 || 4 * PART <= (EARLY ? ST * STAGE : LDS), "a wave's part");
};
template <typename T, typename W, int EPI, bool DMA>
__global__ __launch_bounds__(256, W::LDS > 81920 ? 1 : 2) void ffn_wide_kernel(FfnArgs a) {
  constexpr int E = 16 / (int)sizeof(T), BK = kRow / (int)sizeof(T);
  constexpr int FB = W::FB, RB = W::RB, STAGE = W::STAGE, ST = W::ST;
  constexpr int LF = W::F / 32, LD = LF + W::R / 32;  // copies a thread and step
  constexpr bool CODES = EPI == EPI_BACK && FB == 4;
  __shared__ __align__(16) char smem[CODES ? W::LDS : ST * STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int tx, ty;
  tile_of(a, &tx, &ty);
  const int r0 = tx * W::R, f0 = ty * (EPI == EPI_GATE ? W::F / 2 : W::F);
  const int steps = (a.depth + BK - 1) / BK;
  // rows tid / 8 + 32 j of each operand, one vector each, to slot tid % 8
  const int br = tid >> 3, vec = (tid & 7) ^ ((tid >> 4) & 7);
  uint32_t off[LD];
  const int first = min(r0, a.rows - 1);
#pragma unroll
  for (int j = 0; j < LF; ++j) {
    const int t = br + 32 * j;
    int64_t f;
    if constexpr (EPI == EPI_GATE) {
      const int h = f0 + t / 64 * 32 + (t & 31);  // blocks of u and v in turn
      f = min(h, a.feats - 1) + ((t >> 5) & 1 ? (int64_t)a.feats : 0);
    } else {
      f = min(f0 + t, a.feats - 1);
    }
    off[j] = (uint32_t)((f * a.depth + vec * E) * (int64_t)sizeof(T));
  }
#pragma unroll
  for (int j = LF; j < LD; ++j) {
    const int t = br + 32 * (j - LF);
    off[j] = (uint32_t)(((int64_t)(min(r0 + t, a.rows - 1) - first) * a.x.ld + vec * E) *
                        (int64_t)sizeof(T));
  }
  const char *gw = a.w, *gx = a.x.p + (int64_t)first * a.x.ld * (int64_t)sizeof(T);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem +
                        wave * 8 * kRow;
  int kpos = 0;  // of the step to copy
  // Not aligned: a step's copy j is a load and, a step later, in the place where the
  // next one's is issued, a write to LDS.
  typedef std::conditional_t<sizeof(T) == 2, u32x4_a2, u32x4_a4> u32x4_a;
  u32x4 held[DMA ? 1 : LD];
  auto pull = [&](int j, auto whole) {
    typedef __attribute__((address_space(1))) const char g_char;
    g_char *p = (g_char *)(j < LF ? gw : gx) + off[j];
    const int n = a.depth - kpos - vec * E;
    if (decltype(whole)::value || n >= E) {
      held[j] = *(__attribute__((address_space(1))) const u32x4_a *)p;
    } else {
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e < n) {
          const T v = ((__attribute__((address_space(1))) const T *)p)[e];
          if constexpr (sizeof(T) == 2) w[e / 2] |= (uint32_t)v << (16 * (e & 1));
          else w[e] = __float_as_uint(v);
        }
      held[j] = (u32x4){w[0], w[1], w[2], w[3]};
    }
  };
  typedef __attribute__((address_space(3))) u32x4 lds_vec;
  lds_char *const mine = (lds_char *)smem + br * kRow + (tid & 7) * 16;
  // WHOLE: the step's depth is there to its end
  auto bring = [&](int st, int j, auto whole) {
    const uint32_t to = lds0 + st * STAGE + 32 * kRow * j;
    if constexpr (!DMA) {
      *(lds_vec *)(mine + st * STAGE + 32 * kRow * j) = held[j];
      pull(j, whole);
    } else if constexpr (decltype(whole)::value) {
      copy16(j < LF ? gw : gx, off[j], to);
    } else {
      const bool ok = kpos + vec * E < a.depth;
      copy16(ok ? (j < LF ? gw : gx) + off[j] : (const char *)&g_zero16[0], to);
    }
  };
  auto advance = [&]() {
    kpos += BK, gw += kRow, gx += kRow;
    asm volatile("" : "+s"(gw), "+s"(gx));
  };
  f32x16 acc[FB][RB];
#pragma unroll
  for (int i = 0; i < FB; ++i)
#pragma unroll
    for (int j = 0; j < RB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  const int wf = wave & 1, wr = wave >> 1;
  typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
  lds_char *lds = (lds_char *)smem;
  // a fragment of slice q: vector 4 (lane / 32) + q of row lane % 32 of its block
  int pw[4], px[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int r = lane & 31, at = r * kRow + swz<8>(r, 4 * (lane >> 5) + q) * 16;
    pw[q] = at + wf * 32 * FB * kRow;
    px[q] = at + (W::F + wr * 32 * RB) * kRow;
  }
  u32x4 fw[4][FB], fx[4][RB];  // by slice
  constexpr int S = FB * RB, N = FB + RB;  // slots of a slice, its fragments
  // fragment k of slice q: the first weights', the rows', then the other weights'
  auto fragment = [&](int st, auto q_, auto k_) {
    constexpr int q = decltype(q_)::value, k = decltype(k_)::value;
    if constexpr (k == 0) fw[q][0] = *(lds_u32x4 *)(lds + st * STAGE + pw[q]);
    else if constexpr (k <= RB)
      fx[q][k - 1] = *(lds_u32x4 *)(lds + st * STAGE + px[q] + (k - 1) * 32 * kRow);
    else fw[q][k - RB] = *(lds_u32x4 *)(lds + st * STAGE + pw[q] + (k - RB) * 32 * kRow);
  };
  using std::integral_constant;
  // Slice q: reads READS slices' fragments from slice `from` on out of stage sr; copies
  // the copies C0 .. C1 of a step to stage sc
  auto slice = [&](auto q_, auto from, auto reads, int sr, auto c0, auto c1, int sc, auto whole) {
    constexpr int q = decltype(q_)::value, K = decltype(reads)::value * N;
    constexpr int B = decltype(c0)::value, C = decltype(c1)::value - B;
    constexpr int L = S > 8 ? 3 * S / 4 : S;  // the reads in the first L slots
    each<0, S>([&](auto m_) {
      constexpr int m = decltype(m_)::value, i = m / RB, j = m % RB;
      if constexpr (sizeof(T) == 2) {
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fw[q][i]),
                                                            __builtin_bit_cast(bf16x8, fx[q][j]),
                                                            acc[i][j], 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(fw[q][i][e]),
                                                           __uint_as_float(fx[q][j][e]),
                                                           acc[i][j], 0, 0, 0);
      }
      each<K * least(m, L) / L, K * least(m + 1, L) / L>([&](auto k) {
        constexpr int x = decltype(k)::value;
        fragment(sr, integral_constant<int, (decltype(from)::value + x / N) % 4>(),
                 integral_constant<int, x % N>());
      });
      each<B + C * m / S, B + C * (m + 1) / S>([&](auto j) { bring(sc, j, whole); });
      __builtin_amdgcn_sched_barrier(0);
    });
  };
#define I(x) integral_constant<int, (x)>()
  // From a step's third slice to the next one's second. LAST: there is no next one.
  int st = 0;
  auto turn = [&](auto whole, auto last) {
    constexpr bool LAST = decltype(last)::value;
    const int nx = st == ST - 1 ? 0 : st + 1;
    if constexpr (ST == 2) {
      constexpr int C = LAST ? 0 : LD, C2 = 3 * C / 8, C3 = (C - C2) / 2 + C2;
      __syncthreads();
      slice(I(2), I(0), I(0), nx, I(0), I(C2), st, whole);
      if constexpr (DMA) wait_vmcnt<C2>();
      __syncthreads();
      slice(I(3), I(0), I(LAST ? 0 : 1), nx, I(C2), I(C3), st, whole);
      if constexpr (!LAST) {
        slice(I(0), I(1), I(2), nx, I(C3), I(C), st, whole);
        slice(I(1), I(3), I(1), nx, I(0), I(0), st, whole);
      }
    } else {
      constexpr int C = LAST ? 0 : LD, R1 = LAST ? 0 : 1;
      if constexpr (DMA) wait_vmcnt<(ST - 2) * LD>();
      __syncthreads();
      slice(I(2), I(0), I(R1), nx, I(0), I(C / 4), st, whole);
      slice(I(3), I(1), I(R1), nx, I(C / 4), I(C / 2), st, whole);
      if constexpr (!LAST) {
        slice(I(0), I(2), I(1), nx, I(C / 2), I(3 * C / 4), st, whole);
        slice(I(1), I(3), I(1), nx, I(3 * C / 4), I(C), st, whole);
      }
    }
    if constexpr (!LAST) advance();
    st = nx;
  };
  using std::false_type;
  if constexpr (!DMA) {
#pragma unroll
    for (int j = 0; j < LD; ++j) pull(j, false_type());
    advance();
  }
#pragma unroll 1
  for (int i = 0; i < ST; ++i) {
#pragma unroll
    for (int j = 0; j < LD; ++j) bring(i, j, false_type());
    advance();
  }
  // EPI_BACK from checkpoints: the codes of this wave's rows 32 j on, 1 KB a copy, and
  // exponents of rows lane and lane + 64
  const int wrow = r0 + wr * 32 * RB, wcol = f0 + wf * 128;
  constexpr int HR = (RB + 1) / 2;
  uint32_t eu[HR], ev[HR];
  // (EARLY: a wave's part is the codes of j = 1 .. RB - 1, then the strip; else the strip first)
  auto codes_at = [&](int j) {
    const int at = wave * W::PART + 8192 * (W::EARLY ? j - 1 : j + 1);
    return (lds_char *)smem + (W::EARLY && j == 0 ? ST * STAGE + wave * 8192 : at);
  };
  auto bring_codes = [&](int j) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 32 * j + 8 * i + lane / 8, c = wcol + ((lane & 7) ^ (row & 7)) * 16;
      const int64_t r = min(wrow + row, a.rows - 1);
      const bool ok = c < a.ku.pitch;
      const uint32_t to = (uint32_t)(uintptr_t)codes_at(j) + i * 1024;
      const char *const zero = (const char *)&g_zero16[0];
      copy16(ok ? (const char *)a.ku.q + r * a.ku.pitch + c : zero, to);
      copy16(ok ? (const char *)a.kv.q + r * a.kv.pitch + c : zero, to + 4096);
    }
  };
  const bool ck = CODES && a.ku.q && wcol < a.feats;
  if constexpr (CODES) {
#pragma unroll
    for (int h = 0; h < HR; ++h) eu[h] = ev[h] = 0;
    if (ck) {
      if constexpr (W::EARLY) bring_codes(0);
#pragma unroll
      for (int h = 0; h < HR; ++h) {
        const int64_t r = min(wrow + 64 * h + lane, a.rows - 1);
        eu[h] = exponents4(a.ku, r, wcol);
        ev[h] = exponents4(a.kv, r, wcol);
      }
    }
  }
  if constexpr (DMA) wait_vmcnt<(ST - 1) * LD>();
  __syncthreads();
  each<0, N>([&](auto k) { fragment(0, I(0), k); });
  if constexpr (ST == 2) {
    slice(I(0), I(1), I(2), 0, I(0), I(0), 0, false_type());
    slice(I(1), I(3), I(1), 0, I(0), I(0), 0, false_type());
  } else {
    each<0, N>([&](auto k) { fragment(0, I(1), k); });
    slice(I(0), I(2), I(1), 0, I(0), I(0), 0, false_type());
    slice(I(1), I(3), I(1), 0, I(0), I(0), 0, false_type());
  }
  int t = 0;
  for (; kpos + BK <= a.depth; ++t) turn(std::true_type(), false_type());
  for (; t + 1 < steps; ++t) turn(false_type(), false_type());
  turn(false_type(), std::true_type());
#undef I
  if constexpr (DMA || CODES) wait_vmcnt<0>();
  __syncthreads();
  if constexpr (!CODES) {
    const int c0 = f0 + wf * Lanes<EPI, FB>::WIDTH, k = lane % Lanes<EPI, FB>::PER;
    Bias bias;
    bias.load<EPI>(a, c0 + 8 * k);
    lds_char *const strip = (lds_char *)smem + wave * 32 * 32 * FB * 4;
    const bool whole = wrow + 32 * RB <= a.rows && c0 + Lanes<EPI, FB>::WIDTH <= a.feats;
#pragma unroll 1
    for (int j = 0; j < RB; ++j) {
      each<0, RB>([&](auto j_) {
        if (j == j_) {
          each<0, FB>([&](auto i) { strip_put<FB>(strip, i, acc[i][j_]); });
          own_branch<j_>();
        }
      });
      wave_meets();
      strip_out<T, EPI, FB, true>(a, strip, wrow + 32 * j, c0, bias, whole);
      wave_meets();
    }
  } else {
    // The first rows' codes are there; the others' are on their way while the strips of
    // the first are worked on. (A wait for a load waits for the stores before it, so none
    // is loaded later.)
    lds_char *const strip = codes_at(W::EARLY ? RB : -1);
    const bool whole = wrow + 32 * RB <= a.rows && wcol + 128 <= a.feats;
    if (ck) {
      for (int j = W::EARLY; j < RB; ++j) bring_codes(j);
      if constexpr (!W::EARLY) wait_vmcnt<0>();
    }
#pragma unroll 1
    for (int jh = 0; jh < 2 * RB; ++jh) {
      if (W::EARLY && ck && jh == 2) {
        // (two whole strips have at least 16 stores, newer than the codes)
        if (whole) wait_vmcnt<16>();
        else wait_vmcnt<0>();
      }
      each<0, 2 * RB>([&](auto x) {
        constexpr int j = decltype(x)::value / 2, h = decltype(x)::value % 2;
        if (jh == x) {
          each<0, 2>([&](auto i) { strip_put<2>(strip, i, acc[2 * h + i][j]); });
          own_branch<x>();
        }
      });
      wave_meets();
      const int j = jh >> 1, h = jh & 1, rj = wrow + 32 * j;
      const uint32_t wu = j < 2 ? eu[0] : eu[HR - 1], wv = j < 2 ? ev[0] : ev[HR - 1];
      const lds_char *const held = codes_at(j);
      const int k = lane & 7;
      auto codes = [&](int row, float (&u)[8], float (&v)[8]) {
        const int at = row * 128 + ((4 * h + k / 2) ^ (row & 7)) * 16 + k % 2 * 8;
        const int from = (32 * j + row) & 63, by = 8 * (2 * h + k / 4);
        decode8(lds_pair(held + at), (__shfl(wu, from) >> by) & 255u, u);
        decode8(lds_pair(held + at + 4096), (__shfl(wv, from) >> by) & 255u, v);
      };
      if (whole) {
        auto all = [&](int row, auto &u, auto &v) {
          if (ck) {
#pragma unroll
            for (int p = 0; p < 4; ++p) codes(row + 8 * p, u[p], v[p]);
          } else {
            read_whole<T>(a, (int64_t)rj + row, 8, wcol + 64 * h + 8 * k, u, v);
          }
        };
        with_kind(a.kind, [&](auto K) {
          strip_whole<T, EPI, 2, decltype(K)::value>(a, strip, rj, wcol + 64 * h, Bias(), all);
        });
      } else {
        strip_rows<T, EPI, 2>(a, strip, rj, wcol + 64 * h, Bias(),
                              [&](int row, float (&u)[8], float (&v)[8]) {
                                if (ck) codes(row, u, v);
                                else read_uv<T>(a, rj + row, wcol + 64 * h + 8 * k, u, v);
                              });
      }
      wave_meets();
    }
  }
}

// Few rows (up to 16 NC): the weights' bytes bound it. 16 NF features (EPI_GATE: of u and
// of v) a workgroup, eight waves that take turns along the depth, 128 bytes of a weight
// row a step, straight into registers. NF 1 where that is all, 2 where checkpoints
// are written or read: their groups of 32 leave by a strip.
template <typename T, int NC, int EPI, int NF>
__global__ __launch_bounds__(512) void ffn_few_kernel(FfnArgs a) {
  constexpr int E = 16 / (int)sizeof(T), BK = kRow / (int)sizeof(T);
  constexpr int H = EPI == EPI_GATE ? 2 : 1, W = 8, U = 4 / (H * NF);
  __shared__ float red[W][H][NF][NC][64][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int f0 = blockIdx.x * 16 * NF, g = lane >> 4;
  const T *w[H][NF], *x[NC];
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int f = 0; f < NF; ++f)
      w[h][f] = (const T *)a.w + g * 2 * E +
                (min(f0 + 16 * f + (lane & 15), a.feats - 1) + (int64_t)h * a.feats) * a.depth;
#pragma unroll
  for (int c = 0; c < NC; ++c)
    x[c] = (const T *)a.x.p + (int64_t)min(16 * c + (lane & 15), a.rows - 1) * a.x.ld + g * 2 * E;
  f32x4 acc[H][NF][NC];
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[h][f][c] = (f32x4){0.f, 0.f, 0.f, 0.f};
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
    u32x4 fw[N][H][NF][2], fx[N][NC][2];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int at = k + n * W * BK + q * E, left = a.depth - at - g * 2 * E;
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int f = 0; f < NF; ++f) fw[n][h][f][q] = load(w[h][f] + at, left, whole);
#pragma unroll
        for (int c = 0; c < NC; ++c) fx[n][c][q] = load(x[c] + at, left, whole);
      }
    auto one = [&](f32x4 &d, u32x4 p, u32x4 q) {
      if constexpr (sizeof(T) == 2) {
        d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p),
                                                    __builtin_bit_cast(bf16x8, q), d, 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          d = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(p[e]), __uint_as_float(q[e]), d,
                                                   0, 0, 0);
      }
    };
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int c = 0; c < NC; ++c) one(acc[h][f][c], fw[n][h][f][q], fx[n][c][q]);
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
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int c = 0; c < NC; ++c) *(f32x4 *)red[wave][h][f][c][lane] = acc[h][f][c];
  __syncthreads();
  if constexpr (NF == 2) {
    __shared__ __align__(16) char strip_[32 * 32 * H * 4];
    lds_char *const strip = (lds_char *)strip_;
    for (int t = threadIdx.x; t < H * 2 * NC * 64; t += 512) {
      const int l = t & 63, c = t / 64 % NC, f = t / (64 * NC) % 2, h = t / (128 * NC);
      f32x4 s = *(const f32x4 *)red[0][h][f][c][l];
#pragma unroll
      for (int i = 1; i < W; ++i) s += *(const f32x4 *)red[i][h][f][c][l];
      *(lds_f32x4 *)slot_of<H>(strip, 16 * c + (l & 15), 8 * h + 4 * f + (l >> 4)) = s;
    }
    __syncthreads();
    if (wave) return;
    const int c = f0 + 8 * (lane % Lanes<EPI, H>::PER);
    Bias bias;
    bias.load<EPI>(a, c);
    strip_rows<T, EPI, H>(a, strip, 0, f0, bias, [&](int row, float (&u)[8], float (&v)[8]) {
      read_uv<T>(a, row, c, u, v);
    });
  } else {
    for (int t = threadIdx.x; t < 256 * NC; t += 512) {
      const int ft = t & 15, row = t >> 4, c = row >> 4, l = (ft >> 2) * 16 + (row & 15);
      if (row >= a.rows || f0 + ft >= a.feats) continue;
      float s[H];
#pragma unroll
      for (int h = 0; h < H; ++h) {
        s[h] = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) s[h] += red[i][h][0][c][l][ft & 3];
        if (a.bias) s[h] += a.bias[h * a.feats + f0 + ft];
      }
      if constexpr (EPI == EPI_GATE) {
        if (a.uv.p) {
          T *p = (T *)a.uv.p + row * a.uv.ld + f0 + ft;
          put(p, s[0]);
          put(p + a.feats, s[1]);
        }
        float fu[1], df[1];
        const float u[1] = {s[0]};
        activate_all(a.kind, u, fu, df);
        s[0] = fu[0] * s[1];
      }
      put((T *)a.out.p + row * a.out.ld + f0 + ft, s[0]);
    }
  }
}

// ------------------------------------------------------------- launches
typedef Wide<4, 4, 2> Big;                // 256 features x 256 rows
typedef Wide<4, 2, 3> Half;               // 256 x 128
typedef Wide<2, 2, 2> Mid;                // 128 x 128
typedef Wide<2, 2, 4> Deep;               // 128 x 128, one workgroup a CU
typedef Tile<2, 2, 3> Small;              // 64 x 64
typedef Tile<2, 1, 3> Tiny;               // 64 x 32
typedef Tile<1, 1, 3> Least;              // 32 x 32, one block of features
// One limit for all products. 32 rows, few and the best tile, us: 2048 x 8192 bf16 z 23 and
// 28, backward from checkpoints 12.8 and 12.4, dx 44 and 52; 512 x 2048 float32 z 12.5 and 29,
// backward 8.7 and 8.8, dx 23 and 37. The forward pass' first kernel gains nothing (float32
// 11.2 and 11.5) and loses in bfloat16 over a wide block: 18.2 and 14.6 at 32 rows, 17.1 and
// 13.8 at 16, so there the limit is not the faster choice.
constexpr int kFewRows = 32;

void lay_out(FfnArgs &a, int rows, int feats) {
  a.gx = (a.rows + rows - 1) / rows;
  a.gy = (a.feats + feats - 1) / feats;
  a.panel = fast_div(8 * (uint32_t)a.gy);
  a.rest = fast_div((uint32_t)std::max(a.gx & 7, 1));
}
template <typename T, typename TL, int EPI, bool DMA>
void launch(FfnArgs &a, hipStream_t s) {
  lay_out(a, TL::R, EPI == EPI_GATE ? TL::F / 2 : TL::F);
  ffn_kernel<T, TL, EPI, DMA><<<(unsigned)(a.gx * a.gy), TL::THREADS, 0, s>>>(a);
}

template <typename T, typename W, int EPI, bool DMA>
void launch_wide(FfnArgs &a, hipStream_t s) {
  lay_out(a, W::R, EPI == EPI_GATE ? W::F / 2 : W::F);
  ffn_wide_kernel<T, W, EPI, DMA><<<(unsigned)(a.gx * a.gy), 256, 0, s>>>(a);
}

template <typename T, int EPI>
void product(FfnArgs a, hipStream_t s) {
  constexpr int H = EPI == EPI_GATE ? 2 : 1;
  constexpr int kFew = 7;  // number of the variant for few rows; the others: costs below
  const int forced = g_ffn_tile;
  if (a.rows <= kFewRows && (forced < 0 || forced == kFew)) {
    auto few = [&](auto nc, auto nf) {
      const unsigned g = (unsigned)((a.feats + 16 * nf.value - 1) / (16 * nf.value));
      ffn_few_kernel<T, nc.value, EPI, nf.value><<<g, 512, 0, s>>>(a);
    };
    using std::integral_constant;
    const integral_constant<int, 1> one;
    const integral_constant<int, 2> two;
    if constexpr (EPI != EPI_PLAIN)
      if (EPI == EPI_BACK || a.ku.q || a.kv.q) return a.rows <= 16 ? few(one, two) : few(two, two);
    if constexpr (EPI != EPI_BACK) return a.rows <= 16 ? few(one, one) : few(two, one);
  }
  constexpr int E = 16 / (int)sizeof(T);
  const bool dma = ((uintptr_t)a.x.p | (uintptr_t)a.w) % 16 == 0 && a.x.ld % E == 0 &&
                   a.depth % E == 0;
  auto tiles = [&](int64_t f, int64_t r) {
    return (((int64_t)a.feats * H + f - 1) / f) * ((a.rows + r - 1) / r);
  };
  // (the wide tiles' copies have 32-bit offsets)
  const bool near = (int64_t)a.feats * H * a.depth * (int64_t)sizeof(T) < (int64_t)1 << 32 &&
                    Big::R * a.x.ld * (int64_t)sizeof(T) < (int64_t)1 << 32;
  // The variant of the least estimated time: for n tiles on the busiest of 256 CUs,
  // steps * max(alone, n * busy) + n * finish, in ns measured with one tile on a CU, with
  // many, and for the results. Measured by variant at thirteen sizes from 33 x 2048 x 8192 and
  // 392 x 512 x 2048 to 12000 x 512 x 2048, the pick is within 13% of the best (the first
  // kernel of 256 x 2048 x 8192 24.3 us against 21.5, z of 2000 x 512 x 2048 13.8 against
  // 12.2) and mostly within 5%: 3136 x 1024 x 2736 bf16 in tiles of 256 x 256, 256 x 128, 128
  // x 128 two and one a CU, 64 x 64, 64 x 32: first kernel 64, 56, 48, 54, 77, 83 us, z 55, 40,
  // 32, 28, 47, 57, backward 46, 49, 42, 47, 53, 59; picked 48, 29 and 42. (The times for the
  // results are from before the strips' passes ran side by side: too long for some tiles.)
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int G = EPI == EPI_GATE ? 0 : EPI == EPI_BACK ? 1 : 2;
  struct Cost {
    int f, r, alone, busy, finish[3];
    bool wide;
  };
  constexpr Cost costs[] = {
      {Big::F, Big::R, F32 ? 7100 : 1100, F32 ? 7100 : 1150, {20000, 40000, 6000}, true},
      {Half::F, Half::R, F32 ? 3600 : 800, F32 ? 3600 : 900, {9000, 18000, 3000}, true},
      {Mid::F, Mid::R, F32 ? 1850 : 620, F32 ? 1850 : 530, {1500, 5000, 1500}, true},
      {Deep::F, Deep::R, F32 ? 1850 : 550, F32 ? 1850 : 550, {6000, 10000, 3000}, true},
      {Small::F, Small::R, F32 ? 690 : 290, F32 ? 630 : 220, {2200, 4000, 1000}, false},
      {Tiny::F, Tiny::R, F32 ? 440 : 220, F32 ? 370 : 160, {1400, 2500, 700}, false},
      {Least::F, Least::R, F32 ? 300 : 170, F32 ? 190 : 100, {0, 1300, 400}, false}};
  const int64_t steps = ((int64_t)a.depth * (int64_t)sizeof(T) + kRow - 1) / kRow;
  int pick = -1;
  int64_t least_time = 0;
  for (int i = 0; i < 7; ++i) {
    const Cost &c = costs[i];
    // (half-sized tiles through registers are not built: never the best by a tenth)
    if (c.wide && (!near || (!dma && i == 1))) continue;
    if ((i == 6 && EPI == EPI_GATE) || tiles(c.f, c.r) > kMostTiles) continue;
    if (forced == i) {
      pick = i;
      break;
    }
    const int64_t n = (tiles(c.f, c.r) + 255) / 256;
    // (through registers, smaller tiles take half as long again)
    const int64_t step = std::max<int64_t>(c.alone, n * c.busy) * (i > 3 && !dma ? 3 : 2) / 2;
    const int64_t time = steps * step + n * c.finish[G];
    if (pick < 0 || time < least_time) pick = i, least_time = time;
  }
  auto small = [&](auto tile) {
    using TL = decltype(tile);
    return dma ? launch<T, TL, EPI, true>(a, s) : launch<T, TL, EPI, false>(a, s);
  };
  auto wide = [&](auto tile) {
    using W = decltype(tile);
    return dma ? launch_wide<T, W, EPI, true>(a, s) : launch_wide<T, W, EPI, false>(a, s);
  };
  switch (pick) {
    case 0: return wide(Big());
    case 1: return launch_wide<T, Half, EPI, true>(a, s);
    case 2: return wide(Mid());
    case 3: return wide(Deep());
    case 4: return small(Small());
    case 5: return small(Tiny());
  }
  if constexpr (EPI != EPI_GATE) small(Least());
}

template <typename T>
void products_of(Epi epi, const FfnArgs &a, hipStream_t s) {
  if (epi == EPI_GATE) product<T, EPI_GATE>(a, s);
  else if (epi == EPI_BACK) product<T, EPI_BACK>(a, s);
  else product<T, EPI_PLAIN>(a, s);
}

}  // namespace
#endif  // LRCNN_FFN_KERNELS

}  // namespace act8
}  // namespace lrcnn
