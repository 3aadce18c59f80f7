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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int64_t kMaxFeatures = 1 << 24;  // 31 rows within 32-bit offsets
constexpr int64_t kMaxWgradRows = 1 << 30;
constexpr int kStep = 32;  // rows of dy and of the checkpoint per step

struct WgArgs {
  int rows, n, k;       // n outputs, k inputs
  int splits;           // split z takes the steps z, z + splits, ...
  int gx, gy;           // tiles of n and of k
  FastDiv tiles, panel, rest, stride;  // by gx gy, 8 gy, gx mod 8, 32 splits
  Mat dy;
  Ckpt q;
  const float *scale, *shift;
  float *dw, *db;
  float *part, *dbpart;  // [splits][n][k], [splits][n]; null with one split
  int accumulate;
};

// hi + mid + lo == v (hi alone where v is not finite). As bfloat16 the low one is
// exact above 2^-110, where all its bits are multiples of 2^-133; below, it is
// rounded to one.
__device__ __forceinline__ void cut3(float v, float (&p)[3]) {
  p[0] = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
  float r = v - p[0];
  r = r == r ? r : 0.f;
  p[1] = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
  p[2] = r - p[1];
}
__device__ __forceinline__ uint4 bf_vec(const float *v) {
  return make_uint4(bf_pair(v[0], v[1]), bf_pair(v[2], v[3]), bf_pair(v[4], v[5]),
                    bf_pair(v[6], v[7]));
}

// Eight columns moved down by d < 8, per lane: a vector read d columns early
// so as to end with the last column.
__device__ __forceinline__ Raw8<bf16> moved_down(const Raw8<bf16> &r, int d) {
  const bool b4 = d & 4, b2 = d & 2, b1 = d & 1;
  const uint32_t x0 = b4 ? r.w[2] : r.w[0], x1 = b4 ? r.w[3] : r.w[1], x2 = r.w[2], x3 = r.w[3];
  const uint32_t y0 = b2 ? x1 : x0, y1 = b2 ? x2 : x1, y2 = b2 ? x3 : x2;
  Raw8<bf16> o;
  o.w[0] = b1 ? __builtin_amdgcn_alignbit(y1, y0, 16) : y0;
  o.w[1] = b1 ? __builtin_amdgcn_alignbit(y2, y1, 16) : y1;
  o.w[2] = b1 ? __builtin_amdgcn_alignbit(x3, y2, 16) : y2;
  o.w[3] = b1 ? x3 >> 16 : x3;
  return o;
}
__device__ __forceinline__ Raw8<float> moved_down(const Raw8<float> &r, int d) {
  const bool b4 = d & 4, b2 = d & 2, b1 = d & 1;
  const float x0 = b4 ? r.b[0] : r.a[0], x1 = b4 ? r.b[1] : r.a[1];
  const float x2 = b4 ? r.b[2] : r.a[2], x3 = b4 ? r.b[3] : r.a[3];
  const float y0 = b2 ? x2 : x0, y1 = b2 ? x3 : x1, y2 = b2 ? r.b[0] : x2;
  const float y3 = b2 ? r.b[1] : x3, y4 = b2 ? r.b[2] : r.b[0], y5 = b2 ? r.b[3] : r.b[1];
  Raw8<float> o;
  o.a = (f32x4_a4){b1 ? y1 : y0, b1 ? y2 : y1, b1 ? y3 : y2, b1 ? y4 : y3};
  o.b = (f32x4_a4){b1 ? y5 : y4, b1 ? r.b[2] : y5, b1 ? r.b[3] : r.b[2], r.b[3]};
  return o;
}

// f(0), f(1), ... f(N - 1), the index a constant
template <int B, int E, typename F>
__device__ __forceinline__ void each(F &&f) {
  if constexpr (B < E) {
    f(std::integral_constant<int, B>());
    each<B + 1, E>(f);
  }
}

// The tile of this workgroup. Workgroups go to the eight XCDs in turn; each XCD
// gets one run of tiles in order: splits last, and within one split through a
// panel of eight tiles of n before the next k, so that the tiles an XCD works
// on share rows of both operands in its L2.
__device__ __forceinline__ TileId panel_tile(const WgArgs &a) {
  const uint32_t total = gridDim.x, w = blockIdx.x;
  const uint32_t q = total >> 3, o = total & 7, c = w & 7, k = w >> 3;
  const uint32_t id = c < o ? c * (q + 1) + k : o * (q + 1) + (c - o) * q + k;
  uint32_t z, t, p, r, x, y;
  fdiv_qr(id, a.tiles, z, t);
  fdiv_qr(t, a.panel, p, r);
  if (8 * p + 8 <= (uint32_t)a.gx) y = r >> 3, x = r & 7;
  else fdiv_qr(r, a.rest, y, x);
  return TileId{(int)(8 * p + x), (int)y, (int)z};
}

// The workgroup's waves wait for each other, their LDS accesses before done. Unlike
// __syncthreads, which all threads have to reach at one place, this is the hardware's
// barrier, which counts waves: each may come from code of its own, so long as
// all come equally often and a whole wave at once.
__device__ __forceinline__ void waves_meet() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

constexpr int least(int a, int b) { return a < b ? a : b; }

// How a thread reads its eight columns of dy.
enum Cols {
  COLS_WHOLE,  // n a multiple of 8: a vector has all its columns or none
  COLS_SHIFT,  // the vector with the last column is read earlier and moved
  COLS_EACH    // n < 8: one by one
};

// A W x W tile of S by four waves of W/2 x W/2. Both operands go through
// registers into k-major LDS tiles (the codes as bfloat16, dy as it is or in
// three pieces), and to the matrix cores by transposing reads. A step's loads
// are issued ST steps before its tile is written to LDS, the tile is written
// one step before it is multiplied, and a unit's fragments (16 rows; one
// piece of dy) are read one unit before their MFMAs.
//
// There is one kind of step in the loop. Rows left over from whole steps are
// taken first, as the matrix' last 32 rows of which those that a whole step
// has count as zeros, and the steps that fill up the last round of ST multiply
// by zero; so the code that runs once is short, which a small call notices: its
// instructions come from memory (64 x 2048 x 1000 bf16 13.6 us with guarded steps
// for the ends, 7.6 as here). Columns past the matrix are read from its first
// ones: what they give is never stored.
//
// 67800 x 2048 x 8192 bf16 (2.27 TFLOP) takes 2.03 to 2.2 ms, 1030 to 1120
// TFLOP/s: 4.3 million cycles, the matrix pipes busy in 50% of them, at a clock
// that its own power brings down to 1.7 to 2.0 GHz (2.3 in the small calls); this
// card's library product of the size runs at 1142 with 54% busy. float32
// 67800 x 2048 x 2048 takes 1.69 ms, three products, 1009 TFLOP/s. Long and
// narrow calls (540000 x 256 x 173 bf16: 102 us and 8.9 for the join) take one and
// a half times what reading dy and the codes takes (68 us): 3.8 TB/s with the matrix
// pipes 29% busy, a third of that on columns past the 173rd. Small float32 ones
// (392 x 512 x 2048: 19 us) run 13 steps one after the other on 64 of the CUs, one wave
// a SIMD with its matrix pipe a quarter and its vector instructions a third of the time.
template <typename T, int W, int COLS>
__global__ __launch_bounds__(256, W == 256 ? 1 : 2) void wgrad8_kernel(WgArgs a) {
  constexpr int P = std::is_same<T, float>::value ? 3 : 1;  // pieces of dy
  constexpr int ST = W == 256 ? 3 : 2;                       // LDS tiles and load slots
  constexpr int NB = W / 64;                                 // 32 x 32 blocks per wave and side
  constexpr int U = 2 * P;                                   // units per step
  constexpr int LA = W / 8, RA = 256 / LA, NA = kStep / RA;  // dy: lanes, rows, passes
  constexpr int LB = W / 16, RB = 256 / LB, NQ = kStep / RB; // codes
  using M = KM<bf16, W>;
  constexpr int TB = kStep * W * 2;  // bytes of an LDS tile
  constexpr int EP = W / 2 + 8;      // float pitch of the epilogue's 32-row strips
  constexpr int LDS = ST * (P + 1) * TB > 512 * EP ? ST * (P + 1) * TB : 512 * EP;
  __shared__ __align__(16) char smem[LDS];
  __shared__ float dbs[W];
  const int tid = threadIdx.x, lane = tid & 63,
            wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const TileId tl = panel_tile(a);
  const int n0 = tl.x * W, k0 = tl.y * W;
  // This split's steps: every splits-th run of kStep rows, so that the
  // workgroups together read one window of rows that moves on
  const int stride = a.splits * kStep, first = tl.z * kStep;
  const int steps = first < a.rows ? (int)fdiv_q(a.rows - 1 - first, a.stride) + 1 : 0;
  const int some = min(a.rows, kStep);  // rows a step can read
  const int ar = tid / LA, ac = n0 + (tid % LA) * 8;
  const int br = tid / LB, bc = k0 + (tid % LB) * 16;
  int al = ac < a.n ? ac : 0, down = 0;
  if (COLS == COLS_SHIFT && ac < a.n && ac + 8 > a.n) al = a.n - 8, down = ac + 8 - a.n;
  const int bl = bc < a.q.pitch ? bc : 0;
  const int64_t pe_ld = a.q.pitch / kGroup;
  uint32_t oa[NA], oq[NQ], oe[NQ];  // bytes from a step's first row
#pragma unroll
  for (int i = 0; i < NA; ++i)
    oa[i] = (uint32_t)((min(ar + RA * i, some - 1) * a.dy.ld + al) * sizeof(T));
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const int r = min(br + RB * i, some - 1);
    oq[i] = (uint32_t)(r * a.q.pitch + bl);
    oe[i] = (uint32_t)(r * pe_ld + bl / kGroup);
  }
  struct Slot {
    Raw8<T> a[NA];
    uint4 q[NQ];
    uint32_t e[NQ];
    float live;  // 1, or 0 in a step that only fills up the last round
  } slot[ST];
  // The step to load: its number and its first row in the three arrays
  const int64_t ia = stride * a.dy.ld * (int64_t)sizeof(T), iq = stride * a.q.pitch,
                ie = stride * pe_ld;
  int nt = 0;
  float live = 1.f;
  const char *ga, *gq, *ge;
  auto place = [&](int64_t m) {
    ga = a.dy.p + m * a.dy.ld * (int64_t)sizeof(T);
    gq = (const char *)a.q.q + m * a.q.pitch;
    ge = (const char *)a.q.e + m * pe_ld;
  };
  // this split's last step is not whole: it comes first, `zero` rows early
  const int over = first + (steps - 1) * stride + kStep - a.rows;
  const bool odd = over > 0;
  const int zero = odd && a.rows >= kStep ? over : 0;
  place(odd ? max(a.rows - kStep, 0) : first);
  // (past the end the last step again. Scalar bases that the compiler may not
  // fold into one address per lane and load.)
  auto advance = [&]() {
    ++nt;
    const bool on = nt < steps;
    ga += on ? ia : 0, gq += on ? iq : 0, ge += on ? ie : 0;
    live = on ? 1.f : 0.f;
    asm volatile("" : "+s"(ga), "+s"(gq), "+s"(ge));
  };
  typedef __attribute__((address_space(1))) const char g_char;
  auto gload_dy = [&](Slot &s, int i) {
    uint32_t o = oa[i];
    asm volatile("" : "+v"(o));
    g_char *p = (g_char *)ga + o;
    if constexpr (COLS == COLS_EACH) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        v[e] = to_f(((__attribute__((address_space(1))) const T *)p)[min(e, a.n - 1)]);
      if constexpr (P == 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s.a[i].w[e] = bf_pair(v[2 * e], v[2 * e + 1]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) s.a[i].a[e] = v[e], s.a[i].b[e] = v[4 + e];
      }
    } else if constexpr (P == 1) {
      s.a[i].w = *(__attribute__((address_space(1))) const u32x4_a2 *)p;
    } else {
      s.a[i].a = *(__attribute__((address_space(1))) const f32x4_a4 *)p;
      s.a[i].b = *(__attribute__((address_space(1))) const f32x4_a4 *)(p + 16);
    }
  };
  auto gload_q = [&](Slot &s, int i) {
    uint32_t o = oq[i], oe_ = oe[i];
    asm volatile("" : "+v"(o), "+v"(oe_));
    const u32x4 v = *(__attribute__((address_space(1))) const u32x4 *)((g_char *)gq + o);
    s.q[i] = make_uint4(v.x, v.y, v.z, v.w);
    s.e[i] = *(__attribute__((address_space(1))) const uint8_t *)((g_char *)ge + oe_);
  };
  // LDS bytes of this thread's writes; passes are whole swizzle periods apart
  typedef __attribute__((address_space(3))) char lds_char;
  lds_char *lds = (lds_char *)smem;
  const int wa = 2 * M::off(ar, (tid % LA) * 8);
  const int wq = ST * P * TB + 2 * M::off(br, (tid % LB) * 16);
  auto put = [&](int at, uint4 v) {
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    *(lds_u32x4 *)(lds + at) = (u32x4){v.x, v.y, v.z, v.w};
  };
  // One of the eight columns of pass i of dy: with one piece the last one
  // writes them all; with three each is cut, and the last one writes.
  // FIRST: rows that do not count become zeros.
  uint32_t cut[P][4];
  float even[P];
  auto put_dy = [&](const Slot &s, int st, auto k, auto first_) {
    constexpr int i = decltype(k)::value / 8, e = decltype(k)::value % 8;
    const int at = wa + st * P * TB + 2 * RA * W * i;
    const int r = ar + RA * i;
    const bool in = !decltype(first_)::value || (r >= zero && r < some);
    if constexpr (P == 1) {
      if constexpr (e == 7) {
        const Raw8<T> x = COLS == COLS_SHIFT ? moved_down(s.a[i], down) : s.a[i];
        put(at, make_uint4(in ? x.w[0] : 0, in ? x.w[1] : 0, in ? x.w[2] : 0, in ? x.w[3] : 0));
      }
    } else {
      const Raw8<T> x = COLS == COLS_SHIFT ? moved_down(s.a[i], down) : s.a[i];
      float t[3];
      cut3(in ? e < 4 ? x.a[e & 3] : x.b[e & 3] : 0.f, t);
#pragma unroll
      for (int p = 0; p < P; ++p) {
        if constexpr (e % 2 == 0) even[p] = t[p];
        else cut[p][e / 2] = bf_pair(even[p], t[p]);
        if constexpr (e == 7)
          put(at + p * TB, make_uint4(cut[p][0], cut[p][1], cut[p][2], cut[p][3]));
      }
    }
  };
  // One of the sixteen codes of pass i
  float qstep, qeven;
  uint32_t qw[4];
  auto put_q = [&](const Slot &s, int st, auto k) {
    constexpr int i = decltype(k)::value / 16, c = decltype(k)::value % 16;
    if constexpr (c == 0) qstep = step_of(s.e[i]) * s.live;
    const uint32_t w = c < 4 ? s.q[i].x : c < 8 ? s.q[i].y : c < 12 ? s.q[i].z : s.q[i].w;
    const float v = (float)(int8_t)(w >> (8 * (c % 4))) * qstep;
    if constexpr (c % 2 == 0) qeven = v;
    else qw[c / 2 % 4] = bf_pair(qeven, v);
    if constexpr (c % 8 == 7)
      put(wq + st * TB + 2 * RB * W * i + 2 * (c - 7), make_uint4(qw[0], qw[1], qw[2], qw[3]));
  };

  f32x16 acc[NB][NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  const int wn = (wave & 1) * (W / 2), wk = (wave >> 1) * (W / 2);
  // fragments of the unit being multiplied and of the next one, as the two
  // reads that fetch them; b by slice
  bf16x4 fa[2][NB][2], fb[2][NB][2];
#pragma unroll
  for (int i = 0; i < 2 * NB; ++i)
    fa[1][i / 2][i % 2] = fb[1][i / 2][i % 2] =
        (bf16x4){(__bf16)0.f, (__bf16)0.f, (__bf16)0.f, (__bf16)0.f};
  float dbv[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) dbv[i] = 0.f;
  // A transposing read hands lane 16 G + 4 r + c of a wave the elements of
  // column 16 (G & 1) + its own place in the 16 lanes, of the K rows
  // 16 (G >> 1) + 8 s + [0, 4); a second one, four rows on, the next four.
  // The row's swizzle depends on r alone, so blocks of 32 columns are an
  // address each, and everything else is a constant.
  int pa_[NB], pb_[NB];
  {
    const int G = lane >> 4, r = (lane >> 2) & 3, c = 16 * (G & 1) + 4 * (lane & 3);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      pa_[i] = 2 * M::off(16 * (G >> 1) + r, wn + 32 * i + c);
      pb_[i] = ST * P * TB + 2 * M::off(16 * (G >> 1) + r, wk + 32 * i + c);
    }
  }
  auto read = [&](int at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(lds + at));
  };
  auto whole8 = [&](const bf16x4 (&h)[2]) {
    return __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
  };
  using std::integral_constant;
  // A step on LDS tile st. Its order is laid down instruction by
  // instruction: a slot is one MFMA, which holds the matrix pipe for eight
  // issue slots of the only wave on it, and a share of everything else -- the
  // LDS reads of the next unit's fragments, the next step's tile written from
  // its load slot, the loads that take the slot's place. Left to itself the
  // compiler puts the MFMAs in runs, and the matrix pipe idles between them.
  // The last slots before the barrier have no LDS access to wait for.
  // D: the slice whose fragments of dy this wave sums for db (two waves hold
  // the same dy and take one each), or 2: db is not wanted here.
  uint32_t one_now = 0x3f803f80u, one_was = 0x3f803f80u;  // bfloat16 ones, or zeros
  auto step = [&](auto sc, auto d, int t_) {
    one_was = one_now;
    one_now = t_ < steps ? 0x3f803f80u : 0u;
    constexpr int st = decltype(sc)::value, nx = (st + 1) % ST, D = decltype(d)::value;
    constexpr int MF = NB * NB, S = U * MF, Q = MF / 4;  // slots of a unit, of the step
    each<0, S>([&](auto slot_) {
      constexpr int t = decltype(slot_)::value, u = t / MF, m = t % MF;
      // multiply: the unit before u
      constexpr int v = (u + U - 1) % U, s = v / P, i = m / NB, j = m % NB;
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(whole8(fa[v & 1][i]), whole8(fb[s][j]),
                                                          acc[i][j], 0, 0, 0);
      if constexpr (D == s) {
        const bf16x2 one = __builtin_bit_cast(bf16x2, u ? one_now : one_was);
        each<4 * NB * m / MF, 4 * NB * (m + 1) / MF>([&](auto x) {
          constexpr int k = decltype(x)::value, e = k % 4;
          const bf16x4 h = fa[v & 1][k / 4][e / 2];
          dbv[k / 4] = __builtin_amdgcn_fdot2_f32_bf16((bf16x2){h[2 * (e % 2)], h[2 * (e % 2) + 1]},
                                                       one, dbv[k / 4], false);
        });
      }
      // read: unit u
      constexpr int su = u / P, p = u % P, R = (p == 0 ? 4 : 2) * NB, L = MF - Q;
      each<R * least(m, L) / L, R * least(m + 1, L) / L>([&](auto x) {
        constexpr int k = decltype(x)::value, h = k % 2, f = k / 2 % NB;
        const int at = 16 * W * su + 8 * W * h;
        // b first: the first MFMAs of a unit take all of b and a's first
        if constexpr (p == 0 && k < 2 * NB) fb[su][f][h] = read(pb_[f] + st * TB + at);
        else fa[u & 1][f][h] = read(pa_[f] + (st * P + p) * TB + at);
      });
      // write the next step's tile and load into its slot
      constexpr int N = S - Q;
      constexpr int SA = P == 1 ? N / 2 : 2 * N / 3, S0 = P == 1 ? 0 : SA;  // dy until, codes from
      each<8 * NA * least(t, SA) / SA, 8 * NA * least(t + 1, SA) / SA>([&](auto x) {
        put_dy(slot[nx], nx, x, std::false_type());
        if constexpr (decltype(x)::value % 8 == 7) gload_dy(slot[nx], decltype(x)::value / 8);
      });
      constexpr int q0 = t < S0 ? 0 : least(t, N) - S0, q1 = t < S0 ? 0 : least(t + 1, N) - S0;
      each<16 * NQ * q0 / (N - S0), 16 * NQ * q1 / (N - S0)>([&](auto x) {
        put_q(slot[nx], nx, x);
        if constexpr (decltype(x)::value % 16 == 15) gload_q(slot[nx], decltype(x)::value / 16);
      });
      // the step to load next, once this one's loads are out
      if constexpr (t == S - 2) {
        slot[nx].live = live;
        advance();
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    waves_meet();
  };
  auto all_steps = [&](auto d) {
    for (int t = 0; t < steps; t += ST) {
      step(integral_constant<int, 0>(), d, t);
      step(integral_constant<int, 1>(), d, t + 1);
      if constexpr (ST == 3) step(integral_constant<int, 2>(), d, t + 2);
    }
    // the last unit of the last step
#pragma unroll
    for (int i = 0; i < NB; ++i) {
#pragma unroll
      for (int j = 0; j < NB; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(whole8(fa[1][i]), whole8(fb[1][j]),
                                                            acc[i][j], 0, 0, 0);
      if constexpr (decltype(d)::value == 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dbv[i] += one_now ? (float)fa[1][i][e / 4][e % 4] : 0.f;
      }
    }
  };
  if (steps > 0) {
#pragma unroll
    for (int t = 0; t <= ST; ++t) {
      if (t == ST) {
        each<0, 8 * NA>([&](auto x) { put_dy(slot[0], 0, x, std::true_type()); });
        each<0, 16 * NQ>([&](auto x) { put_q(slot[0], 0, x); });
      }
      Slot &s = slot[t % ST];
      // (in the order in which the steps take them)
#pragma unroll
      for (int i = 0; i < NA; ++i) gload_dy(s, i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < NQ; ++i) gload_q(s, i);
      __builtin_amdgcn_sched_barrier(0);
      s.live = live;
      advance();
      if (t == 0 && odd && steps > 1) place(first);
    }
    __syncthreads();
    // Waves run copies of the loop that differ in the slice summed for db (`wave`
    // is a scalar: no wave splits). `steps` is the workgroup's, and so is the
    // number of times that each copy meets the others. (One copy that sums both
    // slices, one of them times zero, takes 67800 x 2048 x 8192 from 2.07 to 2.26 ms;
    // one loop that branches at each step spills 2500 registers.)
    const bool want_db = tl.y == 0 || (a.shift && !a.part);
    if (!want_db) all_steps(integral_constant<int, 2>());
    else if (wave < 2) all_steps(integral_constant<int, 0>());
    else all_steps(integral_constant<int, 1>());
  }
  __syncthreads();
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
    dbs[tid] = a.shift ? s : 0.f;
    const int nn = n0 + tid;
    if (tl.y == 0 && nn < a.n) {
      if (a.part) a.dbpart[(int64_t)tl.z * a.n + nn] = s;
      else if (a.db) a.db[nn] = a.accumulate ? a.db[nn] + s : s;
    }
  }
  __syncthreads();
  // dW by rows: a wave turns 32 rows of its part at a time in its own LDS
  // (lane l holds column l & 31 of rows 4 (l >> 5) + constants of a block)
  constexpr int V = W / 128;
  float *own = (float *)smem + wave * 32 * EP;
  float *out = a.part ? a.part + (int64_t)tl.z * a.n * a.k : a.dw;
  typedef __attribute__((address_space(1))) float g_float;
  const bool acc_in = a.accumulate && !a.part;
  float sc[V], sh[V];
#pragma unroll
  for (int c = 0; c < V; ++c) {
    const int kk = k0 + wk + 64 * c + lane;
    sc[c] = kk < a.k && !a.part && a.scale ? a.scale[kk] : 1.f;
    sh[c] = kk < a.k && !a.part && a.shift ? a.shift[kk] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) own[acc_row(v, lane) * EP + 32 * j + (lane & 31)] = acc[i][j][v];
    __builtin_amdgcn_wave_barrier();
    const int nb = wn + 32 * i, rows = min(32, a.n - n0 - nb);
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const int kk = k0 + wk + 64 * c + lane;
      if (kk >= a.k) continue;
      const float *from = own + 64 * c + lane, *db = dbs + nb;
      g_float *to = (g_float *)out + (int64_t)(n0 + nb) * a.k + kk;
      int r = 0;
#pragma unroll 1
      for (; r + 8 <= rows; r += 8) {  // eight rows on their way at a time
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(sh[c], db[r + e], from[(r + e) * EP] * sc[c]);
        if (acc_in) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] += to[e * (int64_t)a.k];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e * (int64_t)a.k] = x[e];
        to += 8 * (int64_t)a.k;
      }
#pragma unroll 1
      for (; r < rows; ++r) {
        const float x = fmaf(sh[c], db[r], from[r * EP] * sc[c]);
        *to = acc_in ? *to + x : x;
        to += a.k;
      }
    }
  }
}

// dW and db from the splits' sums, added in a fixed order: G groups of 256 / G
// threads take the splits z = g, g + G, ... of as many vectors of V columns,
// then the groups' sums are added in order.
template <int V, int G>
__global__ __launch_bounds__(256) void wgrad8_join_kernel(WgArgs a, int splits) {
  constexpr int E = 256 / G;
  __shared__ float red[G][E][V + 1];
  const int g = threadIdx.x / E, e = threadIdx.x % E;
  const int64_t nk = (int64_t)a.n * a.k, i = ((int64_t)blockIdx.x * E + e) * V;
  float s[V], d = 0.f;
  const int n = i < nk ? (int)(i / a.k) : 0, k = (int)(i - (int64_t)n * a.k);
#pragma unroll
  for (int c = 0; c < V; ++c) s[c] = 0.f;
  if (i < nk) {
#pragma unroll 4
    for (int z = g; z < splits; z += G) {
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
  if constexpr (G > 1) {
#pragma unroll
    for (int c = 0; c < V; ++c) red[g][e][c] = s[c];
    red[g][e][V] = d;
    __syncthreads();
    if (g) return;
#pragma unroll
    for (int z = 1; z < G; ++z) {
#pragma unroll
      for (int c = 0; c < V; ++c) s[c] += red[z][e][c];
      d += red[z][e][V];
    }
  }
  if (i >= nk) return;
  float o[V];
#pragma unroll
  for (int c = 0; c < V; ++c) {
    o[c] = s[c];
    if (a.scale) o[c] *= a.scale[k + c];
    if (a.shift) o[c] = fmaf(a.shift[k + c], d, o[c]);
    if (a.accumulate) o[c] += a.dw[i + c];
  }
#pragma unroll
  for (int c = 0; c < V; ++c) a.dw[i + c] = o[c];
  if (k == 0 && a.db) a.db[n] = a.accumulate ? a.db[n] + d : d;
}

// Tile width and splits of the rows: the least of
//   steps of a workgroup x time of a step x workgroups of a CU, and, if split,
//   the join's launch and the partial sums written and read,
// in us. The launch, the first loads and the epilogue, 7 to 9 us of a short call, are
// left out, as every choice has them: it ranks choices and is no call's time.
// A step of 32 rows takes 0.98 (256-wide bf16 tile, one workgroup a CU), 0.35
// (128-wide) or 0.82 (128-wide float32); two workgroups a CU share it at 0.85 of
// twice the time. Measured for splits of the 128-wide tile (us): 1568 x 256 x
// 256 bf16 by 3 15.2, 6 12.7, 12 11.3, 24 12.3; 392 x 512 x 2048 bf16 by 1 11.8,
// 3 17.3, 6 23.4; 784 x 64 x 64 float32 by 1 28.1, 3 17.1, 12 12.2; for the tiles:
// 67800 x 2048 x 8192 bf16 2784 and 2083, 67800 x 512 x 2048 195 and 188,
// 540000 x 256 x 256 117 and 113; float32 67800 x 512 x 512 137 and 151 (a
// 256-wide float32 tile spills registers and is not kept).
//
// The choice goes up and down with the rows, so a workspace that serves any
// smaller number of rows too is one for `most` splits: the largest count that
// can be chosen for these rows or fewer. At t <= steps a count s takes at least
// t p / s + d, p a step's time over all of a CU's workgroups and d what the
// split costs. So it is never chosen if steps (p1 - p / s) < d, with p1 the p of
// one split, nor if the count that fills the CUs once or twice, at most
// t p' / s' + p' + d', is always less.
struct Split {
  int tile, splits, most;
};
Split split_of(int64_t rows, int64_t n, int64_t k, int32_t dtype) {
  const int64_t steps = (rows + kStep - 1) / kStep;
  Split best{128, 1, 1};
  double least_us = -1;
  struct Rate {
    int64_t tiles;
    double step_us;
    int tile;
    double p(int64_t s, int64_t times = 1) const {
      const double per_cu = (double)((tiles * s + 255) / 256);
      return (double)times * step_us * per_cu * (tile == 128 && per_cu > 1 ? 0.85 : 1.0);
    }
  } rate[2];
  auto d = [&](int64_t s) {
    return s > 1 ? 2.5 + 2.2e-6 * (double)s * (double)n * (double)k : 0.0;
  };
  // (of a 256-wide tile half would be empty at 128 columns or fewer)
  const int widths = dtype == LRCNN_BF16 && n > 128 && k > 128 ? 2 : 1;
  double p1 = 0;
  for (int i = 0; i < widths; ++i) {
    const int tile = 128 << i;
    rate[i].tile = tile;
    rate[i].tiles = ((n + tile - 1) / tile) * ((k + tile - 1) / tile);
    rate[i].step_us = tile == 256 ? 0.98 : dtype == LRCNN_BF16 ? 0.35 : 0.82;
    p1 = i ? std::min(p1, rate[i].p(1)) : rate[i].p(1);
  }
  auto never = [&](int64_t s, double p) {
    if ((double)steps * (p1 - p / (double)s) < d(s) - 1e-6) return true;
    for (int i = 0; i < widths; ++i)
      for (const int64_t f : {256 / rate[i].tiles, 512 / rate[i].tiles})
        if (f >= 1 && f < s && p * (double)f >= rate[i].p(f) * (double)s &&
            rate[i].p(f) + d(f) <= d(s))
          return true;
    return false;
  };
  for (int i = 0; i < widths; ++i) {
    const Rate &r = rate[i];
    auto consider = [&](int64_t s) {
      if (s < 1 || (s > 1 && (s > steps || s * r.tiles > 1024))) return;
      const double us = r.p(s, (steps + s - 1) / s) + d(s);
      if (least_us < 0 || us < least_us) least_us = us, best.tile = r.tile, best.splits = (int)s;
      if (s > best.most && !never(s, r.p(s))) best.most = (int)s;
    };
    for (int64_t s = 1; s <= 512; s += s < 8 ? 1 : s / 4) consider(s);
    consider(256 / r.tiles), consider(512 / r.tiles);  // one or two workgroups on every CU
  }
  return best;
}
size_t wgrad_ws(int64_t splits, int64_t n, int64_t k) {
  return splits == 1 ? 0 : a256((size_t)splits * n * k * 4) + a256((size_t)splits * n * 4);
}

int wgrad_shape(int64_t rows, int64_t n_in, int64_t n_out, int32_t dtype) {
  int st = take_shape(rows, n_in, dtype);
  if (st == LRCNN_OK) st = take_shape(rows, n_out, dtype);
  if (st == LRCNN_OK) st = take_shape(n_out, n_in, dtype);
  if (st == LRCNN_OK && (n_in > kMaxFeatures || n_out > kMaxFeatures))
    st = refuse(LRCNN_ESHAPE, "more than 2^24 features");
  if (st == LRCNN_OK && rows > kMaxWgradRows)
    st = refuse(LRCNN_ESHAPE, "weight gradient over more than 2^30 rows");
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
  if (!bytes) return refuse(LRCNN_EINVAL, "null output");
  TRY(wgrad_shape(rows, n_in, n_out, dtype));
  *bytes = wgrad_ws(split_of(rows, n_out, n_in, dtype).most, n_out, n_in);
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
  if (rows > 0 && a.dy.ld > kMaxFeatures)
    return refuse(LRCNN_ESHAPE, "dy: row stride of more than 2^24");
  TRY(take_ckpt("ckpt", ckpt, rows > 0));
  TRY(take_f32("scale", scale, false));
  TRY(take_f32("shift", shift, false));
  TRY(take_f32("dw", dw, true));
  TRY(take_f32("db", db, false));
  const Split sp = split_of(rows, n_out, n_in, dtype);
  const size_t need = sp.splits == 1 ? 0 : wgrad_ws(sp.most, n_out, n_in);
  if (need && (!workspace || ((uintptr_t)workspace & 15)))
    return refuse(LRCNN_EINVAL, "workspace null or misaligned");
  if (ws_bytes < need)
    return refuse(LRCNN_EWORKSPACE, "workspace needs ", need, " bytes, got ", ws_bytes);
  a.rows = (int)rows, a.n = (int)n_out, a.k = (int)n_in, a.splits = sp.splits;
  a.q = ckpt_of(ckpt, rows, n_in);
  a.q.pitch = pitch_of(n_in);
  a.scale = scale, a.shift = shift, a.dw = dw, a.db = db, a.accumulate = accumulate != 0;
  if (sp.splits > 1) {
    a.part = (float *)workspace;
    a.dbpart = (float *)((char *)workspace + a256((size_t)sp.splits * n_out * n_in * 4));
  }
  const int64_t gx = (n_out + sp.tile - 1) / sp.tile, gy = (n_in + sp.tile - 1) / sp.tile;
  if (gx * gy * sp.splits >= (1 << 24)) return refuse(LRCNN_ESHAPE, "too many features");
  a.gx = (int)gx, a.gy = (int)gy;
  a.tiles = lrcnn::fast_div((uint32_t)(gx * gy));
  a.panel = lrcnn::fast_div((uint32_t)(8 * gy));
  a.rest = lrcnn::fast_div((uint32_t)(gx % 8 ? gx % 8 : 8));
  a.stride = lrcnn::fast_div((uint32_t)(lrcnn::act8::kStep * sp.splits));
  const dim3 grid((unsigned)(gx * gy * sp.splits));
  hipStream_t s = (hipStream_t)stream;
  auto run = [&](auto *t) {
    using T = std::remove_pointer_t<decltype(t)>;
    auto go = [&](auto w, auto c) {
      wgrad8_kernel<T, w.value, c.value><<<grid, 256, 0, s>>>(a);
    };
    std::integral_constant<int, 256> w256;
    std::integral_constant<int, 128> w128;
    std::integral_constant<int, COLS_WHOLE> whole;
    std::integral_constant<int, COLS_SHIFT> shift;
    std::integral_constant<int, COLS_EACH> each;
    if constexpr (std::is_same<T, bf16>::value) {
      if (sp.tile == 256) {
        if (n_out % 8 == 0) go(w256, whole);
        else go(w256, shift);
        return;
      }
    }
    if (n_out < 8) go(w128, each);
    else if (n_out % 8 == 0) go(w128, whole);
    else go(w128, shift);
  };
  if (dtype == LRCNN_BF16) run((bf16 *)nullptr);
  else run((float *)nullptr);
  if (sp.splits > 1) {
    const int64_t nk = n_out * n_in;
    auto join = [&](auto v, auto g) {
      constexpr int E = 256 / g.value * v.value;
      const unsigned blocks = (unsigned)((nk + E - 1) / E);
      wgrad8_join_kernel<v.value, g.value><<<blocks, 256, 0, s>>>(a, sp.splits);
    };
    auto by_groups = [&](auto v) {
      if (sp.splits <= 8) join(v, std::integral_constant<int, 1>());
      else join(v, std::integral_constant<int, 8>());
    };
    if (n_in % 4 == 0) by_groups(std::integral_constant<int, 4>());
    else by_groups(std::integral_constant<int, 1>());
  }
  return launched("linear_wgrad");
}
