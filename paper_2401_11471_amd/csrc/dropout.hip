// Dropout from a counter-based generator: y = x keep / (1 - p) [+ residual].
//
// The random bits of an element are a function of the seed, the offset, the site
// and the element's place, so the backward pass draws the forward pass' again and no
// mask is stored or read. Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel
// random numbers: as easy as 1, 2, 3", SC 2011): ten rounds of two 32 x 32 bit
// products on a counter of four words, under a key of two words that advances by a
// constant each round. One counter gives 128 bits, 16 for each of the eight
// columns of a thread: the rounds' twenty wide products (a quarter of the rate of
// others) then take less time than the row's bytes. Bound by HBM: 67800 x 2048 bf16 with
// residual 143 to 150 us, 5.6 to 5.8 TB/s, at 0.14 vector instructions a cycle and SIMD; 392 x
// 512 float32 2.7 us, a launch's time. Threads of a row are a power of two: of 199014 x 316
// bf16, 40 vectors a row, 24 of 64 lanes are idle, 69 us against 42 at 6 TB/s.
#include "act8.hpp"

#include <type_traits>

namespace lrcnn {
namespace act8 {
namespace {

struct DropArgs {
  int64_t rows, cols, vecs;  // vecs: counters of a row
  int64_t first;             // the first row's number
  int tpr, rpb;              // threads of a row, rows of a block
  uint32_t site, least;      // site << 16; kept from this value on
  float scale;
  const uint64_t *rng;
  Mat x, res, y;
};

struct Words {
  uint32_t w[4];
};
__device__ __forceinline__ Words philox(uint64_t seed, Words c) {
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p = (uint64_t)c.w[0] * 0xD2511F53u, q = (uint64_t)c.w[2] * 0xCD9E8D57u;
    c = Words{{(uint32_t)(q >> 32) ^ c.w[1] ^ k0, (uint32_t)q,
               (uint32_t)(p >> 32) ^ c.w[3] ^ k1, (uint32_t)p}};
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

template <typename T, bool RES>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs a) {
  const uint64_t seed = a.rng[0], offset = a.rng[1];
  const int64_t v = (int64_t)blockIdx.x * a.tpr + threadIdx.x % a.tpr, c = v * kVec;
  if (v >= a.vecs) return;
  for (int64_t r = (int64_t)blockIdx.y * a.rpb + threadIdx.x / a.tpr; r < a.rows;
       r += (int64_t)gridDim.y * a.rpb) {
    const int64_t n = a.cols - c;
    const Raw8<T> rx = load8((const T *)a.x.p + r * a.x.ld + c, n);
    float x[8], z[8];
    if constexpr (RES) load8((const T *)a.res.p + r * a.res.ld + c, n).get(z);
    const uint64_t g = (uint64_t)(a.first + r) * (uint64_t)a.vecs + (uint64_t)v;
    const Words w = philox(seed, Words{{(uint32_t)g, (uint32_t)(g >> 32) | a.site,
                                        (uint32_t)offset, (uint32_t)(offset >> 32)}});
    rx.get(x);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t bits = i & 1 ? w.w[i / 2] >> 16 : w.w[i / 2] & 0xffffu;
      x[i] = bits >= a.least ? x[i] * a.scale : 0.f;
      if constexpr (RES) x[i] += z[i];
    }
    store8((T *)a.y.p + r * a.y.ld + c, n, x);
  }
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

extern "C" int lrcnn_dropout(int64_t rows, int64_t cols, int32_t dtype, const void *x, int64_t ldx,
                             const void *residual, int64_t ldr, double p, const uint64_t *rng,
                             int32_t site, int64_t first_row, void *y, int64_t ldy, void *stream) {
  TRY(take_shape(rows, cols, dtype));
  if (!(p >= 0.0) || !(p <= 1.0)) return refuse(LRCNN_EINVAL, "p must be in [0, 1]");
  if (site < 0 || site > 65535) return refuse(LRCNN_EINVAL, "site must be in [0, 65536)");
  const int64_t vecs = (cols + kVec - 1) / kVec;
  if (first_row < 0 || first_row > (((int64_t)1 << 48) / vecs) - rows)
    return refuse(LRCNN_ESHAPE, "first_row negative or too large");
  if (rows == 0) return LRCNN_OK;
  const int es = dtype == LRCNN_BF16 ? 2 : 4;
  DropArgs a{};
  TRY(take("x", x, ldx, cols, es, true, &a.x));
  TRY(take("residual", residual, ldr, cols, es, false, &a.res));
  TRY(take("y", y, ldy, cols, es, true, &a.y));
  TRY(same_rows("y", a.y, a.x, rows));
  TRY(same_rows("y", a.y, a.res, rows));
  if (!rng) return refuse(LRCNN_EINVAL, "rng is null");
  if ((uintptr_t)rng & 7) return refuse(LRCNN_EINVAL, "rng is misaligned");
  a.rows = rows, a.cols = cols, a.vecs = vecs, a.first = first_row;
  a.site = (uint32_t)site << 16;
  a.least = (uint32_t)__builtin_rint(p * 65536.0);
  a.scale = a.least < 65536u ? (float)(65536.0 / (65536.0 - a.least)) : 0.f;
  a.rng = rng;
  a.tpr = 1;
  while (a.tpr < 256 && a.tpr < vecs) a.tpr *= 2;
  a.rpb = 256 / a.tpr;
  const int64_t by = (rows + a.rpb - 1) / a.rpb;
  const dim3 grid((unsigned)((vecs + a.tpr - 1) / a.tpr), (unsigned)(by < 65535 ? by : 65535));
  hipStream_t s = (hipStream_t)stream;
  auto run = [&](auto *t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (residual) dropout_kernel<T, true><<<grid, 256, 0, s>>>(a);
    else dropout_kernel<T, false><<<grid, 256, 0, s>>>(a);
  };
  if (dtype == LRCNN_BF16) run((bf16 *)nullptr);
  else run((float *)nullptr);
  return launched("dropout");
}
