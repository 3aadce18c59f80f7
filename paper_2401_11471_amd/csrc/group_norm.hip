// Group norm with an activation over an NHWC map, forward and backward.
//
//   forward   xh = (x - mean) rstd over the pixels and channels of a group of an
//             image, y = f(gamma xh + beta)
//   backward  e = dy f'(gamma xh + beta), q = gamma e,
//             dx = rstd (q - mean(q) - xh mean(q xh)),
//             dgamma = sum of e xh, dbeta = sum of e
//
// A group's sums need all its pixels before the first result. A map whose groups fit
// the registers of a block is read once, in one launch: 1 x 49 x 512 bf16 6.9 us, 7 x 169
// x 510 float32 10.5 (three launches: 13.8 and 19.2), a chain of loads, two reductions and
// a store each. Other maps are read twice: a pass that leaves, for every channel of a
// slab of pixels, two numbers (forward: mean and centred sum of squares; backward: sums of e
// and e xh), a small kernel that joins them by group (and by channel for dgamma, dbeta),
// and a pass that applies the result. A channel's two numbers serve every way of
// grouping, whatever the group's width and alignment, and in the backward pass both
// the groups' means (weighted by gamma) and the parameters' gradients.
//
// Large maps are bound by HBM: 8 x 135000 x 512 bf16 with relu and checkpoint 238 to 256 us
// for the sums (4.4 to 4.6 TB/s), 9 for the join, 530 to 543 for the result (5.2 TB/s);
// backward from the checkpoint with silu, 8 x 8475 x 2048 bf16, 109 to 125 and 121 to 129 us
// (3.6 to 4.1 and 5.7 TB/s; the first also by its vector instructions, 0.19 a cycle and
// SIMD), from the map itself 285 in all. Small parts of a batch at a time,
// so that the second pass finds the map in the Infinity Cache, took longer (1317 us and
// 1078 with the unpack): what the pass before has written goes to memory meanwhile.
//
// Statistics: eight pixels at a time are centred in registers (their mean
// corrected by the centred sum), then joined with
//   n = na + nb, d = mb - ma, mean = ma + d nb / n, M2 = Ma + Mb + d^2 na nb / n,
// so that a mean far from zero costs the variance no digits; across slabs
// and channels in 64 bits, as dgamma and dbeta across slabs and images.
#include "activation.hpp"
#include "kernels.hpp"

#include <algorithm>
#include <type_traits>

namespace lrcnn {
namespace act8 {
namespace {

constexpr int64_t kMaxImages = 1 << 20, kMaxChannels = 1 << 20;
constexpr int kBatch = 8;         // pixels that a thread holds at a time
// Pixels a thread, where the CUs have no work else (8 x 784 x 96 float32 backward: 8 pixels
// 18.8 us, 2 pixels 14.6; but with blocks for all CUs a thread's constants for its channels
// take as long as a few pixels: 25 x 185 x 2023 bf16 backward 76 and 64 us)
constexpr int kLeast = 2;
constexpr int kUnits = 2048;      // blocks of a pass, where there are as many
constexpr int kApplyPixels = 4;   // applying passes: pixels in flight a thread

struct GnArgs {
  int64_t pixels, slab;  // pixels of an image and of a slab
  int64_t units;         // images times slabs
  int slabs, batch, cols, pitch, groups, per;  // per: channels of a group
  int tpr, ctiles;       // threads of a pixel's channels; tiles of 8 tpr channels
  float eps;
  double inv;            // 1 / (pixels of an image times channels of a group)
  Mat x, y;              // backward: y is dy
  Mat dx;
  const float *gamma, *beta;
  const float *mean, *rstd;  // [batch][groups]
  float *mean_out, *rstd_out;
  float2 *part;          // [units][cols]
  float2 *chan;          // [batch][cols]
  float2 *stat;          // [batch][groups]: (mean, rstd), backward the two means
  float *dgamma, *dbeta;
  int accumulate;
  FastDiv by_per;
  int width;             // channels of a block that holds its groups whole
  Ckpt k;
};

// Slab s of image b and the channels of this thread.
struct Place {
  int64_t b, p0, p1;  // the slab's pixels within the image
  int64_t unit;
  int c, n, row, rows;  // first channel, channels left, this thread's row and rows a block
};
// BACK: the units from the last one on, in the second pass: it begins with what the first
// one left in the Infinity Cache.
template <bool BACK = false>
__device__ __forceinline__ Place place(const GnArgs &a) {
  Place q;
  const uint32_t block = BACK ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
  const int ct = block % a.ctiles;
  q.unit = block / a.ctiles;
  q.b = q.unit / a.slabs;
  q.p0 = (q.unit - q.b * a.slabs) * a.slab;
  q.p1 = min(q.p0 + a.slab, a.pixels);
  q.c = (ct * a.tpr + (int)(threadIdx.x % a.tpr)) * kVec;
  q.n = a.cols - q.c;
  q.row = threadIdx.x / a.tpr;
  q.rows = blockDim.x / a.tpr;
  return q;
}

// A thread's eight channels of a float vector, `other` where there is none
__device__ __forceinline__ void channel8(const float *p, const Place &q, float other,
                                         float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = other;
  if (p && q.n > 0) load8(p + q.c, q.n).get(v);
}
// The two numbers of each channel's group
__device__ __forceinline__ void group8(const GnArgs &a, const float2 *stat, const Place &q,
                                       float (&s)[8], float (&t)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = min(q.c + i, a.cols - 1);
    const float2 v = stat[q.b * a.groups + fdiv_q((uint32_t)c, a.by_per)];
    s[i] = v.x, t[i] = v.y;
  }
}
__device__ __forceinline__ void group8(const GnArgs &a, const float *stat, const Place &q,
                                       float (&s)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    s[i] = stat[q.b * a.groups + fdiv_q((uint32_t)min(q.c + i, a.cols - 1), a.by_per)];
}

// Joins the block's rows by halves, in LDS; the first row's threads have the result.
template <typename F>
__device__ __forceinline__ void join_rows_lds(const Place &q, int tpr, F &&halve) {
  for (int s = q.rows / 2; s >= 1; s /= 2) halve(s, s * tpr);
}

template <typename T>
__global__ __launch_bounds__(256) void gn_stats_kernel(GnArgs a) {
  __shared__ float lm[8][256], lq[8][256], ln[256];
  const Place q = place(a);
  float mean[8], m2[8], n = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) mean[i] = m2[i] = 0.f;
  if (q.n > 0) {
    const T *x = (const T *)a.x.p + (q.b * a.pixels) * a.x.ld + q.c;
    for (int64_t p = q.p0 + q.row; p < q.p1; p += (int64_t)q.rows * kBatch) {
      Raw8<T> r[kBatch];
      const int k = (int)min((q.p1 - p + q.rows - 1) / q.rows, (int64_t)kBatch);
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        r[j] = load8(x + (p + (int64_t)q.rows * min(j, k - 1)) * a.x.ld, q.n);
      const float nk = (float)k, nn = n + nk, inv = 1.f / nk;
      const float wb = nk / nn, wm = n * wb;
      float s[8], off[8], sq[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] = off[i] = sq[i] = 0.f;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        float v[8];
        r[j].get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += j < k ? v[i] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] *= inv;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        float v[8];
        r[j].get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float d = j < k ? v[i] - s[i] : 0.f;
          off[i] += d;
          sq[i] = fmaf(d, d, sq[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float o = off[i] * inv;
        const float m = s[i] + o;
        const float d = m - mean[i];
        mean[i] = n == 0.f ? m : fmaf(d, wb, mean[i]);
        m2[i] += fmaf(-o, off[i], sq[i]) + (n == 0.f ? 0.f : d * d * wm);
      }
      n = nn;
    }
  }
  const int t = threadIdx.x;
#pragma unroll
  for (int i = 0; i < 8; ++i) lm[i][t] = mean[i], lq[i][t] = m2[i];
  ln[t] = n;
  __syncthreads();
  join_rows_lds(q, a.tpr, [&](int s, int step) {
    if (q.row < s) {
      const float nb = ln[t + step], nn = n + nb;
      const float wb = nb > 0.f ? nb / nn : 0.f, wm = n * wb;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = lm[i][t + step] - mean[i];
        if (nb > 0.f) {
          mean[i] = n == 0.f ? lm[i][t + step] : fmaf(d, wb, mean[i]);
          m2[i] += lq[i][t + step] + (n == 0.f ? 0.f : d * d * wm);
        }
        lm[i][t] = mean[i], lq[i][t] = m2[i];
      }
      n = nn;
      ln[t] = n;
    }
    __syncthreads();
  });
  if (q.row == 0 && q.n > 0) {
    float2 *o = a.part + q.unit * a.cols + q.c;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < q.n) o[i] = make_float2(mean[i], m2[i]);
  }
}

// Sum over the block in a fixed order, the same in every thread
__device__ __forceinline__ double block_sum(double v, double *red) {
#pragma unroll
  for (int s = 1; s < 64; s *= 2) v += __shfl_xor(v, s);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) v += red[w];
  return v;
}

// Block (image, group): mean and rstd of a group from its slabs' channels
__global__ __launch_bounds__(1024) void gn_group_kernel(GnArgs a) {
  __shared__ double red[16];
  const int64_t b = blockIdx.x / a.groups;
  const int g = blockIdx.x % a.groups;
  const uint32_t all = (uint32_t)a.slabs * (uint32_t)a.per;
  const float2 *part = a.part + b * a.slabs * (int64_t)a.cols + (int64_t)g * a.per;
  auto count = [&](uint32_t s) { return (double)min(a.slab, a.pixels - s * a.slab); };
  auto at = [&](uint32_t e, uint32_t &s) {
    uint32_t c;
    fdiv_qr(e, a.by_per, s, c);
    return part[(int64_t)s * a.cols + c];
  };
  double sum = 0;
#pragma unroll 4
  for (uint32_t e = threadIdx.x; e < all; e += blockDim.x) {
    uint32_t s;
    const float2 v = at(e, s);
    sum += count(s) * v.x;
  }
  const double mean = block_sum(sum, red) * a.inv;
  double m2 = 0;
#pragma unroll 4
  for (uint32_t e = threadIdx.x; e < all; e += blockDim.x) {
    uint32_t s;
    const float2 v = at(e, s);
    const double d = v.x - mean;
    m2 += v.y + count(s) * d * d;
  }
  double var = block_sum(m2, red) * a.inv;
  var = var < 0 ? 0 : var;  // (NaN stays)
  if (threadIdx.x == 0) {
    const float m = (float)mean, r = rsqrt_rounded((float)var + a.eps);
    a.stat[blockIdx.x] = make_float2(m, r);
    if (a.mean_out) a.mean_out[blockIdx.x] = m;
    if (a.rstd_out) a.rstd_out[blockIdx.x] = r;
  }
}

template <typename T, int KIND>
__global__ __launch_bounds__(256) void gn_apply_kernel(GnArgs a) {
  const Place q = place<true>(a);
  if (q.c >= a.pitch) return;
  float ga[8], be[8], mu[8], rs[8];
  channel8(a.gamma, q, 1.f, ga);
  channel8(a.beta, q, 0.f, be);
  group8(a, a.stat, q, mu, rs);
  for (int64_t p = q.p0 + q.row; p < q.p1; p += (int64_t)q.rows * kApplyPixels) {
    Raw8<T> r[kApplyPixels];
    int64_t at[kApplyPixels];
#pragma unroll
    for (int j = 0; j < kApplyPixels; ++j) {
      at[j] = q.b * a.pixels + min(p + (int64_t)q.rows * j, q.p1 - 1);
      r[j] = load8((const T *)a.x.p + at[j] * a.x.ld + q.c, q.n);
    }
#pragma unroll
    for (int j = 0; j < kApplyPixels; ++j) {
      if (p + (int64_t)q.rows * j >= q.p1) continue;
      float v[8], y[8], df;
      r[j].get(v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = i < q.n ? (v[i] - mu[i]) * rs[i] : 0.f;
        activate<KIND>(fmaf(v[i], ga[i], be[i]), y[i], df);
      }
      if (q.n > 0) store8((T *)a.y.p + at[j] * a.y.ld + q.c, q.n, y);
      if (a.k.q) put8(a.k, at[j], q.c, v);
    }
  }
}

// ---------------------------------------------------------------- backward
// xh and e of eight channels of one pixel
template <typename T, int KIND, bool CK>
struct Back {
  float ga[8], be[8], mu[8], rs[8];
  __device__ __forceinline__ void init(const GnArgs &a, const Place &q) {
    channel8(a.gamma, q, 1.f, ga);
    channel8(a.beta, q, 0.f, be);
    group8(a, a.rstd, q, rs);
    if constexpr (!CK) group8(a, a.mean, q, mu);
  }
  struct Raw {
    Raw8<T> dy, x;
    uint2 code;
    uint32_t ex;
  };
  __device__ __forceinline__ Raw load(const GnArgs &a, const Place &q, int64_t at) const {
    Raw r;
    r.dy = load8((const T *)a.y.p + at * a.y.ld + q.c, q.n);
    if constexpr (CK) {
      r.code = *(const uint2 *)(a.k.q + at * a.k.pitch + q.c);
      r.ex = a.k.e[at * (a.k.pitch / kGroup) + q.c / kGroup];
    } else {
      r.x = load8((const T *)a.x.p + at * a.x.ld + q.c, q.n);
    }
    return r;
  }
  __device__ __forceinline__ void get(const Place &q, const Raw &r, float (&xh)[8],
                                      float (&e)[8]) const {
    r.dy.get(e);
    if constexpr (CK) {
      decode8(r.code, r.ex, xh);
    } else {
      r.x.get(xh);
#pragma unroll
      for (int i = 0; i < 8; ++i) xh[i] = (xh[i] - mu[i]) * rs[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float f, df;
      activate<KIND>(fmaf(xh[i], ga[i], be[i]), f, df);
      e[i] *= df;
    }
  }
};

template <typename T, int KIND, bool CK>
__global__ __launch_bounds__(256) void gn_sums_kernel(GnArgs a) {
  __shared__ float l1[8][256], l2[8][256];
  constexpr int R = kApplyPixels;
  const Place q = place(a);
  float s1[8], s2[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) s1[i] = s2[i] = 0.f;
  if (q.n > 0) {
    Back<T, KIND, CK> back;
    back.init(a, q);
    for (int64_t p = q.p0 + q.row; p < q.p1; p += (int64_t)q.rows * R) {
      typename Back<T, KIND, CK>::Raw r[R];
#pragma unroll
      for (int j = 0; j < R; ++j)
        r[j] = back.load(a, q, q.b * a.pixels + min(p + (int64_t)q.rows * j, q.p1 - 1));
      float t1[8], t2[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) t1[i] = t2[i] = 0.f;
#pragma unroll
      for (int j = 0; j < R; ++j) {
        float xh[8], e[8];
        back.get(q, r[j], xh, e);
        const bool in = p + (int64_t)q.rows * j < q.p1;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (in) {
            t1[i] += e[i];
            t2[i] = fmaf(e[i], xh[i], t2[i]);
          }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s1[i] += t1[i], s2[i] += t2[i];
    }
  }
  const int t = threadIdx.x;
#pragma unroll
  for (int i = 0; i < 8; ++i) l1[i][t] = s1[i], l2[i][t] = s2[i];
  __syncthreads();
  join_rows_lds(q, a.tpr, [&](int s, int step) {
    if (q.row < s) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s1[i] += l1[i][t + step], s2[i] += l2[i][t + step];
        l1[i][t] = s1[i], l2[i][t] = s2[i];
      }
    }
    __syncthreads();
  });
  if (q.row == 0 && q.n > 0) {
    float2 *o = a.part + q.unit * a.cols + q.c;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < q.n) o[i] = make_float2(s1[i], s2[i]);
  }
}

// A channel's slabs joined to one entry [image][channel], 32 channels a block of an
// image: for groups whose slabs and channels are too many for the block that joins a group.
// SUMS: sums, else mean and centred sum of squares.
template <bool SUMS>
__global__ __launch_bounds__(1024) void gn_channel_kernel(GnArgs a, float2 *out) {
  __shared__ double l1[32][33], l2[32][33];
  const uint32_t blocks = (uint32_t)(a.cols + 31) / 32, b = blockIdx.x / blocks;
  const int x = threadIdx.x & 31, r = threadIdx.x >> 5, c = (int)(blockIdx.x - b * blocks) * 32 + x;
  const float2 *part = a.part + (int64_t)b * a.slabs * a.cols + c;
  auto count = [&](int s) { return (double)min(a.slab, a.pixels - s * a.slab); };
  // the sums over r of the threads of a column, the same in each
  auto total = [&](double (&l)[32][33], double v) {
    l[r][x] = v;
    __syncthreads();
    double t = 0;
    for (int k = 0; k < 32; ++k) t += l[k][x];
    return t;
  };
  double s1 = 0, s2 = 0;
  if (c < a.cols) {
#pragma unroll 4
    for (int s = r; s < a.slabs; s += 32) {
      const float2 v = part[(int64_t)s * a.cols];
      s1 += SUMS ? v.x : count(s) * v.x;
      if (SUMS) s2 += v.y;
    }
  }
  s1 = total(l1, s1);
  if constexpr (!SUMS) {
    s1 /= (double)a.pixels;
    if (c < a.cols) {
#pragma unroll 4
      for (int s = r; s < a.slabs; s += 32) {
        const float2 v = part[(int64_t)s * a.cols];
        const double d = v.x - s1;
        s2 += v.y + count(s) * d * d;
      }
    }
  }
  s2 = total(l2, s2);
  if (r == 0 && c < a.cols) out[(int64_t)b * a.cols + c] = make_float2((float)s1, (float)s2);
}

// dgamma and dbeta of kChans channels: thread (r, c) takes every kRows-th unit from r
// on, one wave joins a channel's sums of a kind. In 64 bits: a thread of the most images
// adds 2^13 units, whose terms may cancel (262144 x 8 in float32: off by 7e-2 where the sum
// is 1e4). Few channels a block, so that the conversions and the loads' latency are spread
// (the whole backward pass with blocks of 32 channels and of 8: 51 x 5823 x 32 bf16 37.2 and
// 35.0 us; with 32 and float32 sums 34.9, and 64 x 49 x 512 11.0 to 11.7 now).
constexpr int kChans = 8, kRows = 1024 / kChans;
__device__ __forceinline__ void channel_grads(const GnArgs &a, int block) {
  __shared__ double l[2][kChans][kRows + 8];
  const int r = threadIdx.x / kChans, x = threadIdx.x % kChans, c = block * kChans + x;
  double s1 = 0, s2 = 0;
  if (c < a.cols) {
#pragma unroll 8
    for (int64_t u = r; u < a.units; u += kRows) {
      const float2 v = a.part[u * a.cols + c];
      s1 += v.x, s2 += v.y;
    }
  }
  l[0][x][r] = s1, l[1][x][r] = s2;
  __syncthreads();
  static_assert(kRows == 128 && 2 * kChans == 1024 / 64, "a wave joins 128 sums");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, gamma = wave / kChans;
  const int to = block * kChans + wave % kChans;
  double s = l[gamma][wave % kChans][lane] + l[gamma][wave % kChans][lane + 64];
#pragma unroll
  for (int k = 1; k < 64; k *= 2) s += __shfl_xor(s, k);
  float *const out = gamma ? a.dgamma : a.dbeta;
  if (lane == 0 && to < a.cols && out) out[to] = (float)(a.accumulate ? out[to] + s : s);
}
__global__ __launch_bounds__(1024) void gn_grads_kernel(GnArgs a) {
  channel_grads(a, blockIdx.x);
}

// Block (image, group): a group's two means, of q and q xh; the blocks behind these:
// the parameters' gradients of kChans channels each.
__global__ __launch_bounds__(1024) void gn_join_kernel(GnArgs a) {
  __shared__ double red[16];
  const int bg = a.batch * a.groups;
  if ((int)blockIdx.x >= bg) return channel_grads(a, blockIdx.x - bg);
  const int64_t b = blockIdx.x / a.groups;
  const int g = blockIdx.x % a.groups;
  const uint32_t all = (uint32_t)a.slabs * (uint32_t)a.per;
  const float2 *part = a.part + b * a.slabs * (int64_t)a.cols + (int64_t)g * a.per;
  double s1 = 0, s2 = 0;
#pragma unroll 4
  for (uint32_t e = threadIdx.x; e < all; e += blockDim.x) {
    uint32_t s, c;
    fdiv_qr(e, a.by_per, s, c);
    const float2 v = part[(int64_t)s * a.cols + c];
    const double ga = a.gamma ? (double)a.gamma[g * a.per + c] : 1.0;
    s1 += ga * v.x, s2 += ga * v.y;
  }
  s1 = block_sum(s1, red);
  s2 = block_sum(s2, red);
  if (threadIdx.x == 0) a.stat[blockIdx.x] = make_float2((float)(s1 * a.inv), (float)(s2 * a.inv));
}

template <typename T, int KIND, bool CK>
__global__ __launch_bounds__(256) void gn_dx_kernel(GnArgs a) {
  constexpr int R = kApplyPixels;
  const Place q = place<true>(a);
  if (q.n <= 0) return;
  Back<T, KIND, CK> back;
  back.init(a, q);
  float m1[8], m2[8];
  group8(a, a.stat, q, m1, m2);
  for (int64_t p = q.p0 + q.row; p < q.p1; p += (int64_t)q.rows * R) {
    typename Back<T, KIND, CK>::Raw r[R];
    int64_t at[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      at[j] = q.b * a.pixels + min(p + (int64_t)q.rows * j, q.p1 - 1);
      r[j] = back.load(a, q, at[j]);
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if (p + (int64_t)q.rows * j >= q.p1) continue;
      float xh[8], e[8];
      back.get(q, r[j], xh, e);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        e[i] = back.rs[i] * (fmaf(e[i], back.ga[i], -m1[i]) - xh[i] * m2[i]);
      store8((T *)a.dx.p + at[j] * a.dx.ld + q.c, q.n, e);
    }
  }
}

// ------------------------------------------------- maps that a block can hold
// One pass: a block has some whole groups of an image, all their pixels in registers
// (R a thread). `width` channels from its first on, eight to a thread; threads past the
// width or the pixels hold zeros.
struct Whole {
  int64_t b;
  int c0, c, n, row, rows;  // first channel of the block, of the thread; channels left
};
__device__ __forceinline__ Whole whole(const GnArgs &a) {
  Whole w;
  w.b = blockIdx.x / a.ctiles;
  w.c0 = (int)(blockIdx.x % a.ctiles) * a.width;
  const int k = threadIdx.x % a.tpr * kVec;
  w.c = w.c0 + k;
  w.n = min(a.width - k, a.cols - w.c);
  w.row = threadIdx.x / a.tpr, w.rows = blockDim.x / a.tpr;
  return w;
}
// Sums of M values a channel over the block's rows, then over each group's channels
// weighted by `weigh`, of the channel within the block. chan [waves][M][8 tpr]: each
// channel's sums of a wave, then of the block in [M][8 tpr]; the channels are added in
// 64 bits, by 16 or 64 threads a group, the first of which makes of them what all
// threads find in stat[local group].
constexpr int kWide = 512;  // channels of a block at most
// Waves whose sums of a channel are still apart in chan after group_sums' first step
__device__ __forceinline__ int waves_left() { return blockDim.x > 256 ? 1 : blockDim.x >> 6; }
template <int M, typename F, typename G>
__device__ __forceinline__ void group_sums(const GnArgs &a, const Whole &w, float (&v)[M][8],
                                           float *chan, float2 *stat, F &&weigh, G &&make) {
  const int wide = a.tpr * kVec;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  for (int s = a.tpr; s < 64; s *= 2) {  // (all values at a step: a move takes a while)
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[m][i] += __shfl_xor(v[m][i], s);
  }
  __syncthreads();
  if (lane < a.tpr) {
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int i = 0; i < 8; ++i) chan[(wave * M + m) * wide + lane * 8 + i] = v[m][i];
  }
  __syncthreads();
  // many waves' in order, one thread a channel and value; the first wave's place takes them
  const int left = waves_left();
  if (left == 1) {
    for (int c = threadIdx.x; c < M * wide; c += blockDim.x) {
      float t = chan[c];
#pragma unroll 4
      for (int k = 1; k < waves; ++k) t += chan[k * M * wide + c];
      chan[c] = t;
    }
    __syncthreads();
  }
  const int here = (int)fdiv_q((uint32_t)min(a.width, a.cols - w.c0), a.by_per);
  // (one group a wave while there are waves for all, else four)
  const int lanes = here <= waves ? 64 : 16, in = threadIdx.x & (lanes - 1);
  for (int g = threadIdx.x / lanes; g < here; g += blockDim.x / lanes) {
    double t[M];
#pragma unroll
    for (int m = 0; m < M; ++m) t[m] = 0;
    for (int c = g * a.per + in; c < (g + 1) * a.per; c += lanes) {
      const double wt = weigh(c);
#pragma unroll
      for (int m = 0; m < M; ++m) {
        float x = chan[m * wide + c];
        for (int k = 1; k < left; ++k) x += chan[(k * M + m) * wide + c];
        t[m] += wt * x;
      }
    }
#pragma unroll
    for (int m = 0; m < M; ++m)
      for (int s = 1; s < lanes; s *= 2) t[m] += __shfl_xor(t[m], s);
    if (in == 0) make(g, t);
  }
  __syncthreads();
}
// A thread's channels' local groups
__device__ __forceinline__ int local_group(const GnArgs &a, const Whole &w, int i) {
  return (int)fdiv_q((uint32_t)(min(w.c + i, w.c0 + min(a.width, a.cols - w.c0) - 1) - w.c0),
                     a.by_per);
}

// Keeps the eight columns as they are stored: converted ones, kept for a later use, take
// twice the registers.
__device__ __forceinline__ void as_stored(Raw8<bf16> &r) { asm volatile("" : "+v"(r.w)); }
__device__ __forceinline__ void as_stored(Raw8<float> &) {}

template <typename T, int KIND, int R>
__global__ __launch_bounds__(1024) void gn_whole_kernel(GnArgs a) {
  extern __shared__ float2 stat[];  // [8 tpr], then chan (and, backward, gamma)
  const int wide = a.tpr * kVec;
  float *const chan = (float *)(stat + wide);
  const Whole w = whole(a);
  Raw8<T> r[R];
  float v[2][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[0][i] = v[1][i] = 0.f;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int64_t p = w.row + (int64_t)j * w.rows;
    const bool in = p < a.pixels;
    r[j] = load8((const T *)a.x.p + (w.b * a.pixels + (in ? p : 0)) * a.x.ld + w.c, in ? w.n : 0);
  }
#pragma unroll
  for (int j = 0; j < R; ++j) {
    float x[8];
    r[j].get(x);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[0][i] += x[i];
  }
  auto one = [](int) { return 1.0; };
  {
    float t[1][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[0][i] = v[0][i];
    group_sums<1>(a, w, t, chan, stat, one, [&](int g, const double (&t)[1]) {
      stat[g].x = (float)(t[0] * a.inv);
    });
  }
  int lg[8];
  float mu[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lg[i] = local_group(a, w, i);
    mu[i] = stat[lg[i]].x;
    v[0][i] = 0.f;
  }
  // the centred values' own sum corrects the mean
#pragma unroll
  for (int j = 0; j < R; ++j) {
    as_stored(r[j]);
    const bool in = w.row + (int64_t)j * w.rows < a.pixels;
    float x[8];
    r[j].get(x);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = in && i < w.n ? x[i] - mu[i] : 0.f;
      v[0][i] += d;
      v[1][i] = fmaf(d, d, v[1][i]);
    }
  }
  group_sums<2>(a, w, v, chan, stat, one, [&](int g, const double (&t)[2]) {
    const double off = t[0] * a.inv;
    double var = t[1] * a.inv - off * off;
    var = var < 0 ? 0 : var;  // (NaN stays)
    const float2 s = make_float2((float)((double)stat[g].x + off),
                                 rsqrt_rounded((float)var + a.eps));
    stat[g] = s;
    const int64_t at = w.b * a.groups + w.c0 / a.per + g;
    if (a.mean_out) a.mean_out[at] = s.x;
    if (a.rstd_out) a.rstd_out[at] = s.y;
  });
  float ga[8], be[8], rs[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 s = stat[lg[i]];
    mu[i] = s.x, rs[i] = s.y;
    ga[i] = 1.f, be[i] = 0.f;
  }
  if (a.gamma && w.n > 0) load8(a.gamma + w.c, w.n).get(ga);
  if (a.beta && w.n > 0) load8(a.beta + w.c, w.n).get(be);
  // (with a checkpoint the block's channels start and end with its groups of 32)
  const int wide_end = w.c0 + (a.k.q ? (a.width + kGroup - 1) / kGroup * kGroup : a.width);
  if (w.c >= wide_end || w.c >= a.pitch) return;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int64_t p = w.row + (int64_t)j * w.rows;
    if (p >= a.pixels) continue;
    const int64_t at = w.b * a.pixels + p;
    float x[8], y[8], df;
    as_stored(r[j]);
    r[j].get(x);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = i < w.n ? (x[i] - mu[i]) * rs[i] : 0.f;
      activate<KIND>(fmaf(x[i], ga[i], be[i]), y[i], df);
    }
    if (w.n > 0) store8((T *)a.y.p + at * a.y.ld + w.c, w.n, y);
    if (a.k.q) put8(a.k, at, w.c, x);
  }
}

template <typename T, int KIND, bool CK, int R>
__global__ __launch_bounds__(1024) void gn_whole_back_kernel(GnArgs a) {
  extern __shared__ float2 stat[];  // [8 tpr], then chan (and, backward, gamma)
  const int wide = a.tpr * kVec;
  float *const chan = (float *)(stat + wide);
  const Whole w = whole(a);
  Place q;  // as Back reads it
  q.b = w.b, q.c = w.c, q.n = w.n;
  Back<T, KIND, CK> back;
  back.init(a, q);
  float xh[R][8], e[R][8], v[2][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[0][i] = v[1][i] = 0.f;
  typename Back<T, KIND, CK>::Raw r[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int64_t p = w.row + (int64_t)j * w.rows;
    if (w.n > 0) r[j] = back.load(a, q, w.b * a.pixels + min(p, a.pixels - 1));
  }
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const bool in = w.row + (int64_t)j * w.rows < a.pixels && w.n > 0;
    if (in) back.get(q, r[j], xh[j], e[j]);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (in && i < w.n) {
        v[0][i] += e[j][i];
        v[1][i] = fmaf(e[j][i], xh[j][i], v[1][i]);
      }
  }
  float *const gam = chan + (blockDim.x >> 6) * 2 * wide;
  if (w.row == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) gam[w.c - w.c0 + i] = back.ga[i];
  }
  group_sums<2>(a, w, v, chan, stat, [&](int c) { return (double)gam[c]; },
                [&](int g, const double (&t)[2]) {
                  stat[g] = make_float2((float)(t[0] * a.inv), (float)(t[1] * a.inv));
                });
  // the image's sums of each channel, for dgamma and dbeta
  if (a.part) {
    const int here = min(a.width, a.cols - w.c0);
    for (int c = threadIdx.x; c < here; c += blockDim.x) {
      float s1 = chan[c], s2 = chan[wide + c];
      for (int k = 1; k < waves_left(); ++k)
        s1 += chan[2 * k * wide + c], s2 += chan[(2 * k + 1) * wide + c];
      if (a.batch == 1) {
        const int at = w.c0 + c;
        if (a.dbeta) a.dbeta[at] = a.accumulate ? a.dbeta[at] + s1 : s1;
        if (a.dgamma) a.dgamma[at] = a.accumulate ? a.dgamma[at] + s2 : s2;
      } else {
        a.part[w.b * a.cols + w.c0 + c] = make_float2(s1, s2);
      }
    }
  }
  if (w.n <= 0) return;
  float m1[8], m2[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 m = stat[local_group(a, w, i)];
    m1[i] = m.x, m2[i] = m.y;
  }
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int64_t p = w.row + (int64_t)j * w.rows;
    if (p >= a.pixels) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      e[j][i] = back.rs[i] * (fmaf(e[j][i], back.ga[i], -m1[i]) - xh[j][i] * m2[i]);
    store8((T *)a.dx.p + (w.b * a.pixels + p) * a.dx.ld + w.c, w.n, e[j]);
  }
}

// ------------------------------------------------------------------- plan
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
struct Split {
  int tpr, ctiles;
  int64_t slabs, slab;
};
Split split_of(int64_t batch, int64_t pixels, int64_t cols) {
  Split s;
  const int64_t vecs = pitch_of(cols) / kVec;
  s.tpr = 4;
  while (s.tpr < 64 && s.tpr < vecs) s.tpr *= 2;
  s.ctiles = (int)up(vecs, s.tpr);
  pixels = std::max<int64_t>(pixels, 1);
  batch = std::max<int64_t>(batch, 1);
  // (a thread's eight channels' constants take as long as a few pixels)
  auto cut = [&](int64_t blocks, int64_t least) {
    return std::min(blocks / s.ctiles / batch, up(pixels, 256 / s.tpr * least));
  };
  s.slab = up(pixels, std::max<int64_t>(std::max(cut(kUnits, kBatch), cut(kUnits / 4, kLeast)), 1));
  s.slabs = up(pixels, s.slab);
  return s;
}
// Never fewer units than split_of makes of as many images or fewer
int64_t most_units(int64_t batch, int64_t cols) {
  return std::max<int64_t>(batch, kUnits / split_of(1, 1, cols).ctiles);
}

// The block of a call whose groups fit into one: whole groups, at least 64 bytes of
// a pixel, few idle lanes, where there is a checkpoint whole groups of 32 channels (or all
// channels); two pixels a thread where there are as many threads (7 x 169 x 510 float32: one
// 12.5 us, two 10.3), at most most_r, which the registers hold. width 0: they do not fit.
struct Block {
  int width = 0, tpr = 0, threads = 0, r = 0;
};
Block block_of(int64_t batch, int64_t pixels, int64_t cols, int64_t per, int es, bool ckpt,
               int most_r) {
  Block best;
  double score = 0;
  for (int64_t w = per; w <= cols && w <= kWide; w += per) {
    if (ckpt && w % kGroup && w != cols) continue;
    int tpr = 4;
    while (tpr * kVec < w) tpr *= 2;
    if (pixels > (int64_t)most_r * (1024 / tpr)) break;
    const double line = std::min(1.0, (double)w * es / 64), full = (double)w / (tpr * kVec);
    if (line * full <= score + 0.1) continue;
    score = line * full;
    best.width = (int)w, best.tpr = tpr;
  }
  if (!best.width) return best;
  best.threads = 256;
  while (best.threads < 1024 && pixels > 2 * (best.threads / best.tpr)) best.threads *= 2;
  const int64_t r = up(pixels, best.threads / best.tpr);
  best.r = r <= 1 ? 1 : r <= 2 ? 2 : r <= 4 ? 4 : 8;
  // few large blocks leave most of the CUs idle for longer than two more launches take
  // (backward 8 x 784 x 96 float32, 32 blocks: 20.4 us, by slabs 14.6)
  if (batch * up(cols, best.width) < 128 && best.threads * best.r > 1024) best.width = 0;
  return best;
}

size_t part_bytes(int64_t units, int64_t cols) {
  return a256((size_t)units * (size_t)cols * 8);
}
// units' channels, images' channels, images' groups
size_t need_bytes(int64_t batch, int64_t cols, int64_t groups) {
  return part_bytes(most_units(batch, cols), cols) + part_bytes(batch, cols) +
         a256((size_t)batch * (size_t)groups * 8);
}

int gn_shape(int64_t batch, int64_t pixels, int64_t channels, int64_t groups, int32_t dtype) {
  if (batch < 0 || pixels < 0) return refuse(LRCNN_ESHAPE, "need batch >= 0 and pixels >= 0");
  if (batch > kMaxImages || channels > kMaxChannels)
    return refuse(LRCNN_ESHAPE, "group norm takes at most ", kMaxImages, " images and ",
                  kMaxChannels, " channels");
  if (pixels > kMaxRows || (batch && pixels > kMaxRows / batch))
    return refuse(LRCNN_ESHAPE, "matrix too large");
  const int st = take_shape(batch * pixels, channels, dtype);
  if (st != LRCNN_OK) return st;
  if (groups < 1 || channels % groups)
    return refuse(LRCNN_ESHAPE, "channels must be a multiple of groups");
  // (a grid has fewer than 2^32 threads; dividing by 512: a tile's channels)
  if (batch * groups > (int64_t)1 << 21 || batch * (channels / 512 + 1) > (int64_t)1 << 23)
    return refuse(LRCNN_ESHAPE, "too many images and groups or channels");
  return LRCNN_OK;
}

int gn_args(int64_t batch, int64_t pixels, int64_t channels, int64_t groups, void *ws,
            size_t ws_bytes, GnArgs *a) {
  if (!ws || ((uintptr_t)ws & 15)) return refuse(LRCNN_EINVAL, "workspace null or misaligned");
  const size_t need = need_bytes(batch, channels, groups);
  if (ws_bytes < need)
    return refuse(LRCNN_EWORKSPACE, "workspace needs ", need, " bytes, got ", ws_bytes);
  a->pixels = pixels, a->batch = (int)batch;
  a->cols = (int)channels, a->pitch = (int)pitch_of(channels);
  a->groups = (int)groups, a->per = (int)(channels / groups);
  a->by_per = fast_div((uint32_t)a->per);
  a->inv = 1.0 / ((double)pixels * (double)a->per);
  a->part = (float2 *)ws;
  a->chan = (float2 *)((char *)ws + part_bytes(most_units(batch, channels), channels));
  a->stat = (float2 *)((char *)a->chan + part_bytes(batch, channels));
  return LRCNN_OK;
}
// The passes over slabs
void cut(GnArgs *a) {
  const Split s = split_of(a->batch, a->pixels, a->cols);
  a->slab = s.slab, a->slabs = (int)s.slabs, a->units = a->batch * s.slabs;
  a->tpr = s.tpr, a->ctiles = s.ctiles;
}

// The arguments of the kernel that joins by group: where a group has many slabs and
// channels these are joined by channel first (one block of 1024 threads reads 850000
// entries, 512 slabs of 1659 channels, in 130 us).
template <bool SUMS>
GnArgs by_channel(GnArgs a, hipStream_t s) {
  if (a.slabs == 1 || (int64_t)a.slabs * a.per <= 32768) return a;
  gn_channel_kernel<SUMS><<<(unsigned)(a.batch * up(a.cols, 32)), 1024, 0, s>>>(a, a.chan);
  a.part = a.chan, a.slabs = 1, a.slab = a.pixels, a.units = a.batch;
  return a;
}
// Threads that join a group
unsigned join_threads(const GnArgs &a) {
  unsigned t = 64;
  while (t < 1024 && t * 2 < (int64_t)a.slabs * a.per) t *= 2;
  return t;
}

unsigned blocks_of(GnArgs *a, const Block &b) {
  a->width = b.width, a->tpr = b.tpr;
  a->ctiles = (int)up(a->cols, b.width);
  return (unsigned)((int64_t)a->batch * a->ctiles);
}
size_t lds_of(const Block &b) {
  return (size_t)b.tpr * kVec * (8 + b.threads / 64 * 2 * 4 + 4);
}
template <int MOST, typename F>
void by_r(int r, F &&f) {
  using std::integral_constant;
  if (r == 1) f(integral_constant<int, 1>());
  else if (r == 2) f(integral_constant<int, 2>());
  else if (r == 4 || MOST == 4) f(integral_constant<int, 4>());
  else f(integral_constant<int, MOST>());
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

extern "C" int lrcnn_group_norm_workspace_bytes(int64_t batch, int64_t pixels, int64_t channels,
                                                int64_t groups, size_t *bytes) {
  if (!bytes) return refuse(LRCNN_EINVAL, "null output");
  TRY(gn_shape(batch, pixels, channels, groups, LRCNN_F32));
  *bytes = need_bytes(batch, channels, groups);
  return LRCNN_OK;
}

extern "C" int lrcnn_group_norm_forward(int64_t batch, int64_t pixels, int64_t channels,
                                        int64_t groups, int32_t dtype, int32_t kind,
                                        const void *x, int64_t ldx, const float *gamma,
                                        const float *beta, float eps, void *y, int64_t ldy,
                                        float *mean, float *rstd, void *ckpt, void *workspace,
                                        size_t ws_bytes, void *stream) {
  TRY(gn_shape(batch, pixels, channels, groups, dtype));
  if (kind < LRCNN_ACT_NONE || kind > LRCNN_ACT_SILU)
    return refuse(LRCNN_EINVAL, "unknown activation");
  if (!(eps >= 0.f) || !(eps < INFINITY))
    return refuse(LRCNN_EINVAL, "eps must be finite and not negative");
  if (batch == 0 || pixels == 0) return LRCNN_OK;
  const int es = dtype == LRCNN_BF16 ? 2 : 4;
  GnArgs a{};
  TRY(take("x", x, ldx, channels, es, true, &a.x));
  TRY(take("y", y, ldy, channels, es, true, &a.y));
  TRY(same_rows("y", a.y, a.x, batch * pixels));
  TRY(take_f32("gamma", gamma, false));
  TRY(take_f32("beta", beta, false));
  TRY(take_f32("mean", mean, false));
  TRY(take_f32("rstd", rstd, false));
  TRY(take_ckpt("ckpt", ckpt, false));
  TRY(gn_args(batch, pixels, channels, groups, workspace, ws_bytes, &a));
  a.eps = eps, a.gamma = gamma, a.beta = beta, a.mean_out = mean, a.rstd_out = rstd;
  a.k = ckpt_of(ckpt, batch * pixels, channels);
  hipStream_t s = (hipStream_t)stream;
  const Block one = block_of(batch, pixels, channels, a.per, es, ckpt != nullptr, es == 2 ? 8 : 4);
  return by_kind_or_none(kind, [&](auto K) {
    auto run = [&](auto *t) {
      using T = std::remove_pointer_t<decltype(t)>;
      if (one.width) {
        GnArgs w = a;
        const unsigned g = blocks_of(&w, one);
        by_r<sizeof(T) == 2 ? 8 : 4>(one.r, [&](auto r) {
          gn_whole_kernel<T, K.value, r.value><<<g, one.threads, lds_of(one), s>>>(w);
        });
        return;
      }
      GnArgs w = a;
      cut(&w);
      const unsigned grid = (unsigned)(w.units * w.ctiles);
      gn_stats_kernel<T><<<grid, 256, 0, s>>>(w);
      const GnArgs j = by_channel<false>(w, s);
      gn_group_kernel<<<(unsigned)(batch * groups), join_threads(j), 0, s>>>(j);
      gn_apply_kernel<T, K.value><<<grid, 256, 0, s>>>(w);
    };
    if (dtype == LRCNN_BF16) run((bf16 *)nullptr);
    else run((float *)nullptr);
    return launched("group_norm_forward");
  });
}

extern "C" int lrcnn_group_norm_backward(int64_t batch, int64_t pixels, int64_t channels,
                                         int64_t groups, int32_t dtype, int32_t kind,
                                         const void *dy, int64_t lddy, const void *x, int64_t ldx,
                                         const float *mean, const void *ckpt, const float *rstd,
                                         const float *gamma, const float *beta, void *dx,
                                         int64_t lddx, float *dgamma, float *dbeta,
                                         int32_t accumulate, void *workspace, size_t ws_bytes,
                                         void *stream) {
  TRY(gn_shape(batch, pixels, channels, groups, dtype));
  if (kind < LRCNN_ACT_NONE || kind > LRCNN_ACT_SILU)
    return refuse(LRCNN_EINVAL, "unknown activation");
  const int es = dtype == LRCNN_BF16 ? 2 : 4;
  GnArgs a{};
  TRY(take_f32("dgamma", dgamma, false));
  TRY(take_f32("dbeta", dbeta, false));
  const bool some = batch && pixels;
  if (some) {
    if ((x != nullptr) == (ckpt != nullptr) || (x != nullptr) != (mean != nullptr))
      return refuse(LRCNN_EINVAL, "give x with mean, or ckpt");
    TRY(take("dy", dy, lddy, channels, es, true, &a.y));
    TRY(take("x", x, ldx, channels, es, false, &a.x));
    TRY(take("dx", dx, lddx, channels, es, true, &a.dx));
    TRY(same_rows("dx", a.dx, a.y, batch * pixels));
    TRY(same_rows("dx", a.dx, a.x, batch * pixels));
    TRY(take_f32("mean", mean, false));
    TRY(take_f32("rstd", rstd, true));
    TRY(take_f32("gamma", gamma, false));
    TRY(take_f32("beta", beta, false));
    TRY(take_ckpt("ckpt", ckpt, false));
  }
  const bool grads = dgamma || dbeta;
  if (!some && (!grads || accumulate)) return LRCNN_OK;
  TRY(gn_args(batch, pixels, channels, groups, workspace, ws_bytes, &a));
  a.mean = mean, a.rstd = rstd, a.gamma = gamma, a.beta = beta;
  a.dgamma = dgamma, a.dbeta = dbeta, a.accumulate = accumulate != 0;
  a.k = ckpt_of(ckpt, batch * pixels, channels);
  hipStream_t s = (hipStream_t)stream;
  const unsigned chans = (unsigned)up(channels, kChans);
  if (!some) {  // no rows: the gradients are zero
    a.units = 0;
    gn_grads_kernel<<<chans, 1024, 0, s>>>(a);
    return launched("group_norm_backward");
  }
  const Block one = block_of(batch, pixels, channels, a.per, es, ckpt != nullptr, 4);
  return by_kind_or_none(kind, [&](auto K) {
    auto run = [&](auto *t, auto ck) {
      using T = std::remove_pointer_t<decltype(t)>;
      if (one.width) {
        GnArgs w = a;
        const unsigned g = blocks_of(&w, one);
        if (!grads) w.part = nullptr;
        by_r<4>(one.r, [&](auto r) {
          gn_whole_back_kernel<T, K.value, ck.value, r.value><<<g, one.threads, lds_of(one), s>>>(w);
        });
        w.units = batch;
        if (grads && batch > 1) gn_grads_kernel<<<chans, 1024, 0, s>>>(w);
        return;
      }
      GnArgs w = a;
      cut(&w);
      const unsigned grid = (unsigned)(w.units * w.ctiles);
      gn_sums_kernel<T, K.value, ck.value><<<grid, 256, 0, s>>>(w);
      const GnArgs j = by_channel<true>(w, s);
      if (join_threads(j) == 1024 || batch * groups < 512) {
        gn_join_kernel<<<(unsigned)(batch * groups) + (grads ? chans : 0), 1024, 0, s>>>(j);
      } else {
        gn_join_kernel<<<(unsigned)(batch * groups), join_threads(j), 0, s>>>(j);
        if (grads) gn_grads_kernel<<<chans, 1024, 0, s>>>(j);
      }
      gn_dx_kernel<T, K.value, ck.value><<<grid, 256, 0, s>>>(w);
    };
    auto typed = [&](auto *t) {
      if (ckpt) run(t, std::true_type());
      else run(t, std::false_type());
    };
    if (dtype == LRCNN_BF16) typed((bf16 *)nullptr);
    else typed((float *)nullptr);
    return launched("group_norm_backward");
  });
}
