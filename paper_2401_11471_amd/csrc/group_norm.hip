// Group norm with an activation over an NHWC map, forward and backward.
//
//   forward   xh = (x - mean) rstd over the pixels and channels of a group of an
//             image, y = f(gamma xh + beta)
//   backward  e = dy f'(gamma xh + beta), q = gamma e,
//             dx = rstd (q - mean(q) - xh mean(q xh)),
//             dgamma = sum of e xh, dbeta = sum of e
//
// A group's sums need all its pixels before the first result, so a map is read
// twice: a pass that leaves, for every channel of a slab of pixels, two numbers
// (forward: mean and centred sum of squares; backward: sums of e and e xh), a small
// kernel that joins them by group (and by channel for dgamma, dbeta), and a pass
// that applies the result. A channel's two numbers serve every way of
// grouping, whatever the group's width and alignment, and in the backward pass both
// the groups' means (weighted by gamma) and the parameters' gradients.
//
// Statistics: eight pixels at a time are centred in registers (their mean
// corrected by the centred sum), then joined with
//   n = na + nb, d = mb - ma, mean = ma + d nb / n, M2 = Ma + Mb + d^2 na nb / n,
// so that a mean far from zero costs the variance no digits; across slabs
// and channels in 64 bits.
#include "activation.hpp"

#include <algorithm>
#include <type_traits>

namespace lrcnn {
namespace act8 {
namespace {

constexpr int64_t kMaxImages = 1 << 20, kMaxChannels = 1 << 20;
constexpr int kBatch = 8;         // pixels that a thread holds at a time
constexpr int kUnits = 2048;      // blocks of a pass, where there are as many
constexpr int kApplyPixels = 4;   // applying passes: pixels in flight a thread

struct GnArgs {
  int64_t pixels, slab;  // pixels of an image and of a slab
  int64_t units;         // images times slabs
  int slabs, batch, cols, pitch, groups, per;  // per: channels of a group
  int tpr, ctiles;       // threads of a pixel's channels; tiles of 8 tpr channels
  float eps;
  Mat x, y;              // backward: y is dy
  Mat dx;
  const float *gamma, *beta;
  const float *mean, *rstd;  // [batch][groups]
  float *mean_out, *rstd_out;
  float2 *part;          // [units][cols]
  float2 *stat;          // [batch][groups]: (mean, rstd), backward the two means
  float *dgamma, *dbeta;
  int accumulate;
  Ckpt k;
};

// Slab s of image b and the channels of this thread.
struct Place {
  int64_t b, p0, p1;  // the slab's pixels within the image
  int64_t unit;
  int c, n, row, rows;  // first channel, channels left, this thread's row and rows a block
};
__device__ __forceinline__ Place place(const GnArgs &a) {
  Place q;
  const int ct = blockIdx.x % a.ctiles;
  q.unit = blockIdx.x / a.ctiles;
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
    const float2 v = stat[q.b * a.groups + c / a.per];
    s[i] = v.x, t[i] = v.y;
  }
}
__device__ __forceinline__ void group8(const GnArgs &a, const float *stat, const Place &q,
                                       float (&s)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    s[i] = stat[q.b * a.groups + min(q.c + i, a.cols - 1) / a.per];
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
__global__ __launch_bounds__(256) void gn_group_kernel(GnArgs a) {
  __shared__ double red[4];
  const int64_t b = blockIdx.x / a.groups;
  const int g = blockIdx.x % a.groups;
  const int64_t all = (int64_t)a.slabs * a.per;
  const float2 *part = a.part + b * a.slabs * (int64_t)a.cols + (int64_t)g * a.per;
  const double total = (double)a.pixels * a.per;
  auto count = [&](int64_t s) { return (double)min(a.slab, a.pixels - s * a.slab); };
  double sum = 0;
  for (int64_t e = threadIdx.x; e < all; e += 256) {
    const int64_t s = e / a.per;
    sum += count(s) * part[s * a.cols + (e - s * a.per)].x;
  }
  const double mean = block_sum(sum, red) / total;
  double m2 = 0;
  for (int64_t e = threadIdx.x; e < all; e += 256) {
    const int64_t s = e / a.per;
    const float2 v = part[s * a.cols + (e - s * a.per)];
    const double d = v.x - mean;
    m2 += v.y + count(s) * d * d;
  }
  double var = block_sum(m2, red) / total;
  var = var < 0 ? 0 : var;  // (NaN stays)
  if (threadIdx.x == 0) {
    const float m = (float)mean, r = (float)(1 / sqrt(var + (double)a.eps));
    a.stat[blockIdx.x] = make_float2(m, r);
    if (a.mean_out) a.mean_out[blockIdx.x] = m;
    if (a.rstd_out) a.rstd_out[blockIdx.x] = r;
  }
}

template <typename T, int KIND>
__global__ __launch_bounds__(256) void gn_apply_kernel(GnArgs a) {
  const Place q = place(a);
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

// The first batch * groups blocks: a group's two means, of q and q xh. Then one
// block for 32 channels: dgamma and dbeta, thread (r, c) taking every 32nd unit
// from r on, the 32 sums joined in order.
__global__ __launch_bounds__(1024) void gn_join_kernel(GnArgs a) {
  __shared__ double red[16];
  __shared__ float l1[32][33], l2[32][33];
  const int64_t bg = (int64_t)a.batch * a.groups;
  if (blockIdx.x < bg) {
    const int64_t b = blockIdx.x / a.groups;
    const int g = blockIdx.x % a.groups;
    const int64_t all = (int64_t)a.slabs * a.per;
    const float2 *part = a.part + b * a.slabs * (int64_t)a.cols + (int64_t)g * a.per;
    double s1 = 0, s2 = 0;
    for (int64_t e = threadIdx.x; e < all; e += 1024) {
      const int64_t s = e / a.per, c = e - s * a.per;
      const float2 v = part[s * a.cols + c];
      const double ga = a.gamma ? (double)a.gamma[g * a.per + c] : 1.0;
      s1 += ga * v.x, s2 += ga * v.y;
    }
    const double total = (double)a.pixels * a.per;
    s1 = block_sum(s1, red);
    s2 = block_sum(s2, red);
    if (threadIdx.x == 0) a.stat[blockIdx.x] = make_float2((float)(s1 / total), (float)(s2 / total));
    return;
  }
  const int r = threadIdx.x >> 5, c = (int)(blockIdx.x - bg) * 32 + (threadIdx.x & 31);
  float s1 = 0.f, s2 = 0.f;
  if (c < a.cols) {
#pragma unroll 8
    for (int64_t u = r; u < a.units; u += 32) {
      const float2 v = a.part[u * a.cols + c];
      s1 += v.x, s2 += v.y;
    }
  }
  l1[r][threadIdx.x & 31] = s1;
  l2[r][threadIdx.x & 31] = s2;
  __syncthreads();
  if (r == 0 && c < a.cols) {
    for (int k = 1; k < 32; ++k) s1 += l1[k][threadIdx.x], s2 += l2[k][threadIdx.x];
    if (a.dbeta) a.dbeta[c] = a.accumulate ? a.dbeta[c] + s1 : s1;
    if (a.dgamma) a.dgamma[c] = a.accumulate ? a.dgamma[c] + s2 : s2;
  }
}

template <typename T, int KIND, bool CK>
__global__ __launch_bounds__(256) void gn_dx_kernel(GnArgs a) {
  constexpr int R = kApplyPixels;
  const Place q = place(a);
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

// ------------------------------------------------------------------- plan
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
struct Split {
  int tpr, ctiles;
  int64_t slabs, slab;
  int64_t most_units;  // of any call with as many images and pixels, or fewer
};
Split split_of(int64_t batch, int64_t pixels, int64_t cols) {
  Split s;
  const int64_t vecs = pitch_of(cols) / kVec;
  s.tpr = 4;
  while (s.tpr < 64 && s.tpr < vecs) s.tpr *= 2;
  s.ctiles = (int)up(vecs, s.tpr);
  const int64_t least = 256 / s.tpr * kBatch;  // pixels worth a block
  const int64_t units = std::max<int64_t>(kUnits / s.ctiles, 1);
  const int64_t by_pixels = up(std::max<int64_t>(pixels, 1), least);
  const int64_t n = std::max<int64_t>(std::min(units / std::max<int64_t>(batch, 1), by_pixels), 1);
  s.slab = up(std::max<int64_t>(pixels, 1), n);
  s.slabs = up(std::max<int64_t>(pixels, 1), s.slab);
  s.most_units = std::max(batch, by_pixels >= units ? units : std::min(units, batch * by_pixels));
  return s;
}

size_t part_bytes(const Split &s, int64_t cols) {
  return a256((size_t)s.most_units * (size_t)cols * 8);
}
size_t need_bytes(const Split &s, int64_t batch, int64_t cols, int64_t groups) {
  return part_bytes(s, cols) + a256((size_t)batch * (size_t)groups * 8);
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
            size_t ws_bytes, GnArgs *a, Split *s) {
  if (!ws || ((uintptr_t)ws & 15)) return refuse(LRCNN_EINVAL, "workspace null or misaligned");
  *s = split_of(batch, pixels, channels);
  const size_t need = need_bytes(*s, batch, channels, groups);
  if (ws_bytes < need)
    return refuse(LRCNN_EWORKSPACE, "workspace needs ", need, " bytes, got ", ws_bytes);
  a->pixels = pixels, a->slab = s->slab, a->slabs = (int)s->slabs, a->batch = (int)batch;
  a->units = batch * s->slabs;
  a->cols = (int)channels, a->pitch = (int)pitch_of(channels);
  a->groups = (int)groups, a->per = (int)(channels / groups);
  a->tpr = s->tpr, a->ctiles = s->ctiles;
  a->part = (float2 *)ws;
  a->stat = (float2 *)((char *)ws + part_bytes(*s, channels));
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

extern "C" int lrcnn_group_norm_workspace_bytes(int64_t batch, int64_t pixels, int64_t channels,
                                                int64_t groups, size_t *bytes) {
  if (!bytes) return refuse(LRCNN_EINVAL, "null output");
  TRY(gn_shape(batch, pixels, channels, groups, LRCNN_F32));
  *bytes = need_bytes(split_of(batch, pixels, channels), batch, channels, groups);
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
  TRY(take_f32("gamma", gamma, false));
  TRY(take_f32("beta", beta, false));
  TRY(take_f32("mean", mean, false));
  TRY(take_f32("rstd", rstd, false));
  TRY(take_ckpt("ckpt", ckpt, false));
  Split sp;
  TRY(gn_args(batch, pixels, channels, groups, workspace, ws_bytes, &a, &sp));
  a.eps = eps, a.gamma = gamma, a.beta = beta, a.mean_out = mean, a.rstd_out = rstd;
  a.k = ckpt_of(ckpt, batch * pixels, channels);
  hipStream_t s = (hipStream_t)stream;
  const unsigned grid = (unsigned)(a.units * a.ctiles);
  return by_kind_or_none(kind, [&](auto K) {
    auto run = [&](auto *t) {
      using T = std::remove_pointer_t<decltype(t)>;
      gn_stats_kernel<T><<<grid, 256, 0, s>>>(a);
      gn_group_kernel<<<(unsigned)(batch * groups), 256, 0, s>>>(a);
      gn_apply_kernel<T, K.value><<<grid, 256, 0, s>>>(a);
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
    TRY(take_f32("mean", mean, false));
    TRY(take_f32("rstd", rstd, true));
    TRY(take_f32("gamma", gamma, false));
    TRY(take_f32("beta", beta, false));
    TRY(take_ckpt("ckpt", ckpt, false));
  }
  const bool grads = dgamma || dbeta;
  if (!some && (!grads || accumulate)) return LRCNN_OK;
  Split sp;
  TRY(gn_args(batch, pixels, channels, groups, workspace, ws_bytes, &a, &sp));
  a.mean = mean, a.rstd = rstd, a.gamma = gamma, a.beta = beta;
  a.dgamma = dgamma, a.dbeta = dbeta, a.accumulate = accumulate != 0;
  a.k = ckpt_of(ckpt, batch * pixels, channels);
  hipStream_t s = (hipStream_t)stream;
  if (!some) a.batch = 0, a.units = 0;
  const unsigned join = (unsigned)(a.batch * (int64_t)groups + (grads ? up(channels, 32) : 0));
  if (!some) {  // no rows: the gradients are zero
    gn_join_kernel<<<join, 1024, 0, s>>>(a);
    return launched("group_norm_backward");
  }
  const unsigned grid = (unsigned)(a.units * a.ctiles);
  return by_kind_or_none(kind, [&](auto K) {
    auto run = [&](auto *t, auto ck) {
      using T = std::remove_pointer_t<decltype(t)>;
      gn_sums_kernel<T, K.value, ck.value><<<grid, 256, 0, s>>>(a);
      gn_join_kernel<<<join, 1024, 0, s>>>(a);
      gn_dx_kernel<T, K.value, ck.value><<<grid, 256, 0, s>>>(a);
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
