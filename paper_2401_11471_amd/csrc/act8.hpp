// 8-bit activation checkpoints: the buffer's layout, the code of a group and
// the row accesses shared by the kernels that write or read one (pack and
// unpack, layer norm, activations, the linear layer's weight gradient).
//
// A group is 32 consecutive columns of a row. With m its largest magnitude,
//   E = max((bits(m) + 2^16) >> 23, 7),   x ~ q 2^(E - 133),
//   q = rint(x 2^(133 - E)), |q| <= 127.
// Adding 2^16 to the bits of m carries into the exponent exactly where m's
// mantissa is 2 - 2^-7 or more, so that no value rounds to 128 steps. The step
// is a power of two: x 2^(133 - E) is exact, so a code is one correctly
// rounded integer whatever kernel forms it, and q 2^(E - 133), of 7 bits or
// fewer, is a bfloat16 number: what reads a checkpoint as bfloat16 rounds
// nothing.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "lrcnn.h"

int lrcnn_fail(int code, const std::string &msg);

namespace lrcnn {
namespace act8 {

typedef uint16_t bf16;
constexpr int kGroup = 32;  // columns that share an exponent
constexpr int kVec = 8;     // columns per thread and step: four lanes make a group
constexpr int64_t kMaxCols = (int64_t)1 << 30;
constexpr int64_t kMaxRows = (int64_t)1 << 40;
constexpr int64_t kMaxElems = (int64_t)1 << 44;

// Codes [rows][pitch], then, from the next multiple of 256 bytes, exponent
// bytes [rows][pitch / 32].
struct Ckpt {
  int8_t *q = nullptr;
  uint8_t *e = nullptr;
  int64_t pitch = 0;
};
inline int64_t pitch_of(int64_t cols) { return (cols + kGroup - 1) / kGroup * kGroup; }
inline size_t a256(size_t n) { return (n + 255) & ~(size_t)255; }
inline size_t ckpt_bytes(int64_t rows, int64_t cols) {
  const size_t n = (size_t)rows * (size_t)pitch_of(cols);
  return a256(n) + a256(n / kGroup);
}
inline Ckpt ckpt_of(const void *p, int64_t rows, int64_t cols) {
  Ckpt c;
  if (!p) return c;
  c.pitch = pitch_of(cols);
  c.q = (int8_t *)p;
  c.e = (uint8_t *)p + a256((size_t)rows * (size_t)c.pitch);
  return c;
}

// ------------------------------------------------------ argument checks
// The code of a refusal, its message kept; no exception (memory for the message)
// leaves a C entry.
inline void put_part(std::string &m, const char *p) { m += p; }
template <typename N>
void put_part(std::string &m, N n) {
  m += std::to_string(n);
}
template <typename... P>
int refuse(int code, P... parts) noexcept {
  try {
    std::string m;
    (put_part(m, parts), ...);
    return lrcnn_fail(code, m);
  } catch (...) {
    return code;
  }
}
// A row-major matrix of the caller: rows at `ld` elements from each other
// (0: dense). Any alignment of a whole element will do.
struct Mat {
  char *p = nullptr;
  int64_t ld = 0;
};
// The matrix, or a refusal in *err (st < 0): null where it must not be, a
// pointer that cuts an element, or rows that overlap.
inline int take(const char *what, const void *p, int64_t ld, int64_t cols, int es, bool must,
                Mat *m) {
  if (!p && must) return refuse(LRCNN_EINVAL, what, " is null");
  if ((uintptr_t)p % es) return refuse(LRCNN_EINVAL, what, " is misaligned");
  if (p && ld != 0 && ld < cols)
    return refuse(LRCNN_ESHAPE, what, ": row stride smaller than a row");
  if (p && ld > ((int64_t)1 << 40))
    return refuse(LRCNN_ESHAPE, what, ": row stride too large");
  m->p = (char *)p;
  m->ld = ld ? ld : cols;
  return LRCNN_OK;
}
// An output in place of an input is that matrix: its rows are written where the same
// rows are read, not where others still are.
inline int same_rows(const char *what, const Mat &out, const Mat &in, int64_t rows) {
  if (out.p && out.p == in.p && out.ld != in.ld && rows > 1)
    return refuse(LRCNN_EINVAL, what, " is an input's memory with another row stride");
  return LRCNN_OK;
}
inline int take_f32(const char *what, const void *p, bool must) {
  if (!p && must) return refuse(LRCNN_EINVAL, what, " is null");
  if ((uintptr_t)p & 3) return refuse(LRCNN_EINVAL, what, " is misaligned");
  return LRCNN_OK;
}
inline int take_ckpt(const char *what, const void *p, bool must) {
  if (!p && must) return refuse(LRCNN_EINVAL, what, " is null");
  if ((uintptr_t)p & 15)
    return refuse(LRCNN_EINVAL, what, " is not 16-byte aligned");
  return LRCNN_OK;
}
inline int take_shape(int64_t rows, int64_t cols, int32_t dtype) {
  if (dtype != LRCNN_F32 && dtype != LRCNN_BF16)
    return refuse(LRCNN_EDTYPE, "dtype must be LRCNN_F32 or LRCNN_BF16");
  if (rows < 0 || cols < 1) return refuse(LRCNN_ESHAPE, "need rows >= 0 and cols >= 1");
  if (rows > kMaxRows || cols > kMaxCols || (rows && cols > kMaxElems / rows))
    return refuse(LRCNN_ESHAPE, "matrix too large");
  return LRCNN_OK;
}
inline int launched(const char *what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return LRCNN_OK;
  return refuse(LRCNN_EHIP, what, ": ", hipGetErrorString(e));
}

#ifdef __HIPCC__
// ------------------------------------------------------------- row access
// Eight consecutive columns as 16-byte accesses at the element's own
// alignment (rows of odd width, slices): gfx950 takes such addresses, an
// unaligned access costs a second cache line at most.
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16 v) { return __uint_as_float((uint32_t)v << 16); }
// (v_cvt_pk_bf16_f32: round to nearest, ties to even)
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16 *p, float v) {
  *p = __builtin_bit_cast(bf16, (__bf16)v);
}
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf_pair(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
}

// What a thread holds of a row: eight columns as stored.
template <typename T>
struct Raw8;
template <>
struct Raw8<bf16> {
  u32x4_a2 w;
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};
template <>
struct Raw8<float> {
  f32x4_a4 a, b;
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  }
};

// Columns [c, c + 8) of a row of n = columns left from c on; zeros past them.
__device__ __forceinline__ Raw8<bf16> load8(const bf16 *p, int64_t n) {
  Raw8<bf16> r;
  if (n >= 8) {
    r.w = *(const u32x4_a2 *)p;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = 2 * i < n ? p[2 * i] : 0, hi = 2 * i + 1 < n ? p[2 * i + 1] : 0;
      r.w[i] = lo | (hi << 16);
    }
  }
  return r;
}
__device__ __forceinline__ Raw8<float> load8(const float *p, int64_t n) {
  Raw8<float> r;
  if (n >= 8) {
    r.a = *(const f32x4_a4 *)p;
    r.b = *(const f32x4_a4 *)(p + 4);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.a[i] = i < n ? p[i] : 0.f;
      r.b[i] = 4 + i < n ? p[4 + i] : 0.f;
    }
  }
  return r;
}
__device__ __forceinline__ void store8(bf16 *p, int64_t n, const float (&v)[8]) {
  if (n >= 8) {
    u32x4_a2 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = bf_pair(v[2 * i], v[2 * i + 1]);
    *(u32x4_a2 *)p = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) put(p + i, v[i]);
  }
}
__device__ __forceinline__ void store8(float *p, int64_t n, const float (&v)[8]) {
  if (n >= 8) {
    f32x4_a4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = v[i], b[i] = v[4 + i];
    *(f32x4_a4 *)p = a;
    *(f32x4_a4 *)(p + 4) = b;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = v[i];
  }
}

// 1 / sqrt(x) to the last bit but for near ties: the instruction's value, an ulp off
// in one row of seven (an error that a whole row and its checkpoint share), and
// one Newton step y + y (1 - x y^2) / 2, x y as a sum of two floats. Zero and
// infinity, where the step is NaN, keep their limits.
__device__ __forceinline__ float rsqrt_rounded(float x) {
  const float y = rsqrtf(x);
  const float h = x * y, l = fmaf(x, y, -h);
  const float e = fmaf(-l, y, fmaf(-h, y, 1.f));
  const float z = fmaf(0.5f * e, y, y);
  return z == z ? z : y;
}

// ------------------------------------------------------------- the codes
// quad_perm moves inside the four lanes that hold one group
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xb1, 0xf, 0xf, true));  // lane ^ 1
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4e, 0xf, 0xf, true));  // lane ^ 2
  return m;
}
// Codes of eight columns whose group is held by this lane's quad, and the
// group's exponent byte. All four lanes take part. Adding 1.5 2^23 rounds to
// the nearest integer, ties to even, and leaves it in the low byte; the
// product before it is exact, so one FMA does both.
__device__ __forceinline__ uint32_t largest_of(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return quad_max(m);
}
__device__ __forceinline__ uint32_t exponent_of(uint32_t m) {
  return max((m + 0x10000u) >> 23, 7u);
}
// below the top binade's last step
__device__ __forceinline__ uint2 codes_of(const float (&v)[8], uint32_t E) {
  const float inv = __uint_as_float((260u - E) << 23);
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(fmaf(v[i], inv, 12582912.f));
  // low bytes of four words into one
  const uint32_t lo0 = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u);
  const uint32_t hi0 = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
  const uint32_t lo1 = __builtin_amdgcn_perm(b[5], b[4], 0x0c0c0400u);
  const uint32_t hi1 = __builtin_amdgcn_perm(b[7], b[6], 0x04000c0cu);
  return make_uint2(lo0 | hi0, lo1 | hi1);
}
// The top binade's last step (the type's lowest value as a mask): held to +-127
// steps of 2^121; infinity or NaN: the group stands for NaN
__device__ __forceinline__ bool at_top(uint32_t m) { return m >= 0x7f7f0000u; }
__device__ __forceinline__ uint2 top_codes_of(const float (&v)[8], uint32_t m, uint32_t *E) {
  const bool bad = m >= 0x7f800000u;
  *E = bad ? 255u : 254u;
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float s = fminf(fmaxf(v[i] * 0x1p-121f, -127.f), 127.f);
    const uint32_t b = bad ? 0 : __float_as_uint(s + 12582912.f) & 0xffu;
    w[i >> 2] |= b << (8 * (i & 3));
  }
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint2 encode8(const float (&v)[8], uint32_t *exponent) {
  const uint32_t m = largest_of(v);
  *exponent = exponent_of(m);
  if (__builtin_expect(at_top(m), 0)) return top_codes_of(v, m, exponent);
  return codes_of(v, *exponent);
}
// 2^(E - 133) (NaN for E = 255); subnormal steps do not occur (E >= 7)
__device__ __forceinline__ float step_of(uint32_t E) {
  return E == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float((E - 6u) << 23);
}
// Four codes times the step, exact
__device__ __forceinline__ void decode4(uint32_t w, float step, float *v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (float)((int32_t)(w << (24 - 8 * i)) >> 24) * step;
}
__device__ __forceinline__ void decode8(uint2 q, uint32_t E, float (&v)[8]) {
  const float s = step_of(E);
  decode4(q.x, s, v);
  decode4(q.y, s, v + 4);
}
// Columns c .. c + 7 of row r into / out of a checkpoint (c a multiple of 8
// below the pitch)
__device__ __forceinline__ void put8(const Ckpt &k, int64_t r, int64_t c, const float (&v)[8]) {
  uint32_t E;
  const uint2 q = encode8(v, &E);
  *(uint2 *)(k.q + r * k.pitch + c) = q;
  if ((c & (kGroup - 1)) == 0) k.e[r * (k.pitch / kGroup) + c / kGroup] = (uint8_t)E;
}
__device__ __forceinline__ void get8(const Ckpt &k, int64_t r, int64_t c, float (&v)[8]) {
  decode8(*(const uint2 *)(k.q + r * k.pitch + c), k.e[r * (k.pitch / kGroup) + c / kGroup], v);
}
#endif  // __HIPCC__

}  // namespace act8
}  // namespace lrcnn
