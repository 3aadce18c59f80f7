// Entries of the gated feed-forward block: their checks, and the products that they are.
#include "gated_ffn.hpp"

#include <algorithm>
#include <initializer_list>

namespace lrcnn {
namespace act8 {

std::atomic<int> g_ffn_tile{-1};

namespace {

void run(int32_t dtype, Epi epi, const FfnArgs &a, void *stream) {
  (dtype == LRCNN_BF16 ? ffn_bf16 : ffn_f32)(epi, a, (hipStream_t)stream);
}

// n: the block's input or output features. The products that this call makes with them
// have at most 2 hidden or n features.
int ffn_shape(int64_t rows, int64_t n, int64_t hidden, int32_t dtype, int32_t kind) {
  const int st = take_shape(rows, n, dtype);
  if (st != LRCNN_OK) return st;
  if (hidden < 1) return refuse(LRCNN_ESHAPE, "need hidden >= 1");
  if (n > kMaxFeatures || hidden > kMaxFeatures / 2 || rows > kMaxFfnRows)
    return refuse(LRCNN_ESHAPE, "gated_ffn takes at most 2^24 features and 2^30 rows");
  if (((rows + 127) / 128) * ((std::max(n, 2 * hidden) + 127) / 128) > kMostMidTiles)
    return refuse(LRCNN_ESHAPE, "gated_ffn takes fewer than 2^22 tiles of 128 x 128");
  if (kind < LRCNN_ACT_RELU || kind > LRCNN_ACT_SILU)
    return refuse(LRCNN_EINVAL, "unknown activation");
  return LRCNN_OK;
}

// A product reads all of its inputs for each part of its result: what it writes has to
// be other memory.
int apart(const char *what, const void *out, std::initializer_list<const void *> in) {
  if (out)
    for (const void *p : in)
      if (p == out) return refuse(LRCNN_EINVAL, what, " is an input of its product");
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

extern "C" void lrcnn_debug_ffn_tile(int32_t tile) { g_ffn_tile = tile; }

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
  TRY(apart("a", a, {x, w1, b1, z ? w2 : nullptr, z ? (const void *)b2 : nullptr}));
  TRY(apart("uv", uv, {x, w1, b1, a}));
  if (z) TRY(apart("z", z, {a, w2, b2}));
  g.rows = (int)rows, g.depth = (int)n_in, g.feats = (int)hidden, g.kind = kind;
  g.w = w.p, g.bias = b1;
  g.ku = ckpt_of(ckpt_u, rows, hidden);
  g.kv = ckpt_of(ckpt_v, rows, hidden);
  run(dtype, EPI_GATE, g, stream);
  if (z) {
    FfnArgs d{};
    d.rows = (int)rows, d.depth = (int)hidden, d.feats = (int)n_out;
    d.x = g.out, d.w = w2m.p, d.bias = b2, d.out = zm;
    run(dtype, EPI_PLAIN, d, stream);
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
  TRY(apart("duv", duv, {dz, w2t, dx ? w1t : nullptr}));
  TRY(same_rows("duv", g.out, g.uv, rows));
  if (dx) TRY(apart("dx", dx, {duv, w1t}));
  g.rows = (int)rows, g.depth = (int)n_out, g.feats = (int)hidden, g.kind = kind;
  g.w = w.p;
  g.ku = ckpt_of(ckpt_u, rows, hidden);
  g.kv = ckpt_of(ckpt_v, rows, hidden);
  g.ka = ckpt_of(ckpt_a, rows, hidden);
  run(dtype, EPI_BACK, g, stream);
  if (dx) {
    FfnArgs d{};
    d.rows = (int)rows, d.depth = (int)(2 * hidden), d.feats = (int)n_in;
    d.x = g.out, d.w = w1m.p, d.out = xm;
    run(dtype, EPI_PLAIN, d, stream);
  }
  return launched("gated_ffn_backward");
}
