// Products of the gated feed-forward block in float32.
#define LRCNN_FFN_KERNELS
#include "gated_ffn.hpp"

namespace lrcnn {
namespace act8 {
void ffn_f32(Epi epi, const FfnArgs &a, hipStream_t s) { products_of<float>(epi, a, s); }
}  // namespace act8
}  // namespace lrcnn
