// Products of the gated feed-forward block in bfloat16.
#define LRCNN_FFN_KERNELS
#include "gated_ffn.hpp"

namespace lrcnn {
namespace act8 {
void ffn_bf16(Epi epi, const FfnArgs &a, hipStream_t s) { products_of<bf16>(epi, a, s); }
}  // namespace act8
}  // namespace lrcnn
