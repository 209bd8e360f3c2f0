// The product's kernels with epilogues of their own for f16 operands.
#include "product_modes_launch.h"

namespace som {

hipError_t launch_modes_f16(int mode, int shape, const ProductArgs& a, hipStream_t stream) {
  return launch_mode_elem<kF16>(mode, shape, a, stream);
}

hipError_t launch_mirror_f16(int shape, const ExtraArgs& a, hipStream_t stream) {
  return a.p_kc ? launch_square<kF16, true, kMirror>(shape, a, stream) : launch_square<kF16, false, kMirror>(shape, a, stream);
}

}  // namespace som
