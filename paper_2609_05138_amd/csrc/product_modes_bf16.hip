// The product's kernels with epilogues of their own for bf16 operands.
#include "product_modes_launch.h"

namespace som {

hipError_t launch_modes_bf16(int mode, int shape, const ProductArgs& a, hipStream_t stream) {
  return launch_mode_elem<kBF16>(mode, shape, a, stream);
}

}  // namespace som
