// The matrix product's kernels for f16 operands.
#include "product_launch.h"

namespace som {

hipError_t launch_product_f16(int shape, const ProductArgs& a, hipStream_t stream) {
  return launch_elem<kF16>(shape, a, stream);
}

}  // namespace som
