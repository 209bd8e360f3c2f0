// The matrix product's kernels for bf16 operands.
#include "product_launch.h"

namespace som {

hipError_t launch_product_bf16(int shape, const ProductArgs& a, hipStream_t stream) {
  return launch_elem<kBF16>(shape, a, stream);
}

}  // namespace som
