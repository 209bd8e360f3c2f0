// The matrix product's kernels for 8-bit (E4M3) operands.
#include "product_launch.h"

namespace som {

hipError_t launch_product_e4m3(int shape, const ProductArgs& a, hipStream_t stream) {
  return launch_elem<kE4M3>(shape, a, stream);
}

}  // namespace som
