// The instantiations of the product's kernel for one element type.
#pragma once

#include "product.h"

namespace som {

template <int SHAPE, int E, bool PKC, bool QKC, int WI, int WJ, int TI, int TJ, int NS>
hipError_t launch_one(const ProductArgs& a, hipStream_t stream) {
  static_assert(kInfo[SHAPE].bi == WI * TI * 16 && kInfo[SHAPE].bj == WJ * TJ * 16, "the grid is laid out for these tiles");
  constexpr size_t lds = static_cast<size_t>(NS) * (WI * TI + WJ * TJ) * 16 * kStepBytes;
  if constexpr (lds > 64 * 1024) {
    const hipError_t e = allow_lds(k_product<E, PKC, QKC, WI, WJ, TI, TJ, NS>, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_product<E, PKC, QKC, WI, WJ, TI, TJ, NS>), dim3(a.per_xcd * kXcds), dim3(WI * WJ * 64), lds,
                     stream, a);
  return hipGetLastError();
}

template <int E, bool PKC, bool QKC>
hipError_t launch_shape(int shape, const ProductArgs& a, hipStream_t stream) {
  switch (shape) {
    case kShape256:
      return launch_one<kShape256, E, PKC, QKC, 2, 4, 8, 4, 2>(a, stream);
    case kShape256x128:
      return launch_one<kShape256x128, E, PKC, QKC, 4, 2, 4, 4, 3>(a, stream);
    case kShape128:
      return launch_one<kShape128, E, PKC, QKC, 2, 4, 4, 2, 4>(a, stream);
    case kShape64:
      return launch_one<kShape64, E, PKC, QKC, 2, 4, 2, 2, 3>(a, stream);
    default:
      // few rows: their operand has k contiguous in every product that has few
      if constexpr (PKC)
        return shape == kShape32 ? launch_one<kShape32, E, PKC, QKC, 1, 4, 2, 2, 4>(a, stream)
                                 : launch_one<kShape16, E, PKC, QKC, 1, 4, 1, 2, 4>(a, stream);
      else
        return hipErrorInvalidValue;
  }
}

template <int E>
hipError_t launch_elem(int shape, const ProductArgs& a, hipStream_t stream) {
  if constexpr (E == kE4M3) {
    if (a.p_kc && a.q_kc) return launch_shape<E, true, true>(shape, a, stream);
  } else {
    if (a.p_kc) return a.q_kc ? launch_shape<E, true, true>(shape, a, stream) : launch_shape<E, true, false>(shape, a, stream);
    if (!a.q_kc) return launch_shape<E, false, false>(shape, a, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace som
