// The instantiations of the product's kernel with epilogues of its own for one element type.
#pragma once

#include "product_launch.h"
#include "product_modes.h"

namespace som {

template <int E, int MODE>
hipError_t launch_layout(int shape, const typename ModeArgs<MODE>::type& a, hipStream_t stream) {
  if (a.p_kc)
    return a.q_kc ? launch_shape<E, true, true, MODE>(shape, a, stream) : launch_shape<E, true, false, MODE>(shape, a, stream);
  if constexpr (MODE == kExtra)
    if (!a.q_kc) return launch_shape<E, false, false, MODE>(shape, a, stream);
  return hipErrorInvalidValue;
}

// Square tiles, both operands laid out alike.
template <int E, bool KC, int MODE>
hipError_t launch_square(int shape, const typename ModeArgs<MODE>::type& a, hipStream_t stream) {
  if (shape == kShape256) return launch_one<kShape256, E, KC, KC, MODE, 2, 4, 8, 4, 2>(a, stream);
  if (shape == kShape128) return launch_one<kShape128, E, KC, KC, MODE, 2, 4, 4, 2, 4>(a, stream);
  return hipErrorInvalidValue;
}

// `a` is the mode's arguments.
template <int E>
hipError_t launch_mode_elem(int mode, int shape, const ProductArgs& a, hipStream_t stream) {
  if (mode == kExtra) return launch_layout<E, kExtra>(shape, static_cast<const ModeArgs<kExtra>::type&>(a), stream);
  if (mode == kLoss) return launch_layout<E, kLoss>(shape, static_cast<const ModeArgs<kLoss>::type&>(a), stream);
  if (mode == kGradFew) return launch_layout<E, kGradFew>(shape, static_cast<const ModeArgs<kGradFew>::type&>(a), stream);
  return launch_layout<E, kGrad>(shape, static_cast<const ModeArgs<kGrad>::type&>(a), stream);
}

}  // namespace som
