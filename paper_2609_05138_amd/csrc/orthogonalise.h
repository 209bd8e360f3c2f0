// An update orthogonalised by Newton-Schulz steps: call and workspace.
#pragma once

#include "dense.h"

namespace som {

struct OrthoCall {
  const void* G;
  void* y;                   // bf16
  int64_t ldg, ldy, rows, cols;
  int dtype, steps;
  float a, b, c;
};
struct OrthoWs {
  size_t parts, x, half[2], half_t[2], gram, poly, partial, total;
  int64_t rows, cols, short_side;      // rounded up to 64
  int64_t ldx, ldt, ldm;               // strides of X, its transpose, and A
  bool small, low;
};
OrthoWs ortho_ws(int64_t rows, int64_t cols);
hipError_t launch_orthogonalise(const OrthoCall& c, void* ws, hipStream_t stream);

}  // namespace som
