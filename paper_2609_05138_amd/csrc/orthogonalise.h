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
  size_t parts, x, half[2], gram, poly, partial, total;
  int64_t rows, ldx, ldm;    // of X and of A, rounded up
};
OrthoWs ortho_ws(int64_t rows, int64_t cols);
hipError_t launch_orthogonalise(const OrthoCall& c, void* ws, hipStream_t stream);

}  // namespace som
