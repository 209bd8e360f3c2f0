// Softmax cross entropy of rows against a matrix product's columns: calls and workspaces.
#pragma once

#include "dense.h"

namespace som {

struct LossCall {
  const void *x, *W;
  const int32_t* labels;
  const float* bias;
  float *loss, *lse;
  int64_t ldx, ldw, M, N, K;
  int dtype;
  bool units;
  float alpha;
};
struct LossWs {
  size_t label_score, part, scores, total;
};
LossWs loss_ws(int64_t M, int64_t N, int64_t K, int elem);
hipError_t launch_loss(const LossCall& c, void* ws, hipStream_t stream);

struct GradCall {
  const void *x, *W;
  const int32_t* labels;
  const float *bias, *lse, *dloss;
  void *dx, *dW;             // each may be nullptr
  float* dbias;
  int64_t ldx, ldw, lddx, lddw, M, N, K;
  int dtype;
  bool units;
  float alpha;
};
// `clean`, `dx`: M rows of ldx; `g`: M rows of ldg, a piece of the classes
struct GradWs {
  size_t head, g, clean, dx, column, common, lost, flags, lost_part, rest, partial, total;
  bool few;                  // what rounding takes from labels' entries is kept in `rest`
  int64_t piece, ldg, ldx, ld_column;
};
GradWs grad_ws(int64_t M, int64_t N, int64_t K, int elem);
hipError_t launch_loss_back(const GradCall& c, void* ws, hipStream_t stream);

}  // namespace som
