// C ABI of what the dense layer is trained by and served with (declared in include/som.h):
// blocks of 8 bits and their product, cross entropy, orthogonalised updates.
#include <cmath>

#include "api_dense.h"
#include "cross_entropy.h"
#include "orthogonalise.h"
#include "product_blocks.h"

namespace {

using namespace som::api;

constexpr int64_t kBlock = 128;

int64_t blocks(int64_t n) { return (n + kBlock - 1) / kBlock; }

// Factors [rows][cols] of an output, at strides that keep them apart.
som_status check_scale_out(const float* p, int64_t rows, int64_t cols, int64_t row, int64_t col) {
  if (!p) return fail(SOM_ERR_INVALID_ARG, "scale is NULL");
  SOM_CHECK(check_vector("scale", p));
  if (row < 1 || col < 1 || row > kMaxLd || col > kMaxLd)
    return fail(SOM_ERR_INVALID_ARG, "scale's strides must be in [1, 2^40]");
  if (row / cols < col && col / rows < row && rows > 1 && cols > 1)
    return fail(SOM_ERR_INVALID_ARG, "scale's strides make its entries overlap");
  if (row > (int64_t(1) << 58) / rows || col > (int64_t(1) << 58) / cols)
    return fail(SOM_ERR_INVALID_ARG, "scale exceeds the addressable range");
  return SOM_OK;
}

bool is_half(int32_t t) { return t == SOM_F16 || t == SOM_BF16; }

// A vector that has to be there.
som_status need_vector(const char* name, const void* p) {
  if (!p) return fail(SOM_ERR_INVALID_ARG, std::string(name) + " is NULL");
  if (!aligned(p, 4)) return fail(SOM_ERR_INVALID_ARG, std::string(name) + " must be 4-byte aligned");
  return SOM_OK;
}

som_status check_scores(int32_t w_units, int32_t dtype, int64_t M, int64_t N, int64_t K, float alpha) {
  if (!is_half(dtype)) return fail(SOM_ERR_INVALID_ARG, "dtype must be SOM_F16 or SOM_BF16");
  if (w_units != 0 && w_units != 1) return fail(SOM_ERR_INVALID_ARG, "w_units must be 0 or 1");
  SOM_CHECK(check_sizes(M, N, K));
  if (!std::isfinite(alpha)) return fail(SOM_ERR_INVALID_ARG, "alpha must be finite");
  if (!launchable(M, N)) return fail(SOM_ERR_INVALID_ARG, "M * N is too large for one call");
  return SOM_OK;
}

// Factors [rows / s->rows][k / 128] of an operand.
som_status check_scale(const char* name, const som_block_scale* s, int64_t rows, int64_t k) {
  const std::string n(name);
  if (!s) return fail(SOM_ERR_INVALID_ARG, n + " is NULL");
  if (s->rows != 1 && s->rows != kBlock) return fail(SOM_ERR_INVALID_ARG, n + ": rows must be 1 or 128");
  if (s->reserved != 0) return fail(SOM_ERR_INVALID_ARG, n + ": reserved must be 0");
  if (!s->p) return fail(SOM_ERR_INVALID_ARG, n + ": p is NULL");
  SOM_CHECK(check_vector(name, s->p));
  const int64_t r = s->rows == 1 ? rows : blocks(rows);
  if (s->row_stride < 0 || s->block_stride < 0 || s->row_stride > (int64_t(1) << 58) / r ||
      s->block_stride > (int64_t(1) << 58) / blocks(k))
    return fail(SOM_ERR_INVALID_ARG, n + ": the strides must be >= 0, and its entries addressable");
  return SOM_OK;
}

constexpr int64_t kMaxSide = int64_t(1) << 24, kMaxShort = int64_t(1) << 15;

bool ortho_sizes(int64_t rows, int64_t cols) {
  return rows >= 1 && cols >= 1 && rows <= kMaxSide && cols <= kMaxSide && (rows <= kMaxShort || cols <= kMaxShort) &&
         launchable(rows, cols);
}

}  // namespace

extern "C" {

size_t som_cross_entropy_workspace_bytes(int64_t M, int64_t N, int64_t K, int32_t dtype) {
  if (M < 1 || M > kI32Max || N < 1 || N > kMaxK || K < 1 || K > kMaxK || !is_half(dtype)) return 0;
  return som::loss_ws(M, N, K, dtype).total;
}

som_status som_cross_entropy(const void* x, int64_t ldx, const void* W, int64_t ldw, int32_t w_units, int32_t dtype,
                             int64_t M, int64_t N, int64_t K, const int32_t* labels, const float* bias, float alpha,
                             float* loss, float* lse, void* ws, size_t ws_bytes, hipStream_t stream) {
  SOM_CHECK(check_scores(w_units, dtype, M, N, K, alpha));
  if (M == 0) return ok();
  SOM_CHECK(check_matrix("x", x, ldx, M, K, dtype));
  SOM_CHECK(check_matrix("W", W, ldw, w_units ? N : K, w_units ? K : N, dtype));
  SOM_CHECK(need_vector("labels", labels));
  SOM_CHECK(check_vector("bias", bias));
  SOM_CHECK(need_vector("loss", loss));
  SOM_CHECK(need_vector("lse", lse));
  SOM_CHECK(check_ws(ws, ws_bytes, som_cross_entropy_workspace_bytes(M, N, K, dtype)));
  som::LossCall c{};
  c.x = x;
  c.ldx = ldx;
  c.W = W;
  c.ldw = ldw;
  c.units = w_units != 0;
  c.dtype = dtype;
  c.M = M;
  c.N = N;
  c.K = K;
  c.labels = labels;
  c.bias = bias;
  c.alpha = alpha;
  c.loss = loss;
  c.lse = lse;
  const hipError_t e = som::launch_loss(c, ws, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "cross entropy launch");
}

size_t som_cross_entropy_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, int32_t dtype) {
  if (M < 1 || M > kMaxK || N < 1 || N > kMaxK || K < 1 || K > kMaxK || !is_half(dtype)) return 0;
  return som::grad_ws(M, N, K, dtype).total;
}

som_status som_cross_entropy_backward(const float* dloss, const void* x, int64_t ldx, const void* W, int64_t ldw,
                                      int32_t w_units, int32_t dtype, int64_t M, int64_t N, int64_t K,
                                      const int32_t* labels, const float* bias, float alpha, const float* lse, void* dx,
                                      int64_t lddx, void* dW, int64_t lddw, float* dbias, void* ws, size_t ws_bytes,
                                      hipStream_t stream) {
  SOM_CHECK(check_scores(w_units, dtype, M, N, K, alpha));
  if (M > kMaxK) return fail(SOM_ERR_INVALID_ARG, "M must be in [0, 2^30]");
  if (!launchable(M, K) || !launchable(K, N) || !launchable(N, K))
    return fail(SOM_ERR_INVALID_ARG, "a product is too large for one call");
  const int64_t wr = w_units ? N : K, wc = w_units ? K : N;
  if (dW) SOM_CHECK(check_matrix("dW", dW, lddw, wr, wc, dtype));
  SOM_CHECK(check_vector("dbias", dbias));
  if (M == 0) {
    hipError_t e = hipSuccess;
    if (dW) e = som::launch_zero(dW, lddw * 2, wr, wc * 2, stream);
    if (e == hipSuccess && dbias) e = som::launch_zero(dbias, 0, 1, N * 4, stream);
    return e == hipSuccess ? ok() : hip_fail(e, "zero launch");
  }
  SOM_CHECK(need_vector("dloss", dloss));
  SOM_CHECK(check_matrix("x", x, ldx, M, K, dtype));
  SOM_CHECK(check_matrix("W", W, ldw, wr, wc, dtype));
  SOM_CHECK(need_vector("labels", labels));
  SOM_CHECK(check_vector("bias", bias));
  SOM_CHECK(need_vector("lse", lse));
  if (dx) SOM_CHECK(check_matrix("dx", dx, lddx, M, K, dtype));
  if (!dx && !dW && !dbias) return ok();
  SOM_CHECK(check_ws(ws, ws_bytes, som_cross_entropy_backward_workspace_bytes(M, N, K, dtype)));
  som::GradCall c{};
  c.dloss = dloss;
  c.x = x;
  c.ldx = ldx;
  c.W = W;
  c.ldw = ldw;
  c.units = w_units != 0;
  c.dtype = dtype;
  c.M = M;
  c.N = N;
  c.K = K;
  c.labels = labels;
  c.bias = bias;
  c.alpha = alpha;
  c.lse = lse;
  c.dx = dx;
  c.lddx = lddx;
  c.dW = dW;
  c.lddw = lddw;
  c.dbias = dbias;
  const hipError_t e = som::launch_loss_back(c, ws, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "cross entropy gradient launch");
}

som_status som_quantise(const void* x, int64_t ldx, int32_t dtype, int64_t rows, int64_t cols, int32_t block_rows,
                        int32_t transpose, void* q, int64_t ldq, float* scale, int64_t scale_row,
                        int64_t scale_block, hipStream_t stream) {
  if (!is_float(dtype)) return fail(SOM_ERR_INVALID_ARG, "dtype must be SOM_F32, SOM_F16 or SOM_BF16");
  SOM_CHECK(check_rows(rows, cols));
  if (block_rows != 1 && block_rows != kBlock) return fail(SOM_ERR_INVALID_ARG, "block_rows must be 1 or 128");
  if (transpose != 0 && transpose != 1) return fail(SOM_ERR_INVALID_ARG, "transpose must be 0 or 1");
  if (rows == 0) return ok();
  const int64_t qr = transpose ? cols : rows, qc = transpose ? rows : cols;
  SOM_CHECK(check_matrix("x", x, ldx, rows, cols, dtype));
  SOM_CHECK(check_matrix("q", q, ldq, qr, qc, SOM_E4M3));
  SOM_CHECK(check_scale_out(scale, block_rows == 1 ? qr : blocks(qr), blocks(qc), scale_row, scale_block));
  som::QuantiseArgs a{};
  a.x = x;
  a.q = static_cast<uint8_t*>(q);
  a.scale = scale;
  a.ldx = ldx;
  a.ldq = ldq;
  a.rows = rows;
  a.cols = cols;
  a.scale_row = scale_row;
  a.scale_block = scale_block;
  a.dtype = dtype;
  a.block_rows = block_rows;
  a.transpose = transpose != 0;
  const hipError_t e = som::launch_quantise(a, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "quantise launch");
}

size_t som_product_blocks_workspace_bytes(int64_t M, int64_t N, int64_t K, int32_t y_dtype) {
  if (M < 1 || M > kI32Max || N < 1 || N > kMaxK || K < 1 || K > kMaxK || !is_float(y_dtype)) return 0;
  const bool exact = y_dtype == SOM_F32;
  const size_t on = som::plan_blocks(M, N, K, true, exact).partial_floats;
  const size_t off = som::plan_blocks(M, N, K, false, exact).partial_floats;
  return som::align_up(sizeof(float) * (on > off ? on : off), 256);
}

som_status som_product_blocks(const void* x, int64_t ldx, const som_block_scale* x_scale, const void* W, int64_t ldw,
                              const som_block_scale* w_scale, int64_t M, int64_t N, int64_t K, void* y, int64_t ldy,
                              int32_t y_dtype, const som_epilogue* e, void* ws, size_t ws_bytes, hipStream_t stream) {
  const som_epilogue plain = {SOM_ACT_NONE, 0, 1.0f, nullptr, nullptr, nullptr, nullptr, 0, nullptr, 0};
  if (!e) e = &plain;
  if (!is_float(y_dtype)) return fail(SOM_ERR_INVALID_ARG, "y_dtype must be SOM_F32, SOM_F16 or SOM_BF16");
  SOM_CHECK(check_sizes(M, N, K));
  if (e->act < SOM_ACT_NONE || e->act > SOM_ACT_SILU) return fail(SOM_ERR_INVALID_ARG, "unknown activation");
  if (e->reserved != 0) return fail(SOM_ERR_INVALID_ARG, "reserved must be 0");
  if (e->x_scale || e->w_scale) return fail(SOM_ERR_INVALID_ARG, "the epilogue's x_scale and w_scale must be NULL: the factors are the blocks'");
  if (!launchable(M, N)) return fail(SOM_ERR_INVALID_ARG, "M * N is too large for one call");
  if (M == 0) return ok();
  SOM_CHECK(check_matrix("x", x, ldx, M, K, SOM_E4M3));
  SOM_CHECK(check_matrix("W", W, ldw, N, K, SOM_E4M3));
  SOM_CHECK(check_scale("x_scale", x_scale, M, K));
  SOM_CHECK(check_scale("w_scale", w_scale, N, K));
  SOM_CHECK(check_matrix("y", y, ldy, M, N, y_dtype));
  if (e->residual) SOM_CHECK(check_matrix("residual", e->residual, e->ldr, M, N, y_dtype));
  if (e->pre) SOM_CHECK(check_matrix("pre", e->pre, e->ldp, M, N, y_dtype));
  SOM_CHECK(check_vector("bias", e->bias));
  SOM_CHECK(check_ws(ws, ws_bytes, som_product_blocks_workspace_bytes(M, N, K, y_dtype)));
  som::BlockArgs a{};
  a.P = x;
  a.ldp = ldx;
  a.p_kc = true;
  a.Q = W;
  a.ldq = ldw;
  a.q_kc = true;
  a.I = M;
  a.J = N;
  a.K = K;
  a.elem = SOM_E4M3;
  a.alpha = e->alpha;
  a.act = e->act;
  a.bias = e->bias;
  a.residual = e->residual;
  a.ldr = e->ldr;
  a.pre = e->pre;
  a.ldpre = e->ldp;
  a.out = y;
  a.ldo = ldy;
  a.out_type = y_dtype;
  a.xs = x_scale->p;
  a.xs_row = x_scale->row_stride;
  a.xs_k = x_scale->block_stride;
  a.xs_shift = x_scale->rows == 1 ? 0 : 7;
  a.ws = w_scale->p;
  a.ws_row = w_scale->row_stride;
  a.ws_k = w_scale->block_stride;
  a.ws_shift = w_scale->rows == 1 ? 0 : 7;
  a.exact = y_dtype == SOM_F32;
  const hipError_t err = som::launch_blocks(a, static_cast<float*>(ws), stream);
  return err == hipSuccess ? ok() : hip_fail(err, "product launch");
}

size_t som_orthogonalise_workspace_bytes(int64_t rows, int64_t cols) {
  return ortho_sizes(rows, cols) ? som::ortho_ws(rows, cols).total : 0;
}

som_status som_orthogonalise(const void* G, int64_t ldg, int32_t dtype, int64_t rows, int64_t cols, int32_t steps,
                             float a, float b, float c, void* y, int64_t ldy, void* ws, size_t ws_bytes,
                             hipStream_t stream) {
  if (!is_float(dtype)) return fail(SOM_ERR_INVALID_ARG, "dtype must be SOM_F32, SOM_F16 or SOM_BF16");
  if (!ortho_sizes(rows, cols))
    return fail(SOM_ERR_INVALID_ARG, "rows and cols must be in [1, 2^24], one of them up to 2^15, and launchable");
  if (steps < 1 || steps > 64) return fail(SOM_ERR_INVALID_ARG, "steps must be in [1, 64]");
  for (const float v : {a, b, c})
    if (!(std::fabs(v) <= 64.0f)) return fail(SOM_ERR_INVALID_ARG, "the coefficients must be in [-64, 64]");
  SOM_CHECK(check_matrix("G", G, ldg, rows, cols, dtype));
  SOM_CHECK(check_matrix("y", y, ldy, rows, cols, SOM_BF16));
  SOM_CHECK(check_ws(ws, ws_bytes, som_orthogonalise_workspace_bytes(rows, cols)));
  som::OrthoCall o{};
  o.G = G;
  o.y = y;
  o.ldg = ldg;
  o.ldy = ldy;
  o.rows = rows;
  o.cols = cols;
  o.dtype = dtype;
  o.steps = steps;
  o.a = a;
  o.b = b;
  o.c = c;
  const hipError_t e = som::launch_orthogonalise(o, ws, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "orthogonalise launch");
}

}  // extern "C"
