// C ABI of the dense-document operators (declared in include/som.h): argument
// checks, workspace carving and launches.
#include <cmath>

#include "api_common.h"
#include "product.h"

namespace {

using namespace som::api;

static_assert(som::kF32 == SOM_F32 && som::kF16 == SOM_F16 && som::kBF16 == SOM_BF16 && som::kE4M3 == SOM_E4M3,
              "element types");
static_assert(som::kActNone == SOM_ACT_NONE && som::kActRelu == SOM_ACT_RELU && som::kActGelu == SOM_ACT_GELU &&
                  som::kActGeluTanh == SOM_ACT_GELU_TANH && som::kActSilu == SOM_ACT_SILU,
              "activations");

constexpr int64_t kMaxK = int64_t(1) << 30;       // a step past the end stays an int32
constexpr int64_t kMaxLd = int64_t(1) << 40;      // row offsets stay inside 64-bit bytes
constexpr int64_t kMaxTiles = (int64_t(1) << 23) - 8;   // of 512 threads, under a launch's 2^32

bool is_float(int32_t t) { return t == SOM_F32 || t == SOM_F16 || t == SOM_BF16; }

// A [rows][ld] matrix of `cols` columns: present, strided and aligned as its type
// needs, and its last byte within 2^62.
som_status check_matrix(const char* name, const void* p, int64_t ld, int64_t rows, int64_t cols, int32_t dtype) {
  const std::string n(name);
  if (!p) return fail(SOM_ERR_INVALID_ARG, n + " is NULL");
  if (ld < cols || ld > kMaxLd) return fail(SOM_ERR_INVALID_ARG, n + ": the row stride must be in [columns, 2^40]");
  if (rows > 0 && ld > (int64_t(1) << 60) / rows) return fail(SOM_ERR_INVALID_ARG, n + " exceeds the addressable range");
  if (!aligned(p, som::dtype_bytes(dtype))) return fail(SOM_ERR_INVALID_ARG, n + " must be aligned to its elements");
  return SOM_OK;
}

som_status check_vector(const char* name, const float* p) {
  if (p && !aligned(p, 4)) return fail(SOM_ERR_INVALID_ARG, std::string(name) + " must be 4-byte aligned");
  return SOM_OK;
}

som_status check_ws(const void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return SOM_OK;
  if (!ws) return fail(SOM_ERR_WORKSPACE, "ws is NULL: need " + std::to_string(need) + " bytes");
  if (!aligned(ws, 256)) return fail(SOM_ERR_INVALID_ARG, "ws must be 256-byte aligned");
  if (ws_bytes < need)
    return fail(SOM_ERR_WORKSPACE, "workspace too small: need " + std::to_string(need) + " bytes");
  return SOM_OK;
}

som_status check_rows(int64_t rows, int64_t cols) {
  if (rows < 0 || rows > kI32Max) return fail(SOM_ERR_INVALID_ARG, "rows must be in [0, 2^31)");
  if (cols < 1 || cols > kI32Max) return fail(SOM_ERR_INVALID_ARG, "cols must be in [1, 2^31)");
  return SOM_OK;
}

som_status check_sizes(int64_t M, int64_t N, int64_t K) {
  if (M < 0 || M > kI32Max) return fail(SOM_ERR_INVALID_ARG, "M must be in [0, 2^31)");
  if (N < 1 || N > kMaxK) return fail(SOM_ERR_INVALID_ARG, "N must be in [1, 2^30]");
  if (K < 1 || K > kMaxK) return fail(SOM_ERR_INVALID_ARG, "K must be in [1, 2^30]");
  return SOM_OK;
}

// Workgroups of C [I][J]: 256 x 256, or up to 64 rows by 128 columns (then of a strip).
// Smaller tiles and splits are for launches of a few thousand.
bool launchable(int64_t I, int64_t J) { return (I + 255) / 256 <= kMaxTiles / ((J + 127) / 128); }

#define SOM_CHECK(call)                 \
  do {                                  \
    const som_status s_ = (call);       \
    if (s_ != SOM_OK) return s_;        \
  } while (0)

}  // namespace

extern "C" {

som_status som_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight,
                        int32_t dtype, int64_t rows, int64_t cols, float eps, int32_t q8, void* y, int64_t ldy,
                        void* h, int64_t ldh, float* scale, hipStream_t stream) {
  if (!is_float(dtype)) return fail(SOM_ERR_INVALID_ARG, "dtype must be SOM_F32, SOM_F16 or SOM_BF16");
  SOM_CHECK(check_rows(rows, cols));
  if (!(eps >= 0) || !std::isfinite(eps)) return fail(SOM_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (q8 != 0 && q8 != 1) return fail(SOM_ERR_INVALID_ARG, "q8 must be 0 or 1");
  if (rows == 0) return ok();
  SOM_CHECK(check_matrix("x", x, ldx, rows, cols, dtype));
  if (residual) SOM_CHECK(check_matrix("residual", residual, ldr, rows, cols, dtype));
  if (weight && !aligned(weight, som::dtype_bytes(dtype)))
    return fail(SOM_ERR_INVALID_ARG, "weight must be aligned to its elements");
  SOM_CHECK(check_matrix("y", y, ldy, rows, cols, q8 ? SOM_E4M3 : dtype));
  if (h) SOM_CHECK(check_matrix("h", h, ldh, rows, cols, dtype));
  if (q8 ? !scale : scale != nullptr) return fail(SOM_ERR_INVALID_ARG, "scale goes with an output in 8 bits");
  SOM_CHECK(check_vector("scale", scale));
  som::RmsNormArgs a{};
  a.x = x;
  a.residual = residual;
  a.weight = weight;
  a.y = y;
  a.h = h;
  a.scale = scale;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldy = ldy;
  a.ldh = ldh;
  a.rows = rows;
  a.cols = cols;
  a.dtype = dtype;
  a.q8 = q8 != 0;
  a.eps = eps;
  const hipError_t e = som::launch_rms_norm(a, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "norm launch");
}

size_t som_rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || rows > kI32Max || cols < 1 || cols > kI32Max) return 0;
  if (rows == 0) return 0;
  return som::align_up(sizeof(float) * som::rms_norm_back_ws_floats(rows, cols), 256);
}

som_status som_rms_norm_backward(const void* dy, int64_t lddy, const void* h, int64_t ldh, const void* weight,
                                 const void* dh, int64_t lddh, int32_t dtype, int64_t rows, int64_t cols,
                                 float eps, void* dx, int64_t lddx, float* dweight, void* ws, size_t ws_bytes,
                                 hipStream_t stream) {
  if (!is_float(dtype)) return fail(SOM_ERR_INVALID_ARG, "dtype must be SOM_F32, SOM_F16 or SOM_BF16");
  SOM_CHECK(check_rows(rows, cols));
  if (!(eps >= 0) || !std::isfinite(eps)) return fail(SOM_ERR_INVALID_ARG, "eps must be finite and >= 0");
  SOM_CHECK(check_vector("dweight", dweight));
  if (rows == 0) {
    if (!dweight) return ok();
    const hipError_t e = som::launch_zero(dweight, 0, 1, cols * 4, stream);
    return e == hipSuccess ? ok() : hip_fail(e, "zero launch");
  }
  SOM_CHECK(check_matrix("dy", dy, lddy, rows, cols, dtype));
  SOM_CHECK(check_matrix("h", h, ldh, rows, cols, dtype));
  if (weight && !aligned(weight, som::dtype_bytes(dtype)))
    return fail(SOM_ERR_INVALID_ARG, "weight must be aligned to its elements");
  if (dh) SOM_CHECK(check_matrix("dh", dh, lddh, rows, cols, dtype));
  SOM_CHECK(check_matrix("dx", dx, lddx, rows, cols, dtype));
  SOM_CHECK(check_ws(ws, ws_bytes, som_rms_norm_backward_workspace_bytes(rows, cols)));
  som::RmsNormBackArgs a{};
  a.dy = dy;
  a.h = h;
  a.weight = weight;
  a.dh = dh;
  a.dx = dx;
  a.dweight = dweight;
  a.ws = static_cast<float*>(ws);
  a.lddy = lddy;
  a.ldh = ldh;
  a.lddh = lddh;
  a.lddx = lddx;
  a.rows = rows;
  a.cols = cols;
  a.dtype = dtype;
  a.eps = eps;
  const hipError_t e = som::launch_rms_norm_back(a, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "norm gradient launch");
}

size_t som_product_workspace_bytes(int64_t M, int64_t N, int64_t K, int32_t x_dtype) {
  if (M < 1 || M > kI32Max || N < 1 || N > kMaxK || K < 1 || K > kMaxK || x_dtype < SOM_F16 || x_dtype > SOM_E4M3)
    return 0;
  // rows on 16 bytes or not; unit-major weights take the same shapes, or need nothing
  const size_t on = som::plan_product(M, N, K, x_dtype, true, false, true).partial_floats;
  const size_t off = som::plan_product(M, N, K, x_dtype, true, false, false).partial_floats;
  const size_t most = on > off ? on : off;
  return som::align_up(sizeof(float) * most, 256);
}

som_status som_product(const void* x, int64_t ldx, const void* W, int64_t ldw, int32_t w_units, int32_t x_dtype,
                       int64_t M, int64_t N, int64_t K, void* y, int64_t ldy, int32_t y_dtype,
                       const som_epilogue* e, void* ws, size_t ws_bytes, hipStream_t stream) {
  const som_epilogue plain = {SOM_ACT_NONE, 0, 1.0f, nullptr, nullptr, nullptr, nullptr, 0, nullptr, 0};
  if (!e) e = &plain;
  if (x_dtype != SOM_F16 && x_dtype != SOM_BF16 && x_dtype != SOM_E4M3)
    return fail(SOM_ERR_INVALID_ARG, "x_dtype must be SOM_F16, SOM_BF16 or SOM_E4M3");
  if (!is_float(y_dtype) || (x_dtype != SOM_E4M3 && y_dtype != SOM_F32 && y_dtype != x_dtype))
    return fail(SOM_ERR_INVALID_ARG, "y_dtype must be x's type or SOM_F32 (8-bit x: SOM_F32, SOM_F16 or SOM_BF16)");
  if (w_units != 0 && w_units != 1) return fail(SOM_ERR_INVALID_ARG, "w_units must be 0 or 1");
  if (x_dtype == SOM_E4M3 && !w_units) return fail(SOM_ERR_INVALID_ARG, "8-bit weights must be unit-major");
  SOM_CHECK(check_sizes(M, N, K));
  if (e->act < SOM_ACT_NONE || e->act > SOM_ACT_SILU) return fail(SOM_ERR_INVALID_ARG, "unknown activation");
  if (e->reserved != 0) return fail(SOM_ERR_INVALID_ARG, "reserved must be 0");
  if (!launchable(M, N)) return fail(SOM_ERR_INVALID_ARG, "M * N is too large for one call");
  if (M == 0) return ok();
  SOM_CHECK(check_matrix("x", x, ldx, M, K, x_dtype));
  SOM_CHECK(check_matrix("W", W, ldw, w_units ? N : K, w_units ? K : N, x_dtype));
  SOM_CHECK(check_matrix("y", y, ldy, M, N, y_dtype));
  if (e->residual) SOM_CHECK(check_matrix("residual", e->residual, e->ldr, M, N, y_dtype));
  if (e->pre) SOM_CHECK(check_matrix("pre", e->pre, e->ldp, M, N, y_dtype));
  SOM_CHECK(check_vector("x_scale", e->x_scale));
  SOM_CHECK(check_vector("w_scale", e->w_scale));
  SOM_CHECK(check_vector("bias", e->bias));
  SOM_CHECK(check_ws(ws, ws_bytes, som_product_workspace_bytes(M, N, K, x_dtype)));
  som::ProductArgs a{};
  a.P = x;
  a.ldp = ldx;
  a.p_kc = true;
  a.Q = W;
  a.ldq = ldw;
  a.q_kc = w_units != 0;
  a.I = M;
  a.J = N;
  a.K = K;
  a.elem = x_dtype;
  a.alpha = e->alpha;
  a.act = e->act;
  a.p_scale = e->x_scale;
  a.q_scale = e->w_scale;
  a.bias = e->bias;
  a.residual = e->residual;
  a.ldr = e->ldr;
  a.pre = e->pre;
  a.ldpre = e->ldp;
  a.out = y;
  a.ldo = ldy;
  a.out_type = y_dtype;
  const hipError_t err = som::launch_product(a, static_cast<float*>(ws), stream);
  return err == hipSuccess ? ok() : hip_fail(err, "product launch");
}

// dP, its column sums' parts, and the larger of the two products' partial sums.
struct BackwardWs {
  size_t dp, part, partial, total;
  int64_t lddp;
};

static BackwardWs backward_ws(int64_t M, int64_t N, int64_t K, int32_t dtype) {
  BackwardWs w{};
  w.lddp = static_cast<int64_t>(som::align_up(static_cast<size_t>(N), 8));
  size_t o = som::align_up(static_cast<size_t>(M) * w.lddp * som::dtype_bytes(dtype), 256);
  w.part = o;
  o += som::align_up(sizeof(float) * som::act_grad_ws_floats(M, N), 256);
  w.partial = o;
  size_t most = 0;
  for (const bool dma : {true, false})   // rows on 16 bytes or not; either layout of W
    for (const size_t n : {som::plan_product(M, K, N, dtype, true, false, dma).partial_floats,
                           som::plan_product(K, N, M, dtype, false, false, dma).partial_floats,
                           som::plan_product(N, K, M, dtype, false, false, dma).partial_floats})
      if (n > most) most = n;
  w.total = o + som::align_up(sizeof(float) * most, 256);
  return w;
}

size_t som_product_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, int32_t dtype) {
  if (M < 1 || M > kMaxK || N < 1 || N > kMaxK || K < 1 || K > kMaxK || (dtype != SOM_F16 && dtype != SOM_BF16))
    return 0;
  return backward_ws(M, N, K, dtype).total;
}

som_status som_product_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* W, int64_t ldw,
                                int32_t w_units, int32_t dtype, int64_t M, int64_t N, int64_t K, int32_t act,
                                const void* pre, int64_t ldp, float alpha, void* dx, int64_t lddx, void* dW,
                                int64_t lddw, float* dbias, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (dtype != SOM_F16 && dtype != SOM_BF16) return fail(SOM_ERR_INVALID_ARG, "dtype must be SOM_F16 or SOM_BF16");
  if (w_units != 0 && w_units != 1) return fail(SOM_ERR_INVALID_ARG, "w_units must be 0 or 1");
  SOM_CHECK(check_sizes(M, N, K));
  if (M > kMaxK) return fail(SOM_ERR_INVALID_ARG, "M must be in [0, 2^30]");
  if (act < SOM_ACT_NONE || act > SOM_ACT_SILU) return fail(SOM_ERR_INVALID_ARG, "unknown activation");
  if (!launchable(M, K) || !launchable(K, N) || !launchable(N, K)) return fail(SOM_ERR_INVALID_ARG, "a product is too large for one call");
  const int64_t wr = w_units ? N : K, wc = w_units ? K : N;
  if (dW) SOM_CHECK(check_matrix("dW", dW, lddw, wr, wc, dtype));
  SOM_CHECK(check_vector("dbias", dbias));
  if (M == 0) {
    hipError_t e = hipSuccess;
    const int64_t es = som::dtype_bytes(dtype);
    if (dW) e = som::launch_zero(dW, lddw * es, wr, wc * es, stream);
    if (e == hipSuccess && dbias) e = som::launch_zero(dbias, 0, 1, N * 4, stream);
    return e == hipSuccess ? ok() : hip_fail(e, "zero launch");
  }
  SOM_CHECK(check_matrix("dy", dy, lddy, M, N, dtype));
  if (act != SOM_ACT_NONE) SOM_CHECK(check_matrix("pre", pre, ldp, M, N, dtype));
  if (dx) {
    SOM_CHECK(check_matrix("W", W, ldw, wr, wc, dtype));
    SOM_CHECK(check_matrix("dx", dx, lddx, M, K, dtype));
  }
  if (dW) SOM_CHECK(check_matrix("x", x, ldx, M, K, dtype));
  const BackwardWs w = backward_ws(M, N, K, dtype);
  SOM_CHECK(check_ws(ws, ws_bytes, w.total));

  // dP is rounded to x's type because the matrix cores take 16 bits: an fp32 dP would be two
  // products each (dx is 1.4 times as far from 64 bits so).  Its column sums are not.
  const bool rounded = act != SOM_ACT_NONE && (dx || dW);
  if (rounded || dbias) {
    som::ActGradArgs g{};
    g.dy = dy;
    g.lddy = lddy;
    g.pre = pre;
    g.ldpre = ldp;
    g.dp = rounded ? at<void>(ws, w.dp) : nullptr;
    g.lddp = w.lddp;
    g.dbias = dbias;
    g.part = at<float>(ws, w.part);
    g.M = M;
    g.N = N;
    g.elem = dtype;
    g.act = act;
    const hipError_t e = som::launch_act_grad(g, stream);
    if (e != hipSuccess) return hip_fail(e, "activation gradient launch");
  }
  const void* dp = rounded ? at<void>(ws, w.dp) : dy;
  const int64_t lddp = rounded ? w.lddp : lddy;
  som::ProductArgs a{};
  a.elem = dtype;
  a.alpha = alpha;
  a.act = SOM_ACT_NONE;
  a.out_type = dtype;
  if (dx) {
    a.P = dp;
    a.ldp = lddp;
    a.p_kc = true;
    a.Q = W;
    a.ldq = ldw;
    a.q_kc = !w_units;
    a.I = M;
    a.J = K;
    a.K = N;
    a.out = dx;
    a.ldo = lddx;
    const hipError_t e = som::launch_product(a, at<float>(ws, w.partial), stream);
    if (e != hipSuccess) return hip_fail(e, "product launch (dx)");
  }
  if (dW) {
    a.P = w_units ? dp : x;
    a.ldp = w_units ? lddp : ldx;
    a.p_kc = false;
    a.Q = w_units ? x : dp;
    a.ldq = w_units ? ldx : lddp;
    a.q_kc = false;
    a.I = wr;
    a.J = wc;
    a.K = M;
    a.out = dW;
    a.ldo = lddw;
    const hipError_t e = som::launch_product(a, at<float>(ws, w.partial), stream);
    if (e != hipSuccess) return hip_fail(e, "product launch (dW)");
  }
  return ok();
}

som_status som_dropout(const void* x, int64_t ldx, const void* residual, int64_t ldr, int32_t dtype, int64_t rows,
                       int64_t cols, double p, uint64_t seed, uint64_t offset, void* y, int64_t ldy,
                       hipStream_t stream) {
  if (!is_float(dtype)) return fail(SOM_ERR_INVALID_ARG, "dtype must be SOM_F32, SOM_F16 or SOM_BF16");
  if (rows < 0 || rows > 4294967295ll) return fail(SOM_ERR_INVALID_ARG, "rows must be in [0, 2^32)");
  if (cols < 1 || cols > kI32Max) return fail(SOM_ERR_INVALID_ARG, "cols must be in [1, 2^31)");
  if (!(p >= 0.0 && p <= 1.0)) return fail(SOM_ERR_INVALID_ARG, "p must be in [0, 1]");
  if (rows == 0) return ok();
  SOM_CHECK(check_matrix("x", x, ldx, rows, cols, dtype));
  if (residual) SOM_CHECK(check_matrix("residual", residual, ldr, rows, cols, dtype));
  SOM_CHECK(check_matrix("y", y, ldy, rows, cols, dtype));
  som::DropoutArgs a{};
  a.x = x;
  a.residual = residual;
  a.y = y;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldy = ldy;
  a.rows = rows;
  a.cols = cols;
  a.dtype = dtype;
  a.threshold = static_cast<uint32_t>(std::nearbyint(p * 65536.0));
  a.seed = seed;
  a.offset = offset;
  const hipError_t e = som::launch_dropout(a, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "dropout launch");
}

}  // extern "C"
