// An update orthogonalised by Newton-Schulz steps, of the shorter side m against the longer n:
//
//   X = G / |G|;  each step  A = X X^T,  B = b A + c A A,  X = a X + B X
//
// (a tall G without being transposed: A = X^T X, X = a X + X B).  Three products a step on the
// fp16 matrix cores, each with the polynomial's terms in its epilogue.
//
// What is rounded: X is kept in fp32, which the term a X takes as it is; the products take X, A and
// B in fp16, whose 11 bits and not bf16's 8 are what the steps, which amplify small directions 3.4
// times each, leave as errors: 1e-3 to 2e-3 of the result (2-norm; half of what bf16's rounding of y
// adds), with bf16 between the steps 1e-2, with X in fp16 too 5e-3 where singular values spread
// over 10^4.  X's fp16 copy is scaled by a power of two that makes its elements' size about 1,
// since they are 1 / sqrt(m n) of the norm and would lie among fp16's subnormal numbers.
// The norm is summed in fp64, so no gradient is too small or large for its squares.
//
// X lies in rows and columns rounded up to 64 (a step of the product), with zeros, which stay
// zeros: no product but the last, whose result is y, has a partial step or column.
//
// Bound: the matrix cores for sides of 2,048 and more; else 3 launches a step.
#include "orthogonalise.h"

#include <cmath>

#include "product_modes.h"

namespace som {
namespace {

constexpr int kParts = 512;            // sums of squares, one a workgroup

// Sum over the workgroup's 256 threads, in a fixed order.
__device__ __forceinline__ double sum256(double v, double* part) {
#pragma unroll
  for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  return part[0] + part[1] + part[2] + part[3];
}

// Groups of eight columns, dealt to the workgroups in turn.
template <typename T>
__global__ void __launch_bounds__(256) k_ortho_squares(const T* G, int64_t ldg, int64_t rows, int64_t cols,
                                                       double* parts) {
  __shared__ double part[4];
  const int64_t groups = (cols + 7) / 8, all = groups * rows;
  double s = 0.0;
  for (int64_t g = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; g < all; g += int64_t(gridDim.x) * 256) {
    const int64_t row = g / groups, col = (g - row * groups) * 8;
    float v[8];
    load8(G + row * ldg + col, cols - col >= 8 ? 8 : static_cast<int>(cols - col), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fma(static_cast<double>(v[e]), static_cast<double>(v[e]), s);
  }
  s = sum256(s, part);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// X and its fp16 copy, [all_rows][ldx], zeros beyond G.
template <typename T>
__global__ void __launch_bounds__(256) k_ortho_start(const T* G, int64_t ldg, int64_t rows, int64_t cols,
                                                     const double* parts, int nparts, float* X, f16* half,
                                                     int64_t all_rows, int64_t ldx, float scale) {
  __shared__ double part[4];
  double s = 0.0;
  for (int p = threadIdx.x; p < nparts; p += 256) s += parts[p];
  s = sum256(s, part);
  const double inverse = s == 0.0 ? 0.0 : 1.0 / sqrt(s);
  const int64_t groups = ldx / 8, all = groups * all_rows;
  for (int64_t g = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; g < all; g += int64_t(gridDim.x) * 256) {
    const int64_t row = g / groups, col = (g - row * groups) * 8;
    float v[8];
    const int n = row >= rows || col >= cols ? 0 : cols - col >= 8 ? 8 : static_cast<int>(cols - col);
    load8(G + row * ldg + col, n, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? static_cast<float>(v[e] * inverse) : 0.0f;
    store8(X + row * ldx + col, 8, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= scale;
    store8(half + row * ldx + col, 8, v);
  }
}

int64_t round64(int64_t n) { return (n + 63) / 64 * 64; }

template <typename P>
P* at(void* base, size_t off) {
  return reinterpret_cast<P*>(static_cast<char*>(base) + off);
}

int norm_groups(int64_t rows, int64_t cols) {
  const int64_t g = ((cols + 7) / 8 * rows + 255) / 256;
  return static_cast<int>(g < kParts ? g : kParts);
}

// The three products of a step, without their places; rows and cols are rounded up.
struct Step {
  ExtraArgs gram, poly, update;
};
Step step_of(int64_t rows, int64_t cols, bool tall) {
  const int64_t m = tall ? cols : rows, n = tall ? rows : cols;
  Step s{};
  for (ExtraArgs* p : {&s.gram, &s.poly, &s.update}) {
    p->elem = kF16;
    p->alpha = 1.0f;
    p->out_type = kF16;
  }
  s.gram.I = s.gram.J = s.poly.I = s.poly.J = s.poly.K = m;
  s.gram.K = n;
  s.gram.p_kc = s.gram.q_kc = !tall;
  s.poly.p_kc = s.poly.q_kc = true;            // A and B are symmetric
  s.update.I = rows;
  s.update.J = cols;
  s.update.K = m;
  s.update.p_kc = true;
  s.update.q_kc = tall;
  return s;
}

size_t partial_floats(const ExtraArgs& a) {
  return plan_extra(a.I, a.J, a.K, a.elem, a.p_kc, a.q_kc, true).partial_floats;
}

}  // namespace

OrthoWs ortho_ws(int64_t rows, int64_t cols) {
  OrthoWs w{};
  const bool tall = rows > cols;
  w.rows = round64(rows);
  w.ldx = round64(cols);
  w.ldm = tall ? w.ldx : w.rows;
  size_t o = sizeof(double) * kParts;
  w.x = o;
  o += align_up(sizeof(float) * w.rows * w.ldx, 256);
  for (size_t& h : w.half) {
    h = o;
    o += align_up(2 * w.rows * w.ldx, 256);
  }
  for (size_t* g : {&w.gram, &w.poly}) {
    *g = o;
    o += align_up(2 * w.ldm * w.ldm, 256);
  }
  w.partial = o;
  const Step s = step_of(w.rows, w.ldx, tall);
  size_t need = 0;
  for (const ExtraArgs* p : {&s.gram, &s.poly, &s.update}) {
    const size_t f = partial_floats(*p);
    if (f > need) need = f;
  }
  ExtraArgs last = s.update;           // of y's own rows and columns
  last.I = rows;
  last.J = cols;
  const size_t f = partial_floats(last);
  w.total = o + align_up(sizeof(float) * (f > need ? f : need), 256);
  return w;
}

template <typename T>
static hipError_t start(const OrthoCall& c, const OrthoWs& w, float scale, void* ws, hipStream_t stream) {
  const int groups = norm_groups(c.rows, c.cols);
  hipLaunchKernelGGL(k_ortho_squares<T>, dim3(groups), dim3(256), 0, stream, static_cast<const T*>(c.G), c.ldg, c.rows,
                     c.cols, at<double>(ws, w.parts));
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t all = (w.ldx / 8 * w.rows + 255) / 256;
  hipLaunchKernelGGL(k_ortho_start<T>, dim3(static_cast<uint32_t>(all < 2048 ? all : 2048)), dim3(256), 0, stream,
                     static_cast<const T*>(c.G), c.ldg, c.rows, c.cols, at<double>(ws, w.parts), groups,
                     at<float>(ws, w.x), at<f16>(ws, w.half[0]), w.rows, w.ldx, scale);
  return hipGetLastError();
}

hipError_t launch_orthogonalise(const OrthoCall& c, void* ws, hipStream_t stream) {
  const OrthoWs w = ortho_ws(c.rows, c.cols);
  // |X| stays below 4: fp16's largest value is 65,504
  int log = static_cast<int>(std::lround(0.5 * std::log2(static_cast<double>(c.rows) * static_cast<double>(c.cols))));
  if (log > 14) log = 14;
  const float scale = std::ldexp(1.0f, log), inverse = std::ldexp(1.0f, -log);
  hipError_t e = c.dtype == kF32 ? start<float>(c, w, scale, ws, stream)
                 : c.dtype == kF16 ? start<f16>(c, w, scale, ws, stream)
                                   : start<bf16>(c, w, scale, ws, stream);
  if (e != hipSuccess) return e;
  const bool tall = c.rows > c.cols;
  float* const partial = at<float>(ws, w.partial);
  f16 *const A = at<f16>(ws, w.gram), *const B = at<f16>(ws, w.poly);
  float* const X = at<float>(ws, w.x);
  for (int t = 0; t < c.steps; ++t) {
    f16 *const now = at<f16>(ws, w.half[t & 1]), *const next = at<f16>(ws, w.half[~t & 1]);
    Step s = step_of(w.rows, w.ldx, tall);
    s.gram.P = s.gram.Q = now;
    s.gram.ldp = s.gram.ldq = w.ldx;
    s.gram.alpha = inverse * inverse;
    s.gram.out = A;
    s.gram.ldo = w.ldm;
    e = launch_extra(s.gram, partial, stream);
    if (e != hipSuccess) return e;
    const f16* poly = A;
    if (c.c != 0.0f) {
      s.poly.P = s.poly.Q = A;
      s.poly.ldp = s.poly.ldq = s.poly.ldr = s.poly.ldo = w.ldm;
      s.poly.alpha = c.c;
      s.poly.beta = c.b;
      s.poly.residual = A;
      s.poly.res_type = kF16;
      s.poly.out = B;
      e = launch_extra(s.poly, partial, stream);
      if (e != hipSuccess) return e;
      poly = B;
    }
    s.update.P = tall ? now : poly;
    s.update.ldp = tall ? w.ldx : w.ldm;
    s.update.Q = tall ? poly : now;
    s.update.ldq = tall ? w.ldm : w.ldx;
    s.update.alpha = inverse * (c.c != 0.0f ? 1.0f : c.b);
    s.update.beta = c.a;
    s.update.residual = X;
    s.update.res_type = kF32;
    s.update.ldr = w.ldx;
    if (t + 1 < c.steps) {
      s.update.out = X;
      s.update.out_type = kF32;
      s.update.ldo = w.ldx;
      s.update.half = next;
      s.update.ldh = w.ldx;
      s.update.half_scale = scale;
    } else {
      s.update.I = c.rows;
      s.update.J = c.cols;
      s.update.out = c.y;
      s.update.out_type = kBF16;
      s.update.ldo = c.ldy;
    }
    e = launch_extra(s.update, partial, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace som
