// An update orthogonalised by Newton-Schulz steps, of the shorter side m against the longer n:
//
//   X = G / |G|;  each step  A = X X^T,  B = b A + c A A,  X = a X + B X
//
// (a tall G without being transposed: A = X^T X, X = a X + X B).  Three products a step on the
// fp16 matrix cores, each with the polynomial's terms in its epilogue.
//
// What is rounded: X is kept in fp32, which the term a X takes as it is; the products take X, A and
// B in fp16, whose 11 bits and not bf16's 8 are what the steps, which amplify small directions 3.4
// times each, leave as errors: 1e-3 to 2e-3 of the result after 5 steps of (3.4445, -4.7750, 2.0315)
// (2-norm; bf16's rounding of y adds 1.7e-3), 3e-3 to 4e-3 after 10, 2e-2 after 64, and more with
// coefficients whose map is steeper about 1; with bf16 between the steps 1e-2, with X in fp16 too
// 5e-3 where singular values spread over 10^4.  X's fp16 copy is scaled by a power of two that makes its elements' size about 1,
// since they are 1 / sqrt(m n) of the norm and would lie among fp16's subnormal numbers.
// The norm is summed in fp64, so no gradient is too small or large for its squares.
//
// X lies in rows and columns rounded up to 64 (a step of the product), with zeros, which stay
// zeros: no product but the last, whose result is y, has a partial step or column.
//
// Small matrices take products of their own: tiles of 32 x 32, whose eight waves share the k axis
// and read their fragments from the L2 without LDS, so that a product is little more than a launch
// and two memory latencies.  They read rows of k only, so X's fp16 copy is kept transposed too.  Of
// sides up to kLowSide, which average less of it out, what rounding leaves of B is kept and
// multiplied as well (5 steps, before y's rounding: 32 x 1,000 3.1e-3 without and 1.8e-3 with it, 153 x 221
// 1.8e-3 and 1.4e-3).
//
// Bound: the matrix cores for sides of 2,048 and more (4,096 x 4,096, 5 steps: 1,613 us; the symmetric
// products 88 to 97 us each on the 136 tiles that they need, the update 116 to 126, of which 25 are
// X's reading and writing in fp32); else 3 launches a step (1,024 x 512: 104 us, 15 products of 4
// to 8).
#include "orthogonalise.h"

#include <cmath>

#include "product_modes.h"

namespace som {
namespace {

constexpr int kParts = 512;            // sums of squares, one a workgroup
// Up to this size the small products are taken (us a call, theirs and the large ones': 64 x 64 46
// and 51, 512 x 512 81 and 86, 1,024 x 512 105 and 112): 2^19 elements are 512 tiles, two a CU.  One more
// is a round more (640 x 832 149 and 112, 768 x 768 186 and 128, 1,024 x 1,024 272 and 150, 256 x 4,096
// 147 and 118, since their fragments come from the L2 64 bytes a row).
constexpr int64_t kSmall = 1 << 19, kSmallSide = 1024;
constexpr int64_t kLowSide = 256;      // what rounding leaves of B is kept up to this (512 x 512: 82 us, with it 94)

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

// X and its fp16 copy, all_rows x all_cols, zeros beyond G.
template <typename T>
__global__ void __launch_bounds__(256) k_ortho_start(const T* G, int64_t ldg, int64_t rows, int64_t cols,
                                                     const double* parts, int nparts, float* X, f16* half,
                                                     int64_t all_rows, int64_t all_cols, int64_t ldx,
                                                     float scale) {
  __shared__ double part[4];
  double s = 0.0;
  for (int p = threadIdx.x; p < nparts; p += 256) s += parts[p];
  s = sum256(s, part);
  const double inverse = s == 0.0 ? 0.0 : 1.0 / sqrt(s);
  const int64_t groups = all_cols / 8, all = groups * all_rows;
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

// ---------------------------------------------------------------------------
// Small products
// ---------------------------------------------------------------------------

constexpr int kSmallWaves = 8;

// C[i][j] = alpha sum_k P[i][k] Q[j][k] + beta residual; I, J and K are multiples of 64.
struct SmallArgs {
  const f16 *P, *Q;
  int64_t ldp, ldq;
  int32_t I, J, K;
  int32_t wrap_p, wrap_q;    // steps of 64 after which the operand starts again
  float alpha, beta;
  const void* residual;      // fp32 (or fp16 with res_half), or nullptr
  bool res_half;
  int64_t ldr;
  void* out;                 // of out_type, rows x cols of it; or nullptr
  int out_type;
  int64_t ldo, rows, cols;
  f16 *half, *half_t;        // [I][ldh] and its transpose [J][ldt], times half_scale; or nullptr
  int32_t low;               // columns further on: what half's rounding leaves (0: nowhere)
  int64_t ldh, ldt;
  float half_scale;
};

// 32 x 32 a workgroup; wave w takes the steps w, w + 8, ... of 64 of k.
__global__ void __launch_bounds__(kSmallWaves * 64) k_ortho_small(const SmallArgs a) {
  constexpr int TT = 2, kSide = TT * 16, kRow = kSide + 4;     // floats; 4 more: other banks
  __shared__ __align__(16) float sums[kSmallWaves * kSide * kRow];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
  const int tiles_j = a.J / kSide;
  const int ti = blockIdx.x / tiles_j, tj = blockIdx.x - ti * tiles_j;
  const f16* const p = a.P + static_cast<int64_t>(ti * kSide + r) * a.ldp + g * 8;
  const f16* const q = a.Q + static_cast<int64_t>(tj * kSide + r) * a.ldq + g * 8;
  const int steps = a.K / 64, active = min(steps, kSmallWaves);
  f4 acc[TT][TT];
#pragma unroll
  for (int x = 0; x < TT; ++x)
#pragma unroll
    for (int y = 0; y < TT; ++y) acc[x][y] = f4{0.0f, 0.0f, 0.0f, 0.0f};
  struct Step {
    h8 p[TT][2], q[TT][2];
  };
  auto load = [&](Step& s, int step) __attribute__((always_inline)) {
    const int at_p = (step < a.wrap_p ? step : step - a.wrap_p) * 64, at_q = (step < a.wrap_q ? step : step - a.wrap_q) * 64;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
#pragma unroll
      for (int h = 0; h < 2; ++h) s.p[t][h] = *reinterpret_cast<const h8*>(p + t * 16 * a.ldp + at_p + h * 32);
#pragma unroll
      for (int h = 0; h < 2; ++h) s.q[t][h] = *reinterpret_cast<const h8*>(q + t * 16 * a.ldq + at_q + h * 32);
    }
  };
  auto multiply = [&](const Step& s) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int x = 0; x < TT; ++x)
#pragma unroll
        for (int y = 0; y < TT; ++y)
          acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(s.q[y][h], s.p[x][h], acc[x][y], 0, 0, 0);
  };
  typedef f16 h4 __attribute__((ext_vector_type(4)));
  // four columns of C, of half the threads; the residual, asked for before anything is waited for
  const bool mine = threadIdx.x < kSide * kSide / 4;
  const int row = threadIdx.x / (kSide / 4), col = threadIdx.x % (kSide / 4) * 4;
  const int64_t i = ti * kSide + row, j = tj * kSide + col;
  f4 res = {0.0f, 0.0f, 0.0f, 0.0f};
  if (mine && a.residual && !a.res_half)
    res = *reinterpret_cast<const f4*>(static_cast<const float*>(a.residual) + i * a.ldr + j);
  if (mine && a.residual && a.res_half) {
    const h4 h = *reinterpret_cast<const h4*>(static_cast<const f16*>(a.residual) + i * a.ldr + j);
#pragma unroll
    for (int e = 0; e < 4; ++e) res[e] = static_cast<float>(h[e]);
  }
  if (wave < steps) {
    constexpr int kDeep = 2;           // steps on their way
    Step some[kDeep];
    for (int s0 = wave; s0 < steps; s0 += kSmallWaves * kDeep) {
#pragma unroll
      for (int d = 0; d < kDeep; ++d)
        if (s0 + d * kSmallWaves < steps) load(some[d], s0 + d * kSmallWaves);
#pragma unroll
      for (int d = 0; d < kDeep; ++d)
        if (s0 + d * kSmallWaves < steps) multiply(some[d]);
    }
#pragma unroll
    for (int x = 0; x < TT; ++x)
#pragma unroll
      for (int y = 0; y < TT; ++y)
        *reinterpret_cast<f4*>(&sums[(wave * kSide + x * 16 + r) * kRow + y * 16 + g * 4]) = acc[x][y];
  }
  __syncthreads();
  f4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  if (mine) {
    for (int w = 0; w < active; ++w) v += *reinterpret_cast<const f4*>(&sums[(w * kSide + row) * kRow + col]);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(a.beta, res[e], a.alpha * v[e]);
    if (a.out && i < a.rows) {
      if (a.out_type == kF32) {          // X, whose rows are padded
        *reinterpret_cast<f4*>(static_cast<float*>(a.out) + i * a.ldo + j) = v;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (j + e < a.cols) static_cast<bf16*>(a.out)[i * a.ldo + j + e] = static_cast<bf16>(v[e]);
      }
    }
    if (a.half) {
      h4 h;
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = static_cast<f16>(v[e] * a.half_scale);
      *reinterpret_cast<h4*>(a.half + i * a.ldh + j) = h;
      if (a.low) {
        h4 low;
#pragma unroll
        for (int e = 0; e < 4; ++e) low[e] = static_cast<f16>(v[e] * a.half_scale - static_cast<float>(h[e]));
        *reinterpret_cast<h4*>(a.half + i * a.ldh + j + a.low) = low;
      }
    }
  }
  if (!a.half_t) return;
  // the transpose, by way of the first wave's place
  __syncthreads();
  if (mine) {
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[(col + e) * kRow + row] = v[e] * a.half_scale;
  }
  __syncthreads();
  if (mine) {
    const f4 s = *reinterpret_cast<const f4*>(&sums[row * kRow + col]);
    const h4 h = {static_cast<f16>(s[0]), static_cast<f16>(s[1]), static_cast<f16>(s[2]), static_cast<f16>(s[3])};
    *reinterpret_cast<h4*>(a.half_t + static_cast<int64_t>(tj * kSide + row) * a.ldt + ti * kSide + col) = h;
  }
}

hipError_t launch_small(const SmallArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(k_ortho_small, dim3(static_cast<uint32_t>((a.I / 32) * (a.J / 32))), dim3(kSmallWaves * 64), 0, stream,
                     a);
  return hipGetLastError();
}

// X, its fp16 copy and that copy's transpose, 64 x 64 a workgroup.
template <typename T>
__global__ void __launch_bounds__(256) k_ortho_start_small(const T* G, int64_t ldg, int64_t rows, int64_t cols,
                                                           const double* parts, int nparts, float* X, f16* half,
                                                           int64_t ldx, f16* half_t, int64_t ldt, int64_t all_cols, float scale) {
  __shared__ double part[4];
  __shared__ float tile[64][65];
  const int64_t across = all_cols / 64, ti = blockIdx.x / across, tj = blockIdx.x - ti * across;
  float all[2][8];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int at = n * 256 + threadIdx.x, r = at >> 3, c = (at & 7) * 8;
    const int64_t row = ti * 64 + r, col = tj * 64 + c;
    const int some = row >= rows || col >= cols ? 0 : cols - col >= 8 ? 8 : static_cast<int>(cols - col);
    load8(G + row * ldg + col, some, all[n]);                  // (zeros beyond)
  }
  double s = 0.0;
  for (int p = threadIdx.x; p < nparts; p += 256) s += parts[p];
  s = sum256(s, part);
  const double inverse = s == 0.0 ? 0.0 : 1.0 / sqrt(s);
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int at = n * 256 + threadIdx.x, r = at >> 3, c = (at & 7) * 8;
    const int64_t row = ti * 64 + r, col = tj * 64 + c;
    float v[8];
    // (beyond G zeros, also where the norm is not a number)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e] = row < rows && col + e < cols ? static_cast<float>(all[n][e] * inverse) : 0.0f;
    store8(X + row * ldx + col, 8, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] *= scale;
      tile[c + e][r] = v[e];
    }
    store8(half + row * ldx + col, 8, v);
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int at = n * 256 + threadIdx.x, r = at >> 3, c = (at & 7) * 8;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = tile[r][c + e];
    store8(half_t + (tj * 64 + r) * ldt + ti * 64 + c, 8, v);
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
  s.gram.symmetric = s.poly.symmetric = true;
  s.update.I = rows;
  s.update.J = cols;
  s.update.K = m;
  s.update.p_kc = true;
  s.update.q_kc = tall;
  return s;
}

// (rows longer than a tile's offsets span go through registers, by a plan of their own)
size_t partial_floats(const ExtraArgs& a) {
  size_t most = 0;
  for (const bool dma : {true, false}) {
    const size_t f = plan_extra(a.I, a.J, a.K, a.elem, a.p_kc, a.q_kc, dma, a.symmetric).partial_floats;
    if (f > most) most = f;
  }
  return most;
}

}  // namespace

OrthoWs ortho_ws(int64_t rows, int64_t cols) {
  OrthoWs w{};
  const bool tall = rows > cols;
  w.rows = round64(rows);
  w.cols = round64(cols);
  w.short_side = tall ? w.cols : w.rows;
  w.ldx = w.cols;
  w.ldt = w.rows;
  size_t o = sizeof(double) * kParts;
  w.x = o;
  o += align_up(sizeof(float) * w.rows * w.ldx, 256);
  for (size_t& h : w.half) {
    h = o;
    o += align_up(2 * w.rows * w.ldx, 256);
  }
  // (a rule for both sides, so that a matrix and its transpose are made alike)
  w.small = w.rows * w.cols <= kSmall && w.rows <= kSmallSide && w.cols <= kSmallSide;
  w.low = w.small && w.short_side <= kLowSide;
  w.ldm = w.low ? 2 * w.short_side : w.short_side;
  if (w.small)
    for (size_t& h : w.half_t) {
      h = o;
      o += align_up(2 * w.cols * w.ldt, 256);
    }
  for (size_t* g : {&w.gram, &w.poly}) {
    *g = o;
    o += align_up(2 * w.short_side * w.ldm, 256);
  }
  w.partial = w.total = o;
  if (w.small) return w;
  const Step s = step_of(w.rows, w.cols, tall);
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
  const T* const G = static_cast<const T*>(c.G);
  double* const parts = at<double>(ws, w.parts);
  float* const X = at<float>(ws, w.x);
  f16* const half = at<f16>(ws, w.half[0]);
  hipLaunchKernelGGL(k_ortho_squares<T>, dim3(groups), dim3(256), 0, stream, G, c.ldg, c.rows, c.cols, parts);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (w.small) {
    hipLaunchKernelGGL(k_ortho_start_small<T>, dim3(static_cast<uint32_t>(w.rows / 64 * (w.cols / 64))), dim3(256), 0, stream,
                       G, c.ldg, c.rows, c.cols, parts, groups, X, half, w.ldx, at<f16>(ws, w.half_t[0]), w.ldt, w.cols, scale);
  } else {
    const int64_t all = (w.cols / 8 * w.rows + 255) / 256;
    hipLaunchKernelGGL(k_ortho_start<T>, dim3(static_cast<uint32_t>(all < 2048 ? all : 2048)), dim3(256), 0, stream, G, c.ldg,
                       c.rows, c.cols, parts, groups, X, half, w.rows, w.cols, w.ldx, scale);
  }
  return hipGetLastError();
}

static hipError_t small_steps(const OrthoCall& c, const OrthoWs& w, float scale, void* ws, hipStream_t stream) {
  const bool tall = c.rows > c.cols;
  const float inverse = 1.0f / scale;
  f16 *const A = at<f16>(ws, w.gram), *const B = at<f16>(ws, w.poly);
  const int32_t m = static_cast<int32_t>(w.short_side), rows = static_cast<int32_t>(w.rows), cols = static_cast<int32_t>(w.cols);
  for (int t = 0; t < c.steps; ++t) {
    const f16 *const now = at<f16>(ws, w.half[t & 1]), *const now_t = at<f16>(ws, w.half_t[t & 1]);
    SmallArgs s{};
    s.P = s.Q = tall ? now_t : now;
    s.ldp = s.ldq = tall ? w.ldt : w.ldx;
    s.I = s.J = m;
    s.K = tall ? rows : cols;
    s.wrap_p = s.wrap_q = s.K / 64;
    s.alpha = inverse * inverse;
    s.half = A;
    s.low = w.low ? m : 0;
    s.ldh = w.ldm;
    s.half_scale = 1.0f;
    hipError_t e = launch_small(s, stream);
    if (e != hipSuccess) return e;
    const f16* poly = A;
    if (c.c != 0.0f) {
      s.P = s.Q = A;
      s.ldp = s.ldq = s.ldr = w.ldm;
      s.K = m;
      s.wrap_p = s.wrap_q = m / 64;
      s.alpha = c.c;
      s.beta = c.b;
      s.residual = A;
      s.res_half = true;
      s.half = B;
      e = launch_small(s, stream);
      if (e != hipSuccess) return e;
      poly = B;
    }
    SmallArgs u{};
    u.P = tall ? now : poly;
    u.ldp = tall ? w.ldx : w.ldm;
    u.Q = tall ? poly : now_t;
    u.ldq = tall ? w.ldm : w.ldt;
    u.I = rows;
    u.J = cols;
    u.K = w.low ? 2 * m : m;           // the rounded polynomial, then what its rounding left
    u.wrap_p = tall ? m / 64 : u.K / 64;
    u.wrap_q = tall ? u.K / 64 : m / 64;
    u.alpha = inverse * (c.c != 0.0f ? 1.0f : c.b);
    u.beta = c.a;
    u.residual = at<float>(ws, w.x);
    u.ldr = w.ldx;
    if (t + 1 < c.steps) {
      u.out = at<float>(ws, w.x);
      u.out_type = kF32;
      u.ldo = w.ldx;
      u.rows = rows;
      u.cols = cols;
      u.half = at<f16>(ws, w.half[~t & 1]);
      u.ldh = w.ldx;
      u.half_t = at<f16>(ws, w.half_t[~t & 1]);
      u.ldt = w.ldt;
      u.half_scale = scale;
    } else {
      u.out = c.y;
      u.out_type = kBF16;
      u.ldo = c.ldy;
      u.rows = c.rows;
      u.cols = c.cols;
    }
    e = launch_small(u, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
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
  if (w.small) return small_steps(c, w, scale, ws, stream);
  const bool tall = c.rows > c.cols;
  float* const partial = at<float>(ws, w.partial);
  f16 *const A = at<f16>(ws, w.gram), *const B = at<f16>(ws, w.poly);
  float* const X = at<float>(ws, w.x);
  for (int t = 0; t < c.steps; ++t) {
    f16 *const now = at<f16>(ws, w.half[t & 1]), *const next = at<f16>(ws, w.half[~t & 1]);
    Step s = step_of(w.rows, w.cols, tall);
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
