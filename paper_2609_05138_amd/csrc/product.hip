// Host side of the matrix product (tile shape, split of the k axis), the join of a
// split k axis, and the activation's gradient.
#include "product.h"

#include <initializer_list>

namespace som {
namespace {

// C from its partial sums, added in the order of the splits; eight columns a thread.
__global__ void __launch_bounds__(256) k_join(const ProductArgs a) {
  const int64_t ld = (a.J + 7) / 8 * 8, groups = ld / 8;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (at >= groups * a.I) return;
  const int64_t i = at / groups, j = at % groups * 8;
  const float* p = a.partial + i * ld + j;
  float v[8] = {};
  constexpr int kDeep = 8;             // parts on their way
  for (int s0 = 0; s0 < a.splits; s0 += kDeep) {
    float w[kDeep][8];
#pragma unroll
    for (int s = 0; s < kDeep; ++s)
      if (s0 + s < a.splits) load8(p + (s0 + s) * a.I * ld, 8, w[s]);
#pragma unroll
    for (int s = 0; s < kDeep; ++s)
      if (s0 + s < a.splits) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += w[s][e];
      }
  }
  const int n = static_cast<int>(min<int64_t>(8, a.J - j));
  finish8(a, i, j, n, v, column_terms(a, j, n), row_terms(a, i, j, n));
}

// 512 columns (64 lanes of 8) x every (4 gridDim.y)th row; the four waves' column
// sums are added in order, and the workgroups' by launch_column_sums.
template <typename T>
__global__ void __launch_bounds__(256) k_act_grad(const ActGradArgs a) {
  __shared__ float sums[4][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = (static_cast<int64_t>(blockIdx.x) * 64 + lane) * 8;
  const int n = a.N - col >= 8 ? 8 : a.N > col ? static_cast<int>(a.N - col) : 0;
  float db[8] = {};
  for (int64_t row = static_cast<int64_t>(blockIdx.y) * 4 + wave; row < a.M; row += int64_t(gridDim.y) * 4) {
    float g[8];
    load8(static_cast<const T*>(a.dy) + row * a.lddy + col, n, g);
    if (a.act != kActNone) {
      float v[8];
      load8(static_cast<const T*>(a.pre) + row * a.ldpre + col, n, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] *= act_grad(a.act, v[e]);
    }
    if (a.dp) store8(static_cast<T*>(a.dp) + row * a.lddp + col, n, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) db[e] += g[e];
  }
  if (!a.dbias) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[wave][lane * 8 + e] = db[e];
  __syncthreads();
  for (int c = threadIdx.x; c < 512; c += 256) {
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 512 + c;
    if (at < a.N)
      a.part[static_cast<int64_t>(blockIdx.y) * a.N + at] = sums[0][c] + sums[1][c] + sums[2][c] + sums[3][c];
  }
}

int64_t act_grad_groups(int64_t M, int64_t N) {
  const int64_t strips = (N + 511) / 512, rows = (M + 3) / 4;
  int64_t g = (2048 + strips - 1) / strips;        // about eight workgroups per CU
  if (g > 256) g = 256;
  return g < rows ? g : rows;
}

constexpr int64_t kCus = 256;

// Times in us that the choice of a tile shape goes by, measured on MI355X (bf16, replayed
// graphs of 20 products): a workgroup's start, first step and epilogue; a step of 128
// bytes of k alone on a CU, where up to half of the CUs and where all have one; and for two
// workgroups on a CU.  8-bit steps hold twice the products.  Steps of rows off 16 bytes go
// through registers: 1.3 to 1.8 times a step's time in the four wide shapes; in the narrow ones
// 1.0 to 1.4 times, but their whole calls, whose weights the many tiles read again and again,
// are priced right at 1.8 and 2.2 (at 1.4 70 x 5,001 x 3,000 went to 16 x 128, 25.0 us; 64 x
// 128 in three splits takes 17.5).
struct ShapeTime {
  double fixed, half, full, pair, e4m3, off;
};
constexpr ShapeTime kTime[kShapes] = {{11.0, 1.33, 1.50, 0, 1.8, 1.5},   {9.5, 0.58, 0.80, 0, 1.6, 1.5},
                                      {4.4, 0.47, 0.52, 0, 1.4, 1.5},     {4.1, 0.29, 0.33, 0.64, 1.2, 1.5},
                                      {3.4, 0.27, 0.28, 0.59, 1.1, 1.8}, {3.4, 0.20, 0.22, 0.45, 1.1, 2.2}};
// A split k axis: the second launch and its wait, and the parts' bytes per us.
constexpr double kJoinTime = 4.5, kJoinBytes = 6.5e6;
constexpr int64_t kMinSplitSteps = 4;
constexpr int64_t kFewMaxColumns = int64_t(1) << 26;   // 32 threads each at most, of a launch's 2^32

double product_time(int shape, int64_t n, int64_t steps, bool e4m3, bool dma) {
  const ShapeTime& t = kTime[shape];
  const double more = (e4m3 ? t.e4m3 : 1.0) * (dma ? 1.0 : t.off);
  const double fill = n >= kCus ? 1.0 : n <= kCus / 2 ? 0.0 : static_cast<double>(n - kCus / 2) / (kCus / 2);
  const double alone = t.fixed + steps * more * (t.half + (t.full - t.half) * fill);
  const int64_t each = (n + kCus - 1) / kCus;                // workgroups of a CU
  if (kInfo[shape].wgs == 1) return each * alone;
  return each / 2 * (t.fixed + steps * more * t.pair) + each % 2 * alone;
}

}  // namespace

// The shape and split with the least time by the table.  Against the measured best of all
// shapes and splits it chooses within 5% for 2,048^3 (128 x 128, 20.9 us; 256 x 256 in
// two splits 39.3), 4,096^3 (256 x 256, 107; 128 x 128 148), 3,000 x 1,000 x 3,000
// (256 x 256, 33.0; 128 x 128 39.8), 512 x 1,024 x 4,096 (64 x 128, 9.5; 128 x 128 11.8),
// 128 x 4,096 x 4,096 (64 x 128 in four splits, 16.0; unsplit 22.6), 37 x 8,192 x 2,048
// (32 x 128 in eight splits, 12.7; 64 x 128 12.9).  With rows off 16 bytes, 38 sizes from 6 x
// 3,001 x 4,099 to 4,001 x 3,999 x 4,001 in each layout and in 8 bits: 1% off the best in the
// mean, 15% at the most (2,001 x 1,001 x 2,003 64 x 128, 24.3; 128 x 128 in two splits 29.4.
// 333 x 1,023 x 5,001 64 x 128 in four splits, 20.2; 128 x 128 in eight 21.9).
//
// Few rows: with k contiguous in both up to four take the vector kernel (4,096 x 4,096:
// one row 5.8 us, two 7.4, four 10.1; in 16 x 128 tiles and eight splits 9.0, in two
// launches).  With k strided one row does from 8,192 columns on (2,048 x 16,384: 13.4
// against 17.6; two rows are no faster; 4,096 x 4,096: 11.4 against 8.9, since a
// narrow strip's lines are read by several CUs).
ProductPlan plan_product(int64_t I, int64_t J, int64_t K, int elem, bool p_kc, bool q_kc, bool dma) {
  if (p_kc && J <= kFewMaxColumns && (q_kc ? I <= 4 : I == 1 && J >= 8192)) return {kFew, 1, K, 0};
  const int64_t step = elem == kE4M3 ? 128 : 64;
  const int64_t steps = (K + step - 1) / step;
  ProductPlan best{kShape256, 1, steps * step, 0};
  double least = 1e300;
  const int last = p_kc ? kShape16 : kShape64;
  for (int shape = 0; shape <= last; ++shape) {
    const ShapeInfo& s = kInfo[shape];
    // not worth the host's time: tiles of four times the rows, or very many of them unless
    // they are one row (40 x 512 x 1,048,576: 64 x 128 254 us, 128 x 128 338; 16 x 1,024 x
    // 1,048,576: 451, 256 x 256 586)
    if (s.bi >= 4 * I && shape < last) continue;
    const int64_t tiles = ((I + s.bi - 1) / s.bi) * ((J + s.bj - 1) / s.bj);
    if (tiles > 16 * kCus && least < 1e300 && s.bi < I) break;
    for (int64_t want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
      if (want > 1 && (steps < want * kMinSplitSteps || tiles * want > 4 * kCus)) break;
      const int64_t per = (steps + want - 1) / want, splits = (steps + per - 1) / per;
      double t = product_time(shape, tiles * splits, per, elem == kE4M3, dma);
      if (splits > 1) t += kJoinTime + 8.0 * static_cast<double>(splits) * I * J / kJoinBytes;
      if (t < least) {
        least = t;
        best = {shape, static_cast<int>(splits), per * step, 0};
      }
    }
  }
  if (best.splits > 1) best.partial_floats = static_cast<size_t>(best.splits) * I * ((J + 7) / 8 * 8);
  return best;
}

hipError_t launch_product(ProductArgs a, float* partial, hipStream_t stream) {
  const int64_t es = dtype_bytes(a.elem);
  auto whole = [&](const void* p, int64_t ld) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * es % 16 == 0 && ld <= kDmaMaxLd;
  };
  a.dma = whole(a.P, a.ldp) && whole(a.Q, a.ldq);
  const ProductPlan p = plan_product(a.I, a.J, a.K, a.elem, a.p_kc, a.q_kc, a.dma);
  a.splits = p.splits;
  if (p.shape == kFew) return launch_product_few(a, stream);
  const ShapeInfo& s = kInfo[p.shape];
  a.k_split = p.k_split;
  a.partial = partial;
  a.tiles_i = static_cast<uint32_t>((a.I + s.bi - 1) / s.bi);
  a.tiles_j = static_cast<uint32_t>((a.J + s.bj - 1) / s.bj);
  const int64_t wgs = static_cast<int64_t>(a.tiles_i) * a.tiles_j * a.splits;
  a.per_xcd = static_cast<uint32_t>((wgs + kXcds - 1) / kXcds);
  hipError_t e = a.elem == kF16 ? launch_product_f16(p.shape, a, stream)
                 : a.elem == kBF16 ? launch_product_bf16(p.shape, a, stream)
                                   : launch_product_e4m3(p.shape, a, stream);
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t groups = (a.J + 7) / 8 * a.I;
  hipLaunchKernelGGL(k_join, dim3(static_cast<uint32_t>((groups + 255) / 256)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

size_t act_grad_ws_floats(int64_t M, int64_t N) { return static_cast<size_t>(act_grad_groups(M, N) * N); }

hipError_t launch_act_grad(const ActGradArgs& a, hipStream_t stream) {
  const int64_t groups = act_grad_groups(a.M, a.N);
  const dim3 grid(static_cast<uint32_t>((a.N + 511) / 512), static_cast<uint32_t>(groups));
  if (a.elem == kF16)
    hipLaunchKernelGGL(k_act_grad<f16>, grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(k_act_grad<bf16>, grid, dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.dbias) return e;
  return launch_column_sums(a.part, groups, a.N, a.N, a.dbias, stream);
}

}  // namespace som
