// Host side of the matrix product (tile shape, split of the k axis), the join of a
// split k axis, and the activation's gradient.
#include "product.h"

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

constexpr int kCus = 256;

}  // namespace

ProductPlan plan_product(int64_t I, int64_t J, int64_t K, int elem, bool p_kc) {
  const int64_t step = elem == kE4M3 ? 128 : 64;
  const int64_t steps = (K + step - 1) / step;
  auto tiles = [&](int s) { return ((I + kInfo[s].bi - 1) / kInfo[s].bi) * ((J + kInfo[s].bj - 1) / kInfo[s].bj); };
  int shape = kShape256;
  if (p_kc && I <= kFewRows) return {kFew, 1, K, 0};
  if (p_kc && I <= 16)
    shape = kShape16;
  else if (p_kc && I <= 32)
    shape = kShape32;
  else if (I <= 64)
    shape = kShape64;
  else if (tiles(kShape256) < kCus)
    shape = kShape128;
  // few tiles: split k until the device is full, in splits of at least four steps
  int64_t splits = 1;
  const int64_t slots = kCus * kInfo[shape].wgs, n = tiles(shape);
  if (n * 2 <= slots) splits = slots / n;
  if (splits > steps / 4) splits = steps / 4;
  if (splits > 64) splits = 64;
  if (splits < 1) splits = 1;
  const int64_t per = (steps + splits - 1) / splits;
  splits = (steps + per - 1) / per;
  ProductPlan p{shape, static_cast<int>(splits), per * step, 0};
  if (splits > 1) p.partial_floats = static_cast<size_t>(splits) * I * ((J + 7) / 8 * 8);
  return p;
}

hipError_t launch_product(ProductArgs a, float* partial, hipStream_t stream) {
  const ProductPlan p = plan_product(a.I, a.J, a.K, a.elem, a.p_kc);
  a.splits = p.splits;
  if (p.shape == kFew) return launch_product_few(a, stream);
  const ShapeInfo& s = kInfo[p.shape];
  const int64_t es = dtype_bytes(a.elem);
  a.k_split = p.k_split;
  a.partial = partial;
  a.tiles_i = static_cast<uint32_t>((a.I + s.bi - 1) / s.bi);
  a.tiles_j = static_cast<uint32_t>((a.J + s.bj - 1) / s.bj);
  const int64_t wgs = static_cast<int64_t>(a.tiles_i) * a.tiles_j * a.splits;
  a.per_xcd = static_cast<uint32_t>((wgs + kXcds - 1) / kXcds);
  auto whole = [&](const void* p, int64_t ld) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * es % 16 == 0 && ld <= kDmaMaxLd;
  };
  a.dma = whole(a.P, a.ldp) && whole(a.Q, a.ldq);
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
