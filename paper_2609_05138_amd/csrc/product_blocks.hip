// Kernels and host side of the product of 8-bit operands in blocks, and its kernel of few rows.
#include "product_blocks.h"

#include "product_few.h"

namespace som {
namespace {

// One to four rows: as product_few.hip's kernel of unit-major weights (a wave takes two units, 1
// KB of each at a time); the 16 products of a lane's chunk are added before they are multiplied by the
// chunk's two factors, which eight lanes share.  Everything is in fp32, whatever the output.
constexpr int kUnitWaves = 8, kUnits = 2;

template <int MR>
__global__ void __launch_bounds__(kUnitWaves * 64) k_few_blocks(const BlockArgs a) {
  constexpr int kN = 16, kDeep = 4;
  __shared__ float part[MR][kUnitWaves * kUnits];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t j0 = strip_of(a.per_xcd) * (kUnitWaves * kUnits);
  if (j0 >= a.J) return;
  const int64_t j = j0 + wave * kUnits;
  float acc[MR][kUnits] = {};
  for (int64_t k0 = lane * kN; k0 < a.K; k0 += 64 * kN * kDeep) {
    u4 w[kDeep][kUnits], x[kDeep][MR];
    float ws[kDeep][kUnits], xs[kDeep][MR];
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      const int64_t k = k0 + d * 64 * kN, n = a.K - k, b = k >> 7;
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const bool in = j + u < a.J && n > 0;
        w[d][u] = load16<kE4M3>(static_cast<const char*>(a.Q) + (j + u) * a.ldq + k, in ? n : 0);
        ws[d][u] = in ? a.ws[((j + u) >> a.ws_shift) * a.ws_row + b * a.ws_k] : 0.0f;
      }
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        const bool in = m < a.I && n > 0;
        x[d][m] = load16<kE4M3>(static_cast<const char*>(a.P) + m * a.ldp + k, in ? n : 0);
        xs[d][m] = in ? a.xs[(m >> a.xs_shift) * a.xs_row + b * a.xs_k] : 0.0f;
      }
    }
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      float wv[kUnits][kN];
#pragma unroll
      for (int u = 0; u < kUnits; ++u) widen<kE4M3>(w[d][u], wv[u]);
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        float xv[kN];
        widen<kE4M3>(x[d][m], xv);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          float s = 0.0f;
#pragma unroll
          for (int e = 0; e < kN; ++e) s = fmaf(xv[e], wv[u][e], s);
          acc[m][u] = fmaf(s * xs[d][m], ws[d][u], acc[m][u]);
        }
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
#pragma unroll
      for (int off = 32; off; off >>= 1) acc[m][u] += __shfl_xor(acc[m][u], off, 64);
      if (lane == 0) part[m][wave * kUnits + u] = acc[m][u];
    }
  __syncthreads();
  constexpr int kGroups = kUnitWaves * kUnits / 8;
  if (threadIdx.x < kGroups * MR) {
    const int m = threadIdx.x / kGroups, c = threadIdx.x % kGroups * 8;
    const int64_t col = j0 + c;
    if (m < a.I && col < a.J) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = part[m][c + e];
      const int q = static_cast<int>(min<int64_t>(8, a.J - col));
      finish8(a, m, col, q, v, column_terms(a, col, q), row_terms(a, m, col, q));
    }
  }
}

hipError_t launch_few(BlockArgs a, hipStream_t stream) {
  constexpr int kWidth = kUnitWaves * kUnits;
  a.per_xcd = static_cast<uint32_t>(((a.J + kWidth - 1) / kWidth + kXcds - 1) / kXcds);
  const dim3 g(a.per_xcd * kXcds), b(kUnitWaves * 64);
  if (a.I == 1)
    hipLaunchKernelGGL(k_few_blocks<1>, g, b, 0, stream, a);
  else if (a.I == 2)
    hipLaunchKernelGGL(k_few_blocks<2>, g, b, 0, stream, a);
  else
    hipLaunchKernelGGL(k_few_blocks<4>, g, b, 0, stream, a);
  return hipGetLastError();
}

template <int SHAPE, bool EXACT, bool UNITS, int WI, int WJ, int TI, int TJ, int NS>
hipError_t launch_one(const BlockArgs& a, hipStream_t stream) {
  static_assert(kInfo[SHAPE].bi == WI * TI * 16 && kInfo[SHAPE].bj == WJ * TJ * 16, "the grid is laid out for these tiles");
  constexpr size_t lds = static_cast<size_t>(NS) * ((WI * TI + WJ * TJ) * 16 * kStepBytes + WI * WJ * 64 * 4);
  static_assert(lds * kInfo[SHAPE].wgs <= 160 * 1024, "a CU holds the workgroups that the plan counts on");
  if constexpr (lds > 64 * 1024) {
    const hipError_t e = allow_lds(k_product_blocks<EXACT, UNITS, WI, WJ, TI, TJ, NS>, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_product_blocks<EXACT, UNITS, WI, WJ, TI, TJ, NS>), dim3(a.per_xcd * kXcds), dim3(WI * WJ * 64), lds,
                     stream, a);
  return hipGetLastError();
}

template <bool EXACT, bool UNITS>
hipError_t launch_shape(int shape, const BlockArgs& a, hipStream_t stream) {
  switch (shape) {
    case kShape256:
      if constexpr (!EXACT) return launch_one<kShape256, EXACT, UNITS, 2, 4, 8, 4, 2>(a, stream);
      return hipErrorInvalidValue;
    case kShape256x128:
      return launch_one<kShape256x128, EXACT, UNITS, 4, 2, 4, 4, 3>(a, stream);
    case kShape128:
      return launch_one<kShape128, EXACT, UNITS, 2, 4, 4, 2, 4>(a, stream);
    case kShape64:
      return launch_one<kShape64, EXACT, UNITS, 2, 4, 2, 2, 3>(a, stream);
    case kShape32:
      return launch_one<kShape32, EXACT, UNITS, 1, 4, 2, 2, 3>(a, stream);
    default:
      return launch_one<kShape16, EXACT, UNITS, 1, 4, 1, 2, 4>(a, stream);
  }
}

}  // namespace

ProductPlan plan_blocks(int64_t I, int64_t J, int64_t K, bool dma, bool exact) {
  if (exact) return plan_product_by(I, J, K, kE4M3, true, true, dma, {true, kShape256x128, false});
  // a step of the 8-bit instructions takes what one of 16 bits and half the k does
  ProductPlan p = plan_product(I, J, (K + 1) / 2, kBF16, true, true, dma);
  p.k_split *= 2;
  return p;
}

hipError_t launch_blocks(BlockArgs a, float* partial, hipStream_t stream) {
  a.dma = rows_on_16(a);
  const ProductPlan p = plan_blocks(a.I, a.J, a.K, a.dma, a.exact);
  a.splits = p.splits;
  if (p.shape == kFew) return launch_few(a, stream);
  set_launch(a, p, partial);
  const bool units = a.ws_shift == 0;
  const hipError_t e = a.exact ? units ? launch_shape<true, true>(p.shape, a, stream) : launch_shape<true, false>(p.shape, a, stream)
                       : units ? launch_shape<false, true>(p.shape, a, stream) : launch_shape<false, false>(p.shape, a, stream);
  if (e != hipSuccess || p.splits == 1) return e;
  return launch_join(a, stream);
}

}  // namespace som
