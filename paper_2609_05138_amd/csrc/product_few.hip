// The matrix product of one to four rows (a document or a few being served): every
// weight is used that many times only, so the weights' bytes bound it, and it runs on the
// vector units in one launch, without parts to join.
//
//   k strided (feature-major weights), one row: a workgroup of 16 waves takes 8 L
//     columns; its lanes read L pieces of 16 bytes of 64 / L rows of k at a time, eight
//     such loads each on their way.  L = 8 reads whole lines; L = 4 gives twice the
//     workgroups, whose neighbours share lines in the L2 of the XCD that they are dealt
//     to together.
//   k contiguous (unit-major weights): a wave takes two units, 1 KB of each at a time
//     (16,384 x 16,384 in bf16: 91 us, 5.9 TB/s; in 8 bits 40 us, 6.7 TB/s).
//
// The workgroup's sums are joined by shuffles and through LDS in a fixed order.
#include "product.h"

namespace som {
namespace {

constexpr int kFewWaves = 16;

// 16 bytes of weights widened to fp32
template <int E>
struct Wide {
  static constexpr int kN = E == kE4M3 ? 16 : 8;
};
template <int E>
__device__ __forceinline__ void widen(u4 r, float (&v)[Wide<E>::kN]) {
  if constexpr (E == kE4M3) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      typedef float f2 __attribute__((ext_vector_type(2)));
      const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(r[d]), false);
      const f2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(r[d]), true);
      v[4 * d] = lo[0];
      v[4 * d + 1] = lo[1];
      v[4 * d + 2] = hi[0];
      v[4 * d + 3] = hi[1];
    }
  } else if constexpr (E == kF16) {
    const h8 h = __builtin_bit_cast(h8, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(h[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e % 2 ? r[e / 2] & 0xffff0000u : r[e / 2] << 16);
  }
}

// n elements at p (any alignment), the rest zero bits
template <int E>
__device__ __forceinline__ u4 load16(const char* p, int64_t n) {
  if (n >= Wide<E>::kN) return E == kE4M3 ? u4(*reinterpret_cast<const u4_at1*>(p)) : u4(*reinterpret_cast<const u4_at2*>(p));
  u4 r = {0, 0, 0, 0};
  if constexpr (E == kE4M3) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (e < n) r[e / 4] |= static_cast<uint32_t>(reinterpret_cast<const uint8_t*>(p)[e]) << (8 * (e % 4));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) r[e / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(p)[e]) << (16 * (e % 2));
  }
  return r;
}

template <int E>
__device__ __forceinline__ float one(const void* base, int64_t at) {
  if constexpr (E == kF16)
    return static_cast<float>(static_cast<const f16*>(base)[at]);
  else
    return static_cast<float>(static_cast<const bf16*>(base)[at]);
}

// workgroup -> strip of columns: XCD x takes consecutive strips
__device__ __forceinline__ int64_t strip_of(uint32_t per_xcd) {
  return static_cast<int64_t>(blockIdx.x % kXcds) * per_xcd + blockIdx.x / kXcds;
}

template <int E, int L>
__global__ void __launch_bounds__(kFewWaves * 64) k_few_strided(const ProductArgs a) {
  constexpr int kRows = kFewWaves * 64 / L, kDeep = 8;
  __shared__ float part[kFewWaves][L * 8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t j0 = strip_of(a.per_xcd) * (L * 8);
  if (j0 >= a.J) return;
  const int64_t j = j0 + lane % L * 8;
  const int64_t n = a.J - j;
  float acc[8] = {};
  auto add = [&](u4 w, float x) __attribute__((always_inline)) {
    float v[8];
    widen<E>(w, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = fmaf(x, v[e], acc[e]);
  };
  const char* const weights = static_cast<const char*>(a.Q) + j * 2;
  if (n >= 8) {
    for (int64_t k0 = threadIdx.x / L; k0 < a.K; k0 += kRows * kDeep) {
      u4 w[kDeep];
      float x[kDeep];
#pragma unroll
      for (int d = 0; d < kDeep; ++d) {
        // past the last row: that row again, and nothing of it
        const int64_t k = min(k0 + d * kRows, a.K - 1);
        w[d] = *reinterpret_cast<const u4_at2*>(weights + k * a.ldq * 2);
        x[d] = one<E>(a.P, k);
      }
#pragma unroll
      for (int d = 0; d < kDeep; ++d) {
        const bool in = k0 + d * kRows < a.K;
        add(in ? w[d] : u4{0, 0, 0, 0}, in ? x[d] : 0.0f);
      }
    }
  } else if (n > 0) {
    for (int64_t k = threadIdx.x / L; k < a.K; k += kRows) add(load16<E>(weights + k * a.ldq * 2, n), one<E>(a.P, k));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int off = L; off < 64; off <<= 1) acc[e] += __shfl_xor(acc[e], off, 64);
    if (lane < L) part[wave][lane * 8 + e] = acc[e];
  }
  __syncthreads();
  if (threadIdx.x < L * 8) {           // a column each: the waves in order
    float v = part[0][threadIdx.x];
#pragma unroll
    for (int s = 1; s < kFewWaves; ++s) v += part[s][threadIdx.x];
    part[0][threadIdx.x] = v;
  }
  __syncthreads();
  const int64_t col = j0 + threadIdx.x * 8;
  if (threadIdx.x < L && col < a.J) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = part[0][threadIdx.x * 8 + e];
    const int q = static_cast<int>(min<int64_t>(8, a.J - col));
    finish8(a, 0, col, q, v, column_terms(a, col, q), row_terms(a, 0, col, q));
  }
}

constexpr int kUnitWaves = 8, kUnits = 2;       // 16 units per workgroup

template <int E, int MR>
__global__ void __launch_bounds__(kUnitWaves * 64) k_few_contiguous(const ProductArgs a) {
  constexpr int kN = Wide<E>::kN, kES = E == kE4M3 ? 1 : 2, kDeep = 4;
  __shared__ float part[MR][kUnitWaves * kUnits];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t j0 = strip_of(a.per_xcd) * (kUnitWaves * kUnits);
  if (j0 >= a.J) return;
  const int64_t j = j0 + wave * kUnits;
  float acc[MR][kUnits] = {};
  for (int64_t k0 = lane * kN; k0 < a.K; k0 += 64 * kN * kDeep) {
    u4 w[kDeep][kUnits], x[kDeep][MR];
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      const int64_t k = k0 + d * 64 * kN, n = a.K - k;
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
        w[d][u] = load16<E>(static_cast<const char*>(a.Q) + ((j + u) * a.ldq + k) * kES, j + u < a.J ? n : 0);
#pragma unroll
      for (int m = 0; m < MR; ++m)
        x[d][m] = load16<E>(static_cast<const char*>(a.P) + (m * a.ldp + k) * kES, m < a.I ? n : 0);
    }
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      float wv[kUnits][kN];
#pragma unroll
      for (int u = 0; u < kUnits; ++u) widen<E>(w[d][u], wv[u]);
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        float xv[kN];
        widen<E>(x[d][m], xv);
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
          for (int e = 0; e < kN; ++e) acc[m][u] = fmaf(xv[e], wv[u][e], acc[m][u]);
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

template <int E>
void few_of(ProductArgs a, hipStream_t stream) {
  auto grid = [&](int64_t width) {
    a.per_xcd = static_cast<uint32_t>(((a.J + width - 1) / width + kXcds - 1) / kXcds);
    return dim3(a.per_xcd * kXcds);
  };
  if (!a.q_kc) {
    if constexpr (E != kE4M3) {
      const bool lines = a.J >= 16384;           // a workgroup per CU
      const dim3 g = grid(lines ? 64 : 32);
      if (lines)
        hipLaunchKernelGGL((k_few_strided<E, 8>), g, dim3(kFewWaves * 64), 0, stream, a);
      else
        hipLaunchKernelGGL((k_few_strided<E, 4>), g, dim3(kFewWaves * 64), 0, stream, a);
    }
    return;
  }
  const dim3 g = grid(kUnitWaves * kUnits);
  if (a.I == 1)
    hipLaunchKernelGGL((k_few_contiguous<E, 1>), g, dim3(kUnitWaves * 64), 0, stream, a);
  else if (a.I == 2)
    hipLaunchKernelGGL((k_few_contiguous<E, 2>), g, dim3(kUnitWaves * 64), 0, stream, a);
  else
    hipLaunchKernelGGL((k_few_contiguous<E, 4>), g, dim3(kUnitWaves * 64), 0, stream, a);
}

}  // namespace

hipError_t launch_product_few(const ProductArgs& a, hipStream_t stream) {
  if (a.elem == kF16)
    few_of<kF16>(a, stream);
  else if (a.elem == kBF16)
    few_of<kBF16>(a, stream);
  else
    few_of<kE4M3>(a, stream);
  return hipGetLastError();
}

}  // namespace som
