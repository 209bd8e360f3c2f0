// What the kernels of few rows share.
#pragma once

#include "product.h"

namespace som {

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

// workgroup -> strip of columns: XCD x takes consecutive strips
__device__ __forceinline__ int64_t strip_of(uint32_t per_xcd) {
  return static_cast<int64_t>(blockIdx.x % kXcds) * per_xcd + blockIdx.x / kXcds;
}

}  // namespace som
