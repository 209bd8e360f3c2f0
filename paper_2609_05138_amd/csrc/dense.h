// Element types, row reads and reductions shared by the dense-document kernels.
#pragma once

#include "common.h"

namespace som {

// som_dtype (checked against the header where the entry points are).
constexpr int kF32 = 0, kF16 = 1, kBF16 = 2, kE4M3 = 3;
constexpr float kE4M3Max = 448.0f;

typedef __bf16 bf16;
typedef _Float16 f16;

inline int dtype_bytes(int t) { return t == kF32 ? 4 : t == kE4M3 ? 1 : 2; }

// A launch holds fewer than 2^32 threads along x: more than 2^21 workgroups (of up to
// 1,024) lie in several rows of the grid.  The last row may be longer than the work.
inline dim3 groups_grid(int64_t n) {
  constexpr int64_t kMost = int64_t(1) << 21;
  return n <= kMost ? dim3(static_cast<uint32_t>(n)) : dim3(kMost, static_cast<uint32_t>((n + kMost - 1) / kMost));
}
__device__ __forceinline__ int64_t group_index() {
  return static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x;
}

// Eight consecutive elements at any address an element may have.
template <typename T>
struct Eight {
  typedef T vec __attribute__((ext_vector_type(8)));
  typedef vec at __attribute__((aligned(sizeof(T))));
};

// p[0..n) (n >= 8: all eight) widened to fp32; elements from n on are 0.  A whole
// group is one 16-byte read (fp32: two) whatever p's alignment: the hardware
// splits a misaligned one.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float (&v)[8]) {
  if (n >= 8) {
    const typename Eight<T>::vec r = *reinterpret_cast<const typename Eight<T>::at*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(r[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? static_cast<float>(p[e]) : 0.0f;
  }
}

// The same as they lie in memory (zero bits from n on), to be widened where they are
// used: a load on its way takes half the registers.
template <typename T>
__device__ __forceinline__ typename Eight<T>::vec raw8(const T* p, int n) {
  if (n >= 8) return *reinterpret_cast<const typename Eight<T>::at*>(p);
  typename Eight<T>::vec r = {};
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (e < n) r[e] = p[e];
  return r;
}

// Rounds to nearest even, once.
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    typename Eight<T>::vec r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = static_cast<T>(v[e]);
    *reinterpret_cast<typename Eight<T>::at*>(p) = r;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = static_cast<T>(v[e]);
  }
}

// Eight values in E4M3, rounded to nearest even.
__device__ __forceinline__ void store8_e4m3(uint8_t* p, int n, const float (&v)[8]) {
  int w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h], v[4 * h + 1], 0, false);
    w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2], v[4 * h + 3], w[h], true);
  }
  typedef int two __attribute__((ext_vector_type(2)));
  typedef two two_at __attribute__((aligned(1)));
  if (n >= 8) {
    *reinterpret_cast<two_at*>(p) = two{w[0], w[1]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = static_cast<uint8_t>(static_cast<uint32_t>(w[e / 4]) >> (8 * (e % 4)));
  }
}

// The factor of a row's (or block's) 8-bit values from the bits of the largest magnitude (as unsigned
// words NaN is above every number, so a NaN anywhere reaches the factor).  At least the
// smallest normal number, whose inverse is finite.
__device__ __forceinline__ float q8_scale(uint32_t top) {
  constexpr float kLeast = 1.17549435e-38f;             // 2^-126
  const float scale = __uint_as_float(top) / kE4M3Max;
  return top == 0 ? 1.0f : scale < kLeast ? kLeast : scale;
}

// Sum (or maximum of unsigned words) over the G = 64, 256, ... consecutive threads
// that share a row; every one of them gets it.  `part`: a word for each wave of the
// workgroup.  Each wave's sum is a butterfly, the waves are added in order, so the
// result does not depend on timing.  All threads of the workgroup call it.
template <int G>
__device__ __forceinline__ float group_sum(float v, float* part) {
#pragma unroll
  for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off, 64);
  if constexpr (G > 64) {
    const int wave = threadIdx.x >> 6, first = wave / (G / 64) * (G / 64);
    __syncthreads();                       // `part` may still be read for the sum before
    if ((threadIdx.x & 63) == 0) part[wave] = v;
    __syncthreads();
    v = part[first];
#pragma unroll
    for (int w = 1; w < G / 64; ++w) v += part[first + w];
  }
  return v;
}

template <int G>
__device__ __forceinline__ uint32_t group_max(uint32_t v, uint32_t* part) {
#pragma unroll
  for (int off = 32; off; off >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), off, 64)));
  if constexpr (G > 64) {
    const int wave = threadIdx.x >> 6, first = wave / (G / 64) * (G / 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[wave] = v;
    __syncthreads();
    v = part[first];
#pragma unroll
    for (int w = 1; w < G / 64; ++w) v = max(v, part[first + w]);
  }
  return v;
}

// ---------------------------------------------------------------------------
// Launchers
// ---------------------------------------------------------------------------

struct RmsNormArgs {
  const void *x, *residual, *weight;
  void *y, *h;
  float* scale;
  int64_t ldx, ldr, ldy, ldh, rows, cols;
  int dtype;
  bool q8;
  float eps;
};
hipError_t launch_rms_norm(const RmsNormArgs& a, hipStream_t stream);

struct RmsNormBackArgs {
  const void *dy, *h, *weight, *dh;
  void* dx;
  float *dweight, *ws;
  int64_t lddy, ldh, lddh, lddx, rows, cols;
  int dtype;
  float eps;
};
size_t rms_norm_back_ws_floats(int64_t rows, int64_t cols);
hipError_t launch_rms_norm_back(const RmsNormBackArgs& a, hipStream_t stream);

// out[c] = sum over g of part[g * ld + c], in order of g within fixed groups.
hipError_t launch_column_sums(const float* part, int64_t groups, int64_t ld, int64_t cols, float* out,
                              hipStream_t stream);
// Fills out[0..n) with zeros.
hipError_t launch_zero(void* out, int64_t ld_bytes, int64_t rows, int64_t row_bytes, hipStream_t stream);

struct DropoutArgs {
  const void *x, *residual;
  void* y;
  int64_t ldx, ldr, ldy, rows, cols;
  int dtype;
  uint32_t threshold;   // of 65,536
  uint64_t seed, offset;
};
hipError_t launch_dropout(const DropoutArgs& a, hipStream_t stream);

// Factors lie at scale[row / block_rows * scale_row + column / 128 * scale_block], rows and
// columns being those of q (with `transpose` x's columns and rows).
struct QuantiseArgs {
  const void* x;
  uint8_t* q;
  float* scale;
  int64_t ldx, ldq, rows, cols, scale_row, scale_block;
  int dtype, block_rows;       // 1 or 128
  bool transpose;
};
hipError_t launch_quantise(const QuantiseArgs& a, hipStream_t stream);

}  // namespace som
