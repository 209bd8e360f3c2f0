// Dense rows or weights into 8 bits (E4M3) with a factor for each block of 128 elements of
// a row, or of 128 x 128, of the matrix or of its transpose:
//
//   s = max |x| / 448 over the block,  q = x / s
//
// Bound: HBM (a maximum, a quotient and a conversion per element; 16,384 x 8,192 in bf16 72 to 77 us, 5.3
// to 5.6 TB/s, a copy's rate; transposed 88 to 94 us, 4.3 to 4.6; blocks of 128 x 128 77 to 80, and
// transposed 87 to 91).  An element is read once and stays in registers
// while its block's maximum is made.
//
//   rows    a wave takes 512 columns (four blocks) of four rows, 16 lanes a block; the
//           workgroup's 16 rows are next to each other, so that the factors of a block of
//           columns, which lie together in the layout that the product reads best, fill
//           whole pieces of 64 bytes
//   tiles   a workgroup takes 128 x 128, a thread 8 x 8 of it: blocks of 128 rows, and
//           transposed codes, which go through LDS to be written as rows of 128 bytes
#include "dense.h"

namespace som {
namespace {

// x / s for an E4M3 code: the product with the rounded inverse, which is up to 1.5 units of fp32 off,
// and one of Markstein's corrections by its remainder, which leaves 2^-22 of a unit before the
// rounding.  That gives the quotient's code: a tie between two codes has five bits, and no x / s that
// is not one lies so close to the middle between a tie and its neighbour.  (The product alone gives
// another code for 5 of 10,000 values of bf16; the division itself, of some ten instructions, takes 24
// instead of 22 us for 8,192 x 4,096, and 86 instead of 73 for 8,192 x 16,384.)  Small factors are scaled by
// a power of two, or the remainder would lie among the subnormal numbers.
struct Quotient {
  float s, inverse, up;
};
__device__ __forceinline__ Quotient quotient(float scale) {
  Quotient q;
  q.up = scale < 0x1p-60f ? 0x1p64f : 1.0f;
  q.s = scale * q.up;
  q.inverse = 1.0f / q.s;
  if (q.s == INFINITY) q.s = 0.0f;               // (no remainder: finite values over it are 0)
  return q;
}
__device__ __forceinline__ float over(float x, const Quotient& q) {
  x *= q.up;
  const float y = x * q.inverse;
  return fmaf(-fmaf(y, q.s, -x), q.inverse, y);   // (keeps the sign of a zero)
}

template <typename V>
__device__ __forceinline__ uint32_t magnitude(const V& r, int e) {
  return __float_as_uint(static_cast<float>(r[e])) & 0x7fffffffu;
}

__device__ __forceinline__ int left8(int64_t end, int64_t at) {
  return end - at >= 8 ? 8 : end > at ? static_cast<int>(end - at) : 0;
}

constexpr int kRowsWave = 4, kRowsGroup = 16, kTileBand = 8;

template <typename T>
__global__ void __launch_bounds__(256) k_quantise_rows(const QuantiseArgs a, uint32_t col_groups) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // bands of kTileBand row groups: an XCD takes a row group's columns one after the other, and finds
  // the lines that rows off 16 bytes share in its L2 (16,384 x 8,191 155 to 90 us)
  const int64_t g = group_index(), band = g / (int64_t(col_groups) * kTileBand), in = g - band * col_groups * kTileBand;
  const int64_t cg = in / kTileBand, rg = band * kTileBand + in % kTileBand;
  const int64_t row0 = rg * kRowsGroup + wave * kRowsWave, col = cg * 512 + lane * 8;
  const int n = left8(a.cols, col);
  typename Eight<T>::vec v[kRowsWave];
  uint32_t top[kRowsWave];
#pragma unroll
  for (int r = 0; r < kRowsWave; ++r)
    v[r] = raw8(static_cast<const T*>(a.x) + (row0 + r) * a.ldx + col, row0 + r < a.rows ? n : 0);
#pragma unroll
  for (int r = 0; r < kRowsWave; ++r) {
    top[r] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top[r] = max(top[r], magnitude(v[r], e));
#pragma unroll
    for (int off = 8; off; off >>= 1)
      top[r] = max(top[r], static_cast<uint32_t>(__shfl_xor(static_cast<int>(top[r]), off, 64)));
  }
#pragma unroll
  for (int r = 0; r < kRowsWave; ++r) {
    const int64_t row = row0 + r;
    if (row >= a.rows || n == 0) continue;
    const float scale = q8_scale(top[r]);
    const Quotient by = quotient(scale);
    if ((lane & 15) == 0) a.scale[row * a.scale_row + col / 128 * a.scale_block] = scale;
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = over(static_cast<float>(v[r][e]), by);
    store8_e4m3(a.q + row * a.ldq + col, n, w);
  }
}

// Rows and columns are x's; BR128: a factor for the tile, else one for each of its columns
// (blocks of 1 x 128 of the transpose).
template <typename T, bool BR128, bool TRANSPOSE>
__global__ void __launch_bounds__(256) k_quantise_tiles(const QuantiseArgs a, uint32_t tiles_x) {
  static_assert(BR128 || TRANSPOSE, "blocks of one row of x itself are not tiles");
  __shared__ uint32_t tops[4][128];
  __shared__ __align__(16) uint64_t codes[TRANSPOSE ? 128 : 1][16];
  const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  // bands of kTileBand tiles down: what neighbours write of a row of the transpose lies together
  // (16,384 x 8,192 in bf16 99 to 91 us, 16,384 x 8,191 131 to 102)
  const int64_t g = group_index(), band = g / (int64_t(tiles_x) * kTileBand), in = g - band * tiles_x * kTileBand;
  const int64_t tx = in / kTileBand, ty = band * kTileBand + in % kTileBand;
  const int64_t row0 = ty * 128 + rg * 8, col0 = tx * 128 + cg * 8;
  if (ty * 128 >= a.rows) return;
  const int n = left8(a.cols, col0), rows = left8(a.rows, row0);
  typename Eight<T>::vec v[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) v[r] = raw8(static_cast<const T*>(a.x) + (row0 + r) * a.ldx + col0, r < rows ? n : 0);
  uint32_t top[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    top[e] = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) top[e] = max(top[e], magnitude(v[r], e));
  }
  float scale[8];
  Quotient by[8];
  if constexpr (BR128) {
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, top[e]);
    scale[0] = q8_scale(group_max<256>(most, tops[0]));
#pragma unroll
    for (int e = 0; e < 8; ++e) by[e] = quotient(scale[0]);
    // of the matrix that is written: block row, block of 128 columns
    if (threadIdx.x == 0) a.scale[TRANSPOSE ? tx * a.scale_row + ty * a.scale_block : ty * a.scale_row + tx * a.scale_block] = scale[0];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      top[e] = max(top[e], static_cast<uint32_t>(__shfl_xor(static_cast<int>(top[e]), 16, 64)));
      top[e] = max(top[e], static_cast<uint32_t>(__shfl_xor(static_cast<int>(top[e]), 32, 64)));
      if ((threadIdx.x & 48) == 0) tops[wave][cg * 8 + e] = top[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = cg * 8 + e;
      scale[e] = q8_scale(max(max(tops[0][c], tops[1][c]), max(tops[2][c], tops[3][c])));
      by[e] = quotient(scale[e]);
      if (rg == 0 && e < n) a.scale[(col0 + e) * a.scale_row + ty * a.scale_block] = scale[e];
    }
  }
  if constexpr (!TRANSPOSE) {
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      if (r >= rows || n == 0) continue;
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = over(static_cast<float>(v[r][e]), by[e]);
      store8_e4m3(a.q + (row0 + r) * a.ldq + col0, n, w);
    }
  } else {
    // eight rows of a column are eight bytes, at a place that its group of columns turns
    // (else the 16 groups, 1 KB apart, would meet in one bank)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float w[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) w[r] = over(static_cast<float>(v[r][e]), by[e]);
      uint64_t packed;
      store8_e4m3(reinterpret_cast<uint8_t*>(&packed), 8, w);
      codes[cg * 8 + e][rg ^ cg] = packed;
    }
    __syncthreads();
    const int64_t at = ty * 128 + cg * 8;
    const int m = left8(a.rows, at);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = i * 16 + rg;
      const int64_t col = tx * 128 + c;
      if (col >= a.cols || m == 0) continue;
      const uint64_t packed = codes[c][cg ^ (c >> 3)];
      uint8_t* p = a.q + col * a.ldq + at;
      typedef uint64_t u64_at1 __attribute__((aligned(1)));
      if (m == 8) {
        *reinterpret_cast<u64_at1*>(p) = packed;
      } else {
        for (int b = 0; b < m; ++b) p[b] = static_cast<uint8_t>(packed >> (8 * b));
      }
    }
  }
}

template <typename T>
void launch_of(const QuantiseArgs& a, hipStream_t stream) {
  if (a.block_rows == 1 && !a.transpose) {
    const int64_t across = (a.cols + 511) / 512, down = (a.rows + kRowsGroup - 1) / kRowsGroup;
    hipLaunchKernelGGL(k_quantise_rows<T>, groups_grid(across * ((down + kTileBand - 1) / kTileBand * kTileBand)),
                       dim3(256), 0, stream, a, static_cast<uint32_t>(across));
    return;
  }
  const int64_t across = (a.cols + 127) / 128, down = (a.rows + 127) / 128;
  const dim3 grid = groups_grid(across * ((down + kTileBand - 1) / kTileBand * kTileBand));
  const uint32_t x = static_cast<uint32_t>(across);
  if (a.block_rows == 1)
    hipLaunchKernelGGL((k_quantise_tiles<T, false, true>), grid, dim3(256), 0, stream, a, x);
  else if (a.transpose)
    hipLaunchKernelGGL((k_quantise_tiles<T, true, true>), grid, dim3(256), 0, stream, a, x);
  else
    hipLaunchKernelGGL((k_quantise_tiles<T, true, false>), grid, dim3(256), 0, stream, a, x);
}

}  // namespace

hipError_t launch_quantise(const QuantiseArgs& a, hipStream_t stream) {
  if (a.dtype == kF32)
    launch_of<float>(a, stream);
  else if (a.dtype == kF16)
    launch_of<f16>(a, stream);
  else
    launch_of<bf16>(a, stream);
  return hipGetLastError();
}

}  // namespace som
