// Dropout with a mask that is a function of (seed, offset, row, column) and is never
// stored: y = x 65536 / (65536 - t) where the element's 16 random bits are at
// least t, else 0, plus the residual.  The bits are half-words of Philox4x32 with
// ten rounds (Salmon et al., SC 2011): a thread makes the eight of its group of
// columns with one counter (col / 8, row, offset).  Sixteen bits per element and not
// 32: the generator's 20 wide multiplications, which run at a quarter of the vector rate,
// would take longer than the element's bytes.  The rate p is thus a multiple of 2^-16, and
// the kept elements' factor is of that multiple, so the expectation is exact.
// Bound: HBM (16,384 x 8,192 bf16 with a residual 139 us, 5.8 TB/s).
#include "dense.h"

namespace som {
namespace {

__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = static_cast<uint64_t>(c[0]) * 0xD2511F53u, b = static_cast<uint64_t>(c[2]) * 0xCD9E8D57u;
    c[0] = static_cast<uint32_t>(b >> 32) ^ c[1] ^ k0;
    c[1] = static_cast<uint32_t>(b);
    c[2] = static_cast<uint32_t>(a >> 32) ^ c[3] ^ k1;
    c[3] = static_cast<uint32_t>(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

// blockDim (x: groups of eight columns, y: rows); grid-stride over rows.
template <typename T>
__global__ void __launch_bounds__(256) k_dropout(const DropoutArgs a, float keep) {
  const int64_t group = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  const int64_t col = group * 8;
  if (col >= a.cols) return;
  const int n = a.cols - col >= 8 ? 8 : static_cast<int>(a.cols - col);
  const int64_t step = static_cast<int64_t>(gridDim.y) * blockDim.y;
  for (int64_t row = static_cast<int64_t>(blockIdx.y) * blockDim.y + threadIdx.y; row < a.rows; row += step) {
    float v[8], r[8];
    load8(static_cast<const T*>(a.x) + row * a.ldx + col, n, v);
    if (a.residual) load8(static_cast<const T*>(a.residual) + row * a.ldr + col, n, r);
    uint32_t c[4] = {static_cast<uint32_t>(group), static_cast<uint32_t>(row), static_cast<uint32_t>(a.offset),
                     static_cast<uint32_t>(a.offset >> 32)};
    philox(c, static_cast<uint32_t>(a.seed), static_cast<uint32_t>(a.seed >> 32));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t u = e & 1 ? c[e / 2] >> 16 : c[e / 2] & 0xffffu;
      v[e] = u >= a.threshold ? v[e] * keep : 0.0f;
      if (a.residual) v[e] += r[e];
    }
    store8(static_cast<T*>(a.y) + row * a.ldy + col, n, v);
  }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t stream) {
  const int64_t groups = (a.cols + 7) / 8;
  int x = 256;                                   // threads along a row
  while (x > 8 && x / 2 >= groups) x /= 2;
  const int y = 256 / x;
  const int64_t gx = (groups + x - 1) / x;
  int64_t gy = (a.rows + y - 1) / y;
  if (gy > 65535) gy = 65535;
  const dim3 grid(static_cast<uint32_t>(gx), static_cast<uint32_t>(gy)), block(x, y);
  const float keep = a.threshold < 65536 ? 65536.0f / static_cast<float>(65536 - a.threshold) : 0.0f;
  if (a.dtype == kF32)
    hipLaunchKernelGGL(k_dropout<float>, grid, block, 0, stream, a, keep);
  else if (a.dtype == kF16)
    hipLaunchKernelGGL(k_dropout<f16>, grid, block, 0, stream, a, keep);
  else
    hipLaunchKernelGGL(k_dropout<bf16>, grid, block, 0, stream, a, keep);
  return hipGetLastError();
}

}  // namespace som
