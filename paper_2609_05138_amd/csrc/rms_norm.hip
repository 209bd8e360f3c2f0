// Root-mean-square norm of dense rows with the residual's addition, optionally
// into 8 bits with a factor for each row, and its gradient:
//
//   forward   h = x + r;  s = 1 / sqrt(mean h^2 + eps);  y = h s w
//   backward  g = dy w;  dx = s g - h s^3 mean(g h) + dh;  dw_c = sum_rows dy h s
//
// Bound: HBM, a few operations per element (16,384 x 8,192 bf16 with a residual into 8
// bits 169 us, 5.5 TB/s; 8,192 x 8,192 fp32 195 us, 5.5 TB/s; the gradient of 8,192 x 4,096 in
// bf16 46 to 53 us, 5.1 to 5.8 TB/s; one row of 4,096 2.5 us, a launch).  A row is read once and stays in the
// registers of the G threads that share it, 8 elements (16 bytes of a 16-bit type) a
// thread and read, while its sums are made.  Rows too wide for that are read again.
#include "dense.h"

namespace som {
namespace {

template <typename T, bool Q8>
__device__ __forceinline__ void write_y(const RmsNormArgs& a, int64_t row, int64_t c, int n, const float (&y)[8]) {
  if constexpr (Q8)
    store8_e4m3(static_cast<uint8_t*>(a.y) + row * a.ldy + c, n, y);
  else
    store8(static_cast<T*>(a.y) + row * a.ldy + c, n, y);
}

// The sum as the norm sees it: not rounded to T first.
template <typename T>
__device__ __forceinline__ void load_h(const RmsNormArgs& a, int64_t row, int64_t c, int n, float (&v)[8]) {
  load8(static_cast<const T*>(a.x) + row * a.ldx + c, n, v);
  if (a.residual) {
    float r[8];
    load8(static_cast<const T*>(a.residual) + row * a.ldr + c, n, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += r[e];
  }
}

__device__ __forceinline__ int left(int64_t cols, int64_t c) {
  return cols - c >= 8 ? 8 : cols > c ? static_cast<int>(cols - c) : 0;
}

// G threads per row, R rows per workgroup, U groups of eight columns per thread;
// G * U * 8 >= cols.
template <typename T, bool Q8, int G, int R, int U>
__global__ void __launch_bounds__(G* R) k_rms_norm(const RmsNormArgs a) {
  __shared__ float part[G * R / 64];
  __shared__ uint32_t tops[G * R / 64];
  const int t = threadIdx.x % G;
  const int64_t row = group_index() * R + threadIdx.x / G;
  const bool live = row < a.rows;
  float v[U][8], ss = 0.0f;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t c = (static_cast<int64_t>(u) * G + t) * 8;
    load_h<T>(a, row, c, live ? left(a.cols, c) : 0, v[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t c = (static_cast<int64_t>(u) * G + t) * 8;
    if (a.h) store8(static_cast<T*>(a.h) + row * a.ldh + c, live ? left(a.cols, c) : 0, v[u]);
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(v[u][e], v[u][e], ss);
  }
  const float s = rsqrtf(group_sum<G>(ss, part) / static_cast<float>(a.cols) + a.eps);
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t c = (static_cast<int64_t>(u) * G + t) * 8;
    const int n = live ? left(a.cols, c) : 0;
    float w[8];
    if (a.weight) load8(static_cast<const T*>(a.weight) + c, n, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[u][e] = a.weight ? v[u][e] * s * w[e] : v[u][e] * s;
    if constexpr (Q8) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) top = max(top, __float_as_uint(v[u][e]) & 0x7fffffffu);
    } else {
      write_y<T, Q8>(a, row, c, n, v[u]);
    }
  }
  if constexpr (Q8) {
    const float scale = q8_scale(group_max<G>(top, tops)), inv = 1.0f / scale;
    if (live && t == 0) a.scale[row] = scale;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t c = (static_cast<int64_t>(u) * G + t) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] *= inv;
      write_y<T, Q8>(a, row, c, live ? left(a.cols, c) : 0, v[u]);
    }
  }
}

// A workgroup per row of any width, read again for each step.  h is written in the
// last pass: it may be x or the residual.
template <typename T, bool Q8>
__global__ void __launch_bounds__(1024) k_rms_norm_wide(const RmsNormArgs a) {
  __shared__ float part[16];
  __shared__ uint32_t tops[16];
  const int64_t row = group_index();
  if (row >= a.rows) return;
  float v[8], ss = 0.0f;
  for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8192) {
    load_h<T>(a, row, c, left(a.cols, c), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(v[e], v[e], ss);
  }
  const float s = rsqrtf(group_sum<1024>(ss, part) / static_cast<float>(a.cols) + a.eps);
  float inv = 1.0f;
  if constexpr (Q8) {
    uint32_t top = 0;
    for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8192) {
      const int n = left(a.cols, c);
      load_h<T>(a, row, c, n, v);
      float w[8];
      if (a.weight) load8(static_cast<const T*>(a.weight) + c, n, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = a.weight ? v[e] * s * w[e] : v[e] * s;
        if (e < n) top = max(top, __float_as_uint(y) & 0x7fffffffu);
      }
    }
    const float scale = q8_scale(group_max<1024>(top, tops));
    inv = 1.0f / scale;
    if (threadIdx.x == 0) a.scale[row] = scale;
  }
  for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8192) {
    const int n = left(a.cols, c);
    load_h<T>(a, row, c, n, v);
    if (a.h) store8(static_cast<T*>(a.h) + row * a.ldh + c, n, v);
    float w[8];
    if (a.weight) load8(static_cast<const T*>(a.weight) + c, n, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = a.weight ? v[e] * s * w[e] : v[e] * s;
    if constexpr (Q8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= inv;
    }
    write_y<T, Q8>(a, row, c, n, v);
  }
}

// Threads per row: the fewest of 64 to 1024 that hold it with two groups of eight each
// (16,384 x 8,192 into 8 bits with a residual: 512 threads 170 us, 256 of four groups
// 195; 65,536 x 2,048: 128 threads 167, 64 of four 180); with few rows, one, so that more
// of a row's reads are in flight at once.  Wider rows than 1,024 threads hold so, four.
constexpr int64_t kFewRows = 1024;
constexpr int64_t kHeldCols = 1024 * 8 * 4;

template <typename T, bool Q8, int G>
void norm_with(const RmsNormArgs& a, int64_t groups, hipStream_t stream) {
  constexpr int R = G < 256 ? 256 / G : 1;                 // rows per workgroup
  const dim3 grid = groups_grid((a.rows + R - 1) / R), block(G * R);
  if (groups <= G)
    hipLaunchKernelGGL((k_rms_norm<T, Q8, G, R, 1>), grid, block, 0, stream, a);
  else if (groups <= 2 * G)
    hipLaunchKernelGGL((k_rms_norm<T, Q8, G, R, 2>), grid, block, 0, stream, a);
  else if constexpr (G == 1024)
    hipLaunchKernelGGL((k_rms_norm<T, Q8, G, R, 4>), grid, block, 0, stream, a);
}

template <typename T, bool Q8>
void norm_of(const RmsNormArgs& a, hipStream_t stream) {
  const int64_t groups = (a.cols + 7) / 8, most = a.rows < kFewRows ? 1 : 2;
  if (a.cols > kHeldCols)
    hipLaunchKernelGGL((k_rms_norm_wide<T, Q8>), groups_grid(a.rows), dim3(1024), 0, stream, a);
  else if (groups <= 64 * most)
    norm_with<T, Q8, 64>(a, groups, stream);
  else if (groups <= 128 * most)
    norm_with<T, Q8, 128>(a, groups, stream);
  else if (groups <= 256 * most)
    norm_with<T, Q8, 256>(a, groups, stream);
  else if (groups <= 512 * most)
    norm_with<T, Q8, 512>(a, groups, stream);
  else
    norm_with<T, Q8, 1024>(a, groups, stream);
}

// ---------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------

// A workgroup of R groups of G threads takes every (gridDim * R)th row; dweight's terms
// stay in the threads' registers (U * 8 columns each), and each workgroup writes its
// sums, groups added in order, as one row of `part`.  AHEAD: the next row's reads are on
// their way while it works on one (8,192 x 4,096: 52 us; without, 67).  The widest form (above
// 8,192 columns) has no registers for that (4,096 x 16,384 bf16 96 us, 4.2 TB/s), and in fp32
// too few for the row itself (156 spilled; 214 us, 3.8 TB/s).
template <typename T, int G, int R, int U, bool AHEAD>
__global__ void __launch_bounds__(G* R) k_rms_norm_back(const RmsNormBackArgs a, float* __restrict__ part_w) {
  __shared__ float part[G * R / 64], part2[G * R / 64];
  extern __shared__ float cols_sum[];     // R > 1: a row of sums
  const int t = threadIdx.x % G, r = threadIdx.x / G;
  using Raw = typename Eight<T>::vec;
  struct Row {
    Raw h[U], dy[U], dh[U];
  };
  const int64_t step = static_cast<int64_t>(gridDim.x) * R;
  int n[U];
#pragma unroll
  for (int u = 0; u < U; ++u) n[u] = left(a.cols, (static_cast<int64_t>(u) * G + t) * 8);
  auto get = [&](int64_t row, Row& x) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t c = (static_cast<int64_t>(u) * G + t) * 8;
      const int m = row < a.rows ? n[u] : 0;
      x.h[u] = raw8(static_cast<const T*>(a.h) + row * a.ldh + c, m);
      x.dy[u] = raw8(static_cast<const T*>(a.dy) + row * a.lddy + c, m);
      if (a.dh) x.dh[u] = raw8(static_cast<const T*>(a.dh) + row * a.lddh + c, m);
    }
  };
  Raw w[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t c = (static_cast<int64_t>(u) * G + t) * 8;
    if (a.weight) w[u] = raw8(static_cast<const T*>(a.weight) + c, n[u]);
  }
  float dw[U][8] = {};
  Row next;
  get(static_cast<int64_t>(blockIdx.x) * R + r, next);
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * R; first < a.rows; first += step) {
    const int64_t row = first + r;
    const Row now = next;
    if (AHEAD) get(row + step, next);    // on its way while this row's sums are made
    // a group past the last row has zeros: without eps its s would be infinite, and infinity
    // times zero would go into every column's sum
    float ss = R == 1 || row < a.rows ? 0.0f : 1.0f, gh = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float h = static_cast<float>(now.h[u][e]), d = static_cast<float>(now.dy[u][e]);
        ss = fmaf(h, h, ss);
        gh = fmaf(a.weight ? d * static_cast<float>(w[u][e]) : d, h, gh);
      }
    const float s = rsqrtf(group_sum<G>(ss, part) / static_cast<float>(a.cols) + a.eps);
    const float k = group_sum<G>(gh, part2) / static_cast<float>(a.cols) * s * s;   // times s h: the projection
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t c = (static_cast<int64_t>(u) * G + t) * 8;
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float h = static_cast<float>(now.h[u][e]), d = static_cast<float>(now.dy[u][e]);
        dw[u][e] = fmaf(d * h, s, dw[u][e]);
        o[e] = s * ((a.weight ? d * static_cast<float>(w[u][e]) : d) - h * k);
        if (a.dh) o[e] += static_cast<float>(now.dh[u][e]);
      }
      store8(static_cast<T*>(a.dx) + row * a.lddx + c, row < a.rows ? n[u] : 0, o);
    }
    if (!AHEAD) get(row + step, next);
  }
  if (!a.dweight) return;
  if constexpr (R > 1) {
    // the groups in order: the first writes the row of sums, the others add to it
    for (int k = 0; k < R - 1; ++k) {
      if (r == k) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float* at = cols_sum + (u * 8 + e) * G + t;
            *at = k ? *at + dw[u][e] : dw[u][e];
          }
      }
      __syncthreads();
    }
  }
  if (r == R - 1) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t c = (static_cast<int64_t>(u) * G + t) * 8;
      if constexpr (R > 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[u][e] += cols_sum[(u * 8 + e) * G + t];
      }
      store8(part_w + static_cast<int64_t>(blockIdx.x) * a.cols + c, left(a.cols, c), dw[u]);
    }
  }
}

// Wide rows, first step: each row's s and s^2 mean(g h), in stats[2 * row].
template <typename T>
__global__ void __launch_bounds__(1024) k_rms_norm_back_stats(const RmsNormBackArgs a, float* __restrict__ stats) {
  __shared__ float part[16], part2[16];
  const int64_t row = group_index();
  if (row >= a.rows) return;
  float ss = 0.0f, gh = 0.0f;
  for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8192) {
    const int n = left(a.cols, c);
    float h[8], d[8], w[8];
    load8(static_cast<const T*>(a.h) + row * a.ldh + c, n, h);
    load8(static_cast<const T*>(a.dy) + row * a.lddy + c, n, d);
    if (a.weight) load8(static_cast<const T*>(a.weight) + c, n, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      ss = fmaf(h[e], h[e], ss);
      gh = fmaf(a.weight ? d[e] * w[e] : d[e], h[e], gh);
    }
  }
  const float s = rsqrtf(group_sum<1024>(ss, part) / static_cast<float>(a.cols) + a.eps);
  const float k = group_sum<1024>(gh, part2) / static_cast<float>(a.cols) * s * s;
  if (threadIdx.x == 0) {
    stats[2 * row] = s;
    stats[2 * row + 1] = k;
  }
}

// Second step: 2,048 columns a workgroup, every gridDim.y-th row.
template <typename T>
__global__ void __launch_bounds__(256)
k_rms_norm_back_wide(const RmsNormBackArgs a, const float* __restrict__ stats, float* __restrict__ part_w) {
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8;
  const int n = left(a.cols, c);
  float w[8], dw[8] = {};
  if (a.weight) load8(static_cast<const T*>(a.weight) + c, n, w);
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float s = stats[2 * row], k = stats[2 * row + 1];
    float h[8], d[8], o[8];
    load8(static_cast<const T*>(a.h) + row * a.ldh + c, n, h);
    load8(static_cast<const T*>(a.dy) + row * a.lddy + c, n, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dw[e] = fmaf(d[e] * h[e], s, dw[e]);
      o[e] = s * ((a.weight ? d[e] * w[e] : d[e]) - h[e] * k);
    }
    if (a.dh) {
      float dh[8];
      load8(static_cast<const T*>(a.dh) + row * a.lddh + c, n, dh);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += dh[e];
    }
    store8(static_cast<T*>(a.dx) + row * a.lddx + c, n, o);
  }
  if (a.dweight) store8(part_w + static_cast<int64_t>(blockIdx.y) * a.cols + c, n, dw);
}

// Workgroups of the fused form (two of 512 threads per CU) and row groups of the
// wide one; dweight's partial sums take 4 bytes of each per column.
constexpr int64_t kBackGroups = 512, kWideRowGroups = 64;
constexpr int64_t kBackHeldCols = 16384;

struct BackPlan {
  int64_t groups;      // rows of partial sums
  int64_t stats;       // floats before them
};
BackPlan back_plan(int64_t rows, int64_t cols) {
  if (cols > kBackHeldCols) return {rows < kWideRowGroups ? rows : kWideRowGroups, 2 * rows};
  const int64_t per = cols <= 512 ? 8 : cols <= 2048 ? 2 : 1;     // rows per workgroup
  const int64_t all = (rows + per - 1) / per;
  return {all < kBackGroups ? all : kBackGroups, 0};
}

template <typename T>
void back_of(const RmsNormBackArgs& a, hipStream_t stream) {
  const BackPlan p = back_plan(a.rows, a.cols);
  float* part = a.ws + p.stats;
  if (a.cols > kBackHeldCols) {
    hipLaunchKernelGGL((k_rms_norm_back_stats<T>), groups_grid(a.rows), dim3(1024), 0, stream, a, a.ws);
    const dim3 grid(static_cast<uint32_t>((a.cols + 2047) / 2048), static_cast<uint32_t>(p.groups));
    hipLaunchKernelGGL((k_rms_norm_back_wide<T>), grid, dim3(256), 0, stream, a, a.ws, part);
    return;
  }
#define SOM_BACK(G, R, U, AHEAD)                                                                                 \
  hipLaunchKernelGGL((k_rms_norm_back<T, G, R, U, AHEAD>), dim3(static_cast<uint32_t>(p.groups)), dim3(G* R),    \
                     R > 1 ? G * U * 8 * sizeof(float) : 0, stream, a, part)
  if (a.cols <= 512)
    SOM_BACK(64, 8, 1, true);
  else if (a.cols <= 2048)
    SOM_BACK(256, 2, 1, true);
  else if (a.cols <= 4096)
    SOM_BACK(512, 1, 1, true);
  else if (a.cols <= 8192)
    SOM_BACK(512, 1, 2, true);
  else
    SOM_BACK(1024, 1, 2, false);
#undef SOM_BACK
}

// 64 columns a workgroup, 16 waves: wave w adds rows w, w + 16, ..., then the waves
// in order.
__global__ void __launch_bounds__(1024)
k_column_sums(const float* __restrict__ part, int64_t groups, int64_t ld, int64_t cols, float* __restrict__ out) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = group_index() * 64 + lane;
  float s = 0.0f;
  if (c < cols)
    for (int64_t g0 = wave; g0 < groups; g0 += 16 * 8) {
      float v[8];                       // eight on their way
#pragma unroll
      for (int d = 0; d < 8; ++d) v[d] = g0 + 16 * d < groups ? part[(g0 + 16 * d) * ld + c] : 0.0f;
#pragma unroll
      for (int d = 0; d < 8; ++d) s += v[d];
    }
  sums[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < cols) {
    for (int w = 1; w < 16; ++w) s += sums[w][lane];
    out[c] = s;
  }
}

__global__ void __launch_bounds__(256) k_zero(unsigned char* out, int64_t ld_bytes, int64_t row_bytes) {
  unsigned char* row = out + static_cast<int64_t>(blockIdx.y) * ld_bytes;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < row_bytes; i += int64_t(gridDim.x) * 256)
    row[i] = 0;
}

}  // namespace

hipError_t launch_rms_norm(const RmsNormArgs& a, hipStream_t stream) {
  if (a.dtype == kF32)
    a.q8 ? norm_of<float, true>(a, stream) : norm_of<float, false>(a, stream);
  else if (a.dtype == kF16)
    a.q8 ? norm_of<f16, true>(a, stream) : norm_of<f16, false>(a, stream);
  else
    a.q8 ? norm_of<bf16, true>(a, stream) : norm_of<bf16, false>(a, stream);
  return hipGetLastError();
}

size_t rms_norm_back_ws_floats(int64_t rows, int64_t cols) {
  const BackPlan p = back_plan(rows, cols);
  return static_cast<size_t>(p.stats + p.groups * cols);
}

hipError_t launch_rms_norm_back(const RmsNormBackArgs& a, hipStream_t stream) {
  if (a.dtype == kF32)
    back_of<float>(a, stream);
  else if (a.dtype == kF16)
    back_of<f16>(a, stream);
  else
    back_of<bf16>(a, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.dweight) return e;
  const BackPlan p = back_plan(a.rows, a.cols);
  return launch_column_sums(a.ws + p.stats, p.groups, a.cols, a.cols, a.dweight, stream);
}

hipError_t launch_column_sums(const float* part, int64_t groups, int64_t ld, int64_t cols, float* out,
                              hipStream_t stream) {
  hipLaunchKernelGGL(k_column_sums, groups_grid((cols + 63) / 64), dim3(1024), 0, stream, part, groups,
                     ld, cols, out);
  return hipGetLastError();
}

hipError_t launch_zero(void* out, int64_t ld_bytes, int64_t rows, int64_t row_bytes, hipStream_t stream) {
  const int64_t x = (row_bytes + 255) / 256;
  for (int64_t r = 0; r < rows; r += 65535) {
    const int64_t n = rows - r < 65535 ? rows - r : 65535;
    hipLaunchKernelGGL(k_zero, dim3(static_cast<uint32_t>(x < 1024 ? x : 1024), static_cast<uint32_t>(n)), dim3(256), 0,
                       stream, static_cast<unsigned char*>(out) + r * ld_bytes, ld_bytes, row_bytes);
  }
  return hipGetLastError();
}

}  // namespace som
