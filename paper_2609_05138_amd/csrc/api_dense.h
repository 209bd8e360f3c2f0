// Argument checks of the dense-document operators' entry points.
#pragma once

#include "api_common.h"
#include "dense.h"

namespace som::api {

constexpr int64_t kMaxK = int64_t(1) << 30;       // a step past the end stays an int32
constexpr int64_t kMaxLd = int64_t(1) << 40;      // row offsets stay inside 64-bit bytes
constexpr int64_t kMaxTiles = (int64_t(1) << 23) - 8;   // of 512 threads, under a launch's 2^32

inline bool is_float(int32_t t) { return t == SOM_F32 || t == SOM_F16 || t == SOM_BF16; }

// A [rows][ld] matrix of `cols` columns: present, strided and aligned as its type
// needs, and its last byte within 2^62.
inline som_status check_matrix(const char* name, const void* p, int64_t ld, int64_t rows, int64_t cols, int32_t dtype) {
  const std::string n(name);
  if (!p) return fail(SOM_ERR_INVALID_ARG, n + " is NULL");
  if (ld < cols || ld > kMaxLd) return fail(SOM_ERR_INVALID_ARG, n + ": the row stride must be in [columns, 2^40]");
  if (rows > 0 && ld > (int64_t(1) << 60) / rows) return fail(SOM_ERR_INVALID_ARG, n + " exceeds the addressable range");
  if (!aligned(p, som::dtype_bytes(dtype))) return fail(SOM_ERR_INVALID_ARG, n + " must be aligned to its elements");
  return SOM_OK;
}

inline som_status check_vector(const char* name, const float* p) {
  if (p && !aligned(p, 4)) return fail(SOM_ERR_INVALID_ARG, std::string(name) + " must be 4-byte aligned");
  return SOM_OK;
}

inline som_status check_ws(const void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return SOM_OK;
  if (!ws) return fail(SOM_ERR_WORKSPACE, "ws is NULL: need " + std::to_string(need) + " bytes");
  if (!aligned(ws, 256)) return fail(SOM_ERR_INVALID_ARG, "ws must be 256-byte aligned");
  if (ws_bytes < need)
    return fail(SOM_ERR_WORKSPACE, "workspace too small: need " + std::to_string(need) + " bytes");
  return SOM_OK;
}

inline som_status check_rows(int64_t rows, int64_t cols) {
  if (rows < 0 || rows > kI32Max) return fail(SOM_ERR_INVALID_ARG, "rows must be in [0, 2^31)");
  if (cols < 1 || cols > kI32Max) return fail(SOM_ERR_INVALID_ARG, "cols must be in [1, 2^31)");
  return SOM_OK;
}

inline som_status check_sizes(int64_t M, int64_t N, int64_t K) {
  if (M < 0 || M > kI32Max) return fail(SOM_ERR_INVALID_ARG, "M must be in [0, 2^31)");
  if (N < 1 || N > kMaxK) return fail(SOM_ERR_INVALID_ARG, "N must be in [1, 2^30]");
  if (K < 1 || K > kMaxK) return fail(SOM_ERR_INVALID_ARG, "K must be in [1, 2^30]");
  return SOM_OK;
}

// Workgroups of C [I][J]: 256 x 256, or up to 64 rows by 128 columns (then of a strip).
// Smaller tiles and splits are for launches of a few thousand.
inline bool launchable(int64_t I, int64_t J) { return (I + 255) / 256 <= kMaxTiles / ((J + 127) / 128); }

}  // namespace som::api

#define SOM_CHECK(call)                 \
  do {                                  \
    const som_status s_ = (call);       \
    if (s_ != SOM_OK) return s_;        \
  } while (0)
