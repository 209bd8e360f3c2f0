// Host helpers of the C ABI's translation units: the calling thread's last
// error, status returns, workspace addressing.
#pragma once

#include <cstdint>
#include <string>

#include "../../include/som.h"
#include "common.h"

namespace som::api {

inline thread_local std::string g_error;

inline som_status fail(som_status s, const std::string& msg) {
  g_error = msg;
  return s;
}

inline som_status ok() {
  g_error.clear();
  return SOM_OK;
}

inline som_status hip_fail(hipError_t e, const char* where) {
  return fail(SOM_ERR_HIP, std::string(where) + ": " + hipGetErrorString(e));
}

constexpr int64_t kI32Max = 2147483647;

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

template <typename P>
P* at(void* base, size_t off) {
  return reinterpret_cast<P*>(static_cast<char*>(base) + off);
}

template <typename P>
const P* at(const void* base, size_t off) {
  return reinterpret_cast<const P*>(static_cast<const char*>(base) + off);
}

}  // namespace som::api
