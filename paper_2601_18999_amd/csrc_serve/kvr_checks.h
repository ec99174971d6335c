// kvr_checks.h - what the host side of the serving operators checks and
// reports with.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdio>

#include "kvr_serve.h"

namespace kvr {

constexpr int64_t kInt = 0x7fffffff;

inline kvr_status invalid(const char* msg) { return set_error(KVR_EINVAL, msg); }

inline kvr_status hip_failed(hipError_t e, const char* what) {
  char msg[256];
  std::snprintf(msg, sizeof(msg), "%s: %s", what, hipGetErrorString(e));
  return set_error(KVR_EDEVICE, msg);
}

inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

inline size_t round_up(size_t n) { return (n + 255) & ~size_t(255); }

// A stride in bytes; where there is one of a kind there is no next one, and
// whatever the caller's stride is has no meaning.
inline int64_t step(int64_t stride, int64_t n, int size) { return n > 1 ? stride * size : 0; }

inline bool on_chunks(int64_t a, int64_t b, int64_t c = 0) { return ((a | b | c) & 15) == 0; }

}  // namespace kvr
