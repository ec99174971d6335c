// kvr_wave.h - sums and maxima over a wave, and how rows are brought to 8-bit
// integers.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace kvr {
namespace {

// Over the lanes of a wave: within rows of 16 by DPP, then across them.
template <class Op>
__device__ __forceinline__ uint32_t over_wave(uint32_t x, Op op) {
  x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false));   // lane ^ 1
  x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false));   // lane ^ 2
  x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, false));  // mirrored in 8
  x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, false));  // mirrored in 16
  const auto s = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = op(s[0], s[1]);
  const auto t = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return op(t[0], t[1]);
}

__device__ __forceinline__ float wave_sum(float x) {
  return __uint_as_float(over_wave(__float_as_uint(x), [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  return over_wave(x, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// A row's scale from its largest magnitude, given by its bits (NaN is above
// infinity, and that above the rest; kvr_norm in kvr.h has the rules).
struct Quantiser {
  float by, scale;

  explicit __device__ __forceinline__ Quantiser(uint32_t top) {
    const float largest = __uint_as_float(top);
    const bool usual = top < 0x7f800000u && largest >= 0x1p-100f;
    by = usual ? 127.0f / largest : 0.0f;
    scale = usual ? largest / 127.0f : top < 0x7f800000u ? 0.0f : __uint_as_float(0x7fc00000u);
  }

  // (by = 0: 0, whatever x is)
  static __device__ __forceinline__ int8_t integer(float x, float by) {
    return (int8_t)(int)__builtin_rintf(by == 0.0f ? 0.0f : x * by);
  }
};

}  // namespace
}  // namespace kvr
