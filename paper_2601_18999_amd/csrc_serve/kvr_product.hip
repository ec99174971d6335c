// kvr_product.hip - products of 8-bit integers with scales for each token and
// channel (kvr_integer_product; kvr.h has the formula).
//
//   out[t][c] = float(sum_k x[t][k] w[c][k]) * x_scale[t] * w_scale[c] + bias[c]
//
// The sums are exact in 32 bits, so neither their order nor the way they are
// split matters.
#include <hip/hip_runtime.h>

#include "kvr_layer.h"

namespace kvr {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

template <class T>
__device__ __forceinline__ void store_one(const ProductArgs& a, int token, int channel, int sum) {
  if (token >= a.tokens || channel >= a.channels) return;
  float f = (float)sum * a.x_scale[token] * a.w_scale[channel];
  if (a.bias) f += a.bias[channel];
  reinterpret_cast<T*>(a.out + token * a.out_tok)[channel] = (T)f;
}

// A wave has 32 tokens and 32 channels, four waves 32 tokens and 128 channels.
template <class T>
__global__ __launch_bounds__(256) void product_kernel(ProductArgs a, uint32_t across) {
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, n = lane % 32, hh = lane / 32;
  const int t0 = (int)(blockIdx.x / across) * 32, c0 = (int)(blockIdx.x % across) * 128 + wave * 32;
  const char* x = a.x + min(t0 + n, a.tokens - 1) * a.x_tok;
  const char* w = a.w + min(c0 + n, a.channels - 1) * a.w_chan;
  i32x16 sum = {};
  for (int k = hh * 16; k < a.dim + hh * 16; k += 32) {
    i32x4 p = {}, q = {};
    if (k < a.dim) {
      p = *reinterpret_cast<const i32x4*>(w + k);
      q = *reinterpret_cast<const i32x4*>(x + k);
    }
    sum = __builtin_amdgcn_mfma_i32_32x32x32_i8(p, q, sum, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) store_one<T>(a, t0 + n, c0 + 8 * (i / 4) + 4 * hh + i % 4, sum[i]);
}

template <class T>
void launch(const ProductArgs& a, hipStream_t st) {
  const uint32_t across = (uint32_t)((a.channels + 127) / 128), down = (uint32_t)((a.tokens + 31) / 32);
  product_kernel<T><<<across * down, 256, 0, st>>>(a, across);
}

}  // namespace

hipError_t launch_product(const ProductArgs& a, int out, hipStream_t st) {
  if (out == KVR_BF16)
    launch<__bf16>(a, st);
  else if (out == KVR_FP16)
    launch<_Float16>(a, st);
  else
    launch<float>(a, st);
  return hipGetLastError();
}

}  // namespace kvr
