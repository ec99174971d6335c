// kvr_product.hip - products of 8-bit integers with scales for each token and
// channel (kvr_integer_product; kvr.h has the formula).
//
//   out[t][c] = float(sum_k x[t][k] w[c][k]) * x_scale[t] * w_scale[c] + bias[c]
//
// The sums are exact in 32 bits, so neither their order nor the way they are
// split matters.  Everything is computed transposed (channels are the rows of
// the matrix instructions' results, tokens the columns), so that a lane has
// four neighbouring channels of one token at a time.
#include <hip/hip_runtime.h>

#include <atomic>

#include "kvr_layer.h"
#include "kvr_lds.h"

namespace kvr {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 128;  // elements of k that a tile holds
constexpr int kXcds = 8;    // workgroups go to them in turn

// What is read in the place of elements behind the last one.
__device__ const uint32_t kZeros[4] = {0, 0, 0, 0};

template <class T>
struct Four {
  T e[4];
};

// Four neighbouring channels of a token.
template <class T>
__device__ __forceinline__ void store4(const ProductArgs& a, int token, int channel, f32x4 f) {
  T* to = reinterpret_cast<T*>(a.out + token * a.out_tok) + channel;
  if (channel + 4 <= a.channels) {
    Four<T> x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x.e[e] = (T)f[e];
    __builtin_memcpy(to, &x, sizeof(x));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (channel + e < a.channels) to[e] = (T)f[e];
  }
}

// A tile of WC * FC * 32 channels and WT * FT * 32 tokens by WC * WT waves,
// each of which has FC * FT results of 32 x 32.
//
// k passes in steps of 128: rows of 128 bytes of both operands go from memory
// straight to LDS, two steps ahead of their use, into two buffers in turn.
// 16-byte chunks of a row stand at chunk ^ (row / 2 % 8): the reads of one
// chunk of 16 rows fall on different banks.
template <int WC, int WT, int FC, int FT>
struct Shape {
  static constexpr int kWaves = WC * WT, kThreads = 64 * kWaves;
  static constexpr int kChannels = WC * FC * 32, kTokens = WT * FT * 32;
  static constexpr int kRows = kChannels + kTokens;
  static constexpr int kBuffer = kRows * kStep, kBytes = 2 * kBuffer;
  static constexpr int kLoads = kRows / 8 / kWaves;  // of a wave, for a step
  static_assert(kLoads * 8 * kWaves == kRows && kWaves % 2 == 0, "tile shape");
};

__device__ __forceinline__ const i32x4* chunk_at(const char* tile, int row, int chunk) {
  return (const i32x4*)(tile + row * kStep + ((chunk ^ (row >> 1 & 7)) << 4));
}

template <class T, int WC, int WT, int FC, int FT>
__global__ __launch_bounds__(64 * WC * WT, 2) void product_kernel(ProductArgs a, uint32_t across, uint32_t down) {
  typedef Shape<WC, WT, FC, FT> S;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;

  // neighbouring tiles on one XCD, whose cache they share: each takes a run of
  // the tiles, which go through bands of eight token tiles channel by channel
  const uint32_t total = across * down, each = total / kXcds, more = total % kXcds;
  const uint32_t xcd = blockIdx.x % kXcds;
  const uint32_t id = xcd * each + min(xcd, more) + blockIdx.x / kXcds;
  constexpr uint32_t kBand = 8;
  const uint32_t band = id / (kBand * across), in_band = id % (kBand * across);
  const uint32_t high = min(kBand, down - band * kBand);
  const int t0 = (int)(band * kBand + in_band % high) * S::kTokens, c0 = (int)(in_band / high) * S::kChannels;

  // rows 8 (i * waves + wave) + lane / 8 of both operands, the chunk that
  // belongs where the lane writes
  const int chunk = (lane % 8) ^ ((wave & 1) * 4 + lane / 16);
  global_bytes from[S::kLoads];
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) {
    const int row = (i * S::kWaves + wave) * 8 + lane / 8;
    from[i] = (global_bytes)(row < S::kChannels
                                 ? a.w + min(c0 + row, a.channels - 1) * a.w_chan
                                 : a.x + min(t0 + row - S::kChannels, a.tokens - 1) * a.x_tok) +
              chunk * 16;
  }
  const uint32_t to = lds_offset(lds) + wave * 1024;
  const int steps = (a.dim + kStep - 1) / kStep;
  auto load = [&](int s) {
    const bool there = s * kStep + chunk * 16 < a.dim;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i)
      load16_to_lds(there ? from[i] + s * kStep : (global_bytes)kZeros,
                    to + (s & 1) * S::kBuffer + i * S::kWaves * 1024);
  };

  i32x16 sum[FC][FT];
#pragma unroll
  for (int c = 0; c < FC; ++c)
#pragma unroll
    for (int t = 0; t < FT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[c][t][i] = 0;

  load(0);
  if (steps > 1) load(1);
  const int c_row = wave % WC * FC * 32 + n, t_row = S::kChannels + wave / WC * FT * 32 + n;
#pragma unroll 1
  for (int s = 0; s < steps; ++s) {
    if (s + 1 < steps)
      wait_loads<S::kLoads>();
    else
      wait_loads<0>();
    barrier();
    const char* tile = lds + (s & 1) * S::kBuffer;
#pragma unroll
    for (int k = 0; k < kStep / 32; ++k) {
      i32x4 w[FC], x[FT];
#pragma unroll
      for (int c = 0; c < FC; ++c) w[c] = *chunk_at(tile, c_row + c * 32, 2 * k + h);
#pragma unroll
      for (int t = 0; t < FT; ++t) x[t] = *chunk_at(tile, t_row + t * 32, 2 * k + h);
#pragma unroll
      for (int c = 0; c < FC; ++c)
#pragma unroll
        for (int t = 0; t < FT; ++t) sum[c][t] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[c], x[t], sum[c][t], 0, 0, 0);
    }
    if (s + 2 < steps) {
      barrier();
      load(s + 2);
    }
  }

#pragma unroll
  for (int t = 0; t < FT; ++t) {
    const int token = t0 + (wave / WC * FT + t) * 32 + n;
    if (token >= a.tokens) continue;
    const float x_scale = a.x_scale[token];
#pragma unroll
    for (int c = 0; c < FC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int channel = c0 + (wave % WC * FC + c) * 32 + 8 * i + 4 * h;
        if (channel >= a.channels) continue;
        f32x4 f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = min(channel + e, a.channels - 1);
          f[e] = (float)sum[c][t][4 * i + e] * x_scale * a.w_scale[at];
          if (a.bias) f[e] += a.bias[at];
        }
        store4<T>(a, token, channel, f);
      }
  }
}

// Once a device: LDS beyond the default limit.
template <auto Kernel>
hipError_t allow_lds(int bytes) {
  static std::atomic<uint64_t> allowed{0};
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const uint64_t bit = device < 64 ? 1ull << device : 0;
  if (!(allowed.load(std::memory_order_relaxed) & bit)) {
    e = hipFuncSetAttribute((const void*)Kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    allowed.fetch_or(bit, std::memory_order_relaxed);
  }
  return hipSuccess;
}

template <class T, int WC, int WT, int FC, int FT>
hipError_t launch_tiles(const ProductArgs& a, hipStream_t st) {
  typedef Shape<WC, WT, FC, FT> S;
  const hipError_t e = allow_lds<product_kernel<T, WC, WT, FC, FT>>(S::kBytes);
  if (e != hipSuccess) return e;
  const uint32_t across = (uint32_t)((a.channels + S::kChannels - 1) / S::kChannels);
  const uint32_t down = (uint32_t)((a.tokens + S::kTokens - 1) / S::kTokens);
  product_kernel<T, WC, WT, FC, FT><<<across * down, S::kThreads, S::kBytes, st>>>(a, across, down);
  return hipGetLastError();
}

template <class T>
hipError_t launch(const ProductArgs& a, hipStream_t st) {
  if ((int64_t)a.tokens * a.channels >= 200 * 65536) return launch_tiles<T, 2, 4, 4, 2>(a, st);
  return launch_tiles<T, 2, 2, 2, 2>(a, st);
}

}  // namespace

hipError_t launch_product(const ProductArgs& a, int out, hipStream_t st) {
  if (out == KVR_BF16) return launch<__bf16>(a, st);
  if (out == KVR_FP16) return launch<_Float16>(a, st);
  return launch<float>(a, st);
}

}  // namespace kvr
