// kvr_product.hip - products of 8-bit integers with scales for each token and
// channel (kvr_integer_product; kvr.h has the formula).
//
//   out[t][c] = float(sum_k x[t][k] w[c][k]) * x_scale[t] * w_scale[c] + bias[c]
//
// The sums are exact in 32 bits, so neither their order nor the way they are
// split matters.  Everything is computed transposed (channels are the rows of
// the matrix instructions' results, tokens the columns), so that a lane has
// four neighbouring channels of one token at a time.
//
// Two kernels: tiles that pass through LDS, which the matrix units bound (9,216
// tokens x 16,384 channels, k = 4,096: 645 us, 1.92 PFLOP/s; 8,192^3 at 2.05),
// and a direct one for few results, which the weights' bytes bound (16 tokens x
// 16,384 channels, k = 4,096: 16.5 us, 4.1 TB/s).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kvr_layer.h"
#include "kvr_lds.h"
#include "kvr_wave.h"

namespace kvr {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int kStep = 64;   // elements of k that a tile holds
constexpr int kXcds = 8;    // workgroups go to them in turn

// What is read in the place of (16) elements behind the last one.
__device__ const uint32_t kZeros[8] = {0, 0, 0, 0, 0, 0, 0, 0};

template <class T, int N>
struct Some {
  T e[N];
};

// N neighbouring channels of a token, as many as there are.
template <class T, int N>
__device__ __forceinline__ void store(char* row, int channel, int channels, const float (&f)[N]) {
  T* to = reinterpret_cast<T*>(row) + channel;
  if (channel + N <= channels) {
    Some<T, N> x;
#pragma unroll
    for (int e = 0; e < N; ++e) x.e[e] = (T)f[e];
    __builtin_memcpy(to, &x, sizeof(x));
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (channel + e < channels) to[e] = (T)f[e];
  }
}

// A tile of WC * FC * 32 channels and WT * FT * 32 tokens by WC * WT waves,
// each of which has FC * FT results of 32 x 32.
//
// k passes in steps of 64: rows of 64 bytes of both operands go from memory
// straight to LDS, into BUFFERS buffers in turn.  16-byte chunks of a row stand
// at chunk ^ (row / 4 % 4): the reads of one chunk of 16 rows fall on
// different banks.
//
// KS such groups of waves have the steps in turn, and their sums are added at
// the end: the waves that a compute unit needs, where there is one workgroup for
// each.
template <int WC, int WT, int FC, int FT, int BUFFERS, int KS>
struct Shape {
  static constexpr int kGroup = WC * WT, kWaves = kGroup * KS, kThreads = 64 * kWaves;
  static constexpr int kChannels = WC * FC * 32, kTokens = WT * FT * 32;
  static constexpr int kRows = kChannels + kTokens;
  static constexpr int kBuffer = kRows * kStep, kPitch = 4 * kChannels + 16, kResults = WT * 32 * kPitch;
  static constexpr int kTiles = KS * (BUFFERS * kBuffer > kResults ? BUFFERS * kBuffer : kResults);
  static constexpr int kBytes = kTiles + (kTokens + 2 * kChannels) * 4;  // and the tile's scales and biases
  static constexpr int kLoads = kRows / 16 / kGroup;  // of a wave, for a step: 16 rows each
  static_assert(kLoads * 16 * kGroup == kRows && kThreads <= 1024 && kBytes <= 160 * 1024, "tile shape");
};

__device__ __forceinline__ const i32x4* chunk_at(const char* tile, int row, int chunk) {
  return (const i32x4*)(tile + row * kStep + ((chunk ^ (row >> 2 & 3)) << 4));
}

// kinds of instructions for the scheduler
constexpr int kProducts = 0x8, kReads = 0x100;

template <class T, int WC, int WT, int FC, int FT, int BUFFERS, int KS>
__global__ __launch_bounds__(64 * WC * WT * KS, FC * FT > 8 ? 1 : 2) void product_kernel(ProductArgs a, uint32_t across,
                                                                                  uint32_t down) {
  typedef Shape<WC, WT, FC, FT, BUFFERS, KS> S;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, all_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5, part = KS == 1 ? 0 : all_wave / S::kGroup, wave = all_wave - part * S::kGroup;

  // neighbouring tiles on one XCD, whose cache they share: each takes a run of
  // the tiles, which go through bands of eight token tiles channel by channel
  const uint32_t total = across * down, each = total / kXcds, more = total % kXcds;
  const uint32_t xcd = blockIdx.x % kXcds;
  const uint32_t id = xcd * each + min(xcd, more) + blockIdx.x / kXcds;
  constexpr uint32_t kBand = 8;
  const uint32_t band = id / (kBand * across), in_band = id % (kBand * across);
  const uint32_t high = min(kBand, down - band * kBand);
  const int t0 = (int)(band * kBand + in_band % high) * S::kTokens, c0 = (int)(in_band / high) * S::kChannels;

  // rows 16 (i * group + wave) + lane / 4 of both operands, the chunk that
  // belongs where the lane writes
  const int chunk = (lane % 4) ^ (lane / 16);
  global_bytes from[S::kLoads];
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) {
    const int row = (i * S::kGroup + wave) * 16 + lane / 4;
    from[i] = (global_bytes)(row < S::kChannels
                                 ? a.w + min(c0 + row, a.channels - 1) * a.w_chan
                                 : a.x + min(t0 + row - S::kChannels, a.tokens - 1) * a.x_tok) +
              chunk * 16;
  }
  char* buffers = lds + part * BUFFERS * S::kBuffer;
  const uint32_t to = lds_offset(buffers) + wave * 1024;
  // of each group (behind k's end there are zeros)
  const int steps = (a.dim + KS * kStep - 1) / (KS * kStep);
  auto load = [&](int s) {
    const int k = (s * KS + part) * kStep;
    const bool there = k + chunk * 16 < a.dim;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i)
      load16_to_lds(there ? from[i] + k : (global_bytes)kZeros,
                    to + (s % BUFFERS) * S::kBuffer + i * S::kGroup * 1024);
  };
  // waits for step s, where those up to `last` are on their way
  auto wait_for = [&](int s, int last) {
    last = min(last, steps - 1);
    if (last >= s + 2)
      wait_loads<2 * S::kLoads>();
    else if (last == s + 1)
      wait_loads<S::kLoads>();
    else
      wait_loads<0>();
    barrier();
  };

  i32x16 sum[FC][FT];
#pragma unroll
  for (int c = 0; c < FC; ++c)
#pragma unroll
    for (int t = 0; t < FT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[c][t][i] = 0;

  const int c_row = wave % WC * FC * 32 + n, t_row = S::kChannels + wave / WC * FT * 32 + n;
  i32x4 w[2][FC], x[2][FT];
  auto read = [&](int s, int k) {
    const char* tile = buffers + (s % BUFFERS) * S::kBuffer;
#pragma unroll
    for (int c = 0; c < FC; ++c) w[k][c] = *chunk_at(tile, c_row + c * 32, 2 * k + h);
#pragma unroll
    for (int t = 0; t < FT; ++t) x[k][t] = *chunk_at(tile, t_row + t * 32, 2 * k + h);
    __builtin_amdgcn_sched_group_barrier(kReads, FC + FT, 0);
  };
  auto multiply = [&](int k) {
#pragma unroll
    for (int c = 0; c < FC; ++c)
#pragma unroll
      for (int t = 0; t < FT; ++t)
        sum[c][t] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[k][c], x[k][t], sum[c][t], 0, 0, 0);
    __builtin_amdgcn_sched_group_barrier(kProducts, FC * FT, 0);
  };
  // scales and biases, for the end: 64 values a load
  float* scales = (float*)(lds + S::kTiles);
  for (int i = all_wave; i < (S::kTokens + 2 * S::kChannels) / 64; i += S::kWaves) {
    const int first = i * 64, of = first < S::kTokens ? 0 : first < S::kTokens + S::kChannels ? 1 : 2;
    const float* base = of == 0 ? a.x_scale : of == 1 ? a.w_scale : a.bias ? a.bias : a.w_scale;
    const int at = of == 0 ? min(t0 + first + lane, a.tokens - 1)
                           : min(c0 + (first - S::kTokens) % S::kChannels + lane, a.channels - 1);
    load4_to_lds((global_ints)(base + at), lds_offset(scales + first));
  }
#pragma unroll
  for (int s = 0; s < BUFFERS; ++s)
    if (s < steps) load(s);
  wait_for(0, BUFFERS - 1);
  read(0, 0);
  // Half of a step's operands are read while the other half is multiplied, and
  // the barrier stands between: behind it the step before is read by all waves
  // (its buffer is filled again) and the next one is there, and there are
  // products left to do while its first operands are on their way.
#pragma unroll 1
  for (int s = 0; s < steps; ++s) {
    read(s, 1);
    multiply(0);
    if (s + 1 < steps) {
      wait_for(s + 1, s + BUFFERS - 1);
      if (s + BUFFERS < steps) load(s + BUFFERS);
      read(s + 1, 0);
    }
    multiply(1);
  }

  // The sums go through LDS, WT * 32 tokens at a time, so that a thread has
  // eight neighbouring channels and a wave whole rows: rows of 32-bit sums, 16
  // bytes apart beyond their own.
  constexpr int kAcross = S::kChannels / 8, kDown = S::kThreads / kAcross, kPitch = S::kPitch;
  const int col = (int)threadIdx.x % kAcross * 8, channel = c0 + col;
  float w_scale[8], bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    w_scale[e] = scales[S::kTokens + col + e];
    bias[e] = scales[S::kTokens + S::kChannels + col + e];
  }
#pragma unroll
  for (int t = 0; t < FT; ++t) {
    barrier();
    char* row = lds + part * S::kResults + (wave / WC * 32 + n) * kPitch + (wave % WC * FC * 32 + 4 * h) * 4;
#pragma unroll
    for (int c = 0; c < FC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(i32x4*)(row + (c * 32 + 8 * i) * 4) =
            i32x4{sum[c][t][4 * i], sum[c][t][4 * i + 1], sum[c][t][4 * i + 2], sum[c][t][4 * i + 3]};
    barrier();
#pragma unroll 4
    for (int r = (int)threadIdx.x / kAcross; r < WT * 32; r += kDown) {
      const int place = (r / 32 * FT + t) * 32 + r % 32, token = t0 + place;
      if (token >= a.tokens || channel >= a.channels) continue;
      const float x_scale = scales[place];
      i32x4 lo = {0, 0, 0, 0}, hi = lo;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        lo += *(const i32x4*)(lds + k * S::kResults + r * kPitch + col * 4);
        hi += *(const i32x4*)(lds + k * S::kResults + r * kPitch + col * 4 + 16);
      }
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[e] = (float)(e < 4 ? lo[e % 4] : hi[e % 4]) * x_scale * w_scale[e];
        if (a.bias) f[e] += bias[e];
      }
      store<T, 8>(a.out + token * a.out_tok, channel, a.channels, f);
    }
  }
}

// Few results: a workgroup has CT * 16 channels and TT * 16 tokens, and its
// waves have k in turn, 256 elements at a time, from memory straight to the
// registers that the matrix instructions take them from; their sums are added
// in LDS.  Four lanes read 64 neighbouring bytes of a row in one load (16 bytes
// of each 64 a lane, all four in loads of their own, took 27 instead of 14.6 us
// for 8 tokens x 16,384 channels, k = 4,096).
//
// X: int8_t, or the type of few tokens of 16 bits, which each workgroup brings
// to integers for itself: its waves take the rows' largest magnitudes first.
constexpr int kDirectStep = 256;

template <class T, class X, int CT, int TT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void product_direct_kernel(ProductArgs a, uint32_t across) {
  constexpr int kPitch = CT * 64 + 16, kWave = TT * 16 * kPitch;
  constexpr bool kInts = sizeof(X) == 1;
  extern __shared__ __align__(16) char lds[];
  __shared__ float by[TT * 16], scales[TT * 16];  // of the workgroup's tokens
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int t0 = (int)(blockIdx.x / across) * TT * 16, c0 = (int)(blockIdx.x % across) * CT * 16;
  const char *w_from[CT], *x_from[TT];
#pragma unroll
  for (int c = 0; c < CT; ++c) w_from[c] = a.w + min(c0 + c * 16 + n, a.channels - 1) * a.w_chan;
#pragma unroll
  for (int t = 0; t < TT; ++t) x_from[t] = a.x + min(t0 + t * 16 + n, a.tokens - 1) * a.x_tok;
  i32x4 sum[CT][TT];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int t = 0; t < TT; ++t) sum[c][t] = i32x4{0, 0, 0, 0};
  if constexpr (!kInts) {
    for (int t = wave; t < min(TT * 16, a.tokens - t0); t += WAVES) {
      const char* row = a.x + (t0 + t) * a.x_tok;
      uint32_t top = 0;
#pragma unroll 4
      for (int k = lane * 8; k < a.dim; k += 512) {
        Some<X, 8> x;
        __builtin_memcpy(&x, row + k * 2, sizeof(x));
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint((float)x.e[e]) & 0x7fffffffu);
      }
      const Quantiser q(wave_max(top));
      if (lane == 0) {
        by[t] = q.by;
        scales[t] = q.scale;
      }
    }
    __syncthreads();
  }
  auto step = [&](int k0, auto whole) {
    i32x4 w[CT][4], x[TT][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = k0 + j * 64 + g * 16;
      const bool there = whole.value || k < a.dim;
#pragma unroll
      for (int c = 0; c < CT; ++c) w[c][j] = *(const i32x4*)(there ? w_from[c] + k : (const char*)kZeros);
      if constexpr (kInts) {
#pragma unroll
        for (int t = 0; t < TT; ++t) x[t][j] = *(const i32x4*)(there ? x_from[t] + k : (const char*)kZeros);
      }
    }
    if constexpr (!kInts) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = k0 + j * 64 + g * 16;
#pragma unroll
        for (int t = 0; t < TT; ++t) {
          Some<X, 16> y;
          __builtin_memcpy(&y, whole.value || k < a.dim ? x_from[t] + k * 2 : (const char*)kZeros, sizeof(y));
          const float b = by[min(t * 16 + n, a.tokens - t0 - 1)];
          Some<int8_t, 16> q;
#pragma unroll
          for (int e = 0; e < 16; ++e) q.e[e] = Quantiser::integer((float)y.e[e], b);
          x[t][j] = __builtin_bit_cast(i32x4, q);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int t = 0; t < TT; ++t)
          sum[c][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[c][j], x[t][j], sum[c][t], 0, 0, 0);
  };
  int k0 = wave * kDirectStep;
  for (; k0 + kDirectStep <= a.dim; k0 += WAVES * kDirectStep) step(k0, std::true_type());
  if (k0 < a.dim) step(k0, std::false_type());
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int t = 0; t < TT; ++t)
      *(i32x4*)(lds + wave * kWave + (t * 16 + n) * kPitch + c * 64 + g * 16) = sum[c][t];
  __syncthreads();
  for (int i = threadIdx.x; i < TT * 16 * CT * 4; i += 64 * WAVES) {
    const int token = t0 + i / (CT * 4), channel = c0 + i % (CT * 4) * 4;
    if (token >= a.tokens || channel >= a.channels) continue;
    i32x4 all = {0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < WAVES; ++v)
      all += *(const i32x4*)(lds + v * kWave + i / (CT * 4) * kPitch + i % (CT * 4) * 16);
    const float x_scale = kInts ? a.x_scale[token] : scales[token - t0];
    float f[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = min(channel + e, a.channels - 1);
      f[e] = (float)all[e] * x_scale * a.w_scale[at];
      if (a.bias) f[e] += a.bias[at];
    }
    store<T, 4>(a.out + token * a.out_tok, channel, a.channels, f);
  }
}

template <class T, int WC, int WT, int FC, int FT, int BUFFERS, int KS>
hipError_t launch_tiles(const ProductArgs& a, hipStream_t st) {
  typedef Shape<WC, WT, FC, FT, BUFFERS, KS> S;
  const hipError_t e = allow_lds<product_kernel<T, WC, WT, FC, FT, BUFFERS, KS>>(S::kBytes);
  if (e != hipSuccess) return e;
  const uint32_t across = (uint32_t)((a.channels + S::kChannels - 1) / S::kChannels);
  const uint32_t down = (uint32_t)((a.tokens + S::kTokens - 1) / S::kTokens);
  product_kernel<T, WC, WT, FC, FT, BUFFERS, KS><<<across * down, S::kThreads, S::kBytes, st>>>(a, across, down);
  return hipGetLastError();
}

template <class T, class X, int CT, int TT, int WAVES>
hipError_t launch_direct(const ProductArgs& a, hipStream_t st) {
  constexpr int bytes = WAVES * TT * 16 * (CT * 64 + 16);
  const hipError_t e = allow_lds<product_direct_kernel<T, X, CT, TT, WAVES>>(bytes);
  if (e != hipSuccess) return e;
  const uint32_t across = (uint32_t)((a.channels + CT * 16 - 1) / (CT * 16));
  const uint32_t down = (uint32_t)((a.tokens + TT * 16 - 1) / (TT * 16));
  product_direct_kernel<T, X, CT, TT, WAVES><<<across * down, 64 * WAVES, bytes, st>>>(a, across);
  return hipGetLastError();
}

// Which kernel, by what they take (8-bit tokens, bfloat16 results, weights that
// no cache holds, us; direct kernels by tokens x channels of a workgroup, tiles
// by channels x tokens and the groups of waves that have k in turn):
//   tokens x k x channels    direct 16x16  16x32  32x32  64x32   tiles 64x64/2  128x64/2  128x128/1  /2  256x256
//        8 x  4,096 x  4,096      8.0       8.2    9.0    9.8         12.3         18         25      22     57
//        8 x  4,096 x 16,384     19.7      16.5   19.0   18.3         16.9         22         26      24     59
//       16 x 16,384 x  8,192     40.1      35.4   37.5   37.6         41           66         90      77    212
//       64 x 16,384 x  1,024     17.8      25.2   33.6   45.4         43.2
//      532 x  8,592 x    128     14.1      10.5   14.8   18.5         22.6
//       64 x  4,096 x  2,048     10.0       8.5   10.9   14.3         14.4
//      200 x  4,096 x  1,024     16.0      13.1    9.8   13.4         12.0
//       33 x  4,096 x  8,192     23.8      22.1   17.3   12.2         13.6         22         26      24     59
//      333 x  5,008 x  1,001     24.6      18.6   18.9   13.2         15.3         30         45      42     83
//      128 x  4,096 x  8,192     62        50     35     25.1         14.8         22         29      28     62
//      512 x  4,096 x  4,096    117        92     65     47           23.2         20.7       28      27     64
//      256 x  4,096 x 16,384    243       197    133     92           45           44         31.0    31.1   68
//    1,024 x  4,096 x  8,192    456       365    252    178           75           74         53.0    56.1   65
//    2,048 x  4,096 x  8,192    904       727    500    354          143          145        100     109     80
// The direct kernels are taken as long as one round of workgroups does it (up
// to 16 tokens, which weights bound, always), the smallest of those; of the
// tiles product_tile's.  64 x 64 without groups took 18.7 instead of 14.8 us for
// 128 tokens x 8,192 channels, with four of them 15.8.
template <class T, class X>
hipError_t launch_one_round(const ProductArgs& a, hipStream_t st) {
  auto fits = [&](int tokens, int channels) {
    return product_tiles(a.tokens, a.channels, tokens, channels) <= kComputeUnits;
  };
  if (fits(16, 16)) return launch_direct<T, X, 1, 1, 8>(a, st);
  if (a.tokens <= 16 || fits(16, 32)) return launch_direct<T, X, 2, 1, 16>(a, st);
  if (fits(32, 32)) return launch_direct<T, X, 2, 2, 16>(a, st);
  return launch_direct<T, X, 2, 4, 8>(a, st);
}

template <class T>
hipError_t launch(const ProductArgs& a, hipStream_t st) {
  if (a.dtype == KVR_BF16) return launch_one_round<T, __bf16>(a, st);
  if (a.dtype == KVR_FP16) return launch_one_round<T, _Float16>(a, st);
  if (a.tokens <= 16 || product_tiles(a.tokens, a.channels, 64, 32) <= kComputeUnits)
    return launch_one_round<T, int8_t>(a, st);
  const ProductTile tile = product_tile(a.tokens, a.channels);
  if (tile.channels == 64) return launch_tiles<T, 2, 2, 1, 1, 4, 2>(a, st);
  if (tile.tokens == 64) return launch_tiles<T, 2, 2, 2, 1, 4, 2>(a, st);
  if (tile.channels == 256) return launch_tiles<T, 4, 2, 2, 4, 4, 1>(a, st);
  return tile.groups == 2 ? launch_tiles<T, 2, 2, 2, 2, 4, 2>(a, st) : launch_tiles<T, 2, 2, 2, 2, 4, 1>(a, st);
}

}  // namespace

hipError_t launch_product(const ProductArgs& a, int out, hipStream_t st) {
  if (out == KVR_BF16) return launch<__bf16>(a, st);
  if (out == KVR_FP16) return launch<_Float16>(a, st);
  return launch<float>(a, st);
}

}  // namespace kvr
