// kvr_norm.hip - the norms behind and before a block, its gate and residual
// (kvr_block_norm; kvr.h has the formulas).
//
// A row is held in registers (32-bit) from its one reading to its one writing,
// by WAVES waves, V times eight elements a lane; the two means and the largest
// magnitude are sums and maxima over those lanes.  Memory bounds: every input
// is read once and every output written once.
#include <hip/hip_runtime.h>

#include "kvr_layer.h"

namespace kvr {
namespace {

template <class T>
struct Eight {
  T e[8];
};

// Eight elements from `at` on, as many as there are of `n` (behind them: 0).
// Rows start on any element, so the loads may be unaligned, which the memory
// instructions allow.
template <class T>
__device__ __forceinline__ void load8(const char* row, int at, int n, float (&f)[8]) {
  const T* p = reinterpret_cast<const T*>(row) + at;
  if (at + 8 <= n) {
    Eight<T> x;
    __builtin_memcpy(&x, p, sizeof(x));
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)x.e[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = at + i < n ? (float)p[i] : 0.0f;
  }
}

template <class T>
__device__ __forceinline__ void store8(char* row, int at, int n, const float (&f)[8]) {
  T* p = reinterpret_cast<T*>(row) + at;
  if (at + 8 <= n) {
    Eight<T> x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x.e[i] = (T)f[i];
    __builtin_memcpy(p, &x, sizeof(x));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at + i < n) p[i] = (T)f[i];
  }
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
  return x;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int m = 32; m; m >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, m));
  return x;
}

constexpr int kMostBlocks = 1 << 20;  // of a launch; they take the rows in turn

constexpr int row_threads(int waves) { return waves < 4 ? 256 : 64 * waves; }

template <class T, int WAVES, int V>
__global__ __launch_bounds__(row_threads(WAVES)) void norm_kernel(NormArgs a) {
  constexpr int kRows = row_threads(WAVES) / (64 * WAVES);  // of a workgroup
  __shared__ float sums[2][kRows][WAVES];
  __shared__ uint32_t tops[kRows][WAVES];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int mine = wave / WAVES, part = wave % WAVES;
  const int at0 = (part * 64 + lane) * 8;
  constexpr int kNext = WAVES * 512;

  // the sum of f^2 over the row
  auto mean_square = [&](const float(&f)[V][8], int which) {
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) s = __builtin_fmaf(f[v][i], f[v][i], s);
    s = wave_sum(s);
    if constexpr (WAVES > 1) {
      if (lane == 0) sums[which][mine][part] = s;
      __syncthreads();
      s = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s += sums[which][mine][w];
    }
    return s * a.inv_dim;
  };

  for (int64_t row = (int64_t)blockIdx.x * kRows + mine; row < a.tokens; row += (int64_t)gridDim.x * kRows) {
    float f[V][8];
    const char* x = a.x + row * a.x_tok;
#pragma unroll
    for (int v = 0; v < V; ++v) load8<T>(x, at0 + v * kNext, a.dim, f[v]);
    if (a.after) {
      const float by = __builtin_amdgcn_rsqf(mean_square(f, 0) + a.eps);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float w[8];
        load8<T>(a.after, at0 + v * kNext, a.dim, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[v][i] = f[v][i] * by * w[i];
      }
    }
    if (a.gate) {
      const char* gate = a.gate + row * a.gate_tok;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float g[8];
        load8<T>(gate, at0 + v * kNext, a.dim, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (a.activation != KVR_ACT_NONE)
            g[i] = (a.activation == KVR_ACT_SILU ? g[i] : 1.0f) / (1.0f + expf(-g[i]));
          f[v][i] *= g[i];
        }
      }
    }
    if (a.residual) {
      const char* from = a.residual + row * a.res_tok;
      char* to = a.residual_out + row * a.res_out_tok;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int at = at0 + v * kNext;
        float r[8];
        if (a.res32)
          load8<float>(from, at, a.dim, r);
        else
          load8<T>(from, at, a.dim, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[v][i] = __builtin_fmaf(a.residual_scale, f[v][i], r[i]);
        if (at < a.dim) {
          if (a.res32)
            store8<float>(to, at, a.dim, f[v]);
          else
            store8<T>(to, at, a.dim, f[v]);
        }
      }
    }
    if (a.before) {
      const float by = __builtin_amdgcn_rsqf(mean_square(f, 1) + a.eps);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float w[8];
        load8<T>(a.before, at0 + v * kNext, a.dim, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[v][i] = f[v][i] * by * w[i];
      }
    }
    char* out = a.out + row * a.out_tok;
    if (!a.int8) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int at = at0 + v * kNext;
        if (at < a.dim) store8<T>(out, at, a.dim, f[v]);
      }
      if (WAVES > 1) __syncthreads();
      continue;
    }
    // The largest magnitude by its bits: NaN is above infinity, and that above the rest.
    uint32_t top = 0;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[v][i]) & 0x7fffffffu);
    top = wave_max(top);
    if constexpr (WAVES > 1) {
      if (lane == 0) tops[mine][part] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < WAVES; ++w) top = max(top, tops[mine][w]);
    }
    const float largest = __uint_as_float(top);
    const bool usual = top < 0x7f800000u && largest >= 0x1p-100f;
    const float by = usual ? 127.0f / largest : 0.0f;
    if (part == 0 && lane == 0)
      a.out_scale[row] = usual ? largest / 127.0f : top < 0x7f800000u ? 0.0f : __uint_as_float(0x7fc00000u);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int at = at0 + v * kNext;
      if (at >= a.dim) continue;
      Eight<int8_t> q;
#pragma unroll
      for (int i = 0; i < 8; ++i) q.e[i] = usual ? (int8_t)(int)__builtin_rintf(f[v][i] * by) : 0;
      if (at + 8 <= a.dim) {
        __builtin_memcpy(out + at, &q, 8);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (at + i < a.dim) out[at + i] = (char)q.e[i];
      }
    }
    if (WAVES > 1) __syncthreads();  // before the next row's sums
  }
}

template <class T, int WAVES, int V>
void launch(const NormArgs& a, hipStream_t st) {
  constexpr int rows = row_threads(WAVES) / (64 * WAVES);
  const int64_t groups = ((int64_t)a.tokens + rows - 1) / rows;
  const uint32_t blocks = (uint32_t)(groups < kMostBlocks ? groups : kMostBlocks);
  norm_kernel<T, WAVES, V><<<blocks, row_threads(WAVES), 0, st>>>(a);
}

template <class T>
void launch_typed(const NormArgs& a, hipStream_t st) {
  if (a.dim <= 512)
    launch<T, 1, 1>(a, st);
  else if (a.dim <= 1024)
    launch<T, 1, 2>(a, st);
  else if (a.dim <= 2048)
    launch<T, 4, 1>(a, st);
  else if (a.dim <= 4096)
    launch<T, 4, 2>(a, st);
  else if (a.dim <= 8192)
    launch<T, 4, 4>(a, st);
  else if (a.dim <= 16384)
    launch<T, 16, 2>(a, st);
  else if (a.dim <= 32768)
    launch<T, 16, 4>(a, st);
  else
    launch<T, 16, 8>(a, st);
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, bool fp16, hipStream_t st) {
  if (fp16)
    launch_typed<_Float16>(a, st);
  else
    launch_typed<__bf16>(a, st);
  return hipGetLastError();
}

}  // namespace kvr
