// kvr_norm.hip - the norms behind and before a block, its gate and residual
// (kvr_block_norm; kvr.h has the formulas).
//
// A row is held in registers (32-bit) from its one reading to its one writing,
// V times eight elements a lane (rows above 32,768 partly in scratch memory: see
// launch_typed); the two means and the largest magnitude are
// sums and maxima over its lanes, and those of its waves over LDS.  Memory
// bounds long calls, as every input is read once and every output written once:
// 9,216 rows of 4,096 with everything and a 32-bit residual (528 MB) 97 us, 5.4
// TB/s (a copy: 5.1).  Short ones are bound by the row's two or three sums, each of
// which the next step waits for: 777 rows of 5,003 (31 MB) 11.2 us, of 5,000
// 10.5, 8 rows of 4,096 3.5.
#include <hip/hip_runtime.h>

#include "kvr_layer.h"
#include "kvr_wave.h"

namespace kvr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMostWaves = 16;       // of a row
constexpr int kMostBlocks = 1 << 20; // of a launch; they take the rows in turn

template <class T>
struct Eight {
  T e[8];
};

// 16 bytes from any address on (rows start on any element; the memory
// instructions allow it).
__device__ __forceinline__ u32x4 load16(const char* p) {
  u32x4 x;
  __builtin_memcpy(&x, p, sizeof(x));
  return x;
}

// Eight elements of a row of n from `at` on, as they stand in memory; 0 behind
// its end.  EVEN: n is a multiple of 8; no branch stands around its loads, as
// the compiler waits for one that a branch may have made before it goes on (9,216
// rows of 4,096 with everything 105 -> 98 us).  (For other rows to be shifted
// when they are used took 17 instead of 14 us for 777 of 5,003.)
template <class T, bool EVEN>
struct Raw {
  static constexpr int kLoads = sizeof(T) / 2, kEach = 16 / sizeof(T);  // elements of a load
  u32x4 x[kLoads];

  __device__ __forceinline__ void load(const char* row, int at, int n) {
    if constexpr (EVEN) {
      const int from = min(at, n - 8);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) x[i] = load16(row + (from + i * kEach) * (int)sizeof(T));
      return;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) x[i] = u32x4{0, 0, 0, 0};
    if (n >= 8) {
      // those that would end behind the row end with it, and are shifted
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int want = at + i * kEach, from = min(want, n - kEach), by = (want - from) * (int)sizeof(T) * 8;
        x[i] = load16(row + from * (int)sizeof(T));
        if (by) {
          uint64_t lo = x[i][0] | (uint64_t)x[i][1] << 32, hi = x[i][2] | (uint64_t)x[i][3] << 32;
          lo = by >= 128 ? 0 : by >= 64 ? hi >> (by - 64) : lo >> by | hi << (64 - by);
          hi = by >= 64 ? 0 : hi >> by;
          x[i] = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
        }
      }
    } else if (at == 0) {
      Eight<T> e;
#pragma unroll
      for (int i = 0; i < 8; ++i) e.e[i] = i < n ? reinterpret_cast<const T*>(row)[i] : (T)0.0f;
      __builtin_memcpy(x, &e, sizeof(e));
    }
  }

  __device__ __forceinline__ void widen(float (&f)[8], int at, int n) const {
    Eight<T> y;
    __builtin_memcpy(&y, x, sizeof(y));
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = !EVEN || at < n ? (float)y.e[i] : 0.0f;
  }
};

template <class T>
__device__ __forceinline__ void store8(char* row, int at, int n, const float (&f)[8]) {
  T* p = reinterpret_cast<T*>(row) + at;
  if (at + 8 <= n) {
    Eight<T> x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x.e[i] = (T)f[i];
    __builtin_memcpy(p, &x, sizeof(x));
  } else if (at < n) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at + i < n) p[i] = (T)f[i];
  }
}

// One row for each wave (SINGLE: four rows a workgroup), or for a workgroup.
// T: the type of x, R: of the residual.  Several rows a compute unit are on
// their way at once, which takes few registers for each: with 180 instead of
// 64 (eight waves of a row of 4,096, V = 1) 9,216 rows took 144 us.
template <class T, class R, bool SINGLE, int V, bool EVEN>
__global__ __launch_bounds__(SINGLE ? 256 : 64 * kMostWaves, V == 1 ? 8 : 4) void norm_kernel(NormArgs a) {
  __shared__ float sums[2][kMostWaves];
  __shared__ uint32_t tops[kMostWaves];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int waves = SINGLE ? 1 : (int)blockDim.x / 64;
  const int at0 = (SINGLE ? lane : (int)threadIdx.x) * 8, next = waves * 512;
  const int64_t first = SINGLE ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
  const int64_t step = SINGLE ? (int64_t)gridDim.x * 4 : gridDim.x;

  // the mean of f^2 over the row
  auto mean_square = [&](const float(&f)[V][8], int which) {
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) s = __builtin_fmaf(f[v][i], f[v][i], s);
    s = wave_sum(s);
    if (!SINGLE) {
      if (lane == 0) sums[which][wave] = s;
      __syncthreads();
      s = wave_sum(lane < waves ? sums[which][lane % kMostWaves] : 0.0f);
    }
    return s * a.inv_dim;
  };
  auto weigh = [&](float(&f)[V][8], const char* weight, int which) {
    Raw<T, EVEN> raw[V];
    if (V == 1) raw[0].load(weight, at0, a.dim);
    // (the instruction takes a subnormal number for 0)
    const float mean = mean_square(f, which) + a.eps;
    const bool small = mean < 0x1p-126f;
    const float by = __builtin_amdgcn_rsqf(small ? mean * 0x1p64f : mean) * (small ? 0x1p32f : 1.0f);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (V > 1) raw[v].load(weight, at0 + v * next, a.dim);
      float w[8];
      raw[v].widen(w, at0 + v * next, a.dim);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[v][i] = f[v][i] * by * w[i];
    }
  };

#pragma unroll 1
  for (int64_t row = first; row < a.tokens; row += step) {
    // what comes from far is on its way before the first sum is waited for
    Raw<T, EVEN> raw_x[V], raw_gate[V];
    Raw<R, EVEN> raw_res[V];
    const char *gate = a.gate + row * a.gate_tok, *res = a.residual + row * a.res_tok;
#pragma unroll
    for (int v = 0; v < V; ++v) raw_x[v].load(a.x + row * a.x_tok, at0 + v * next, a.dim);
    if (V == 1 && a.gate) raw_gate[0].load(gate, at0, a.dim);
    if (V == 1 && a.residual) raw_res[0].load(res, at0, a.dim);
    float f[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) raw_x[v].widen(f[v], at0 + v * next, a.dim);
    if (a.after) weigh(f, a.after, 0);
    if (a.gate) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (V > 1) raw_gate[v].load(gate, at0 + v * next, a.dim);
        float g[8];
        raw_gate[v].widen(g, at0 + v * next, a.dim);
        if (a.activation != KVR_ACT_NONE) {
          // (an error of the exponent's product is one of |g| half steps)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            g[i] = (a.activation == KVR_ACT_SILU ? g[i] : 1.0f) *
                   __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g[i] * -1.44269504088896340736f));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) f[v][i] *= g[i];
      }
    }
    if (a.residual) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int at = at0 + v * next;
        if (V > 1) raw_res[v].load(res, at, a.dim);
        float r[8];
        raw_res[v].widen(r, at, a.dim);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[v][i] = __builtin_fmaf(a.residual_scale, f[v][i], r[i]);
        store8<R>(a.residual_out + row * a.res_out_tok, at, a.dim, f[v]);
      }
    }
    if (a.before) weigh(f, a.before, 1);
    char* out = a.out + row * a.out_tok;
    if (!a.int8) {
#pragma unroll
      for (int v = 0; v < V; ++v) store8<T>(out, at0 + v * next, a.dim, f[v]);
    } else {
      uint32_t top = 0;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[v][i]) & 0x7fffffffu);
      top = wave_max(top);
      if (!SINGLE) {
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        top = wave_max(lane < waves ? tops[lane % kMostWaves] : 0);
      }
      const Quantiser by(top);
      if (at0 == 0) a.out_scale[row] = by.scale;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int at = at0 + v * next;
        Eight<int8_t> q;
#pragma unroll
        for (int i = 0; i < 8; ++i) q.e[i] = Quantiser::integer(f[v][i], by.by);
        if (at + 8 <= a.dim) {
          __builtin_memcpy(out + at, &q, 8);
        } else if (at < a.dim) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (at + i < a.dim) out[at + i] = (char)q.e[i];
        }
      }
    }
    if (!SINGLE) __syncthreads();  // before the next row's sums
  }
}

template <class T, class R, bool SINGLE, int V>
void launch(const NormArgs& a, hipStream_t st) {
  const int64_t rows = SINGLE ? ((int64_t)a.tokens + 3) / 4 : a.tokens;
  const int threads = SINGLE ? 256 : (a.dim + 512 * V - 1) / (512 * V) * 64;
  const uint32_t blocks = (uint32_t)(rows < kMostBlocks ? rows : kMostBlocks);
  if (a.dim % 8 == 0)
    norm_kernel<T, R, SINGLE, V, true><<<blocks, threads, 0, st>>>(a);
  else
    norm_kernel<T, R, SINGLE, V, false><<<blocks, threads, 0, st>>>(a);
}

// Values of a lane: 16, which have more of a row on its way for each of its
// waits (9,216 rows of 4,096, 16-bit residual and norm before: 61 us with 8, 54
// with 16, 67 with 32), where the residual has 16 bits; with a 32-bit one that
// takes too many registers (9,216 rows with everything: 98 us with 8, 102 with
// 16).  64 values, of rows above 32,768, are more than 128 registers hold beside
// what is on its way: 74 to 257 of them go to scratch memory (16-bit result, norm
// before: 2,048 rows of 32,768 56 us, 4.8 TB/s; 1,024 of 65,536 117, 2.3 TB/s; of
// 65,533 218).
template <class T, class R>
void launch_typed(const NormArgs& a, hipStream_t st) {
  constexpr bool kWide = sizeof(R) == 4;
  if (a.dim <= 512)
    launch<T, R, true, 1>(a, st);
  else if (a.dim <= (kWide ? 512 * kMostWaves : 1024))
    launch<T, R, false, 1>(a, st);
  else if (a.dim <= 1024 * kMostWaves)
    launch<T, R, false, 2>(a, st);
  else if (a.dim <= 2048 * kMostWaves)
    launch<T, R, false, 4>(a, st);
  else
    launch<T, R, false, 8>(a, st);
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, bool fp16, hipStream_t st) {
  if (fp16)
    a.res32 ? launch_typed<_Float16, float>(a, st) : launch_typed<_Float16, _Float16>(a, st);
  else
    a.res32 ? launch_typed<__bf16, float>(a, st) : launch_typed<__bf16, __bf16>(a, st);
  return hipGetLastError();
}

}  // namespace kvr
