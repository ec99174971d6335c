// kvr_linear.hip - linear attention with a decay for each key head
// (kvr_linear_attention; kvr.h has the formulas).
#include <hip/hip_runtime.h>

#include "kvr_layer.h"

namespace kvr {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// The request's first token and its number of tokens, -1 where the slots are
// not the pool's (which is reported).
__device__ __forceinline__ bool slots_fit(const LinearArgs& a, int request, int& read, int& write) {
  read = a.read[request];
  write = a.write[request];
  const bool fit = read >= -1 && read < a.slots && write >= -1 && write < a.slots;
  if (!fit && a.status && threadIdx.x == 0) atomicOr(a.status, (uint32_t)KVR_DEV_BAD_PAGE);
  return fit;
}

// Results of the tokens row0 .. row0 + rows - 1 of a key head's queries: NaN.
template <class T>
__device__ void fill_nan(const LinearArgs& a, int row0, int rows, int head, int dim) {
  const int64_t n = (int64_t)rows * a.share * dim;
  for (int64_t i = threadIdx.x; i < n; i += kThreads) {
    const int64_t r = i / dim;
    char* to = a.out + (row0 + r / a.share) * a.o_tok + (head * a.share + r % a.share) * a.o_head;
    reinterpret_cast<T*>(to)[i % dim] = (T)__uint_as_float(0x7fc00000u);
  }
}

// Checks row_start and lists the segments: one workgroup.
__global__ __launch_bounds__(kThreads) void linear_plan_kernel(LinearArgs a) {
  int bad = 0;
  for (int r = threadIdx.x; r < a.requests; r += kThreads) {
    const int from = a.row_start[r], to = a.row_start[r + 1];
    bad |= from < 0 || to < from || to > a.tokens;
    a.segments[r] = {r, from, to - from, 0};
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) {
    *a.hdr = {a.requests, bad};
    if (bad && a.status) atomicOr(a.status, (uint32_t)KVR_DEV_BAD_LENGTH);
  }
}

// The recurrent form: one workgroup for a request's key head, which holds the
// state in registers: thread t columns 4 (t % (D / 4)) .. + 3 of every
// (1024 / D)th row, and passes over the tokens.
template <int D, class T>
__global__ __launch_bounds__(kThreads) void linear_steps_kernel(LinearArgs a) {
  constexpr int kAcross = D / 4, kDown = kThreads / kAcross, kRows = D / kDown;
  __shared__ float qk[2][D];
  __shared__ f32x4 part[kDown][kAcross];
  const int tid = threadIdx.x, col = tid % kAcross, down = tid / kAcross;
  const uint32_t at = divide(blockIdx.x, a.kv_div);
  const int head = (int)(blockIdx.x - at * a.kv_div.d);
  Segment s = {(int)at, (int)at, 1, 0};
  if (a.row_start) {
    if (a.hdr->rejected) {
      for (int t = (int)at; t < a.tokens; t += a.requests) fill_nan<T>(a, t, 1, head, D);
      return;
    }
    s = a.segments[at];
  }
  int read, write;
  if (!slots_fit(a, s.request, read, write)) {
    fill_nan<T>(a, s.row0, s.rows, head, D);
    return;
  }
  f32x4 state[kRows];
  if (read >= 0) {
    const float* from = a.state + read * a.state_slot + head * a.state_head + 4 * col;
#pragma unroll
    for (int i = 0; i < kRows; ++i) state[i] = *reinterpret_cast<const f32x4*>(from + (down + i * kDown) * D);
  } else {
#pragma unroll
    for (int i = 0; i < kRows; ++i) state[i] = f32x4{0, 0, 0, 0};
  }
  const float decay = expf(a.log_decay[head]);
  for (int t = s.row0; t < s.row0 + s.rows; ++t) {
    const T* k = reinterpret_cast<const T*>(a.k + t * a.k_tok + head * a.k_head);
    const T* v = reinterpret_cast<const T*>(a.v + t * a.v_tok + head * a.v_head) + 4 * col;
    if (tid < D) qk[0][tid] = (float)k[tid];
    f32x4 value;
#pragma unroll
    for (int e = 0; e < 4; ++e) value[e] = (float)v[e];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const float key = qk[0][down + i * kDown];
#pragma unroll
      for (int e = 0; e < 4; ++e) state[i][e] = __builtin_fmaf(key, value[e], decay * state[i][e]);
    }
    for (int h = head * a.share; h < (head + 1) * a.share; ++h) {
      const T* q = reinterpret_cast<const T*>(a.q + t * a.q_tok + h * a.q_head);
      __syncthreads();
      if (tid < D) qk[1][tid] = (float)q[tid] * a.scale;
      __syncthreads();
      f32x4 o = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const float query = qk[1][down + i * kDown];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(query, state[i][e], o[e]);
      }
      part[down][col] = o;
      __syncthreads();
      if (tid < D) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kDown; ++i) sum += part[i][tid / 4][tid % 4];
        reinterpret_cast<T*>(a.out + t * a.o_tok + h * a.o_head)[tid] = (T)sum;
      }
    }
    __syncthreads();
  }
  if (write >= 0 && (s.rows || write != read)) {
    float* to = a.state + write * a.state_slot + head * a.state_head + 4 * col;
#pragma unroll
    for (int i = 0; i < kRows; ++i) *reinterpret_cast<f32x4*>(to + (down + i * kDown) * D) = state[i];
  }
}

template <class T>
void launch(const LinearArgs& a, hipStream_t st) {
  const uint32_t blocks = (uint32_t)a.segment_cap * (uint32_t)a.kv_heads;
  if (a.dim == 64)
    linear_steps_kernel<64, T><<<blocks, kThreads, 0, st>>>(a);
  else
    linear_steps_kernel<128, T><<<blocks, kThreads, 0, st>>>(a);
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, bool fp16, hipStream_t st) {
  if (a.row_start) {
    linear_plan_kernel<<<1, kThreads, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (fp16)
    launch<_Float16>(a, st);
  else
    launch<__bf16>(a, st);
  return hipGetLastError();
}

}  // namespace kvr
