// kvr_linear.hip - linear attention with a decay for each key head
// (kvr_linear_attention; kvr.h has the formulas).
//
// Requests of a few tokens take the recurrent form (linear_steps_kernel): a
// workgroup holds a state in registers from its reading to its writing and
// passes over the tokens; the states' bytes bound it.
//
// Longer ones take the chunked form.  For the tokens i of a chunk, d = e^g,
// and the state S before it
//   out_i = scale * (d^(i+1) q_i S + sum_(j<=i) d^(i-j) (q_i . k_j) v_j),
//   S' = d^n S + sum_j k_j (d^(n-1-j) v_j)^T,
// four matrix products.  A request is cut into segments, which are as many as
// fill the device: one pass adds up what each segment brings to the state, a
// second one turns these into the states before the segments, and the third
// one computes the results of all segments side by side.
#include <hip/hip_runtime.h>

#include <atomic>

#include "kvr_layer.h"

namespace kvr {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kThreads = 256;
constexpr int kChunk = 64;  // tokens

// Whether the request's slots are the pool's (else that is reported).
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
  __shared__ uint64_t ahead[2][kThreads];
  const int tid = threadIdx.x;
  int bad = 0;
  uint64_t base = 0;  // segments of the requests before, and (above 32 bits) slots
  for (int r0 = 0; r0 < a.requests; r0 += kThreads) {
    const int r = r0 + tid;
    int from = 0, rows = 0, parts = 0;
    if (r < a.requests) {
      from = a.row_start[r];
      const int to = a.row_start[r + 1];
      if (from < 0 || to < from || to > a.tokens) bad = 1;
      rows = to - from;
      parts = rows > 0 ? (rows - 1) / a.segment + 1 : 1;
    }
    // (of valid lengths there are no more segments than the list has room for)
    if (__syncthreads_or(bad)) break;
    const uint64_t mine = (uint64_t)(parts > 1 ? parts : 0) << 32 | (uint32_t)parts;
    uint64_t sum = mine;
    ahead[0][tid] = sum;
    __syncthreads();
    int buffer = 0;
    for (int d = 1; d < kThreads; d <<= 1) {
      if (tid >= d) sum += ahead[buffer][tid - d];
      buffer ^= 1;
      ahead[buffer][tid] = sum;
      __syncthreads();
    }
    const uint64_t at = base + sum - mine;
    for (int i = 0; i < parts; ++i)
      a.segments[(uint32_t)at + i] = {r,     from + i * a.segment, min(a.segment, rows - i * a.segment), i,
                                      parts, (int)(at >> 32),      0,                                    0};
    base += ahead[buffer][kThreads - 1];
    __syncthreads();
  }
  bad = __syncthreads_or(bad);
  if (tid == 0) {
    *a.hdr = {(int)(uint32_t)base, bad};
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
  int row0 = (int)at, rows = 1;
  if (a.row_start) {
    if (a.hdr->rejected) {
      for (int t = (int)at; t < a.tokens; t += a.requests) fill_nan<T>(a, t, 1, head, D);
      return;
    }
    row0 = a.row_start[at];
    rows = a.row_start[at + 1] - row0;
    if (rows > kFewTokens) return;
  }
  int read, write;
  if (!slots_fit(a, (int)at, read, write)) {
    fill_nan<T>(a, row0, rows, head, D);
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
  for (int t = row0; t < row0 + rows; ++t) {
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
  if (write >= 0 && (rows || write != read)) {
    float* to = a.state + write * a.state_slot + head * a.state_head + 4 * col;
#pragma unroll
    for (int i = 0; i < kRows; ++i) *reinterpret_cast<f32x4*>(to + (down + i * kDown) * D) = state[i];
  }
}


// ---- the chunked form ----

// Numbers of 32 bits as sums of bfloat16 ones, which the matrix units multiply
// exactly: two hold 16 bits of them (results, which are rounded to 8 or 11
// bits), three all 24 (states).
__device__ __forceinline__ s16x8 rounded(f32x8 x) {
  return __builtin_bit_cast(s16x8, __builtin_convertvector(x, bf16x8));
}
__device__ __forceinline__ f32x8 widened(s16x8 x) {
  return __builtin_convertvector(__builtin_bit_cast(bf16x8, x), f32x8);
}
template <int N>
__device__ __forceinline__ void split(f32x8 x, s16x8 (&part)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    part[i] = rounded(x);
    if (i + 1 < N) x -= widened(part[i]);
  }
}
__device__ __forceinline__ f32x16 multiply(s16x8 a, s16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(s16x8 a, s16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Tokens as the matrix units take them: bfloat16 as they are, halves as two
// bfloat16 (exact but for the smallest).
struct OfBf16 {
  typedef __bf16 Type;
  static constexpr int kParts = 1;
  // the sign bits of a pair's infinities and NaN
  static __device__ __forceinline__ uint32_t odd(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
  static __device__ __forceinline__ f32x8 wide(s16x8 x) { return widened(x); }
  static __device__ __forceinline__ void parts(s16x8 x, s16x8 (&part)[1]) { part[0] = x; }
  static __device__ __forceinline__ s16x4 narrow(f32x4 x) {
    return __builtin_bit_cast(s16x4, __builtin_convertvector(x, bf16x4));
  }
};
struct OfFp16 {
  typedef _Float16 Type;
  static constexpr int kParts = 2;
  static __device__ __forceinline__ uint32_t odd(uint32_t x) { return ((x & 0x7c007c00u) + 0x04000400u) & 0x80008000u; }
  static __device__ __forceinline__ f32x8 wide(s16x8 x) {
    return __builtin_convertvector(__builtin_bit_cast(f16x8, x), f32x8);
  }
  static __device__ __forceinline__ void parts(s16x8 x, s16x8 (&part)[2]) { split<2>(wide(x), part); }
  static __device__ __forceinline__ s16x4 narrow(f32x4 x) {
    return __builtin_bit_cast(s16x4, __builtin_convertvector(x, f16x4));
  }
};

// 16-byte chunks of a row of D elements in LDS stand at chunk ^ swizzle(row):
// the reads of one chunk of 16 rows, and those of 64 bytes of four rows, fall
// on different banks (64 banks of 4 bytes).
template <int D>
__device__ __forceinline__ int swizzle(int row) {
  return D == 64 ? ((row << 1) & 4) | ((row >> 2) & 3) : ((row & 3) << 2) | ((row >> 2) & 3);
}
template <int D>
__device__ __forceinline__ int place(int row, int chunk) {
  return row * 2 * D + ((chunk ^ swizzle<D>(row)) << 4);
}

// Queries and keys stand in LDS in the order in which a state's registers
// hold its rows: of 16 elements the groups of four 0, 2, 1, 3.  A chunk of 16
// bytes, which a half wave takes as an operand, then holds elements 4 h .. and
// 8 + 4 h .. of its 16.
template <int D>
__device__ __forceinline__ void put(char* tile, int row, int chunk, s16x8 x) {
  char* to = tile + (chunk & 1) * 8;
  *(s16x4*)(to + place<D>(row, chunk & ~1)) = __builtin_shufflevector(x, x, 0, 1, 2, 3);
  *(s16x4*)(to + place<D>(row, chunk | 1)) = __builtin_shufflevector(x, x, 4, 5, 6, 7);
}

// Eight rows' elements of one column a lane: rows 16 s + 8 h .., column 32 c +
// lane % 32.  The transposing read: 16 lanes name four rows of 16 elements,
// four lanes a row, and lane i of them gets column i.
template <int D, bool ORDERED>
__device__ __forceinline__ s16x8 column(const char* tile, int s, int c, int lane) {
  const int h = lane >> 5, sl = lane & 15, g = 2 * c + ((lane >> 4) & 1);
  s16x4 x[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = s * 16 + h * 8 + j * 4 + sl / 4;
    const char* p = ORDERED ? tile + place<D>(row, 2 * g + (sl & 1)) + (sl & 2) * 4
                            : tile + place<D>(row, 2 * g + (sl & 2) / 2) + (sl & 1) * 8;
    x[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(lds_char*)p);
  }
  return __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// A lane's share of a tile of 64 tokens on its way to LDS.
template <int D>
struct Tile {
  static constexpr int kChunks = D / 8, kN = kChunk * kChunks / kThreads;
  s16x8 x[kN];

  // rows behind `rows`: zeros
  __device__ __forceinline__ void fetch(const char* from, int64_t stride, int rows, int thread) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int row = (thread + i * kThreads) / kChunks, chunk = thread % kChunks;
      x[i] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
      if (row < rows) x[i] = *(const s16x8*)(from + row * stride + chunk * 16);
    }
  }
  template <class T>
  __device__ __forceinline__ void store_ordered(char* tile, int thread) const {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int row = (thread + i * kThreads) / kChunks, chunk = thread % kChunks;
      s16x8 part[T::kParts];
      T::parts(x[i], part);
#pragma unroll
      for (int k = 0; k < T::kParts; ++k) put<D>(tile + k * kChunk * 2 * D, row, chunk, part[k]);
    }
  }
  __device__ __forceinline__ void store(char* tile, int thread) const {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int row = (thread + i * kThreads) / kChunks, chunk = thread % kChunks;
      *(s16x8*)(tile + place<D>(row, chunk)) = x[i];
    }
  }
};

template <int D, class T, bool OUT>
struct ChunkLds {
  static constexpr int kTile = kChunk * 2 * D;
  static constexpr int kKeys = T::kParts * kTile;
  static constexpr int kQueries = OUT ? T::kParts * kTile : 0;
  static constexpr int kWeights = OUT ? 2 * kChunk * 2 * kChunk : 0;
  static constexpr int kBytes = kKeys + kQueries + kTile + kWeights + 2 * kChunk * 4;
};

// One workgroup for a segment's key head.  Wave w has 32 columns of the state
// (D / 32 column groups; with two groups two waves hold the same) in registers:
// lane n column n, register i row 8 (i / 4) + 4 h + i % 4 of each 32, which is
// an operand of the products with queries as it stands.  OUT: computes the
// results from the state before the segment; else what the segment adds to it.
template <int D, class T, bool OUT>
__global__ __launch_bounds__(kThreads, 2) void linear_chunks_kernel(LinearArgs a) {
  typedef ChunkLds<D, T, OUT> L;
  constexpr int kGroups = D / 32, kRowWaves = 4 / kGroups, kRowTiles = 2 / kRowWaves, kSteps = D / 16, P = T::kParts;
  extern __shared__ __align__(16) char lds[];
  char* keys = lds;
  char* queries = keys + L::kKeys;
  char* values = queries + L::kQueries;
  char* weights = values + L::kTile;
  float* left = (float*)(weights + L::kWeights);  // d^(n - 1 - j)
  float* power = left + kChunk;                   // d^(i + 1)
  int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = wave % kGroups, rw = wave / kGroups;
  if (a.hdr->rejected) return;  // (linear_steps_kernel writes the results)
  const uint32_t at = divide(blockIdx.x, a.kv_div);
  if ((int)at >= a.hdr->segments) return;
  const int head = (int)(blockIdx.x - at * a.kv_div.d);
  const Segment seg = a.segments[at];
  const bool last = seg.index == seg.parts - 1;
  if (seg.parts == 1 && seg.rows <= kFewTokens) return;
  if (!OUT && last) return;
  int read, write;
  if (!slots_fit(a, seg.request, read, write)) {
    if (OUT) fill_nan<typename T::Type>(a, seg.row0, seg.rows, head, D);
    return;
  }
  const float g = a.log_decay[head];
  // d^m; a decay of 0 has d^0 = 1
  auto decay_by = [&](int m) { return m ? expf(g * (float)m) : 1.0f; };

  f32x16 state[kGroups];
  const float* from = nullptr;
  if (OUT && seg.parts > 1)
    from = a.added + ((int64_t)(seg.slot + seg.index) * a.kv_heads + head) * D * D;
  else if (OUT && read >= 0)
    from = a.state + read * a.state_slot + head * a.state_head;
#pragma unroll
  for (int t = 0; t < kGroups; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      state[t][i] = from ? from[(t * 32 + 8 * (i / 4) + 4 * h + i % 4) * D + c * 32 + n] : 0.0f;

  const int chunks = (seg.rows + kChunk - 1) / kChunk;
  const char* k_from = a.k + seg.row0 * a.k_tok + head * a.k_head;
  const char* v_from = a.v + seg.row0 * a.v_tok + head * a.v_head;
  const int q_head0 = head * a.share;
  const char* q_from = a.q + seg.row0 * a.q_tok + q_head0 * a.q_head;

  // d^(i - j) of the scores that this lane computes: queries i = 16 wave +
  // lane % 16, keys j = 16 t + 4 (lane / 16) + e
  float apart[4][4];
  if (OUT) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = 16 * wave + lane % 16 - (16 * t + 4 * (lane / 16) + e);
        apart[t][e] = m >= 0 ? decay_by(m) : -1.0f;
      }
  }
  if (tid < kChunk) power[tid] = decay_by(tid + 1);

  Tile<D> tk, tv, tq;
  tk.fetch(k_from, a.k_tok, seg.rows, tid);
  tv.fetch(v_from, a.v_tok, seg.rows, tid);
  if (OUT) tq.fetch(q_from, a.q_tok, seg.rows, tid);
#pragma unroll 1
  for (int chunk = 0; chunk < chunks; ++chunk) {
    const int row0 = chunk * kChunk, rows = min(kChunk, seg.rows - row0);
    // (places in LDS are computed where they are used: kept over the loop, they take more registers than there are)
    asm volatile("" : "+v"(lane), "+v"(n), "+v"(h), "+v"(tid));
    __syncthreads();  // the tiles of the chunk before are read
    tk.template store_ordered<T>(keys, tid);
    tv.store(values, tid);
    if (tid < kChunk && (chunk == 0 || rows < kChunk)) left[tid] = tid < rows ? decay_by(rows - 1 - tid) : 0.0f;
    const int next = row0 + kChunk;
    if (chunk + 1 < chunks) {
      tk.fetch(k_from + next * a.k_tok, a.k_tok, seg.rows - next, tid);
      tv.fetch(v_from + next * a.v_tok, a.v_tok, seg.rows - next, tid);
    }
    if constexpr (OUT) {
#pragma unroll 1
      for (int s = 0; s < a.share; ++s) {
        if (s) __syncthreads();
        // (nor are the state's parts kept over this loop)
#pragma unroll
        for (int t = 0; t < kGroups; ++t) asm volatile("" : "+v"(state[t]));
        asm volatile("" : "+v"(lane), "+v"(n), "+v"(h), "+v"(tid));
        tq.template store_ordered<T>(queries, tid);
        if (s + 1 < a.share)
          tq.fetch(q_from + row0 * a.q_tok + (s + 1) * a.q_head, a.q_tok, rows, tid);
        else if (chunk + 1 < chunks)
          tq.fetch(q_from + next * a.q_tok, a.q_tok, seg.rows - next, tid);
        __syncthreads();
        // scores, transposed: keys 16 t .. of the wave's 16 queries; those of later keys are 0, and of a later 32
        // queries' keys are not read
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if (t > (wave | 1)) continue;
          f32x4 x = {0, 0, 0, 0};
          if (t <= wave) {
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
              s16x8 kp[P], qp[P];
#pragma unroll
              for (int p = 0; p < P; ++p) {
                kp[p] = *(const s16x8*)(keys + p * L::kTile + place<D>(16 * t + lane % 16, 4 * k + lane / 16));
                qp[p] = *(const s16x8*)(queries + p * L::kTile + place<D>(16 * wave + lane % 16, 4 * k + lane / 16));
              }
#pragma unroll
              for (int p = 0; p < P; ++p)
#pragma unroll
                for (int r = 0; r + p < P; ++r) x = multiply(kp[p], qp[r], x);
            }
          }
          f32x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = apart[t][e] < 0.0f ? 0.0f : x[e] * apart[t][e];
          const bf16x4 hi = __builtin_convertvector(y, bf16x4);
          const bf16x4 lo = __builtin_convertvector(y - __builtin_convertvector(hi, f32x4), bf16x4);
          const int to = place<64>(16 * wave + lane % 16, 2 * t + lane / 32) + ((lane >> 4) & 1) * 8;
          *(bf16x4*)(weights + to) = hi;
          *(bf16x4*)(weights + 2 * kChunk * kChunk + to) = lo;
        }
        // the state's part of the results, transposed: queries 32 (rw * tiles + t) + n, columns as the state's rows
        f32x16 o[kRowTiles];
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          f32x8 x;
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = state[k / 2][8 * (k % 2) + e];
          s16x8 sp[2];
          split<2>(x, sp);
#pragma unroll
          for (int t = 0; t < kRowTiles; ++t) {
            const int row = 32 * (rw * kRowTiles + t) + n;
            s16x8 qp[P];
#pragma unroll
            for (int p = 0; p < P; ++p) qp[p] = *(const s16x8*)(queries + p * L::kTile + place<D>(row, 2 * k + h));
            o[t] = multiply(sp[0], qp[0], o[t]);
            o[t] = multiply(sp[1], qp[0], o[t]);
            if constexpr (P == 2) o[t] = multiply(sp[0], qp[1], o[t]);
          }
        }
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t) {
          const float by = power[32 * (rw * kRowTiles + t) + n];
#pragma unroll
          for (int i = 0; i < 16; ++i) o[t][i] *= by;
        }
        __syncthreads();
        // the chunk's own part
        i32x4 v[4];
        uint32_t some = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[k] = __builtin_bit_cast(i32x4, column<D, false>(values, k, c, lane));
#pragma unroll
          for (int e = 0; e < 4; ++e) some |= T::odd(v[k][e]);
        }
        // An infinity or NaN does not go into the products, where 0 * inf would
        // reach the rows before it.
        const bool odd = __any(some != 0);
        if (odd) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[k][e] &= (int)~((T::odd(v[k][e]) >> 15) * 0xffffu);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          s16x8 vp[P];
          T::parts(__builtin_bit_cast(s16x8, v[k]), vp);
#pragma unroll
          for (int t = 0; t < kRowTiles; ++t) {
            const int tile = rw * kRowTiles + t;
            if (k > 2 * tile + 1) continue;
            const int p = place<64>(32 * tile + n, 2 * k + h);
            const s16x8 hi = *(const s16x8*)(weights + p), lo = *(const s16x8*)(weights + 2 * kChunk * kChunk + p);
            o[t] = multiply(vp[0], hi, o[t]);
            o[t] = multiply(vp[0], lo, o[t]);
            if constexpr (P == 2) o[t] = multiply(vp[1], hi, o[t]);
          }
        }
        if (odd) {
#pragma unroll 1
          for (int j = 0; j < rows; ++j) {
            const char* x_at = values + j * 2 * D;
            const char* w_at = weights + (j % 8) * 2;
            int sw = swizzle<D>(j) << 4, first = c * 64 + 8 * h, chunk_at = (j / 8) << 4;
            asm volatile("" : "+v"(sw), "+v"(first), "+v"(chunk_at));
#pragma unroll
            for (int t = 0; t < kRowTiles; ++t) {
              const int row = 32 * (rw * kRowTiles + t) + n;
              const char* p = w_at + row * 2 * kChunk + (chunk_at ^ swizzle<64>(row) << 4);
              const float w = j <= row ? (float)*(const __bf16*)p + (float)*(const __bf16*)(p + 2 * kChunk * kChunk) : 0.0f;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const s16x4 x = *(const s16x4*)(x_at + (((first & ~15) + i * 16) ^ sw) + (first & 8));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const bool here = T::odd(x[e] & 0xffff) && j <= row;
                  o[t][4 * i + e] += here ? w * (float)__builtin_bit_cast(typename T::Type, (short)x[e]) : 0.0f;
                }
              }
            }
          }
        }
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t) {
          const int row = 32 * (rw * kRowTiles + t) + n;
          if (row < rows) {
            char* to = a.out + (seg.row0 + row0 + row) * a.o_tok + (q_head0 + s) * a.o_head + (c * 32 + 4 * h) * 2;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f32x4 x = {o[t][4 * i] * a.scale, o[t][4 * i + 1] * a.scale, o[t][4 * i + 2] * a.scale,
                               o[t][4 * i + 3] * a.scale};
              *(s16x4*)(to + i * 16) = T::narrow(x);
            }
          }
        }
      }
    } else {
      __syncthreads();
    }
    // the state behind the chunk
    const float by = rows == kChunk ? power[kChunk - 1] : power[rows - 1];
#pragma unroll
    for (int t = 0; t < kGroups; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) state[t][i] *= by;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f32x8 x = T::wide(column<D, false>(values, k, c, lane));
      const f32x4 w0 = *(const f32x4*)(left + 16 * k + 8 * h), w1 = *(const f32x4*)(left + 16 * k + 8 * h + 4);
      x *= __builtin_shufflevector(w0, w1, 0, 1, 2, 3, 4, 5, 6, 7);
      s16x8 vp[3];
      split<3>(x, vp);
#pragma unroll
      for (int t = 0; t < kGroups; ++t) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const s16x8 kp = column<D, true>(keys + p * L::kTile, k, t, lane);
#pragma unroll
          for (int r = 0; r + p < 3; ++r) state[t] = multiply(kp, vp[r], state[t]);
        }
      }
    }
  }

  float* to = nullptr;
  if (!OUT)
    to = a.added + ((int64_t)(seg.slot + seg.index + 1) * a.kv_heads + head) * D * D;
  else if (last && write >= 0)
    to = a.state + write * a.state_slot + head * a.state_head;
  if (to && rw == 0) {
#pragma unroll
    for (int t = 0; t < kGroups; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) to[(t * 32 + 8 * (i / 4) + 4 * h + i % 4) * D + c * 32 + n] = state[t][i];
  }
}

// For each request of several segments, what they add becomes the states
// before them, in place (the first one's is copied: the last segment may write
// the slot that it is read from).  blockIdx.y: part of the state.
template <int D>
__global__ __launch_bounds__(kThreads) void linear_states_kernel(LinearArgs a) {
  if (a.hdr->rejected) return;
  const uint32_t at = divide(blockIdx.x, a.kv_div);
  if ((int)at >= a.hdr->segments) return;
  const int head = (int)(blockIdx.x - at * a.kv_div.d);
  const Segment seg = a.segments[at];
  if (seg.index || seg.parts == 1) return;
  const int read = a.read[seg.request];
  if (read < -1 || read >= a.slots) return;  // (reported by linear_chunks_kernel)
  const int64_t place = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * 4;
  f32x4 state = {0, 0, 0, 0};
  if (read >= 0) state = *(const f32x4*)(a.state + read * a.state_slot + head * a.state_head + place);
  const float by = expf(a.log_decay[head] * (float)a.segment);
  const int64_t next = (int64_t)a.kv_heads * D * D;
  float* to = a.added + ((int64_t)seg.slot * a.kv_heads + head) * D * D + place;
  *(f32x4*)to = state;
  for (int i = 1; i < seg.parts; ++i) {
    to += next;
    const f32x4 x = *(const f32x4*)to;
#pragma unroll
    for (int e = 0; e < 4; ++e) state[e] = __builtin_fmaf(by, state[e], x[e]);
    *(f32x4*)to = state;
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

template <int D, class T, bool OUT>
hipError_t launch_chunks(const LinearArgs& a, hipStream_t st) {
  constexpr int bytes = ChunkLds<D, T, OUT>::kBytes;
  const hipError_t e = allow_lds<linear_chunks_kernel<D, T, OUT>>(bytes);
  if (e != hipSuccess) return e;
  linear_chunks_kernel<D, T, OUT><<<(uint32_t)a.segment_cap * (uint32_t)a.kv_heads, kThreads, bytes, st>>>(a);
  return hipGetLastError();
}

template <int D, class T>
hipError_t launch(const LinearArgs& a, hipStream_t st) {
  hipError_t e = hipSuccess;
  if (a.row_start && a.tokens > kFewTokens) {
    if (a.tokens > a.segment) {
      e = launch_chunks<D, T, false>(a, st);
      if (e != hipSuccess) return e;
      linear_states_kernel<D><<<dim3((uint32_t)a.segment_cap * (uint32_t)a.kv_heads, D * D / 4 / kThreads), kThreads, 0, st>>>(a);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    e = launch_chunks<D, T, true>(a, st);
    if (e != hipSuccess) return e;
  }
  linear_steps_kernel<D, typename T::Type><<<(uint32_t)a.requests * (uint32_t)a.kv_heads, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, bool fp16, hipStream_t st) {
  if (a.row_start) {
    linear_plan_kernel<<<1, kThreads, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dim == 64) return fp16 ? launch<64, OfFp16>(a, st) : launch<64, OfBf16>(a, st);
  return fp16 ? launch<128, OfFp16>(a, st) : launch<128, OfBf16>(a, st);
}

}  // namespace kvr
