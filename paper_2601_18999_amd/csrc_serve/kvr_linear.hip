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
// one computes the results of all segments side by side.  One request of 9,216
// tokens, 32 heads of 128: 38 + 12 + 84 us, where the bytes of the three take 30
// + 13 + 60.  In the last one the matrix units are busy for 28% of the time and
// the vector units, which split the state and weigh the scores, for 38%; two
// waves a SIMD, which is what their registers allow, hide little of the one
// behind the other, or of the loads.
#include <hip/hip_runtime.h>

#include "kvr_layer.h"
#include "kvr_lds.h"

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

constexpr int kThreads = 256;
constexpr int kChunk = 64;  // tokens

// Whether the request's slots are the pool's (else that is reported).
__device__ __forceinline__ bool slots_fit(const LinearArgs& a, int read, int write) {
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

// Whether row_start is not valid: of the plan, or, where there is none (few
// requests, none of which is cut), checked by every workgroup.
__device__ __forceinline__ bool rejected(const LinearArgs& a) {
  if (a.planned) return a.hdr->rejected;
  int bad = 0;
  for (int r = threadIdx.x; r < a.requests; r += kThreads) {
    const int from = a.row_start[r], to = a.row_start[r + 1];
    bad |= from < 0 || to < from || to > a.tokens;
  }
  bad = __syncthreads_or(bad);
  if (bad && a.status && threadIdx.x == 0) atomicOr(a.status, (uint32_t)KVR_DEV_BAD_LENGTH);
  return bad;
}

// Checks row_start and lists the segments: those that others follow, which are
// full (the requests' first ones before the others), then the last ones, the
// longest first (the workgroups that start last then have little to do).  One
// workgroup.
__global__ __launch_bounds__(kThreads) void linear_plan_kernel(LinearArgs a) {
  constexpr int kKinds = 64;  // by chunks, the last one all longer ones
  __shared__ int place[kKinds], followed, cut, slots;
  const int tid = threadIdx.x;
  if (tid < kKinds) place[tid] = 0;
  if (tid == 0) followed = cut = slots = 0;
  __syncthreads();
  auto kind = [&](int rows) { return kKinds - 1 - min((rows + kChunk - 1) / kChunk, kKinds - 1); };
  int bad = 0;
  // (requests of a few tokens are not listed: linear_steps_kernel takes them)
  auto each = [&](auto found) {
    for (int r = tid; r < a.requests; r += kThreads) {
      const int from = a.row_start[r], to = a.row_start[r + 1];
      if (from < 0 || to < from || to > a.tokens)
        bad = 1;
      else if (a.few < 0 || to - from > a.few)
        found(r, from, to - from, to > from ? (to - from - 1) / a.segment + 1 : 1);
    }
  };
  each([&](int, int, int rows, int parts) {
    if (parts > 1) {
      atomicAdd(&followed, parts - 1);
      atomicAdd(&cut, 1);
    }
    atomicAdd(&place[kind(rows - (parts - 1) * a.segment)], 1);
  });
  bad = __syncthreads_or(bad);
  int all = 0;
  const int first = followed, firsts = cut;
  __syncthreads();
  if (tid == 0) {
    followed = firsts;
    cut = 0;
  }
  if (tid < kKinds) {
    const int mine = place[tid];
    int sum = mine;
#pragma unroll
    for (int d = 1; d < kKinds; d <<= 1) {
      const int x = __shfl_up(sum, d);
      if (tid >= d) sum += x;
    }
    place[tid] = first + sum - mine;
    all = first + sum;
  }
  __syncthreads();
  if (tid == kKinds - 1) {
    *a.hdr = {all, first, firsts, bad};
    if (bad && a.status) atomicOr(a.status, (uint32_t)KVR_DEV_BAD_LENGTH);
  }
  if (bad) return;
  each([&](int r, int from, int rows, int parts) {
    const int slot = parts > 1 ? atomicAdd(&slots, parts) : 0;
    if (parts > 1) {
      a.segments[atomicAdd(&cut, 1)] = {r, from, a.segment, 0, parts, slot};
      const int full = atomicAdd(&followed, parts - 2) - 1;
      for (int i = 1; i < parts - 1; ++i)
        a.segments[full + i] = {r, from + i * a.segment, a.segment, i, parts, slot};
    }
    const int rest = rows - (parts - 1) * a.segment;
    a.segments[atomicAdd(&place[kind(rest)], 1)] = {r, from + rows - rest, rest, parts - 1, parts, slot};
  });
}

// The recurrent form: one workgroup for a request's key head, which holds the
// state in registers: thread t columns 4 (t % (D / 4)) .. + 3 of every
// (1024 / D)th row, and passes over the tokens.  The states' bytes bound it (64
// requests of one token, 32 heads of 128: 268 MB, 55 us, 4.9 TB/s); for more
// tokens what comes next is on its way, and the places in LDS are taken in turn
// (256 requests of 8 tokens, 32 heads of 64: 117 -> 104 us).
template <int D, class T>
__global__ __launch_bounds__(kThreads) void linear_steps_kernel(LinearArgs a) {
  constexpr int kAcross = D / 4, kDown = kThreads / kAcross, kRows = D / kDown;
  __shared__ float keys[2][D], queries[2][D];  // of tokens, and of their heads, in turn
  __shared__ f32x4 part[2][kDown][kAcross];
  const int tid = threadIdx.x, col = tid % kAcross, down = tid / kAcross;
  const uint32_t at = divide(blockIdx.x, a.kv_div);
  const int head = (int)(blockIdx.x - at * a.kv_div.d);
  int row0 = (int)at, rows = 1;
  const int read = a.read[at], write = a.write[at];  // (on their way while row_start is checked)
  const float log_decay = a.log_decay[head];
  if (a.row_start) {
    row0 = a.row_start[at];
    rows = a.row_start[at + 1] - row0;
    if (rejected(a)) {
      for (int t = (int)at; t < a.tokens; t += a.requests) fill_nan<T>(a, t, 1, head, D);
      return;
    }
    if (rows > a.few) return;
  }
  if (!slots_fit(a, read, write)) {
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
  const float decay = expf(log_decay);
  // what comes next is on its way (behind the last one that again)
  struct Four {
    T e[4];
  };
  auto key = [&](int t) { return reinterpret_cast<const T*>(a.k + t * a.k_tok + head * a.k_head)[tid % D]; };
  auto value = [&](int t) { return *reinterpret_cast<const Four*>(a.v + t * a.v_tok + head * a.v_head + 8 * col); };
  auto query = [&](int t, int h) {
    return reinterpret_cast<const T*>(a.q + t * a.q_tok + (head * a.share + h) * a.q_head)[tid % D];
  };
  const int last = row0 + rows - 1;
  T next_key, next_query;
  Four next_value;
  if (rows) {
    next_key = key(row0);
    next_value = value(row0);
    next_query = query(row0, 0);
  }
  int turn = 0;
#pragma unroll 1
  for (int t = row0; t <= last; ++t) {
    const int then = min(t + 1, last);
    if (tid < D) keys[t & 1][tid] = (float)next_key;
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)next_value.e[e];
    next_key = key(then);
    next_value = value(then);
#pragma unroll 1
    for (int h = 0; h < a.share; ++h, turn ^= 1) {
      if (tid < D) queries[turn][tid] = (float)next_query * a.scale;
      const bool same = h + 1 < a.share;
      next_query = query(same ? t : then, same ? h + 1 : 0);
      __syncthreads();
      if (h == 0) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const float k = keys[t & 1][down + i * kDown];
#pragma unroll
          for (int e = 0; e < 4; ++e) state[i][e] = __builtin_fmaf(k, v[e], decay * state[i][e]);
        }
      }
      f32x4 o = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const float q = queries[turn][down + i * kDown];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(q, state[i][e], o[e]);
      }
      part[turn][down][col] = o;
      __syncthreads();
      if (tid < D) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kDown; ++i) sum += part[turn][i][tid / 4][tid % 4];
        reinterpret_cast<T*>(a.out + t * a.o_tok + (head * a.share + h) * a.o_head)[tid] = (T)sum;
      }
    }
  }
  if (write >= 0 && (rows || write != read)) {
    float* to = a.state + write * a.state_slot + head * a.state_head + 4 * col;
#pragma unroll
    for (int i = 0; i < kRows; ++i) *reinterpret_cast<f32x4*>(to + (down + i * kDown) * D) = state[i];
  }
}

// ---- the chunked form ----

// Numbers of 32 bits as sums of bfloat16 ones, which the matrix units multiply
// exactly: the first takes the leading 8 bits, the second the next 8, and so
// three hold all 24 (states); of two the second is rounded, so they hold 16
// (results, which are rounded to 8 or 11 bits).
__device__ __forceinline__ float leading(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ int packed(float x, float y) {  // their leading halves
  return (int)__builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
}
template <int N>
__device__ __forceinline__ void split(f32x8 x, s16x8 (&part)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if (N == 2 && k == 1) {
      part[k] = __builtin_bit_cast(s16x8, __builtin_convertvector(x, bf16x8));
    } else {
      i32x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = packed(x[2 * i], x[2 * i + 1]);
      part[k] = __builtin_bit_cast(s16x8, y);
    }
    if (k + 1 < N) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] -= leading(x[i]);
    }
  }
}
__device__ __forceinline__ f32x16 multiply(s16x8 a, s16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}
__device__ __forceinline__ f32x4 multiply(s16x8 a, s16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}

// Tokens as the matrix units take them: bfloat16 as they are, halves as two
// bfloat16, exactly.  (Of the products of such pairs that of the two second parts
// is left out, which is below 2^-14 of the whole; of what is added to a state,
// where one factor has three parts, below 2^-22.)
struct OfBf16 {
  typedef __bf16 Type;
  static constexpr int kParts = 1;
  // the sign bits of a pair's infinities and NaN
  static __device__ __forceinline__ uint32_t odd(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
  static __device__ __forceinline__ f32x8 wide(s16x8 x) {
    return __builtin_convertvector(__builtin_bit_cast(bf16x8, x), f32x8);
  }
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

// A tile of 64 tokens in LDS: rows of D elements, 64 bytes apart beyond their
// own, and 16 more after every four.  The reads of 16 bytes of 16 rows, and
// those of 64 bytes of four rows, then fall on different banks (64 banks of 4
// bytes), and every address is one of the lane and a constant.
template <int D>
struct Rows {
  static constexpr int kPitch = 2 * D + 64, kBytes = kChunk * kPitch + kChunk / 4 * 16;
  static constexpr int of(int rows) { return rows * kPitch + rows / 4 * 16; }  // multiples of four rows
  static __device__ __forceinline__ int at(int row) { return row * kPitch + row / 4 * 16; }
};

// Eight rows' elements of one column a lane: rows 16 s + 8 h .., column 32 c +
// lane % 32.  The transposing read: 16 lanes name four rows of 16 elements,
// four lanes a row, and lane i of them gets column i.  `at`: column_place.
// STATE: of 16 columns the groups of four 0, 2, 1, 3, so that of the products'
// results, whose rows those columns are, a lane holds rows 16 s + 8 h .. + 7 in
// registers 8 s .., as an operand has them.
template <int D, bool STATE>
__device__ __forceinline__ int column_place(int lane) {
  const int sl = lane & 15;
  return Rows<D>::at((lane >> 5) * 8 + sl / 4) + ((lane >> 4) & 1) * 32 +
         (STATE ? (sl & 1) * 16 + (sl & 2) * 4 : (sl & 3) * 8);
}
template <int D>
__device__ __forceinline__ s16x8 column(const char* tile, int at, int s, int c) {
  s16x4 x[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
    x[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(
        lds_char*)(tile + at + Rows<D>::of(16 * s + 4 * j) + c * 64));
  return __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// A lane's share of a tile on its way to LDS: one 16-byte chunk of every
// kStepRows-th row.
template <int D>
struct Tile {
  static constexpr int kChunks = D / 8, kStepRows = kThreads / kChunks, kN = kChunk / kStepRows;
  s16x8 x[kN];

  // `from`: the lane's chunk of row 0.  Rows behind `last` are that one again:
  // nothing branches here, as the compiler waits for loads that a branch may
  // have made before it goes on.
  __device__ __forceinline__ void fetch(const char* from, int64_t stride, int row, int last) {
#pragma unroll
    for (int i = 0; i < kN; ++i) x[i] = *(const s16x8*)(from + min(row + i * kStepRows, last) * stride);
  }
  // in as many parts as the products take (one tile behind the other)
  template <class T>
  __device__ __forceinline__ void store_parts(char* tile, int thread) const {
    char* to = tile + Rows<D>::at(thread / kChunks) + thread % kChunks * 16;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      s16x8 part[T::kParts];
      T::parts(x[i], part);
#pragma unroll
      for (int k = 0; k < T::kParts; ++k) *(s16x8*)(to + Rows<D>::of(i * kStepRows) + k * Rows<D>::kBytes) = part[k];
    }
  }
  __device__ __forceinline__ void store(char* tile, int thread) const {
    char* to = tile + Rows<D>::at(thread / kChunks) + thread % kChunks * 16;
#pragma unroll
    for (int i = 0; i < kN; ++i) *(s16x8*)(to + Rows<D>::of(i * kStepRows)) = x[i];
  }
};

// The scores of a chunk: rows of 64, 16 bytes apart beyond their own.
constexpr int kScorePitch = 2 * kChunk + 16, kScores = kChunk * kScorePitch;

template <int D, class T, bool OUT>
struct ChunkLds {
  static constexpr int kTile = Rows<D>::kBytes;
  static constexpr int kKeys = T::kParts * kTile;
  static constexpr int kQueries = OUT ? T::kParts * kTile : 0;
  static constexpr int kWeights = OUT ? 2 * kScores : 0;
  static constexpr int kBytes = kKeys + kQueries + kTile + kWeights + 2 * kChunk * 4;
};
static_assert(2 * ChunkLds<128, OfBf16, true>::kBytes <= 160 * 1024, "two workgroups a compute unit");

// What is read from LDS above is on its way before anything below begins: a
// read takes as long as several products, and left to itself the compiler puts
// it right before its use.
__device__ __forceinline__ void ahead() { __builtin_amdgcn_sched_barrier(0); }

// One workgroup for a segment's key head.  Wave w has 32 columns of the state
// (D / 32 column groups; with two groups two waves hold the same) in registers:
// lane n column n, register i row 16 (i / 8) + 8 h + i % 8 of each 32, which is
// an operand of the products with queries as it stands.  OUT: computes the
// results from the state before the segment; else what the segment adds to it.
template <int D, class T, bool OUT>
__global__ __launch_bounds__(kThreads, 2) void linear_chunks_kernel(LinearArgs a) {
  typedef ChunkLds<D, T, OUT> L;
  constexpr bool kEarly = D == 64;  // (heads of 128 leave no registers for it)
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
  const uint32_t at = divide(blockIdx.x, a.kv_div);
  const int head = (int)(blockIdx.x - at * a.kv_div.d);
  const float g = a.log_decay[head];
  Segment seg;
  int read = -1, write = -1;
  if (OUT && !a.planned) {  // (on their way while row_start is checked)
    const int row0 = a.row_start[at];
    seg = {(int)at, row0, a.row_start[at + 1] - row0, 0, 1, 0};
    read = a.read[at];
    write = a.write[at];
  }
  if (rejected(a)) {  // (with few >= 0 linear_steps_kernel writes the results)
    if (OUT && a.few < 0 && blockIdx.y == 0)
      for (int t = (int)at; t < a.tokens; t += a.segment_cap) fill_nan<typename T::Type>(a, t, 1, head, D);
    return;
  }
  if (!OUT || a.planned) {
    const int all = OUT ? a.hdr->segments : a.hdr->followed;
    int from = (int)at;
    if (from >= all) return;
    // The list is the longest first.  Where the device takes all at once, two a
    // compute unit, the second ones are the shortest first.
    const int alone = kComputeUnits / a.kv_heads;
    if (OUT && from >= alone && all * a.kv_heads <= kLinearSlots) from = all - 1 - (from - alone);
    seg = a.segments[from];
    read = a.read[seg.request];
    write = a.write[seg.request];
  } else if (a.few >= 0 && seg.rows <= a.few) {
    return;
  }
  const int team = OUT ? (int)blockIdx.y : 0;
  if (!slots_fit(a, read, write)) {
    if (OUT && team == 0) fill_nan<typename T::Type>(a, seg.row0, seg.rows, head, D);
    return;
  }
  // The queries' heads of the key head; with several teams each has its share
  // of them, and all keep the state.  (Where a request's state is read and
  // written in one place, one team has all heads: it could be written before
  // another has read it.)
  const int teams = seg.parts == 1 && read == write && read >= 0 ? 1 : OUT ? a.teams : 1;
  if (team >= teams) return;
  const int s0 = a.share / teams * team, s1 = s0 + a.share / teams;
  // d^m; a decay of 0 has d^0 = 1
  auto decay_by = [&](int m) { return m ? expf(g * (float)m) : 1.0f; };

  f32x16 state[kGroups];
  const float* from = nullptr;
  if (OUT && seg.parts > 1)
    from = a.added + ((int64_t)(seg.slot + seg.index) * a.kv_heads + head) * D * D;
  else if (OUT && read >= 0)
    from = a.state + read * a.state_slot + head * a.state_head;
  const int mine = 8 * h * D + c * 32 + n;  // the lane's first value
  if (from) {
#pragma unroll
    for (int t = 0; t < kGroups; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) state[t][i] = from[mine + (t * 32 + 16 * (i / 8) + i % 8) * D];
  } else {
#pragma unroll
    for (int t = 0; t < kGroups; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) state[t][i] = 0.0f;
  }
  if (tid < kChunk) power[tid] = decay_by(tid + 1);

  const int chunks = (seg.rows + kChunk - 1) / kChunk;
  // Whether the state behind the segment is of use; else the last chunk need not
  // add to it (16 requests of 512 tokens, 32 / 4 heads of 128, heads side by
  // side: 83 -> 79 us).  (To leave out the third part of the values too, where
  // the state is for results only, costs the others more than it saves.)
  const bool kept = !OUT || (team == 0 && seg.index == seg.parts - 1 && write >= 0);
  const int q_head0 = head * a.share + s0;
  const int chunk16 = tid % Tile<D>::kChunks * 16, last = seg.rows - 1;
  const char* k_from = a.k + seg.row0 * a.k_tok + head * a.k_head + chunk16;
  const char* v_from = a.v + seg.row0 * a.v_tok + head * a.v_head + chunk16;
  const char* q_from = a.q + seg.row0 * a.q_tok + q_head0 * a.q_head + chunk16;

  Tile<D> tk, tv, tq;
  if (chunks) {
    const int row = tid / Tile<D>::kChunks;
    tk.fetch(k_from, a.k_tok, row, last);
    tv.fetch(v_from, a.v_tok, row, last);
    if (OUT) tq.fetch(q_from, a.q_tok, row, last);
  }
  // scale * d^(i - j) of the scores that this lane computes: queries i = 16
  // wave + lane % 16, keys j = 16 t + 4 (lane / 16) + e, and of those which are
  // not later ones (bit 4 t + e)
  float apart[4][4];
  int earlier = 0;
  if (OUT) {
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = 16 * wave + lane % 16 - (16 * t + 4 * (lane / 16) + e);
        apart[t][e] = m > 0 ? power[m - 1] * a.scale : a.scale;
        earlier |= (m >= 0) << (4 * t + e);
      }
  }
  int chunk = 0, rows = min(kChunk, seg.rows);
  auto to_lds = [&]() {
    tk.template store_parts<T>(keys, tid);
    tv.store(values, tid);
    if (OUT) tq.template store_parts<T>(queries, tid);
    if (tid < kChunk && (chunk == 0 || rows < kChunk)) left[tid] = tid < rows ? decay_by(rows - 1 - tid) : 0.0f;
  };
  if (chunks) to_lds();
#pragma unroll 1
  while (chunk < chunks) {
    const int row0 = chunk * kChunk;
    // (places in LDS are computed where they are used: kept over the loop, they take more registers than there are)
    asm volatile("" : "+v"(lane), "+v"(n), "+v"(h), "+v"(tid));
    // the next chunk's (behind the last one its last row), and the queries of
    // the next head
    const int row = row0 + tid / Tile<D>::kChunks;
    tk.fetch(k_from, a.k_tok, row + kChunk, last);
    tv.fetch(v_from, a.v_tok, row + kChunk, last);
    auto fetch_queries = [&](int s) {
      const bool here = s < s1 - s0;
      tq.fetch(q_from + (here ? s * a.q_head : 0), a.q_tok, here ? row : row + kChunk, last);
    };
    if (OUT) fetch_queries(1);
    __syncthreads();
    const int v_place = column_place<D, false>(lane) + c * 64;
    if constexpr (OUT) {
#pragma unroll 1
      for (int s = 0;; ++s) {
        // (nor are the state's parts kept over this loop)
#pragma unroll
        for (int t = 0; t < kGroups; ++t) asm volatile("" : "+v"(state[t]));
        asm volatile("" : "+v"(lane), "+v"(n), "+v"(h), "+v"(tid));
        // scores, transposed: keys 16 t .. of the wave's 16 queries; those of later keys are 0, and of a later 32
        // queries' keys are not read
        const char* k_at = keys + Rows<D>::at(lane % 16) + lane / 16 * 16;
        const char* q_at = queries + Rows<D>::at(lane % 16) + lane / 16 * 16 + wave * Rows<D>::of(16);
        char* w_to = weights + (16 * wave + lane % 16) * kScorePitch + lane / 16 * 8;
        s16x8 qp[D / 32][P], kp[2][D / 32][P];
        auto read_keys = [&](int t) {
#pragma unroll
          for (int k = 0; k < D / 32; ++k)
#pragma unroll
            for (int p = 0; p < P; ++p)
              kp[t & 1][k][p] = *(const s16x8*)(k_at + p * L::kTile + Rows<D>::of(16 * t) + k * 64);
        };
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
#pragma unroll
          for (int p = 0; p < P; ++p) qp[k][p] = *(const s16x8*)(q_at + p * L::kTile + k * 64);
        if (kEarly) read_keys(0);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if (t > (wave | 1)) continue;
          f32x4 x = {0, 0, 0, 0};
          if (kEarly && t < wave) read_keys((t + 1) & 3);
          if (kEarly) ahead();
          if (!kEarly && t <= wave) read_keys(t);
          if (t <= wave) {
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
#pragma unroll
              for (int p = 0; p < P; ++p)
#pragma unroll
                for (int r = 0; r + p < P; ++r) x = multiply(kp[t & 1][k][p], qp[k][r], x);
          }
          f32x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            y[e] = x[e] * apart[t][e];
            if (t >= wave) y[e] = earlier >> (4 * t + e) & 1 ? y[e] : 0.0f;
          }
          f32x4 rest;
#pragma unroll
          for (int e = 0; e < 4; ++e) rest[e] = y[e] - leading(y[e]);
          *(i32x2*)(w_to + t * 32) = i32x2{packed(y[0], y[1]), packed(y[2], y[3])};
          *(bf16x4*)(w_to + t * 32 + kScores) = __builtin_convertvector(rest, bf16x4);
        }
        // the state's part of the results, transposed: queries 32 (rw * tiles + t) + n, columns as the state's rows
        f32x16 o[kRowTiles];
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
        const char* q_row = queries + Rows<D>::at(n) + h * 16 + rw * kRowTiles * Rows<D>::of(32);
        s16x8 qs[2][kRowTiles][P];
        auto read_queries = [&](int k) {
#pragma unroll
          for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
            for (int p = 0; p < P; ++p)
              qs[k & 1][t][p] = *(const s16x8*)(q_row + p * L::kTile + Rows<D>::of(32 * t) + k * 32);
        };
        read_queries(0);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          if (k + 1 < kSteps) read_queries(k + 1);
          ahead();
          f32x8 x;
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = state[k / 2][8 * (k % 2) + e];
          s16x8 sp[2];
          split<2>(x, sp);
#pragma unroll
          for (int t = 0; t < kRowTiles; ++t) {
            o[t] = multiply(sp[0], qs[k & 1][t][0], o[t]);
            o[t] = multiply(sp[1], qs[k & 1][t][0], o[t]);
            if constexpr (P == 2) o[t] = multiply(sp[0], qs[k & 1][t][1], o[t]);
          }
        }
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t) {
          const float by = power[32 * (rw * kRowTiles + t) + n] * a.scale;
#pragma unroll
          for (int i = 0; i < 16; ++i) o[t][i] *= by;
        }
        __syncthreads();
        // the chunk's own part
        i32x4 v[4];
        s16x8 wp[2][kRowTiles][2];
        const char* w_row = weights + (rw * kRowTiles * 32 + n) * kScorePitch + h * 16;
        auto read_weights = [&](int k) {
#pragma unroll
          for (int t = 0; t < kRowTiles; ++t) {
            if (k > 2 * (rw * kRowTiles + t) + 1) continue;
#pragma unroll
            for (int p = 0; p < 2; ++p)
              wp[k & 1][t][p] = *(const s16x8*)(w_row + t * 32 * kScorePitch + k * 32 + p * kScores);
          }
        };
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __builtin_bit_cast(i32x4, column<D>(values, v_place, k, 0));
        read_weights(0);
        ahead();
        uint32_t some = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) some |= T::odd(v[k][e]);
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
          if (k + 1 < 4) read_weights(k + 1);
          ahead();
          s16x8 vp[P];
          T::parts(__builtin_bit_cast(s16x8, v[k]), vp);
#pragma unroll
          for (int t = 0; t < kRowTiles; ++t) {
            if (k > 2 * (rw * kRowTiles + t) + 1) continue;
            o[t] = multiply(vp[0], wp[k & 1][t][0], o[t]);
            o[t] = multiply(vp[0], wp[k & 1][t][1], o[t]);
            if constexpr (P == 2) o[t] = multiply(vp[1], wp[k & 1][t][0], o[t]);
          }
        }
        if (odd) {
#pragma unroll 1
          for (int j = 0; j < rows; ++j) {
            const char* x_at = values + Rows<D>::at(j) + c * 64 + h * 8;
#pragma unroll
            for (int t = 0; t < kRowTiles; ++t) {
              const int row = 32 * (rw * kRowTiles + t) + n;
              const char* p = weights + row * kScorePitch + j * 2;
              const float w = j <= row ? (float)*(const __bf16*)p + (float)*(const __bf16*)(p + kScores) : 0.0f;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const s16x4 x = *(const s16x4*)(x_at + i * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const bool here = T::odd(x[e] & 0xffff) && j <= row;
                  o[t][4 * i + e] += here ? w * (float)__builtin_bit_cast(typename T::Type, (short)x[e]) : 0.0f;
                }
              }
            }
          }
        }
        // A wave's results, 64 bytes of each row, go through the queries' place
        // (which all waves have read), so that four lanes write a row's.
        const int first = rw * kRowTiles * 32;
        char* r_to = queries + Rows<D>::at(n) + rw * kRowTiles * Rows<D>::of(32) + c * 64 + h * 8;
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *(s16x4*)(r_to + Rows<D>::of(32 * t) + i * 16) =
                T::narrow(f32x4{o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]});
        // (rows behind the end: the last one again)
        const char* r_from = queries + c * 64 + lane % 4 * 16;
        char* to = a.out + (seg.row0 + row0) * a.o_tok + (q_head0 + s) * a.o_head + c * 64 + lane % 4 * 16;
        if (kRowWaves == 1 || first < rows) {
#pragma unroll
          for (int i = 0; i < 2 * kRowTiles; ++i) {
            const int r = min(first + 16 * i + lane / 4, rows - 1);
            const s16x8 x = *(const s16x8*)(r_from + Rows<D>::at(r));
            __builtin_memcpy(to + r * a.o_tok, &x, sizeof(x));
          }
        }
        if (s + 1 == s1 - s0) break;
        __syncthreads();
        tq.template store_parts<T>(queries, tid);
        fetch_queries(s + 2);
        __syncthreads();
      }
    }
    // the state behind the chunk
    if (!kept && chunk + 1 == chunks) break;
    const int k_place = column_place<D, true>(lane);
    s16x8 vs[2], ks[2][kGroups][P];
    f32x4 ws[2];
    auto read_update = [&](int k) {
      vs[k & 1] = column<D>(values, v_place, k, 0);
      ws[0] = *(const f32x4*)(left + 16 * k + 8 * h);
      ws[1] = *(const f32x4*)(left + 16 * k + 8 * h + 4);
#pragma unroll
      for (int t = 0; t < kGroups; ++t)
#pragma unroll
        for (int p = 0; p < P; ++p) ks[k & 1][t][p] = column<D>(keys + p * L::kTile, k_place, k, t);
    };
    read_update(0);
    const float by = power[rows - 1];
#pragma unroll
    for (int t = 0; t < kGroups; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) state[t][i] *= by;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f32x8 x = T::wide(vs[k & 1]);
      x *= __builtin_shufflevector(ws[0], ws[1], 0, 1, 2, 3, 4, 5, 6, 7);
      if (k + 1 < 4) read_update(k + 1);
      ahead();
      s16x8 vp[3];
      split<3>(x, vp);
#pragma unroll
      for (int r = 0; r < 3; ++r)
#pragma unroll
        for (int t = 0; t < kGroups; ++t)
#pragma unroll
          for (int p = 0; p < P; ++p)
            if (r + p < 3) state[t] = multiply(ks[k & 1][t][p], vp[r], state[t]);
    }
    if (++chunk == chunks) break;
    rows = min(kChunk, seg.rows - chunk * kChunk);
    __syncthreads();  // the tiles are read
    to_lds();
  }

  // (read again: kept over the loop, they are more than the scalar registers hold)
  typedef const __attribute__((address_space(4))) LinearArgs Args;
  const Args* late = (const Args*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(late));
  const Args& z = *late;
  float* to = nullptr;
  if (!OUT) {
    to = z.added + ((int64_t)(seg.slot + seg.index + 1) * z.kv_heads + head) * D * D;
  } else if (team == 0 && seg.index == seg.parts - 1) {
    const int into = z.write[seg.request];
    if (into >= 0 && (seg.rows || into != z.read[seg.request]))
      to = z.state + into * z.state_slot + head * z.state_head;
  }
  if (to && rw == 0) {
#pragma unroll
    for (int t = 0; t < kGroups; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) to[mine + (t * 32 + 16 * (i / 8) + i % 8) * D] = state[t][i];
  }
}

// For each request of several segments, what they add becomes the states
// before them, in place (the first one's is copied: the last segment may write
// the slot that it is read from).  blockIdx.y: part of the state.  Memory bounds
// it: 17 segments of 32 heads of 128, 67 MB, 12 us (16 with the loads one after
// the other).
template <int D>
__global__ __launch_bounds__(kThreads) void linear_states_kernel(LinearArgs a) {
  if (a.hdr->rejected) return;
  const uint32_t at = divide(blockIdx.x, a.kv_div);
  if ((int)at >= a.hdr->cut) return;
  const int head = (int)(blockIdx.x - at * a.kv_div.d);
  const Segment seg = a.segments[at];
  const int read = a.read[seg.request];
  if (read < -1 || read >= a.slots) return;  // (reported by linear_chunks_kernel)
  const int64_t place = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * 4;
  f32x4 state = {0, 0, 0, 0};
  if (read >= 0) state = *(const f32x4*)(a.state + read * a.state_slot + head * a.state_head + place);
  const float by = expf(a.log_decay[head] * (float)a.segment);
  const int64_t next = (int64_t)a.kv_heads * D * D;
  float* to = a.added + ((int64_t)seg.slot * a.kv_heads + head) * D * D + place;
  // (several on their way at once)
  constexpr int kAhead = 8;
  f32x4 x[kAhead];
  for (int i0 = 1; i0 < seg.parts; i0 += kAhead) {
    const int n = min(kAhead, seg.parts - i0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i < n) x[i] = *(const f32x4*)(to + (i0 + i) * next);
    if (i0 == 1) *(f32x4*)to = state;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i >= n) break;
#pragma unroll
      for (int e = 0; e < 4; ++e) state[e] = __builtin_fmaf(by, state[e], x[i][e]);
      *(f32x4*)(to + (i0 + i) * next) = state;
    }
  }
}

template <int D, class T, bool OUT>
hipError_t launch_chunks(const LinearArgs& a, int segments, hipStream_t st) {
  constexpr int bytes = ChunkLds<D, T, OUT>::kBytes;
  const hipError_t e = allow_lds<linear_chunks_kernel<D, T, OUT>>(bytes);
  if (e != hipSuccess) return e;
  const dim3 grid((uint32_t)segments * (uint32_t)a.kv_heads, OUT ? a.teams : 1);
  linear_chunks_kernel<D, T, OUT><<<grid, kThreads, bytes, st>>>(a);
  return hipGetLastError();
}

template <int D, class T>
hipError_t launch(const LinearArgs& a, hipStream_t st) {
  hipError_t e = hipSuccess;
  if (a.row_start && a.tokens > a.few) {
    if (a.tokens > a.segment) {
      const int most = a.tokens / a.segment;  // segments that others follow
      e = launch_chunks<D, T, false>(a, most, st);
      if (e != hipSuccess) return e;
      const dim3 grid((uint32_t)(most < a.requests ? most : a.requests) * (uint32_t)a.kv_heads, D * D / 4 / kThreads);
      linear_states_kernel<D><<<grid, kThreads, 0, st>>>(a);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    e = launch_chunks<D, T, true>(a, a.segment_cap, st);
    if (e != hipSuccess) return e;
  }
  if (a.few < 0) return hipSuccess;
  linear_steps_kernel<D, typename T::Type><<<(uint32_t)a.requests * (uint32_t)a.kv_heads, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, bool fp16, hipStream_t st) {
  if (a.planned) {
    linear_plan_kernel<<<1, kThreads, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dim == 64) return fp16 ? launch<64, OfFp16>(a, st) : launch<64, OfBf16>(a, st);
  return fp16 ? launch<128, OfFp16>(a, st) : launch<128, OfBf16>(a, st);
}

}  // namespace kvr
