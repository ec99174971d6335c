// kvr_attend.h - the attention kernel, a template over the head dimension,
// the type of queries and results, and the type of the cache.
//
//   out[r] = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q_r . k_j - m_r)
//
// over the keys j that row r sees: its group's shared prefix and its own
// tokens up to itself.  A workgroup takes up to 128 rows of one key head and
// a range of keys, passes over the keys once in tiles with a running maximum
// m and sum l, and writes the result, or (o, m, l) where the unit's keys are
// split or the prefix is taken for a whole group; partial results are joined
// by the join kernel.
//
// Everything is computed transposed: S^T = K Q^T and O^T = V^T P^T with
// 32x32x16 matrix instructions, so that a lane holds one row's scores (16 of
// each 32 keys; the other half wave holds the rest).  The maximum and the sum
// are then in-lane but for one exchange of the half waves, and the scores are
// the second product's operand as they stand: operand slot (half, j) of key
// step s is key 16 s + 8 (j / 4) + 4 half + j % 4 for both operands, an order
// that the sum over keys does not care about.  V^T comes out of LDS by the
// transposing reads.
//
// With more than 32 rows each of the four waves has 32 rows (or none) and all
// share a tile of 64 keys; with fewer rows the waves take different tiles of
// 32 keys and are joined in LDS at the end.
//
// Scores, maxima, sums and accumulators are 32-bit.  p is rounded to the
// queries' type for the second product (the matrix instructions take 16-bit
// operands): its relative error, at most 2^-8 (bfloat16) or 2^-11, is that of
// the rounded result; the sum l adds the unrounded p.
#pragma once

#include <type_traits>

#include "kvr_lds.h"
#include "kvr_plan.h"

namespace kvr {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef const __attribute__((address_space(1))) i32x4* global_chunk;

struct Bf16 {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  typedef __bf16 x4 __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ int from_fp8_lo(int w) {
    return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
  }
  static __device__ __forceinline__ int from_fp8_hi(int w) {
    return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
  }
  static constexpr int kExponent = 0x7f80;  // exponent bits: all ones = infinity or NaN
  static constexpr float kLift = 0.0f;
};

struct Fp16 {
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  typedef _Float16 x4 __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ int from_fp8_lo(int w) {
    return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
  }
  static __device__ __forceinline__ int from_fp8_hi(int w) {
    return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
  }
  static constexpr int kExponent = 0x7c00;
  // p is up to 2^kLift at a row's maximum: halves end at 2^-24 below and 2^16 above
  static constexpr float kLift = 7.0f;
};

// 16-byte chunks of a row in LDS stand at chunk ^ swizzle(row).  K is read a
// 16-byte chunk of 16 or more rows at a time, V 64 bytes of four rows at a
// time; either way the lanes that are served together then fall on different
// banks (64 banks of 4 bytes).
template <int D>
__device__ __forceinline__ int swizzle_k(int row) {
  return D == 64 ? (row >> 1) & 7 : row & 15;
}
template <int D>
__device__ __forceinline__ int swizzle_v(int row) {
  return D == 64 ? (row & 2) << 1 : (row & 3) << 2;
}

// the larger (the sum) of a lane's value and that of the same row's lane in the other half wave
__device__ __forceinline__ float half_max(float x) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// The largest of three, or NaN (one instruction; fmaxf's rule for NaN takes two more).
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// RW: waves along the rows; the other 4 / RW are along the keys.
//
// A 16-bit cache goes from memory to LDS without a register in between.  With
// RW > 1 there are two buffers for a tile: while one is worked on, the other
// is filled.  With RW = 1 (a wave has its tile for itself, and memory bounds)
// there is one: K's half is filled again as soon as the scores are computed,
// V's when it has been multiplied, so loads are in flight all the time and
// two workgroups fit a compute unit.  An 8-bit cache is widened on the way,
// through registers, once for all waves that share the tile.
template <int D, int RW>
struct Shape {
  static constexpr int kKeyGroups = 4 / RW;
  static constexpr int kKeys = RW == 4 ? 64 : 32;  // of a tile
  static constexpr int kBuffers = RW == 1 ? 1 : 2;
  static constexpr int kRowBytes = 2 * D;           // of a tile's row in LDS (always 16-bit elements)
  static constexpr int kTileBytes = kKeys * kRowBytes;
  static constexpr int kTiles = kKeyGroups * kBuffers * 2 * kTileBytes;
  // the join of the key groups at the end: maxima and sums, and results
  static constexpr int kJoin = kKeyGroups == 1 ? 0 : kKeyGroups * RW * 32 * (8 + 4 * D);
  static constexpr int kMain = kTiles > kJoin ? kTiles : kJoin;
  static constexpr int kPages = RW == 1 ? 4 * 2 * 256 : 0;  // page numbers of a wave's next two tiles
  static constexpr int kBytes = kMain + kPages;
};

template <int D>
constexpr int attend_lds() {
  return Shape<D, 1>::kBytes > Shape<D, 4>::kBytes ? Shape<D, 1>::kBytes : Shape<D, 4>::kBytes;
}

// What a lane reads in the place of a row behind the last key, and of a row
// whose page number is none.
__device__ const uint32_t kNoRow[4] = {0, 0, 0, 0};
__device__ const uint32_t kBadRow[4] = {~0u, ~0u, ~0u, ~0u};  // NaN in every type

// page * page_bytes + slot * slot_bytes behind base (32-bit factors: two multiply-adds)
__device__ __forceinline__ global_bytes row_address(global_bytes base, int page, int slot, uint32_t page_bytes,
                                                   uint32_t slot_bytes) {
  return base + (uint64_t)(uint32_t)page * page_bytes + (uint64_t)(uint32_t)slot * slot_bytes;
}

// A lane's share of a tile of a 16-bit cache on its way to LDS: kN times 16
// bytes of K and of V.  Load i of a wave fills 1,024 neighbouring bytes, so a
// lane reads the chunk that belongs where it writes.
template <int D, int RW>
struct Direct {
  typedef Shape<D, RW> S;
  static constexpr int kChunks = D / 8;             // of a row
  static constexpr int kRows = 64 / kChunks;        // of one load of a wave
  static constexpr int kN = S::kKeys / (kRows * RW);
  static_assert(kN * kRows * RW == S::kKeys, "tile shape");

  // rows i * RW * kRows + first of the tile, i < kN
  static __device__ __forceinline__ int first(int wave, int lane) { return wave * kRows + lane / kChunks; }

  // whole: every row is a key and every page number is one of the cache
  template <bool KEYS>
  static __device__ __forceinline__ void load(const AttendArgs& a, global_bytes base, const int (&page)[kN], bool whole,
                                              int key0, int end, int wave, int lane, uint32_t to) {
    const uint32_t page_bytes = KEYS ? a.kc_page : a.vc_page, slot_bytes = KEYS ? a.kc_slot : a.vc_slot;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int row = i * RW * kRows + first(wave, lane);
      const int ch = (lane % kChunks) ^ (KEYS ? swizzle_k<D>(row) : swizzle_v<D>(row));
      global_bytes p = row_address(base + ch * 16, page[i], (key0 + row) & a.page_mask, page_bytes, slot_bytes);
      if (!whole) {
        if (key0 + row >= end)
          p = (global_bytes)kNoRow;
        else if ((uint32_t)page[i] >= (uint32_t)a.num_pages)
          p = (global_bytes)kBadRow;
      }
      load16_to_lds(p, to + (i * RW + wave) * 1024);
    }
  }

  // Pages of kRows tokens or more: the rows of one load stand in one page, so
  // a load has one base, in scalar registers, and lane offsets that stay the
  // same from tile to tile but for the swizzle of load i (the rows of one load
  // and i's multiples share no bits, so the swizzles are xored).  The offsets
  // have 32 bits, so the rows have to be near enough (lanes_reach).  Addresses
  // by lane, as other caches need them: 757 instead of 739 us for 9,216 tokens.
  struct Offsets {
    uint32_t k_row, k_chunk, v_row, v_chunk;
  };
  static __device__ __forceinline__ Offsets offsets(const AttendArgs& a, int wave, int lane) {
    const uint32_t row = lane / kChunks, chunk = lane % kChunks;
    return {row * a.kc_slot, (chunk ^ swizzle_k<D>(first(wave, lane))) << 4, row * a.vc_slot,
            (chunk ^ swizzle_v<D>(first(wave, lane))) << 4};
  }
  // page_of(i): the page of load i's rows, the same in all lanes
  template <bool KEYS, class PageOf>
  static __device__ __forceinline__ void load(const AttendArgs& a, global_bytes base, PageOf page_of, const Offsets& o,
                                              int key0, int wave, uint32_t to) {
    const uint32_t page_bytes = KEYS ? a.kc_page : a.vc_page, slot_bytes = KEYS ? a.kc_slot : a.vc_slot;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const uint32_t slot = (uint32_t)(key0 + (i * RW + wave) * kRows) & (uint32_t)a.page_mask;
      const uint64_t from = (uint64_t)base + (uint64_t)(uint32_t)page_of(i) * page_bytes + (uint64_t)slot * slot_bytes;
      const uint32_t swizzle = (uint32_t)(KEYS ? swizzle_k<D>(i * RW * kRows) : swizzle_v<D>(i * RW * kRows)) << 4;
      uint32_t chunk = KEYS ? o.k_chunk : o.v_chunk;
      if (swizzle) asm volatile("" : "+v"(chunk));  // xored here, not kept for each i (and spilled)
      const uint32_t offset = (KEYS ? o.k_row : o.v_row) + (chunk ^ swizzle);
      load16_to_lds(from, offset, to + (i * RW + wave) * 1024);
    }
  }
};

// A lane's share of a tile of an 8-bit cache: kN 16-byte chunks of K and of V
// in registers, at rows i * (threads / chunks of a row) + thread / chunks.
template <int D, class T, int RW>
struct Widened {
  typedef Shape<D, RW> S;
  static constexpr int kThreads = 64 * RW;
  static constexpr int kChunks = D / 16;  // of a row in the cache
  static constexpr int kRows = kThreads / kChunks;
  static constexpr int kN = S::kKeys / kRows;
  static_assert(kThreads % kChunks == 0 && S::kKeys % kRows == 0, "tile shape");
  static_assert(kN <= 4, "addresses that are held at once");

  i32x4 k[kN], v[kN];

  __device__ __forceinline__ void fetch(const AttendArgs& a, global_bytes kc, global_bytes vc, const int (&page)[kN],
                                        bool whole, int key0, int end, int thread) {
    const int at = thread % kChunks * 16;
    auto place = [&](int i, global_bytes& pk, global_bytes& pv) {
      const int slot = (key0 + i * kRows + thread / kChunks) & a.page_mask;
      pk = row_address(kc + at, page[i], slot, a.kc_page, a.kc_slot);
      pv = row_address(vc + at, page[i], slot, a.vc_page, a.vc_slot);
    };
    auto check = [&](int i, global_bytes& pk, global_bytes& pv) {
      if (key0 + i * kRows + thread / kChunks >= end)
        pk = pv = (global_bytes)kNoRow;
      else if ((uint32_t)page[i] >= (uint32_t)a.num_pages)
        pk = pv = (global_bytes)kBadRow;
    };
    global_bytes pk[kN], pv[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) place(i, pk[i], pv[i]);
    if (!whole) {
#pragma unroll
      for (int i = 0; i < kN; ++i) check(i, pk[i], pv[i]);
    }
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      k[i] = *(global_chunk)pk[i];
      v[i] = *(global_chunk)pv[i];
    }
  }

  static __device__ __forceinline__ void widen(i32x4 x, i32x4& lo, i32x4& hi) {
    lo = i32x4{T::from_fp8_lo(x[0]), T::from_fp8_hi(x[0]), T::from_fp8_lo(x[1]), T::from_fp8_hi(x[1])};
    hi = i32x4{T::from_fp8_lo(x[2]), T::from_fp8_hi(x[2]), T::from_fp8_lo(x[3]), T::from_fp8_hi(x[3])};
  }

  __device__ __forceinline__ void store(char* kt, char* vt, int thread) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int row = i * kRows + thread / kChunks, ch = thread % kChunks;
      char* kr = kt + row * S::kRowBytes;
      char* vr = vt + row * S::kRowBytes;
      i32x4 lo, hi;
      widen(k[i], lo, hi);
      *(i32x4*)(kr + (((2 * ch) ^ swizzle_k<D>(row)) << 4)) = lo;
      *(i32x4*)(kr + (((2 * ch + 1) ^ swizzle_k<D>(row)) << 4)) = hi;
      widen(v[i], lo, hi);
      *(i32x4*)(vr + (((2 * ch) ^ swizzle_v<D>(row)) << 4)) = lo;
      *(i32x4*)(vr + (((2 * ch + 1) ^ swizzle_v<D>(row)) << 4)) = hi;
    }
  }
};

template <class T>
__device__ __forceinline__ s16x4 round4(float a, float b, float c, float d) {
  const f32x4 x = {a, b, c, d};
  return __builtin_bit_cast(s16x4, __builtin_convertvector(x, typename T::x4));
}

// kinds of instructions for the scheduler
constexpr int kProducts = 0x8, kReads = 0x100;

constexpr float kSlack = 8.0f;  // p <= 2^(kLift + 8): below the largest half, and l far below the largest float

// A wave's 32 rows: queries, running maximum (log2 units) and sum, results.
template <int D, class T>
struct Rows {
  s16x8 q[D / 16];
  f32x16 o[D / 32];
  float m, l;

  static __device__ __forceinline__ s16x8 key_chunk(const char* kt, int row, int i, int hh) {
    return *(const s16x8*)(kt + row * 2 * D + (((2 * i + hh) ^ swizzle_k<D>(row)) << 4));
  }

  // Elements c * 32 .. of 16 keys (step q of the tile), as the second product
  // takes them.  The transposing read: 16 lanes name four rows of 16 elements,
  // four lanes a row, and lane i of them gets column i.
  static __device__ __forceinline__ s16x8 value_chunk(const char* vt, int q, int c, int lane) {
    const int hh = lane >> 5, sl = lane & 15, dh = (lane >> 4) & 1;
    s16x4 x[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int vr = q * 16 + j * 8 + hh * 4 + sl / 4;
      const int ch = c * 4 + dh * 2 + (sl & 3) / 2;
      const char* p8 = vt + vr * 2 * D + ((ch ^ swizzle_v<D>(vr)) << 4) + (sl & 1) * 8;
      x[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(lds_char*)p8);
    }
    return __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
  }

  // Scores of KB * 32 keys in LDS.  A chunk is read AHEAD products before its
  // own (a read takes as long as several products), and with VALUES the first
  // values while the last products run.
  template <int KB, int AHEAD, bool VALUES>
  __device__ __forceinline__ void scores(const char* kt, const char* vt, f32x16 (&s)[KB], s16x8 (&first)[D / 32], int n,
                                         int hh) {
    constexpr int N = D / 16, F = KB * N, V = VALUES ? D / 32 : 0;
    static_assert(V <= AHEAD && AHEAD <= F, "chunks ahead");
    s16x8 f[F];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) f[i] = key_chunk(kt, i / N * 32 + n, i % N, hh);
    __builtin_amdgcn_sched_group_barrier(kReads, AHEAD, 0);
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
#pragma unroll
    for (int i = 0; i < F; ++i) {
      const int next = i + AHEAD;
      if (next < F)
        f[next] = key_chunk(kt, next / N * 32 + n, next % N, hh);
      else if (next - F < V)
        first[next - F] = value_chunk(vt, 0, next - F, n + 32 * hh);
      s[i / N] = T::mfma(f[i], q[i % N], s[i / N]);
    }
#pragma unroll
    for (int i = 0; i < F; ++i) {
      __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
      if (i + AHEAD < F)
        __builtin_amdgcn_sched_group_barrier(kReads, 1, 0);
      else if (i + AHEAD - F < V)
        __builtin_amdgcn_sched_group_barrier(kReads, 2, 0);
    }
  }

  // Scores to p; keys from `seen` on are hidden where `edge` says that there are such.
  template <int KB>
  __device__ __forceinline__ void softmax(f32x16 (&s)[KB], bool edge, int seen, float scale, int hh) {
    if (edge) {
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          int last = seen - 4 * hh;
          asm("" : "+v"(last));  // each compare by itself: related, they take more masks than there are registers
          if (b * 32 + 8 * (i / 4) + i % 4 >= last) s[b][i] = -INFINITY;
        }
    }
    float top = max3(s[0][0], s[0][1], s[0][2]);
#pragma unroll
    for (int i = 3; i < 16 * KB - 1; i += 2) top = max3(top, s[i / 16][i % 16], s[(i + 1) / 16][(i + 1) % 16]);
    top = max3(top, s[KB - 1][15], s[KB - 1][15]);
    top = half_max(top) * scale;
    // m need not be the maximum, only near it: o and l are scaled when a row's
    // maximum has grown by more than 2^kSlack
    if (__any(top > m + (T::kLift + kSlack))) {
      const float next = fmaxf(m, top - T::kLift);
      // before the first key of a row: nothing to scale
      const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= f;
#pragma unroll
      for (int b = 0; b < D / 32; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] *= f;
      }
    }
    // a row that has seen no key yet has m = -inf: its p are exp2(-inf) = 0
    const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], scale, -base));
        l += s[b][i];
      }
  }

  // O^T += V^T P^T; with VALUES the first step's values are there.
  template <int KB, bool VALUES>
  __device__ __forceinline__ void values(const char* vt, const f32x16 (&s)[KB], const s16x8 (&first)[D / 32],
                                         int lane) {
    constexpr int N = D / 32;
    s16x8 f[2][N];
#pragma unroll
    for (int c = 0; c < N; ++c) f[0][c] = VALUES ? first[c] : value_chunk(vt, 0, c, lane);
#pragma unroll
    for (int q = 0; q < 2 * KB; ++q) {
      const int b = q / 2, st = q % 2;
      const s16x4 lo = round4<T>(s[b][8 * st], s[b][8 * st + 1], s[b][8 * st + 2], s[b][8 * st + 3]);
      const s16x4 hi = round4<T>(s[b][8 * st + 4], s[b][8 * st + 5], s[b][8 * st + 6], s[b][8 * st + 7]);
      const s16x8 p = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
      for (int c = 0; c < N; ++c) {
        if (q + 1 < 2 * KB) f[(q + 1) & 1][c] = value_chunk(vt, q + 1, c, lane);
        o[c] = T::mfma(f[q & 1][c], p, o[c]);
      }
    }
  }

  // The same key by key, for a tile whose V holds an infinity or NaN that some
  // rows do not see: 0 * inf must not reach them.
  template <int KB>
  __device__ __forceinline__ void values_seen(const char* vt, const f32x16 (&s)[KB], int seen, int hh) {
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll 1
      for (int i = 0; i < 16; ++i) {
        float x = s[b][0];  // s[b][i]
#pragma unroll
        for (int j = 1; j < 16; ++j) x = i == j ? s[b][j] : x;
        const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = b * 32 + 8 * (i >> 2) + 4 * h + (i & 3);
          const float p = __uint_as_float(w[h]);
          const char* vr = vt + key * 2 * D + hh * 8;
          int sw = swizzle_v<D>(key) << 4;
          asm("" : "+v"(sw));  // (folded into the unrolled addresses, it keeps the compiler busy without end)
#pragma unroll
          for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const int ch = c * 4 + g;  // 8 elements: this half's four
              const s16x4 x4 = *(const s16x4*)(vr + ((ch << 4) ^ sw));
              const auto y = __builtin_convertvector(__builtin_bit_cast(typename T::x4, x4), f32x4);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (key < seen) o[c][g * 4 + e] = __builtin_fmaf(p, y[e], o[c][g * 4 + e]);
            }
        }
      }
  }
};

// Whether a tile of `bytes` bytes in LDS holds an infinity or NaN, by one wave.
template <class T, int BYTES>
__device__ __forceinline__ bool holds_odd(const char* tile, int lane) {
  bool odd = false;
#pragma unroll 4
  for (int i = lane * 16; i < BYTES; i += 1024) {
    const i32x4 x = *(const i32x4*)(tile + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      odd |= (x[j] & T::kExponent) == T::kExponent;
      odd |= ((x[j] >> 16) & T::kExponent) == T::kExponent;
    }
  }
  return __any(odd);
}

typedef const __attribute__((address_space(4))) AttendArgs Args;

// A tile that every row sees to its end, and one that some may not.
struct Plain {
  static constexpr bool edge = false;
};
struct Edge {
  static constexpr bool edge = true;
};

template <int D, class T, bool FP8, int RW>
__device__ __forceinline__ void attend_item(const AttendArgs& a, const Item& it, int head, float scale, char* lds) {
  typedef Shape<D, RW> S;
  constexpr int KG = S::kKeyGroups, KT = S::kKeys, KB = KT / 32, DB = D / 32;
  // reads ahead, as many as there are registers for (9,216 new tokens: 739 us
  // without, 731 with them)
  constexpr int kAhead = D == 256 || FP8 ? 4 : D == 64 && RW == 1 ? 4 : 8;
  constexpr bool kEarly = RW > 1 && D <= 128 && !FP8;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kg = wave / RW, thread = tid % (64 * RW);
  const int n = lane & 31, hh = lane >> 5;

  // the lane's row: its token, head and query
  const int r = rw * 32 + n;
  const bool live = r < it.rows;
  const uint32_t row = (uint32_t)(it.row0 + (live ? r : 0));
  const uint32_t token = divide(row, a.share);
  const int qhead = head * (int)a.share.d + (int)(row - token * a.share.d);
  Rows<D, T> x;
  // called when the first page numbers are on their way: both arrive together
  auto load_queries = [&]() {
    const char* p = a.q + token * a.q_tok + qhead * a.q_head + hh * 16;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) x.q[i] = *(const s16x8*)(p + i * 32);
    // waited for here: a wait inside the loop would be for the tiles' loads too
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      if constexpr (D == 256)  // in accumulation registers, of which the products take operands too
        asm volatile("" : "+a"(x.q[i]));
      else
        asm volatile("" : "+v"(x.q[i]));
    }
  };
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) x.o[b][i] = 0.0f;
  x.m = -INFINITY;
  x.l = 0.0f;
  const int limit = (int)token + it.limit;                                // own keys that this row sees
  const int limit0 = (int)divide((uint32_t)it.row0, a.share) + it.limit;  // ... and the first row

  const global_bytes kc = (global_bytes)(a.kc + head * a.kc_head);
  const global_bytes vc = (global_bytes)(a.vc + head * a.vc_head);
  const global_ints own_table = (global_ints)(a.table + it.request * a.table_stride);
  const global_ints prefix_table = (global_ints)(a.prefix_table + it.prefix * a.prefix_stride);
  const int tiles = (it.step1 - it.step0) * (kStepKeys / KT);

  // tile t of the item: its first key, the end of its keys, their table, and
  // whether it is the prefix's
  struct Place {
    int key0, end;
    global_ints table;
    bool shared;
  };
  auto place = [&](int t) {
    const int step = it.step0 + t / (kStepKeys / KT), part = t % (kStepKeys / KT);
    Place p;
    p.shared = step < it.prefix_steps;
    p.key0 = (p.shared ? step : step - it.prefix_steps) * kStepKeys + part * KT;
    p.end = t >= tiles ? 0 : p.shared ? it.prefix_len : it.own_end;
    p.table = t >= tiles ? (global_ints)kNoRow : p.shared ? prefix_table : own_table;
    return p;
  };
  // page numbers of rows row0 + i * step (i < N) of a tile (behind its end: the last key's)
  auto pages = [&](const Place& p, int row0, int step, auto& page) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(page) / sizeof(int)); ++i)
      page[i] = p.table[max(0, min(p.key0 + row0 + i * step, p.end - 1)) >> a.page_shift];
  };
  // whether all rows of a tile are keys in pages of the cache; a page outside it is reported
  auto whole_of = [&](const Place& p, const auto& page) {
    uint32_t top = (uint32_t)page[0];
#pragma unroll
    for (int i = 1; i < (int)(sizeof(page) / sizeof(int)); ++i) top = max(top, (uint32_t)page[i]);
    const bool bad = top >= (uint32_t)a.num_pages && p.end > 0;
    if (bad && a.status) atomicOr(a.status, (uint32_t)KVR_DEV_BAD_PAGE);
    return p.key0 + KT <= p.end && !__any(bad);
  };
  // Tiles before `plain` are seen by all rows: no masks in their loop, and no
  // second way to multiply V, which would keep two copies of the results.
  const int plain = max(0, min(tiles, (it.prefix_steps + limit0 / kStepKeys - it.step0) * (kStepKeys / KT)));
  // scores to p
  auto weigh = [&](auto kind, const Place& p, f32x16(&s)[KB]) {
    const int seen = (kind.edge && !p.shared ? min(limit, p.end) : p.end) - p.key0;
    x.softmax(s, kind.edge || p.key0 + KT > p.end, seen, scale, hh);
  };
  // and their product with V
  auto multiply = [&](auto kind, const Place& p, const char* vt, const f32x16(&s)[KB], const s16x8(&first)[DB]) {
    if constexpr (kind.edge) {
      const int seen = (p.shared ? p.end : min(limit, p.end)) - p.key0;
      if (holds_odd<T, S::kTileBytes>(vt, lane)) {
        x.values_seen(vt, s, seen, hh);
        return;
      }
    }
    x.template values<KB, kEarly>(vt, s, first, lane);
  };

  if constexpr (RW == 1 && !FP8) {
    typedef Direct<D, 1> L;
    constexpr int N = L::kN;
    char* kt = lds + wave * 2 * S::kTileBytes;
    char* vt = kt + S::kTileBytes;
    int* ids = (int*)(lds + S::kMain) + wave * 128;
    const uint32_t k_to = lds_offset(kt), v_to = lds_offset(vt), id_to = lds_offset(ids);
    const int mine = (tiles - wave + 3) / 4;  // tiles wave, wave + 4, ..
    auto load_ids = [&](int j) {
      const Place p = place(wave + 4 * j);
      const int key = min(p.key0 + n, p.end - 1);
      load4_to_lds(p.table + (key >> a.page_shift), id_to + (j & 1) * 256);
    };
    const typename L::Offsets offsets = L::offsets(a, 0, lane);
    const bool uniform = a.one_base;
    // whether all rows of tile j are keys in pages of the cache; a page outside it is reported
    auto whole_of_ids = [&](const Place& p, int j) {
      const bool bad = (uint32_t)ids[(j & 1) * 64 + n] >= (uint32_t)a.num_pages;
      if (bad && a.status) atomicOr(a.status, (uint32_t)KVR_DEV_BAD_PAGE);
      return p.key0 + KT <= p.end && !__any(bad);
    };
    auto load = [&](auto keys, const Place& p, int j, bool whole) {
      constexpr bool K = decltype(keys)::value;
      const int* id = ids + (j & 1) * 64;
      if (whole && uniform) {
        const int of_load = id[lane * L::kRows % KT];  // lane i: load i's
        L::template load<K>(a, K ? kc : vc, [&](int i) { return __builtin_amdgcn_readlane(of_load, i); }, offsets,
                            p.key0, 0, K ? k_to : v_to);
      } else {
        int page[N];
#pragma unroll
        for (int i = 0; i < N; ++i) page[i] = id[i * L::kRows + L::first(0, lane)];
        wait_lds();
        L::template load<K>(a, K ? kc : vc, page, whole, p.key0, p.end, 0, lane, K ? k_to : v_to);
      }
    };
    constexpr std::true_type keys{};
    constexpr std::false_type vals{};
    if (mine > 0) {
      Place p = place(wave);
      load_ids(0);
      load_queries();
      wait_loads<0>();
      const bool whole = whole_of_ids(p, 0);
      load(keys, p, 0, whole);
      if (mine > 1) load_ids(1);
      load(vals, p, 0, whole);
      auto round = [&](auto kind, int j) {
        // in flight, oldest first: K of this tile, the next one's page numbers, V of this tile
        const bool more = j + 1 < mine;
        const Place p1 = place(wave + 4 * (j + 1));
        bool whole1 = false;
        wait_loads<N>();
        f32x16 s[KB];
        s16x8 first[DB];
        x.template scores<KB, kAhead, false>(kt, vt, s, first, n, hh);
        if (more) whole1 = whole_of_ids(p1, j + 1);
        wait_lds();
        if (more) {
          load(keys, p1, j + 1, whole1);
          if (j + 2 < mine) load_ids(j + 2);
        }
        weigh(kind, p, s);
        if (j + 2 < mine)
          wait_loads<N + 1>();
        else if (more)
          wait_loads<N>();
        else
          wait_loads<0>();
        multiply(kind, p, vt, s, first);
        wait_lds();
        if (more) load(vals, p1, j + 1, whole1);
        p = p1;
      };
      int j = 0;
      for (; j < mine && wave + 4 * j < plain; ++j) round(Plain(), j);
      for (; j < mine; ++j) round(Edge(), j);
    }
  } else if constexpr (RW == 1) {
    typedef Widened<D, T, 1> L;
    char* kt = lds + wave * 2 * S::kTileBytes;
    char* vt = kt + S::kTileBytes;
    const int mine = (tiles - wave + 3) / 4;
    int page[L::kN];
    L ld;
    const int row0 = lane / L::kChunks;
    Place p = place(wave), p1 = place(wave + 4);
    pages(p, row0, L::kRows, page);
    load_queries();
    ld.fetch(a, kc, vc, page, whole_of(p, page), p.key0, p.end, lane);
    pages(p1, row0, L::kRows, page);
    auto round = [&](auto kind, int j) {
      ld.store(kt, vt, lane);
      ld.fetch(a, kc, vc, page, whole_of(p1, page), p1.key0, p1.end, lane);
      const Place p2 = place(wave + 4 * (j + 2));
      pages(p2, row0, L::kRows, page);
      f32x16 s[KB];
      s16x8 first[DB];
      x.template scores<KB, kAhead, kEarly>(kt, vt, s, first, n, hh);
      weigh(kind, p, s);
      multiply(kind, p, vt, s, first);
      p = p1;
      p1 = p2;
    };
    int j = 0;
    for (; j < mine && wave + 4 * j < plain; ++j) round(Plain(), j);
    for (; j < mine; ++j) round(Edge(), j);
  } else {
    // two buffers; one barrier a tile
    static_assert(KG == 1, "the waves share every tile");
    Place p = place(0), p1 = place(1);
    const bool idle = wave * 32 >= it.rows;  // no row: it only loads
    auto work = [&](auto kind, const char* kt, const char* vt) {
      if (idle) return;
      f32x16 s[KB];
      s16x8 first[DB];
      // a wave that multiplies goes first: two waves of a SIMD else fall into
      // step, and the matrix and the vector unit wait for each other (9,216 new
      // tokens: 731 -> 708 us)
      __builtin_amdgcn_s_setprio(1);
      x.template scores<KB, kAhead, kEarly>(kt, vt, s, first, n, hh);
      __builtin_amdgcn_s_setprio(0);
      weigh(kind, p, s);
      __builtin_amdgcn_s_setprio(1);
      multiply(kind, p, vt, s, first);
      __builtin_amdgcn_s_setprio(0);
    };
    if constexpr (!FP8) {
      typedef Direct<D, RW> L;
      int page[L::kN];
      const int row0 = L::first(rw, lane), step = RW * L::kRows;
      const uint32_t to = lds_offset(lds);
      const typename L::Offsets offsets = L::offsets(a, rw, lane);
      const bool uniform = a.one_base;
      auto load = [&](const Place& q, uint32_t at) {
        const bool whole = whole_of(q, page);
        if (whole && uniform) {
          auto page_of = [&](int i) { return __builtin_amdgcn_readfirstlane(page[i]); };
          L::template load<true>(a, kc, page_of, offsets, q.key0, rw, at);
          L::template load<false>(a, vc, page_of, offsets, q.key0, rw, at + S::kTileBytes);
        } else {
          L::template load<true>(a, kc, page, whole, q.key0, q.end, rw, lane, at);
          L::template load<false>(a, vc, page, whole, q.key0, q.end, rw, lane, at + S::kTileBytes);
        }
      };
      if (tiles > 0) {
        pages(p, row0, step, page);
        load_queries();
        load(p, to);
        pages(p1, row0, step, page);
      }
      auto round = [&](auto kind, int j) {
        wait_loads<0>();
        barrier();
        const uint32_t b1 = (j + 1 & 1) * 2 * S::kTileBytes;
        const char* kt = lds + (j & 1) * 2 * S::kTileBytes;
        const Place p2 = place(j + 2);
        if (j + 1 < tiles) {
          load(p1, to + b1);
          pages(p2, row0, step, page);
        }
        work(kind, kt, kt + S::kTileBytes);
        p = p1;
        p1 = p2;
      };
      int j = 0;
      for (; j < plain; ++j) round(Plain(), j);
      for (; j < tiles; ++j) round(Edge(), j);
    } else {
      typedef Widened<D, T, RW> L;
      int page[L::kN];
      L ld;
      const int row0 = thread / L::kChunks;
      pages(p, row0, L::kRows, page);
      load_queries();
      ld.fetch(a, kc, vc, page, whole_of(p, page), p.key0, p.end, thread);
      pages(p1, row0, L::kRows, page);
      ld.store(lds, lds + S::kTileBytes, thread);
      auto round = [&](auto kind, int j) {
        barrier();
        char* kt = lds + (j & 1) * 2 * S::kTileBytes;
        char* kt1 = lds + (j + 1 & 1) * 2 * S::kTileBytes;
        const Place p2 = place(j + 2);
        ld.fetch(a, kc, vc, page, whole_of(p1, page), p1.key0, p1.end, thread);
        pages(p2, row0, L::kRows, page);
        work(kind, kt, kt + S::kTileBytes);
        ld.store(kt1, kt1 + S::kTileBytes, thread);
        p = p1;
        p1 = p2;
      };
      int j = 0;
      for (; j < plain; ++j) round(Plain(), j);
      for (; j < tiles; ++j) round(Edge(), j);
    }
  }
  const float m = x.m, l = half_sum(x.l);
  auto& o = x.o;
  // what only the end needs is read here, not kept in scalar registers
  const Args* late = (const Args*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(late));
  const Args& z = *late;
  const Divisor share = {z.share.d, z.share.mul, z.share.shift};
  const float vs = z.vs ? z.vs[head] : 1.0f;
  // four consecutive results of a row: the final ones, or the partial ones
  auto emit = [&](int rr, int d, f32x4 y, float ll) {
    const uint32_t R = (uint32_t)(it.row0 + rr);
    if (it.acc < 0) {
      const float f = ll > 0.0f || ll != ll ? vs / ll : 0.0f;
      const uint32_t tk = divide(R, share);
      const int hd = head * (int)share.d + (int)(R - tk * share.d);
      *(s16x4*)(z.out + tk * z.o_tok + hd * z.o_head + d * 2) = round4<T>(y[0] * f, y[1] * f, y[2] * f, y[3] * f);
    } else {
      *(f32x4*)(z.acc + ((int64_t)(it.acc + rr) * z.kv_heads + head) * D + d) = y;
    }
  };
  auto emit_ml = [&](int rr, float mm, float ll) {
    if (it.acc >= 0) {
      z.ml[(int64_t)(it.acc + rr) * z.kv_heads + head] = make_float2(mm, ll);
    } else if (z.lse) {
      const uint32_t R = (uint32_t)(it.row0 + rr);
      const uint32_t tk = divide(R, share);
      const int hd = head * (int)share.d + (int)(R - tk * share.d);
      z.lse[(int64_t)tk * z.heads + hd] = ll > 0.0f || ll != ll ? (mm + __log2f(ll)) * 0.69314718055994530942f
                                                               : -INFINITY;
    }
  };

  if constexpr (KG == 1) {
    if (live) {
#pragma unroll
      for (int c = 0; c < DB; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          emit(r, c * 32 + g * 8 + hh * 4, f32x4{o[c][g * 4], o[c][g * 4 + 1], o[c][g * 4 + 2], o[c][g * 4 + 3]}, l);
      if (hh == 0) emit_ml(r, m, l);
    }
  } else {
    constexpr int ROWS = RW * 32;
    float* jm = (float*)lds;            // [KG][ROWS]
    float* jl = jm + KG * ROWS;         // [KG][ROWS]
    float* jo = jl + KG * ROWS;         // [KG][ROWS][D], 16-byte chunks swizzled by row
    __syncthreads();
    if (hh == 0) {
      jm[kg * ROWS + r] = m;
      jl[kg * ROWS + r] = l;
    }
    __syncthreads();
    float all = -INFINITY;
#pragma unroll
    for (int g = 0; g < KG; ++g) all = fmaxf(all, jm[g * ROWS + r]);
    const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - all);
    if (live) {
#pragma unroll
      for (int c = 0; c < DB; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int ch = (c * 8 + g * 2 + hh) ^ (r & 15);
          *(f32x4*)(jo + (kg * ROWS + r) * D + ch * 4) =
              f32x4{o[c][g * 4] * f, o[c][g * 4 + 1] * f, o[c][g * 4 + 2] * f, o[c][g * 4 + 3] * f};
        }
    }
    __syncthreads();
    for (int i = tid; i < it.rows * (D / 4); i += kAttendThreads) {
      const int rr = i / (D / 4), c = i % (D / 4);
      float mm = -INFINITY, ll = 0.0f;
#pragma unroll
      for (int g = 0; g < KG; ++g) mm = fmaxf(mm, jm[g * ROWS + rr]);
      f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int g = 0; g < KG; ++g) {
        const float mg = jm[g * ROWS + rr];
        // (a group without a maximum has the sum 0, or NaN where a score was)
        ll += mg == -INFINITY ? jl[g * ROWS + rr] : jl[g * ROWS + rr] * __builtin_amdgcn_exp2f(mg - mm);
        y += *(const f32x4*)(jo + (g * ROWS + rr) * D + (c ^ (rr & 15)) * 4);
      }
      emit(rr, c * 4, y, ll);
      if (c == 0) emit_ml(rr, mm, ll);
    }
  }
}

// Many rows: bound by the matrix and the vector unit, whose times add up (9,216
// new tokens of 32 / 8 heads of 128: 695 to 740 us on different devices, 940 to
// 1,000 TFLOP/s, where a library product reaches 1,230 to 1,264; heads of 256,
// 6,000 new tokens of 16 / 4 heads: 480 to 491 us, 600 to 614 TFLOP/s).  Few
// rows: bound by memory (64 requests in four groups, 243 MB: 50 us, 4.9 TB/s,
// where a copy reaches 5.1; 57 us with the plan in each workgroup).
template <int D, class T, bool FP8>
__global__ void __launch_bounds__(kAttendThreads, D == 256 ? 1 : 2) attend_kernel(AttendArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int item = blockIdx.x / a.kv_heads, head = blockIdx.x % a.kv_heads;
  Item it;
  if (a.fused) {
    static_assert(4 * plan_words(kPlanFused) + (int)sizeof(Item) <= attend_lds<D>(), "the plan's LDS");
    Item* mine = (Item*)(lds + 4 * plan_words(kPlanFused));
    const int items = make_plan<kPlanFused>(a, (int*)lds, blockIdx.x == 0, [&](int i, const Item& x) {
      if (i == item) *mine = x;
    });
    if (items < 0 && a.direct) fill_with_nan(a);
    if (item >= items) return;
    __syncthreads();
    it = *mine;
    // the same in all lanes: in scalar registers
#pragma unroll
    for (int i = 0; i < (int)(sizeof(Item) / 4); ++i)
      ((int*)&it)[i] = __builtin_amdgcn_readfirstlane(((int*)&it)[i]);
    __syncthreads();
  } else {
    it = a.items[item];  // (there is room for as many as there are workgroups)
    if (a.direct && a.hdr->rejected) fill_with_nan(a);
    if (item >= a.hdr->items) return;
  }
  const float scale = FP8 && a.ks ? a.scale_log2 * a.ks[head] : a.scale_log2;
  // An 8-bit tile on its way and heads of 256 are more than a wave's registers
  // hold: few rows then share a tile too (64 requests of 2,000 to 4,000 tokens,
  // 16 heads: 272 -> 241 us).
  if constexpr (FP8 && D == 256)
    attend_item<D, T, FP8, 4>(a, it, head, scale, lds);
  else if (it.rows > 32)
    attend_item<D, T, FP8, 4>(a, it, head, scale, lds);
  else  // (sharing tiles here too: 256 requests of one group 196 instead of 183 us)
    attend_item<D, T, FP8, 1>(a, it, head, scale, lds);
}

template <int D, class T, bool FP8>
hipError_t launch_attend_as(const AttendArgs& a, hipStream_t st) {
  constexpr int lds = attend_lds<D>();
  static_assert(lds * (D == 256 ? 1 : 2) <= 160 * 1024, "LDS of a compute unit");
  const hipError_t e = allow_lds<attend_kernel<D, T, FP8>>(lds);
  if (e != hipSuccess) return e;
  attend_kernel<D, T, FP8><<<dim3((uint32_t)a.item_cap * (uint32_t)a.kv_heads), dim3(kAttendThreads), lds, st>>>(a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_attend(const AttendArgs& a, bool fp16, bool fp8, hipStream_t st) {
  if (fp16) return fp8 ? launch_attend_as<D, Fp16, true>(a, st) : launch_attend_as<D, Fp16, false>(a, st);
  return fp8 ? launch_attend_as<D, Bf16, true>(a, st) : launch_attend_as<D, Bf16, false>(a, st);
}

}  // namespace
}  // namespace kvr
