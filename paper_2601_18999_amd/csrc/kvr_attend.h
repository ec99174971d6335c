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
// Four waves share the rows and the keys: with more than 64 rows each wave
// has 32 rows and all share a tile of 64 keys; with fewer rows the waves take
// different tiles of keys and are joined in LDS at the end.
//
// Scores, maxima, sums and accumulators are 32-bit.  p is rounded to the
// queries' type for the second product (the matrix instructions take 16-bit
// operands): its relative error, at most 2^-8 (bfloat16) or 2^-11, is that of
// the rounded result; the sum l adds the unrounded p.
#pragma once

#include "kvr_serve.h"

namespace kvr {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

struct Bf16 {
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
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
};

struct Fp16 {
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
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
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// RW: waves along the rows; the other 4 / RW are along the keys.
template <int D, int RW>
struct Shape {
  static constexpr int kKeyGroups = 4 / RW;
  static constexpr int kKeys = RW == 1 ? 32 : 64;   // of a tile
  static constexpr int kRowBytes = 2 * D;           // of a tile's row in LDS (always 16-bit elements)
  static constexpr int kTileBytes = kKeys * kRowBytes;
  static constexpr int kTiles = kKeyGroups * 2 * kTileBytes;
  // the join of the key groups at the end: maxima and sums, and results
  static constexpr int kJoin = kKeyGroups == 1 ? 0 : kKeyGroups * RW * 32 * (8 + 4 * D);
  static constexpr int kBytes = (kTiles > kJoin ? kTiles : kJoin) + 64;  // + flags
};

template <int D>
constexpr int attend_lds() {
  int n = Shape<D, 1>::kBytes;
  if (Shape<D, 2>::kBytes > n) n = Shape<D, 2>::kBytes;
  if (Shape<D, 4>::kBytes > n) n = Shape<D, 4>::kBytes;
  return n;
}

// A lane's share of a tile on its way from memory to LDS: NI 16-byte chunks of
// K and of V, at rows i * (threads / chunks of a row) + thread / chunks.
template <int D, class T, bool FP8, int RW>
struct Loader {
  typedef Shape<D, RW> S;
  static constexpr int kThreads = 64 * RW;
  static constexpr int kChunks = FP8 ? D / 16 : D / 8;  // of a row in the cache
  static constexpr int kRows = kThreads / kChunks;
  static constexpr int kN = S::kKeys / kRows;
  static_assert(kThreads % kChunks == 0 && S::kKeys % kRows == 0, "tile shape");

  i32x4 k[kN], v[kN];
  int page[kN];  // of the tile that is fetched next; -1: behind the last key

  // The tile's page numbers: keys key0.. of a table's row, `end` keys in all.
  __device__ __forceinline__ void pages(const AttendArgs& a, const int32_t* table, int key0, int end, int thread) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int key = key0 + i * kRows + thread / kChunks;
      page[i] = key < end ? table[key >> a.page_shift] : -1;
    }
  }

  __device__ __forceinline__ void fetch(const AttendArgs& a, const char* kc, const char* vc, int key0, int end,
                                        int thread) {
    const int mask = (1 << a.page_shift) - 1;
    const int64_t at = (int64_t)(thread % kChunks) * 16;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int key = key0 + i * kRows + thread / kChunks;
      const i32x4 zero = {0, 0, 0, 0};
      k[i] = zero;
      v[i] = zero;
      if (key < end) {
        if ((uint32_t)page[i] < (uint32_t)a.num_pages) {
          k[i] = *(const i32x4*)(kc + page[i] * a.kc_page + (key & mask) * a.kc_slot + at);
          v[i] = *(const i32x4*)(vc + page[i] * a.vc_page + (key & mask) * a.vc_slot + at);
        } else {  // no such page: the result is NaN
          const i32x4 nan = {-1, -1, -1, -1};
          k[i] = nan;
          v[i] = nan;
          if (a.status) atomicOr(a.status, (uint32_t)KVR_DEV_BAD_PAGE);
        }
      }
    }
  }

  static __device__ __forceinline__ void widen(i32x4 x, i32x4& lo, i32x4& hi) {
    lo = i32x4{T::from_fp8_lo(x[0]), T::from_fp8_hi(x[0]), T::from_fp8_lo(x[1]), T::from_fp8_hi(x[1])};
    hi = i32x4{T::from_fp8_lo(x[2]), T::from_fp8_hi(x[2]), T::from_fp8_lo(x[3]), T::from_fp8_hi(x[3])};
  }

  // whether one of the 8 16-bit values is infinite or NaN
  static __device__ __forceinline__ bool odd(i32x4 x) {
    bool b = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      b |= (x[j] & T::kExponent) == T::kExponent;
      b |= ((x[j] >> 16) & T::kExponent) == T::kExponent;
    }
    return b;
  }

  // Writes the tile to LDS; with `look`, whether V has an infinity or NaN here.
  __device__ __forceinline__ bool store(char* kt, char* vt, int thread, bool look) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int row = i * kRows + thread / kChunks, ch = thread % kChunks;
      char* kr = kt + row * S::kRowBytes;
      char* vr = vt + row * S::kRowBytes;
      if constexpr (FP8) {
        i32x4 lo, hi;
        widen(k[i], lo, hi);
        *(i32x4*)(kr + (((2 * ch) ^ swizzle_k<D>(row)) << 4)) = lo;
        *(i32x4*)(kr + (((2 * ch + 1) ^ swizzle_k<D>(row)) << 4)) = hi;
        widen(v[i], lo, hi);
        *(i32x4*)(vr + (((2 * ch) ^ swizzle_v<D>(row)) << 4)) = lo;
        *(i32x4*)(vr + (((2 * ch + 1) ^ swizzle_v<D>(row)) << 4)) = hi;
        if (look) bad |= odd(lo) | odd(hi);
      } else {
        *(i32x4*)(kr + ((ch ^ swizzle_k<D>(row)) << 4)) = k[i];
        *(i32x4*)(vr + ((ch ^ swizzle_v<D>(row)) << 4)) = v[i];
        if (look) bad |= odd(v[i]);
      }
    }
    return bad;
  }
};

template <class T>
__device__ __forceinline__ s16x4 round4(float a, float b, float c, float d) {
  const f32x4 x = {a, b, c, d};
  return __builtin_bit_cast(s16x4, __builtin_convertvector(x, typename T::x4));
}

template <int D, class T, bool FP8, int RW>
__device__ __forceinline__ void attend_item(const AttendArgs& a, const Item& it, int head, char* lds) {
  typedef Shape<D, RW> S;
  constexpr int KG = S::kKeyGroups, KT = S::kKeys, KB = KT / 32, DB = D / 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kg = wave / RW, thread = tid % (64 * RW);
  const int n = lane & 31, hh = lane >> 5;
  char* kt = lds + kg * 2 * S::kTileBytes;
  char* vt = kt + S::kTileBytes;
  int* flags = (int*)(lds + (S::kTiles > S::kJoin ? S::kTiles : S::kJoin));

  // the lane's row: its token, head and query
  const int r = rw * 32 + n;
  const bool live = r < it.rows;
  const uint32_t row = (uint32_t)(it.row0 + (live ? r : 0));
  const uint32_t token = divide(row, a.share);
  const int qhead = head * (int)a.share.d + (int)(row - token * a.share.d);
  s16x8 q[D / 16];
  {
    const char* p = a.q + token * a.q_tok + qhead * a.q_head + hh * 16;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) q[i] = *(const s16x8*)(p + i * 32);
  }
  const int limit = (int)token + it.limit;                             // own keys that this row sees
  const int limit0 = (int)divide((uint32_t)it.row0, a.share) + it.limit;  // ... and the first row

  const char* kc = a.kc + head * a.kc_head;
  const char* vc = a.vc + head * a.vc_head;
  const int32_t* own_table = a.table + it.request * a.table_stride;
  const int32_t* prefix_table = it.prefix_steps ? a.prefix_table + it.prefix * a.prefix_stride : nullptr;

  f32x16 o[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[b][i] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  const int tiles = (it.step1 - it.step0) * (kStepKeys / KT);
  const int rounds = (tiles + KG - 1) / KG;
  Loader<D, T, FP8, RW> ld;
  // tile t of the item: its first key, the end of its keys, and the table they come from
  auto place = [&](int t, int& key0, int& end, const int32_t*& table) {
    const int step = it.step0 + t / (kStepKeys / KT), part = t % (kStepKeys / KT);
    const bool shared = step < it.prefix_steps;
    key0 = (shared ? step : step - it.prefix_steps) * kStepKeys + part * KT;
    end = t >= tiles ? 0 : shared ? it.prefix_len : it.own_end;
    table = shared ? prefix_table : own_table;
    return shared;
  };
  int key0 = 0, end = 0, key1 = 0, end1 = 0;
  const int32_t* table;
  bool shared = place(kg, key0, end, table);
  ld.pages(a, table, key0, end, thread);
  ld.fetch(a, kc, vc, key0, end, thread);
  bool shared1 = place(KG + kg, key1, end1, table);
  ld.pages(a, table, key1, end1, thread);
  if (tid < 2 * KG) flags[tid] = 0;

  for (int round = 0; round < rounds; ++round) {
    // a row of this tile may stand before some of its own keys
    const bool edge = !shared && key0 + KT > limit0;
    __syncthreads();
    const bool bad = ld.store(kt, vt, thread, edge);
    if (edge && __any(bad) && lane == 0) flags[(round & 1) * KG + kg] = 1;
    __syncthreads();
    const bool odd = edge && flags[(round & 1) * KG + kg];
    if (tid < KG) flags[((round + 1) & 1) * KG + tid] = 0;
    const int k0 = key0, e0 = end;
    const bool sh0 = shared;
    // the next tile is on its way while this one is worked on
    key0 = key1;
    end = end1;
    shared = shared1;
    ld.fetch(a, kc, vc, key0, end, thread);
    shared1 = place((round + 2) * KG + kg, key1, end1, table);
    ld.pages(a, table, key1, end1, thread);
    if (k0 >= e0) continue;

    f32x16 s[KB];
#pragma unroll
    for (int b = 0; b < KB; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
      const int kr = b * 32 + n;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const s16x8 x = *(const s16x8*)(kt + kr * S::kRowBytes + (((2 * i + hh) ^ swizzle_k<D>(kr)) << 4));
        s[b] = T::mfma(x, q[i], s[b]);
      }
    }
    const int seen = (sh0 ? e0 : min(limit, e0)) - k0;  // keys of this tile that the row sees
    if (edge || k0 + KT > e0) {
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (b * 32 + 8 * (i / 4) + 4 * hh + i % 4 >= seen) s[b][i] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
    top = half_max(top) * a.scale_log2;
    if (__any(top > m)) {
      const float next = fmaxf(m, top);
      // before the first key of a row: nothing to scale
      const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= f;
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] *= f;
    }
    // a row that has seen no key yet has m = -inf: its p are exp2(-inf) = 0
    const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], a.scale_log2, -base));
        l += s[b][i];
      }

    if (__builtin_expect(odd, 0)) {
      // V holds an infinity or NaN and some rows do not see all keys: 0 * inf
      // must not reach them, so the products are taken key by key
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
            const char* vr = vt + key * S::kRowBytes + hh * 8;
            int sw = swizzle_v<D>(key) << 4;
            asm("" : "+v"(sw));  // (folded into the unrolled addresses, it keeps the compiler busy without end)
#pragma unroll
            for (int c = 0; c < DB; ++c)
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
      continue;
    }

    const int sl = lane & 15, dh = (lane >> 4) & 1;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        s16x8 p;
        {
          const s16x4 lo = round4<T>(s[b][8 * st], s[b][8 * st + 1], s[b][8 * st + 2], s[b][8 * st + 3]);
          const s16x4 hi = round4<T>(s[b][8 * st + 4], s[b][8 * st + 5], s[b][8 * st + 6], s[b][8 * st + 7]);
          p = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
#pragma unroll
        for (int c = 0; c < DB; ++c) {
          s16x4 x[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            // the transposing read: 16 lanes name four rows of 16 elements, four
            // lanes a row, and lane i of them gets column i
            const int vr = b * 32 + st * 16 + j * 8 + hh * 4 + sl / 4;
            const int ch = c * 4 + dh * 2 + (sl & 3) / 2;
            const char* p8 = vt + vr * S::kRowBytes + ((ch ^ swizzle_v<D>(vr)) << 4) + (sl & 1) * 8;
            x[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)(lds_char*)p8);
          }
          o[c] = T::mfma(__builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7), p, o[c]);
        }
      }
  }
  l = half_sum(l);

  const float vs = a.vs ? a.vs[head] : 1.0f;
  // four consecutive results of a row: the final ones, or the partial ones
  auto emit = [&](int rr, int d, f32x4 x, float ll) {
    const uint32_t R = (uint32_t)(it.row0 + rr);
    if (it.acc < 0) {
      const float f = ll > 0.0f || ll != ll ? vs / ll : 0.0f;
      const uint32_t tk = divide(R, a.share);
      const int hd = head * (int)a.share.d + (int)(R - tk * a.share.d);
      *(s16x4*)(a.out + tk * a.o_tok + hd * a.o_head + d * 2) = round4<T>(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
    } else {
      *(f32x4*)(a.acc + ((int64_t)(it.acc + rr) * a.kv_heads + head) * D + d) = x;
    }
  };
  auto emit_ml = [&](int rr, float mm, float ll) {
    if (it.acc >= 0) {
      a.ml[(int64_t)(it.acc + rr) * a.kv_heads + head] = make_float2(mm, ll);
    } else if (a.lse) {
      const uint32_t R = (uint32_t)(it.row0 + rr);
      const uint32_t tk = divide(R, a.share);
      const int hd = head * (int)a.share.d + (int)(R - tk * a.share.d);
      a.lse[(int64_t)tk * a.heads + hd] = ll > 0.0f || ll != ll ? (mm + __log2f(ll)) * 0.69314718055994530942f
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
    for (int i = tid; i < it.rows * (D / 4); i += 256) {
      const int rr = i / (D / 4), c = i % (D / 4);
      float mm = -INFINITY, ll = 0.0f;
#pragma unroll
      for (int g = 0; g < KG; ++g) mm = fmaxf(mm, jm[g * ROWS + rr]);
      f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int g = 0; g < KG; ++g) {
        const float mg = jm[g * ROWS + rr];
        if (mg != -INFINITY) ll += jl[g * ROWS + rr] * __builtin_amdgcn_exp2f(mg - mm);
        x += *(const f32x4*)(jo + (g * ROWS + rr) * D + (c ^ (rr & 15)) * 4);
      }
      emit(rr, c * 4, x, ll);
      if (c == 0) emit_ml(rr, mm, ll);
    }
  }
}

template <int D, class T, bool FP8>
__global__ void __launch_bounds__(256, D == 256 ? 1 : 2) attend_kernel(AttendArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int item = blockIdx.x / a.kv_heads, head = blockIdx.x % a.kv_heads;
  if (item >= a.hdr->items) return;
  const Item it = a.items[item];
  AttendArgs b = a;
  if (FP8 && a.ks) b.scale_log2 *= a.ks[head];
  if (it.rows > 64)
    attend_item<D, T, FP8, 4>(b, it, head, lds);
  else if (it.rows > 32)
    attend_item<D, T, FP8, 2>(b, it, head, lds);
  else
    attend_item<D, T, FP8, 1>(b, it, head, lds);
}

template <int D, class T, bool FP8>
hipError_t launch_attend_as(const AttendArgs& a, hipStream_t st) {
  constexpr int lds = attend_lds<D>();
  static_assert(lds * (D == 256 ? 1 : 2) <= 160 * 1024, "LDS of a compute unit");
  static const hipError_t set = hipFuncSetAttribute((const void*)attend_kernel<D, T, FP8>,
                                                    hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (set != hipSuccess) return set;
  attend_kernel<D, T, FP8><<<dim3((uint32_t)a.item_cap * (uint32_t)a.kv_heads), dim3(256), lds, st>>>(a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_attend(const AttendArgs& a, bool fp16, bool fp8, hipStream_t st) {
  if (fp16) return fp8 ? launch_attend_as<D, Fp16, true>(a, st) : launch_attend_as<D, Fp16, false>(a, st);
  return fp8 ? launch_attend_as<D, Bf16, true>(a, st) : launch_attend_as<D, Bf16, false>(a, st);
}

}  // namespace
}  // namespace kvr
