// kvr_serve.hip - kernels of the serving operators but the attention itself:
// page tables and slot maps, the store of new keys and values, and the plan
// and the join of the attention.
#include "kvr_plan.h"

namespace kvr {
namespace {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- page tables

constexpr int kScanThreads = 1024;

struct RowChange {
  int64_t tokens, pages;  // new tokens; pages taken (low word) and given back (high word)
  uint32_t bits;
};

__device__ __forceinline__ RowChange row_change(const TablesArgs& a, int held, int delta) {
  RowChange c = {0, 0, 0};
  const int64_t total = (int64_t)held + delta, page = 1ll << a.page_shift;
  if (held < 0 || total < 0) {
    c.bits = KVR_DEV_BAD_LENGTH;
  } else if (held > ((int64_t)a.width << a.page_shift) || total > ((int64_t)a.width << a.page_shift)) {
    c.bits = KVR_DEV_ROW_FULL;
  } else {
    const int64_t before = (held + page - 1) >> a.page_shift, after = (total + page - 1) >> a.page_shift;
    c.tokens = delta > 0 ? delta : 0;
    c.pages = after > before ? after - before : (before - after) << 32;
  }
  return c;
}

// One workgroup: sums over the rows, the checks, and everything that is one
// value a row.  A thread takes neighbouring rows.  row_start (one more than
// the rows), gain_at and give_at are written for what follows.
__device__ __forceinline__ TablesHdr scan_rows(const TablesArgs& a, int64_t* part, int* row_start, int* gain_at,
                                               int* give_at) {
  const int per = (a.rows + blockDim.x - 1) / blockDim.x;
  const int r0 = min(a.rows, (int)threadIdx.x * per), r1 = min(a.rows, r0 + per);
  const int64_t head = a.state[0], tail = a.state[1], old_bits = a.state[2];
  int64_t tokens = 0, pages = 0;
  uint32_t bits = 0;
  for (int r = r0; r < r1; ++r) {
    const RowChange c = row_change(a, a.held[r], a.delta[r]);
    tokens += c.tokens;
    pages += c.pages;
    bits |= c.bits;
  }
  int64_t all_tokens, all_pages;
  tokens = group_before(tokens, all_tokens, part);
  pages = group_before(pages, all_pages, part);
  const int64_t gain = all_pages & 0xffffffffll, give = all_pages >> 32;
  bits = (__syncthreads_or(bits & KVR_DEV_BAD_LENGTH) ? KVR_DEV_BAD_LENGTH : 0u) |
         (__syncthreads_or(bits & KVR_DEV_ROW_FULL) ? KVR_DEV_ROW_FULL : 0u);
  if (all_tokens > a.num_tokens) bits |= KVR_DEV_BAD_LENGTH;
  if (head < 0 || tail < head || tail - head > a.ring_size || gain > tail - head) bits |= KVR_DEV_PAGES_FULL;
  // more pages free than there are
  if (tail - head + give > a.ring_size) bits |= KVR_DEV_PAGES_FULL;
  for (int r = r0; r < r1; ++r) {
    const int held = a.held[r], delta = a.delta[r];
    const RowChange c = row_change(a, held, delta);
    row_start[r] = bits ? 0 : (int)tokens;
    gain_at[r] = (int)(pages & 0xffffffffll);
    give_at[r] = (int)(pages >> 32);
    a.held_out[r] = bits ? held : held + delta;
    tokens += c.tokens;
    pages += c.pages;
  }
  if (threadIdx.x == 0) row_start[a.rows] = bits ? 0 : (int)all_tokens;
  TablesHdr h;
  h.head = head % a.ring_size;
  h.tail = tail % a.ring_size;
  h.gain = (int)gain;
  h.give = (int)give;
  h.tokens = (int)all_tokens;
  h.rejected = bits != 0;
  __syncthreads();  // every thread has read the state and its rows
  if (threadIdx.x == 0) {
    a.state_out[0] = bits ? head : head + gain;
    a.state_out[1] = bits ? tail : tail + give;
    a.state_out[2] = old_bits | bits;
  }
  return h;
}

// place of page i of the ring counted from `from`; from, i < size
__device__ __forceinline__ int ring_at(int from, int i, int size) {
  const uint32_t at = (uint32_t)from + (uint32_t)i;
  return (int)(at >= (uint32_t)size ? at - size : at);
}

// Slot and position of new token t, of row r.  The first token of a gained
// page writes its table entry (a gained page always has one).
__device__ __forceinline__ void place_token(const TablesArgs& a, const TablesHdr& h, const int* row_start,
                                            const int* gain_at, int t, int r) {
  int slot = -1, position = -1;
  if (!h.rejected && t < h.tokens) {
    const int mask = (1 << a.page_shift) - 1;
    const int held = a.held_out[r] - a.delta[r];
    const int at = held + t - row_start[r];
    const int col = at >> a.page_shift, before = (int)(((int64_t)held + mask) >> a.page_shift);
    int32_t* entry = a.table + r * a.table_stride + col;
    int page;
    if (col < before) {
      page = *entry;
    } else {
      page = a.ring[ring_at((int)h.head, gain_at[r] + col - before, a.ring_size)];
      if ((at & mask) == 0) *entry = page;
    }
    slot = (page << a.page_shift) | (at & mask);
    position = (a.base_held ? held : a.base ? a.base[r] : 0) + at;
  }
  a.slots[t] = slot;
  a.positions[t] = position;
}

// Puts back dropped page g, of row r.
__device__ __forceinline__ void drop_page(const TablesArgs& a, const TablesHdr& h, const int* give_at, int g, int r) {
  const int mask = (1 << a.page_shift) - 1;
  const int after = (int)(((int64_t)a.held_out[r] + mask) >> a.page_shift);
  a.ring[ring_at((int)h.tail, g, a.ring_size)] = a.table[r * a.table_stride + after + g - give_at[r]];
}

__global__ void __launch_bounds__(kScanThreads) tables_scan_kernel(TablesArgs a) {
  __shared__ int64_t part[16];
  const TablesHdr h = scan_rows(a, part, a.row_start, a.gain_at, a.give_at);
  if (threadIdx.x == 0) *a.hdr = h;
}

// Few rows and tokens: all in one workgroup and one launch, the sums in LDS
// (32 rows: 12.5 us a call, 15.5 in two launches).
constexpr int kFusedRows = 1024, kFusedTokens = 4096;
__global__ void __launch_bounds__(kScanThreads) tables_fused_kernel(TablesArgs a) {
  __shared__ int64_t part[16];
  __shared__ int row_start[kFusedRows + 1], gain_at[kFusedRows], give_at[kFusedRows];
  const TablesHdr h = scan_rows(a, part, row_start, gain_at, give_at);
  for (int r = threadIdx.x; r <= a.rows; r += blockDim.x) a.row_start[r] = row_start[r];
  for (int t = threadIdx.x; t < a.num_tokens; t += blockDim.x) place_token(a, h, row_start, gain_at, t, last_at_most(row_start, a.rows, t));
  if (h.rejected) return;
  for (int g = threadIdx.x; g < h.give; g += blockDim.x) drop_page(a, h, give_at, g, last_at_most(give_at, a.rows, g));
}

// last_at_most(start, n, x0 + lane) for a wave's neighbouring values: the wave
// finds the first one's place, 64 probes at a time, and each lane its own among
// the next 64 entries (a search by each lane reads log2(n) times in a row
// instead of three).  All lanes are active.
__device__ __forceinline__ int last_at_most_of_lanes(const int* start, int n, int x0) {
  const int lane = threadIdx.x & 63, x = x0 + lane;
  int lo = 0, len = n;
  while (len > 1) {
    const int step = (len + 63) / 64, at = lane * step;
    const int probe = at < len ? start[lo + at] : 0x7fffffff;
    const int k = max(0, __popcll(__ballot(probe <= x0)) - 1);
    lo += k * step;
    len = min(step, len - k * step);
  }
  const int next = lo + 1 + lane < n ? start[lo + 1 + lane] : 0x7fffffff;
  int k = 0;
#pragma unroll
  for (int s = 32; s; s >>= 1)
    if (__shfl(next, k + s - 1) <= x) k += s;
  // (k = 63: the 64 entries may not reach)
  return k < 63 ? lo + k : lo + k + last_at_most(start + lo + k, n - lo - k, x);
}

constexpr int kFillThreads = 256;

// Slots and positions of the new tokens, the pages they gain, and the pages
// that are given back.
__global__ void __launch_bounds__(kFillThreads) tables_fill_kernel(TablesArgs a) {
  const TablesHdr h = *a.hdr;
  const int lane = threadIdx.x & 63, first = blockIdx.x * kFillThreads + (threadIdx.x - lane);
  if (first < a.num_tokens) {
    const int r = first < h.tokens && !h.rejected ? last_at_most_of_lanes(a.row_start, a.rows, first) : 0;
    if (first + lane < a.num_tokens) place_token(a, h, a.row_start, a.gain_at, first + lane, r);
  }
  if (h.rejected) return;
  // (64 bits: the grid may have 2^31 threads)
  for (int64_t at = first; at < h.give; at += (int64_t)gridDim.x * kFillThreads) {
    const int g = (int)at, r = last_at_most_of_lanes(a.give_at, a.rows, g);
    if (lane < h.give - g) drop_page(a, h, a.give_at, g + lane, r);
  }
}

// ---------------------------------------------------------------- cache store

__device__ __forceinline__ int to_fp8(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// fminf and fmaxf drop a NaN: it stays one
__device__ __forceinline__ float clamp_fp8(float x) { return x != x ? x : fminf(fmaxf(x, -448.0f), 448.0f); }

__device__ __forceinline__ void widen8(i32x4 x, int fp16, float* f) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (fp16) {
      f[2 * j] = (float)__builtin_bit_cast(_Float16, (short)(x[j] & 0xffff));
      f[2 * j + 1] = (float)__builtin_bit_cast(_Float16, (short)((uint32_t)x[j] >> 16));
    } else {
      f[2 * j] = __uint_as_float((uint32_t)x[j] << 16);
      f[2 * j + 1] = __uint_as_float((uint32_t)x[j] & 0xffff0000u);
    }
  }
}

// 8 elements of K and of V a thread.  Bound by memory: 131,072 tokens of 8 heads
// of 128, 1.07 GB read and written in 206 us (5.2 TB/s).
template <bool FP8>
__global__ void __launch_bounds__(256) store_kernel(StoreArgs a) {
  const uint32_t n = blockIdx.x * 256u + threadIdx.x;
  const uint32_t t = divide(n, a.chunks);
  if (t >= (uint32_t)a.tokens) return;
  const int c = (int)(n - t * a.chunks.d) * 8, head = c >> a.dim_shift, d = c & ((1 << a.dim_shift) - 1);
  const int slot = a.slots[t];
  if (slot < 0) return;
  if (slot >= a.slots_limit) {
    if (a.status) atomicOr(a.status, (uint32_t)KVR_DEV_BAD_PAGE);
    return;
  }
  const int64_t page = slot >> a.page_shift, at = slot & ((1 << a.page_shift) - 1);
  const i32x4 k = *(const i32x4*)(a.k + t * a.k_tok + head * a.k_head + d * 2);
  const i32x4 v = *(const i32x4*)(a.v + t * a.v_tok + head * a.v_head + d * 2);
  char* kc = a.kc + page * a.kc_page + at * a.kc_slot + head * a.kc_head;
  char* vc = a.vc + page * a.vc_page + at * a.vc_slot + head * a.vc_head;
  if constexpr (FP8) {
    float f[8];
    const float ks = a.ks ? 1.0f / a.ks[head] : 1.0f, vs = a.vs ? 1.0f / a.vs[head] : 1.0f;
    widen8(k, a.fp16, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = clamp_fp8(f[j] * ks);
    *(i32x2*)(kc + d) = i32x2{to_fp8(f[0], f[1], f[2], f[3]), to_fp8(f[4], f[5], f[6], f[7])};
    widen8(v, a.fp16, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = clamp_fp8(f[j] * vs);
    *(i32x2*)(vc + d) = i32x2{to_fp8(f[0], f[1], f[2], f[3]), to_fp8(f[4], f[5], f[6], f[7])};
  } else {
    *(i32x4*)(kc + d * 2) = k;
    *(i32x4*)(vc + d * 2) = v;
  }
}

// ---------------------------------------------------------------- attention: the plan

// The plan in a launch of its own: the items in memory.
template <bool SMALL>
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(AttendArgs a) {
  __shared__ __attribute__((aligned(8))) int lds[SMALL ? plan_words(kPlanSmall) : plan_words(0)];
  make_plan<SMALL ? kPlanSmall : 0>(a, lds, true, [&](int i, const Item& it) { a.items[i] = it; });
}

// ---------------------------------------------------------------- attention: the join

// (64 requests in four groups: 7 to 9 us, latency.)
// Joins the partial results of a request's unit, its own splits' and those of
// its group's prefix: m = max m_i, l = sum l_i 2^(m_i - m), o likewise.
constexpr int kJoinAtOnce = 4;

template <bool FP16>
__global__ void __launch_bounds__(256) join_kernel(AttendArgs a) {
  const int quads = a.dim / 4;
  if (a.hdr->rejected) {
    fill_with_nan(a);
    return;
  }
  // a block takes 256 quads (four elements of a row) of a unit and head at a time
  const int64_t tasks = (int64_t)a.hdr->joins * a.kv_heads;
  for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int head = (int)(task % a.kv_heads);
    const int2 join = a.joins[task / a.kv_heads];
    const Unit x = a.units[join.x];
    const float vs = a.vs ? a.vs[head] : 1.0f;
    const int i = join.y * 256 + threadIdx.x, r = i / quads, c = i % quads;
    if (r >= x.rows) continue;
    const int row = x.row0 + r;
    float m = -INFINITY, l = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    // n partial results, `step` rows apart; four are on their way at a time
    auto add = [&](int first, int step, int n) {
      for (int s0 = 0; s0 < n; s0 += kJoinAtOnce) {
        float2 ml[kJoinAtOnce];
        f32x4 y[kJoinAtOnce];
#pragma unroll
        for (int k = 0; k < kJoinAtOnce; ++k) {
          const int64_t at = (int64_t)(first + min(s0 + k, n - 1) * step) * a.kv_heads + head;
          ml[k] = a.ml[at];
          y[k] = *(const f32x4*)(a.acc + at * a.dim + c * 4);
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < kJoinAtOnce; ++k) {
          if (s0 + k >= n) ml[k] = make_float2(-INFINITY, 0.0f);
          top = fmaxf(top, ml[k].x);
        }
        const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top);
        // (before the first key of a row l and o are 0, or NaN where a key was)
        l = m == -INFINITY ? l : l * f;
        o = m == -INFINITY ? o : o * f;
        m = top;
#pragma unroll
        for (int k = 0; k < kJoinAtOnce; ++k) {
          if (s0 + k >= n) continue;
          const float h = ml[k].x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ml[k].x - top);
          l += ml[k].y * h;
          o += y[k] * h;
        }
      }
    };
    add(x.acc + r, x.rows, x.splits);
    if (x.group_unit >= 0) {
      const Unit y = a.units[x.group_unit + (row - x.group_row) / kTileRows];
      add(y.acc + row - y.row0, y.rows, y.splits);
    }
    const float f = l > 0.0f || l != l ? vs / l : 0.0f;
    const uint32_t token = divide((uint32_t)row, a.share);
    const int h = head * (int)a.share.d + (int)(row - token * a.share.d);
    char* p = a.out + token * a.o_tok + h * a.o_head + c * 8;
    if (FP16) {
      typedef _Float16 x4 __attribute__((ext_vector_type(4)));
      *(x4*)p = __builtin_convertvector(o * f, x4);
    } else {
      typedef __bf16 x4 __attribute__((ext_vector_type(4)));
      *(x4*)p = __builtin_convertvector(o * f, x4);
    }
    if (a.lse && c == 0)
      a.lse[(int64_t)token * a.heads + h] =
          l > 0.0f || l != l ? (m + __log2f(l)) * 0.69314718055994530942f : -INFINITY;
  }
}

}  // namespace

hipError_t launch_tables(const TablesArgs& a, hipStream_t st) {
  if (a.rows <= kFusedRows && a.num_tokens <= kFusedTokens) {
    tables_fused_kernel<<<dim3(1), dim3(a.rows <= 256 && a.num_tokens <= 1024 ? 256 : kScanThreads), 0, st>>>(a);
    return hipGetLastError();
  }
  tables_scan_kernel<<<dim3(1), dim3(kScanThreads), 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // blocks for the tokens; with few new tokens there may be many pages to give back
  int blocks = (int)(((int64_t)a.num_tokens + kFillThreads - 1) / kFillThreads);
  const int least = a.rows / 16 + 1 < 256 ? a.rows / 16 + 1 : 256;
  if (blocks < least) blocks = least;
  tables_fill_kernel<<<dim3(blocks), dim3(kFillThreads), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_store(const StoreArgs& a, hipStream_t st) {
  const uint32_t blocks = (uint32_t)(((int64_t)a.tokens * a.chunks.d + 255) / 256);
  if (a.fp8)
    store_kernel<true><<<dim3(blocks), dim3(256), 0, st>>>(a);
  else
    store_kernel<false><<<dim3(blocks), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

// Each workgroup plans for itself, which saves a launch, while the device holds
// most of them at once (eight requests, 18.8 -> 15.9 us; 64 requests, 77.5 ->
// 76.3; 157 requests of one key head, 20.8 -> 18.8).  Where they come in several
// rounds each round pays (127 requests, eight heads of 256: 90 -> 99 us).
bool attend_fused(const AttendArgs& a) {
  const int64_t held = (a.dim == 256 ? 1 : 2) * kComputeUnits;
  return a.unit_cap <= kPlanFused && a.requests <= kPlanFused && a.groups <= kPlanFused &&
         (int64_t)a.unit_cap * a.kv_heads <= 2 * held;
}

// Where the tables have no room for keys enough that a unit is split or a prefix
// shared, nothing can be joined: no join kernel (eight requests of up to 48 own
// and 64 shared tokens: 16.3 -> 12.9 us a call).
bool attend_direct(const AttendArgs& a) {
  const int64_t own = (a.own_room + kStepKeys - 1) / kStepKeys;
  const int64_t prefix = a.groups ? (a.prefix_room + kStepKeys - 1) / kStepKeys : 0;
  const int64_t waves = (int64_t)a.tokens * a.share.d <= 32 ? a.few_waves : 4;
  return prefix < kMinSharedSteps && (own + prefix) * waves <= kMinSplitCost;
}

hipError_t launch_attend_plan(const AttendArgs& a, hipStream_t st) {
  if (a.fused) return hipSuccess;
  const dim3 threads(a.unit_cap <= 256 ? 256 : kPlanThreads);
  if (a.requests <= kPlanSmall && a.groups <= kPlanSmall)
    plan_kernel<true><<<dim3(1), threads, 0, st>>>(a);
  else
    plan_kernel<false><<<dim3(1), threads, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_attend_join(const AttendArgs& a, bool fp16, hipStream_t st) {
  if (a.direct) return hipSuccess;
  // what there is to join only the plan knows: as many blocks as the device
  // holds at once, or fewer where there cannot be so many parts
  const int64_t parts = (int64_t)a.join_cap * a.kv_heads;
  const dim3 blocks((uint32_t)(parts < 8 * kComputeUnits ? parts : 8 * kComputeUnits));
  if (fp16)
    join_kernel<true><<<blocks, dim3(256), 0, st>>>(a);
  else
    join_kernel<false><<<blocks, dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace kvr
