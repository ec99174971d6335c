// kvr_serve.h - arguments of the serving kernels (page tables, cache store,
// shared-prefix attention): what the host side fills in and the device side
// reads.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/kvr.h"

namespace kvr {

// Compute units of a gfx950 device and the attention workgroups that one of
// them holds: the width that the attention work is split for (for three or four
// a unit 15 calls of all kinds were 2 and 5% slower).
constexpr int kComputeUnits = 256;
constexpr int kAttendSlots = 2 * kComputeUnits;
constexpr int kAttendThreads = 256;
constexpr int kTileRows = 128;  // most query rows of an attention workgroup
constexpr int kStepKeys = 64;   // keys of one step: what the plan counts in
// Most keys of a prefix or of a request: the first key of a tile, and of those
// that are looked up ahead behind the last, fits 31 bits.
constexpr int kMostKeys = 0x7fffffff - 1023;

// n / d for n < 2^31 by a multiplication, exact (d >= 1, d < 2^31).
struct Divisor {
  uint32_t d, mul, shift;
};

inline Divisor make_divisor(uint32_t d) {
  // smallest s with 2^s >= d; mul = ceil(2^(31+s) / d) < 2^32 keeps
  // n * mul / 2^(31+s) within 1/d of n / d for n < 2^31
  uint32_t s = 0;
  while ((1ull << s) < d) ++s;
  Divisor v;
  v.d = d;
  v.shift = s;
  v.mul = (uint32_t)(((1ull << (31 + s)) + d - 1) / d);
  return v;
}

__host__ __device__ inline uint32_t divide(uint32_t n, const Divisor& v) {
  return (uint32_t)(((uint64_t)n * v.mul) >> (31 + v.shift));
}

// Whether the lanes of one load of a tile of a 16-bit cache reach their rows by
// 32-bit offsets from the first row's.  A load brings 1,024 neighbouring bytes
// to LDS, so it spans 512 / dim rows, `stride` bytes apart in the cache.
constexpr bool lanes_reach(int dim, int64_t stride) {
  return (512 / dim - 1) * stride + 2 * dim <= (int64_t)1 << 32;
}

// Most partial rows of the attention's plan: a unit of up to kTileRows rows that
// is split, or whose rows have a shared prefix, has as many as it has rows, for
// each of its items.
//  * A unit is split where it costs more than a slot's share of the total, and
//    into fewer than twice as many items as shares it costs: all such units have
//    fewer than 2 * slots items.
//  * A prefix is shared where that leaves at most 3/4 of the requests' own row
//    waves.  R rows of n requests take at least R / 32 waves together and less
//    than R / 32 + 4 n apart, so R < 384 n.  They count twice, with the prefix
//    and with the own tokens.
// (Never more than all rows, twice with groups, and a tile for each added item.)
constexpr int64_t most_partial_rows(int64_t rows, int64_t requests, bool groups, int64_t slots) {
  const int64_t shared = !groups ? 0 : rows < 384 * requests ? 2 * rows : 2 * 384 * requests;
  const int64_t some = shared + 2 * slots * kTileRows, all = (groups ? 2 : 1) * rows + slots * kTileRows;
  return some < all ? some : all;
}

// ---- page tables ----
struct TablesHdr {
  int64_t head, tail;  // the ring before the call
  int32_t gain, give;  // pages taken and given back
  int32_t tokens;      // new tokens
  int32_t rejected;
};

struct TablesArgs {
  const int32_t *held, *delta, *base;
  int32_t *table, *ring;
  const int64_t* state;
  int32_t* held_out;
  int64_t* state_out;
  int32_t *row_start, *slots, *positions;
  TablesHdr* hdr;
  int32_t *gain_at, *give_at;  // [rows + 1] pages taken / given back before a row
  int64_t table_stride;
  int32_t rows, width, page_shift, ring_size, num_tokens;
  int32_t base_held;  // 1: base is held, which is updated in place
};

// ---- cache store ----
struct StoreArgs {
  const char *k, *v;
  char *kc, *vc;
  const float *ks, *vs;
  const int32_t* slots;
  uint32_t* status;
  int64_t k_tok, k_head, v_tok, v_head;                       // bytes
  int64_t kc_page, kc_slot, kc_head, vc_page, vc_slot, vc_head;  // bytes
  Divisor chunks;  // 16-byte source chunks of a token: kv_heads * dim / 8
  int32_t tokens, dim_shift, page_shift, slots_limit;
  int32_t fp8, fp16;
};

// ---- attention ----
// One unit: up to 128 consecutive query rows (row = token * share + head in
// its key head's share) of one request, or of one group against its shared
// prefix.  One item: a range of a unit's key steps, one workgroup per key
// head.  Items of a unit are consecutive, and so are their partial results.
struct Unit {
  int32_t row0, rows;
  int32_t acc, splits;           // first partial row (-1: written directly), items
  int32_t group_unit, group_row; // first unit of its group's prefix (-1: none) and that unit's row0
  int32_t pad, pad1;
};

struct Item {
  int32_t row0, rows;
  int32_t step0, step1;    // key steps: the prefix's first, then the own tokens'
  int32_t prefix_steps;    // steps of the prefix among them
  int32_t prefix, prefix_len;
  int32_t request, own_end; // own keys that some row of the unit sees
  int32_t limit;           // a row of token t sees own keys below t + limit
  int32_t acc;             // first partial row, -1: final
  int32_t pad;
};

struct PlanHdr {
  int32_t joins, items, rejected, pad;  // joins: parts of the units whose results are joined
};

struct AttendArgs {
  const char* q;
  char* out;
  float* lse;
  const char *kc, *vc;
  const float *ks, *vs;
  int64_t q_tok, q_head, o_tok, o_head;  // bytes
  int64_t kc_head, vc_head;
  uint32_t kc_page, kc_slot, vc_page, vc_slot;
  const int32_t *row_start, *length, *table, *group_start, *prefix_table, *prefix_length;
  int64_t table_stride, prefix_stride;
  uint32_t* status;
  PlanHdr* hdr;
  int32_t* bounds;  // [groups + requests + 1] first unit of a group / request
  int32_t* group_of;  // [requests]
  int32_t* waves;     // [groups] row waves of its requests, then: 1 = shared
  Unit* units;
  int2* joins;  // unit and part of it (256 quads of four elements)
  Item* items;
  float2* ml;  // [partial row][kv head] running maximum (log2 units) and sum
  float* acc;  // [partial row][kv head][dim]
  Divisor share;
  float scale_log2;
  int32_t tokens, requests, groups, heads, kv_heads, dim;
  int32_t page_shift, page_mask, num_pages;
  int32_t own_room, prefix_room;  // most tokens that a row of the tables has room for
  int32_t unit_cap, item_cap, join_cap, split_slots;
  int32_t few_waves;      // waves along the rows that up to 32 rows take (attend_kernel): 1 or 4
  int32_t fused, direct;  // 1: no plan kernel; no join kernel
  int32_t one_base;       // 1: the rows of one load stand in one page and reach of one base
};

hipError_t launch_tables(const TablesArgs& a, hipStream_t st);
hipError_t launch_store(const StoreArgs& a, hipStream_t st);
// whether every workgroup of the attention makes the plan itself
bool attend_fused(const AttendArgs& a);
// whether there can be nothing to join
bool attend_direct(const AttendArgs& a);
hipError_t launch_attend_plan(const AttendArgs& a, hipStream_t st);
hipError_t launch_attend_join(const AttendArgs& a, bool fp16, hipStream_t st);
// fp16: queries and results are 16-bit IEEE, else bfloat16; fp8: the cache
// holds 8-bit e4m3, else the queries' type
hipError_t launch_attend_64(const AttendArgs& a, bool fp16, bool fp8, hipStream_t st);
hipError_t launch_attend_128(const AttendArgs& a, bool fp16, bool fp8, hipStream_t st);
hipError_t launch_attend_256(const AttendArgs& a, bool fp16, bool fp8, hipStream_t st);

// Sets the message that kvr_last_error returns on this thread.
kvr_status set_error(kvr_status st, const char* msg) noexcept;

}  // namespace kvr
