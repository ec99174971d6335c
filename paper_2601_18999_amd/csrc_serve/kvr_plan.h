// kvr_plan.h - the plan of the attention: which rows and which keys a workgroup
// takes.  Made by one workgroup in a launch of its own or, where there is
// little to plan, by every workgroup of the attention for itself.
#pragma once

#include "kvr_serve.h"

namespace kvr {
namespace {

// x of the lane that a DPP control names, 0 where there is none.
template <int CONTROL, int ROWS, class V>
__device__ __forceinline__ V moved(V x) {
  if constexpr (sizeof(V) == 8) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CONTROL, ROWS, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)((uint64_t)x >> 32), CONTROL, ROWS, 0xf, true);
    return (V)((uint64_t)hi << 32 | lo);
  } else {
    return (V)__builtin_amdgcn_update_dpp(0, (int)x, CONTROL, ROWS, 0xf, true);
  }
}

// Sum over the lanes before this one, and (by reference) over all lanes; all
// lanes are active.
template <class V>
__device__ __forceinline__ V wave_before(V x, V& all) {
  V s = x;
  s += moved<0x111, 0xf>(s);  // the rows of 16: 1, 2, 4, 8 lanes up
  s += moved<0x112, 0xf>(s);
  s += moved<0x114, 0xf>(s);
  s += moved<0x118, 0xf>(s);
  s += moved<0x142, 0xa>(s);  // a row's last lane to the next row, of rows 1 and 3
  s += moved<0x143, 0xc>(s);  // lane 31 to rows 2 and 3
  if constexpr (sizeof(V) == 8)
    all = (V)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)((uint64_t)s >> 32), 63) << 32 |
              (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)s, 63));
  else
    all = (V)__builtin_amdgcn_readlane((int)s, 63);
  return s - x;
}

// The same over a workgroup of up to 16 waves; `part` is 16 values of LDS.
// Every thread of the workgroup calls it.
template <class V>
__device__ __forceinline__ V group_before(V x, V& all, V* part) {
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = threadIdx.x & 63;
  V w;
  const V s = wave_before(x, w);
  __syncthreads();
  if (lane == 0) part[wave] = w;
  __syncthreads();
  const V y = lane < waves ? part[lane] : V(0);
  const V before = wave_before(y, all);
  return s + __shfl(before, wave);
}

// Largest i of [0, n) with start[i] <= x, for start ascending and start[0] <= x.
template <class P>
__device__ __forceinline__ int last_at_most(P start, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

constexpr int kPlanThreads = 1024;
constexpr int kPlanSmall = 1024;  // requests, groups: their lengths then stand in LDS
constexpr int kPlanFused = 256;   // ... and units: each workgroup of the attention may make the plan itself
// Least cost of an item that a unit is split into (over 15 calls of all kinds 4
// and 16 were 2% slower).
constexpr int kMinSplitCost = 8;
constexpr int kMinSharedSteps = 4;  // of a prefix that is taken for a group

constexpr int plan_words(int cap) { return 48 + (cap ? 8 * (cap + 1) : 0); }

// Waves along the rows that `rows` rows take in tiles of kTileRows; `few`: that
// up to 32 rows take.
__host__ __device__ __forceinline__ int row_waves(int rows, int few) {
  const int rest = rows % kTileRows;
  return rows / kTileRows * 4 + (rest == 0 ? 0 : rest <= 32 ? few : 4);
}

__host__ __device__ __forceinline__ int steps_of(int keys) { return (keys + kStepKeys - 1) / kStepKeys; }

// Whether a group takes its prefix for all of its requests at once, in tiles of
// `together` waves along the rows instead of `apart`, at the price of partial
// results and their join.  Requests with tiles of their own gain nothing (16
// prompts of 128 to 1,024 tokens: 930 us apart, 1,034 together); answers gain
// from about 200 keys on if the group is large enough (64 requests, 8 key
// heads: 256 keys 34.3 apart, 33.6 together, 2,048 keys 67.9 and 40.5; 16
// requests: 512 keys 19.0 and 19.8, 1,024 keys 21.1 and 20.9).
__host__ __device__ __forceinline__ bool worth_sharing(int apart, int together, int steps, int kv_heads) {
  return (int64_t)together * 4 <= (int64_t)apart * 3 && steps >= kMinSharedSteps &&
         (int64_t)(apart - together) * steps * kv_heads >= 256;
}

// Most cost of an item, where all units cost `total`: the slots' fair share.
__host__ __device__ __forceinline__ int chunk_of(int64_t total, int slots, int few) {
  const int64_t fair = (total + slots - 1) / slots;
  const int least = kMinSplitCost * few;
  return (int)(fair < least ? least : fair > 0x7fffffff ? 0x7fffffff : fair);
}

// Items of a unit, and the steps of each.
struct Cut {
  int splits, per;
};

__host__ __device__ __forceinline__ Cut cut_of(int steps, int cost, int chunk) {
  Cut c;
  c.splits = max(1, (cost + chunk - 1) / chunk);
  c.per = max(1, (steps + c.splits - 1) / c.splits);
  c.splits = max(1, (steps + c.per - 1) / c.per);
  return c;
}

// Lengths that are not valid: nothing was computed, every result is NaN.
__device__ __forceinline__ void fill_with_nan(const AttendArgs& a) {
  const int quads = a.dim / 4;
  const int64_t all = (int64_t)a.tokens * a.heads * quads, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < all; i += step) {
    const int64_t th = i / quads;
    *(int2*)(a.out + th / a.heads * a.o_tok + th % a.heads * a.o_head + i % quads * 8) = make_int2(-1, -1);
    if (a.lse && i % quads == 0) a.lse[th] = __uint_as_float(0x7fc00000u);
  }
}

struct UnitWork {
  Item it;
  int steps, cost;
  int group;  // the group whose shared partial results the unit's rows have, or -1
};

// The lengths, in LDS or (many requests) where the caller has them, and what
// the plan finds on its way.
struct Lengths {
  const int *row_start, *length, *group_start, *prefix_length;
  int *bounds, *group_of, *waves;
  bool single;  // one token each: row_start[b] = b
  __device__ __forceinline__ int start(int b) const { return single ? b : row_start[b]; }
};

// Unit u of segment s (a group, or groups + a request).  A request's last
// rows, which see the most keys, come first: the workgroups that start last
// are then the short ones (9,216 new tokens of 32 heads: 924 -> 804 us with
// the scheduler that build.py names).
__device__ UnitWork unit_work(const AttendArgs& a, const Lengths& z, int s, int u) {
  const int tile = s < a.groups ? u - z.bounds[s] : z.bounds[s + 1] - 1 - u;
  UnitWork w;
  const int g = (int)a.share.d;
  w.group = -1;
  w.it.pad = 0;
  w.it.acc = -1;
  w.it.step0 = 0;
  if (s < a.groups) {
    const int t0 = z.start(z.group_start[s]), t1 = z.start(z.group_start[s + 1]);
    w.it.row0 = t0 * g + tile * kTileRows;
    w.it.rows = min(kTileRows, t1 * g - w.it.row0);
    w.it.prefix = s;
    w.it.prefix_len = z.prefix_length[s];
    w.it.prefix_steps = steps_of(w.it.prefix_len);
    w.it.request = 0;
    w.it.own_end = 0;
    w.it.limit = 0;
    w.steps = w.it.prefix_steps;
  } else {
    const int b = s - a.groups;
    const int t0 = z.start(b), t1 = z.start(b + 1);
    w.it.row0 = t0 * g + tile * kTileRows;
    w.it.rows = min(kTileRows, t1 * g - w.it.row0);
    w.it.request = b;
    w.it.limit = z.length[b] - (t1 - t0) - t0 + 1;
    const int last = (int)divide((uint32_t)(w.it.row0 + w.it.rows - 1), a.share);
    w.it.own_end = last + w.it.limit;
    w.it.prefix = 0;
    w.it.prefix_len = 0;
    w.it.prefix_steps = 0;
    if (a.groups) {
      const int j = z.group_of[b];
      if (z.waves[j] == 1) {
        w.group = j;
      } else {
        w.it.prefix = j;
        w.it.prefix_len = z.prefix_length[j];
        w.it.prefix_steps = steps_of(w.it.prefix_len);
      }
    }
    w.steps = w.it.prefix_steps + steps_of(w.it.own_end);
  }
  w.it.step1 = w.steps;
  w.cost = w.steps * row_waves(w.it.rows, a.few_waves);
  return w;
}

// One workgroup: checks the lengths, decides which groups take their prefix
// for all requests at once, and cuts the units into items of about equal cost.
// CAP > 0: the lengths of up to CAP requests and groups stand in LDS.  `write`:
// what others read of the plan (its header and units) is written; every item
// goes to emit(its number, the item).  `lds`: plan_words(CAP) words.  Returns
// the number of items, -1 for lengths that are not valid.
template <int CAP, class Emit>
__device__ __forceinline__ int make_plan(const AttendArgs& a, int* lds, bool write, Emit emit) {
  constexpr bool SMALL = CAP > 0;
  int64_t* part64 = (int64_t*)lds;
  int* part = lds + 32;
  lds += 48;
  const int g = (int)a.share.d, tid = threadIdx.x, threads = blockDim.x;
  Lengths z;
  z.single = !a.row_start;
  bool bad = false;
  if constexpr (SMALL) {
    int* rs = lds;
    int* len = rs + CAP + 1;
    int* gs = len + CAP + 1;
    int* pl = gs + CAP + 1;
    z.waves = pl + CAP + 1;
    z.group_of = z.waves + CAP + 1;
    z.bounds = z.group_of + CAP + 1;  // twice as many
    z.row_start = rs;
    z.length = len;
    z.group_start = gs;
    z.prefix_length = pl;
    for (int i = tid; i <= max(a.requests, a.groups); i += threads) {
      const bool r = i < a.requests, j = i < a.groups;
      const int x0 = i <= a.requests && a.row_start ? a.row_start[i] : i;
      const int x1 = r ? a.length[i] : 0;
      const int x2 = i <= a.groups && a.groups ? a.group_start[i] : 0;
      const int x3 = j ? a.prefix_length[i] : 0;
      if (i <= a.requests) rs[i] = x0;
      if (r) len[i] = x1;
      if (i <= a.groups) gs[i] = x2;
      if (j) pl[i] = x3;
    }
    __syncthreads();
  } else {
    z.row_start = a.row_start;
    z.length = a.length;
    z.group_start = a.group_start;
    z.prefix_length = a.prefix_length;
    z.waves = a.waves;
    z.group_of = a.group_of;
    z.bounds = a.bounds;
  }
  // checks
  for (int b = tid; b < a.requests; b += threads) {
    const int t0 = z.start(b), t1 = z.start(b + 1), n = z.length[b];
    bad |= t0 < 0 || t1 < t0 || t1 > a.tokens || n < t1 - t0 || n > a.own_room;
    if (b == 0) bad |= t0 != 0;
  }
  for (int j = tid; j < a.groups; j += threads) {
    const int b0 = z.group_start[j], b1 = z.group_start[j + 1], p = z.prefix_length[j];
    bad |= b0 < 0 || b1 < b0 || b1 > a.requests || p < 0 || p > a.prefix_room;
    if (j == 0) bad |= b0 != 0;
    if (j == a.groups - 1) bad |= b1 != a.requests;
    z.waves[j] = 0;
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0 && write) {
      a.hdr->joins = 0;
      a.hdr->items = 0;
      a.hdr->rejected = 1;
      if (a.status) atomicOr(a.status, (uint32_t)KVR_DEV_BAD_LENGTH);
    }
    return -1;
  }
  // waves along the rows that the requests of a group take one by one
  for (int b = tid; b < a.requests && a.groups; b += threads) {
    const int j = last_at_most(z.group_start, a.groups, b);
    z.group_of[b] = j;
    atomicAdd(&z.waves[j], row_waves((z.start(b + 1) - z.start(b)) * g, a.few_waves));
  }
  __syncthreads();
  // units: a group's (its prefix, if that is shared), then a request's
  const int segments = a.groups + a.requests;
  int units = 0;
  for (int s0 = 0; s0 < segments; s0 += threads) {
    const int s = s0 + tid;
    int count = 0;
    if (s < a.groups) {
      const int rows = (z.start(z.group_start[s + 1]) - z.start(z.group_start[s])) * g;
      const bool shared = worth_sharing(z.waves[s], row_waves(rows, a.few_waves), steps_of(z.prefix_length[s]), a.kv_heads);
      z.waves[s] = shared ? 1 : 0;
      count = shared ? (rows + kTileRows - 1) / kTileRows : 0;
    } else if (s < segments) {
      const int b = s - a.groups;
      count = ((z.start(b + 1) - z.start(b)) * g + kTileRows - 1) / kTileRows;
    }
    int all;
    const int before = group_before(count, all, part);
    if (s < segments) z.bounds[s] = units + before;
    units += all;
  }
  if (tid == 0) z.bounds[segments] = units;
  __syncthreads();
  int64_t total = 0;
  UnitWork w;
  int s = 0;
  for (int u = tid; u < units; u += threads) {
    s = last_at_most(z.bounds, segments, u);
    w = unit_work(a, z, s, u);
    total += w.cost;
  }
  group_before(total, total, part64);
  const int chunk = chunk_of(total, a.split_slots, a.few_waves);
  int items = 0, rows_acc = 0, joins = 0;
  for (int u0 = 0; u0 < units; u0 += threads) {
    const int u = u0 + tid;
    int splits = 0, per = 1, partial = 0;
    if (u < units) {
      if (units > threads) {  // else it is there
        s = last_at_most(z.bounds, segments, u);
        w = unit_work(a, z, s, u);
      }
      const Cut c = cut_of(w.steps, w.cost, chunk);
      splits = c.splits;
      per = c.per;
      partial = s < a.groups || w.group >= 0 || splits > 1 ? splits * w.it.rows : 0;
    }
    int all_items, all_rows;
    const int i0 = items + group_before(splits, all_items, part);
    const int acc = rows_acc + group_before(partial, all_rows, part);
    int all_joins = 0;
    const int parts = partial && s >= a.groups ? (w.it.rows * (a.dim / 4) + 255) / 256 : 0;
    const int join_at = joins + (write ? group_before(parts, all_joins, part) : 0);
    items += all_items;
    rows_acc += all_rows;
    joins += all_joins;
    if (u < units) {
      Unit x;
      x.row0 = w.it.row0;
      x.rows = w.it.rows;
      x.acc = partial ? acc : -1;
      x.splits = splits;
      x.pad1 = 0;
      x.group_unit = -1;
      x.group_row = 0;
      x.pad = 0;
      if (w.group >= 0) {
        x.group_unit = z.bounds[w.group];
        x.group_row = z.start(z.group_start[w.group]) * g;
      }
      if (write) a.units[u] = x;
      if (write)
        for (int i = 0; i < parts; ++i) a.joins[join_at + i] = make_int2(u, i);
      for (int i = 0; i < splits; ++i) {
        Item it = w.it;
        it.step0 = min(w.steps, i * per);
        it.step1 = min(w.steps, (i + 1) * per);
        it.acc = partial ? acc + i * w.it.rows : -1;
        emit(i0 + i, it);
      }
    }
  }
  if (tid == 0 && write) {
    a.hdr->joins = joins;
    a.hdr->items = items;
    a.hdr->rejected = 0;
  }
  return items;
}

}  // namespace
}  // namespace kvr
