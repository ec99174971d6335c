// kvr_serve_api.cpp - host side of the serving operators of include/kvr.h:
// checks of the arguments, layout of the workspaces, launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "kvr_checks.h"
#include "kvr_serve.h"

namespace {

using kvr::aligned;
using kvr::hip_failed;
using kvr::invalid;
using kvr::kInt;
using kvr::on_chunks;
using kvr::round_up;
using kvr::set_error;
using kvr::step;

bool power_of_two(int32_t x) { return x > 0 && (x & (x - 1)) == 0; }

int log2_of(int32_t x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

kvr_status check(const kvr_tables* t) {
  if (!t) return invalid("tables is NULL");
  if (t->struct_size != sizeof(kvr_tables)) return invalid("struct_size mismatch (kvr_tables)");
  if (t->rows < 1 || t->rows > (1 << 20)) return invalid("rows must be in 1..2^20");
  if (!power_of_two(t->page_size) || t->page_size > 1024) return invalid("page_size must be a power of two in 1..1024");
  if (t->width < 1 || (int64_t)t->rows * t->width > kInt) return invalid("width must be >= 1, rows * width < 2^31");
  if (t->ring_size < 1 || (int64_t)t->ring_size * t->page_size > kInt)
    return invalid("ring_size must be >= 1, ring_size * page_size < 2^31");
  if (t->num_tokens < 0) return invalid("num_tokens must be >= 0");
  if (t->table_stride < t->width) return invalid("table_stride must be >= width");
  return KVR_OK;
}

size_t tables_bytes(const kvr_tables* t) { return 256 + 2 * round_up(((size_t)t->rows + 1) * 4); }

kvr_status check(const kvr_cache* c) {
  if (!c) return invalid("cache is NULL");
  if (c->struct_size != sizeof(kvr_cache)) return invalid("struct_size mismatch (kvr_cache)");
  if (c->dtype != KVR_BF16 && c->dtype != KVR_FP16 && c->dtype != KVR_FP8) return invalid("unknown cache dtype");
  if (!power_of_two(c->page_size) || c->page_size > 1024) return invalid("page_size must be a power of two in 1..1024");
  if (c->num_pages < 1 || (int64_t)c->num_pages * c->page_size > kInt)
    return invalid("num_pages must be >= 1, num_pages * page_size < 2^31");
  if (c->kv_heads < 1 || c->kv_heads > 1024) return invalid("kv_heads must be in 1..1024");
  if (c->dim != 64 && c->dim != 128 && c->dim != 256) return invalid("dim must be 64, 128 or 256");
  if (c->dtype != KVR_FP8 && (c->d_k_scale || c->d_v_scale)) return invalid("scales are for an 8-bit cache");
  return KVR_OK;
}

// The strides of a cache in bytes.
struct CacheSteps {
  int64_t page, slot, head;
};

CacheSteps steps(const kvr_cache* c, int64_t page, int64_t slot, int64_t head) {
  const int size = c->dtype == KVR_FP8 ? 1 : 2;
  return {step(page, c->num_pages, size), step(slot, c->page_size, size), step(head, c->kv_heads, size)};
}

kvr_status check_buffers(const kvr_cache* c, CacheSteps* k, CacheSteps* v) {
  if (!c->d_k || !c->d_v) return invalid("d_k and d_v are required");
  *k = steps(c, c->k_page, c->k_slot, c->k_head);
  *v = steps(c, c->v_page, c->v_slot, c->v_head);
  if (!aligned(c->d_k, 16) || !aligned(c->d_v, 16) || !on_chunks(k->page, k->slot, k->head) ||
      !on_chunks(v->page, v->slot, v->head))
    return invalid("every head of the cache must start on a 16-byte boundary");
  // the kernels multiply by these in 32 bits
  for (const int64_t stride : {k->page, k->slot, v->page, v->slot})
    if (stride < 0 || stride > kInt) return invalid("strides of pages and slots must be in 0..2^31 - 1 bytes");
  return KVR_OK;
}

// Tokens of a row of a table, at most as many as the kernels count.
int32_t room(int32_t width, int32_t page_size) {
  const int64_t n = (int64_t)width * page_size;
  return (int32_t)(n < kvr::kMostKeys ? n : kvr::kMostKeys);
}

struct AttendLayout {
  size_t bounds, group_of, waves, units, joins, items, ml, acc, bytes;
  int32_t unit_cap, item_cap, join_cap, split_slots;
};

kvr_status check(const kvr_cache* c, const kvr_attention* a) {
  const kvr_status st = check(c);
  if (st != KVR_OK) return st;
  if (!a) return invalid("attention is NULL");
  if (a->struct_size != sizeof(kvr_attention)) return invalid("struct_size mismatch (kvr_attention)");
  if (a->dtype != KVR_BF16 && a->dtype != KVR_FP16) return invalid("queries must be KVR_BF16 or KVR_FP16");
  if (c->dtype != KVR_FP8 && c->dtype != a->dtype) return invalid("queries and a 16-bit cache must have one type");
  if (a->num_tokens < 0) return invalid("num_tokens must be >= 0");
  if (a->num_requests < 1 || a->num_requests > (1 << 20)) return invalid("num_requests must be in 1..2^20");
  if (a->num_groups < 0 || a->num_groups > (1 << 20)) return invalid("num_groups must be in 0..2^20");
  if (a->heads < 1 || a->heads % c->kv_heads) return invalid("heads must be a positive multiple of kv_heads");
  if ((int64_t)a->num_tokens * a->heads > kInt) return invalid("num_tokens * heads must be below 2^31");
  if (a->width < 0 || a->prefix_width < 0) return invalid("width and prefix_width must be >= 0");
  if (!a->d_row_start && a->num_tokens != a->num_requests)
    return invalid("without d_row_start there is one token a request");
  if (!(a->scale > 0.0f) || !std::isfinite(a->scale)) return invalid("scale must be finite and > 0");
  return KVR_OK;
}

// Most units and items that the plan can make: a request's and a group's rows
// end in one tile that is not full each, and the items of the units that are
// split add at most split_slots.
kvr_status lay_out(const kvr_cache* c, const kvr_attention* a, AttendLayout* l) {
  const int64_t rows = (int64_t)a->num_tokens * (a->heads / c->kv_heads);
  const int64_t parts = a->num_groups ? 2 : 1;
  const int64_t units = parts * (rows / kvr::kTileRows) + a->num_requests + a->num_groups;
  l->split_slots = kvr::kAttendSlots / c->kv_heads > 0 ? kvr::kAttendSlots / c->kv_heads : 1;
  const int64_t items = units + l->split_slots;
  // (a launch has fewer than 2^32 threads)
  if (items * c->kv_heads >= (1ll << 32) / kvr::kAttendThreads)
    return invalid("too many heads and requests for one launch: (num_tokens * heads / kv_heads / 128 * (2 with groups) + "
                   "num_requests + num_groups + 512 / kv_heads) * kv_heads must be below 2^24");
  const int64_t partial = kvr::most_partial_rows(rows, a->num_requests, a->num_groups > 0, l->split_slots);
  l->unit_cap = (int32_t)units;
  l->item_cap = (int32_t)items;
  size_t at = 256;
  l->bounds = at;
  at += round_up(((size_t)a->num_groups + a->num_requests + 1) * 4);
  l->group_of = at;
  at += round_up((size_t)a->num_requests * 4);
  l->waves = at;
  at += round_up((size_t)a->num_groups * 4);
  l->units = at;
  at += round_up((size_t)units * sizeof(kvr::Unit));
  l->joins = at;
  const int64_t joins = rows * c->dim / 1024 + units;
  l->join_cap = (int32_t)(joins < kInt ? joins : kInt);
  at += round_up((size_t)joins * sizeof(int2));
  l->items = at;
  at += round_up((size_t)items * sizeof(kvr::Item));
  l->ml = at;
  at += round_up((size_t)partial * c->kv_heads * sizeof(float2));
  l->acc = at;
  at += round_up((size_t)partial * c->kv_heads * c->dim * sizeof(float));
  l->bytes = at;
  return KVR_OK;
}

}  // namespace

extern "C" {

kvr_status kvr_block_tables_workspace(const kvr_tables* t, size_t* bytes) {
  const kvr_status st = check(t);
  if (st != KVR_OK) return st;
  if (!bytes) return invalid("bytes is NULL");
  *bytes = tables_bytes(t);
  return KVR_OK;
}

kvr_status kvr_block_tables(const kvr_tables* t, void* d_workspace, size_t bytes, void* hip_stream) {
  const kvr_status st = check(t);
  if (st != KVR_OK) return st;
  if (!t->d_held || !t->d_delta || !t->d_table || !t->d_ring || !t->d_state || !t->d_held_out || !t->d_state_out ||
      !t->d_row_start || (t->num_tokens && (!t->d_slots || !t->d_positions)))
    return invalid("a required pointer is NULL");
  if (t->d_held_out == t->d_delta || t->d_row_start == t->d_held || t->d_row_start == t->d_delta ||
      t->d_row_start == t->d_base || (t->d_held_out == t->d_base && t->d_held_out != t->d_held))
    return invalid("an output is an input");
  if (!d_workspace || !aligned(d_workspace, 16)) return invalid("the workspace must be on a 16-byte boundary");
  if (bytes < tables_bytes(t)) return set_error(KVR_ENOMEM, "workspace too small (kvr_block_tables_workspace)");
  kvr::TablesArgs a;
  char* ws = static_cast<char*>(d_workspace);
  a.held = t->d_held;
  a.delta = t->d_delta;
  a.base = t->d_base;
  a.table = t->d_table;
  a.ring = t->d_ring;
  a.state = t->d_state;
  a.held_out = t->d_held_out;
  a.state_out = t->d_state_out;
  a.row_start = t->d_row_start;
  a.slots = t->d_slots;
  a.positions = t->d_positions;
  a.hdr = reinterpret_cast<kvr::TablesHdr*>(ws);
  a.gain_at = reinterpret_cast<int32_t*>(ws + 256);
  a.give_at = reinterpret_cast<int32_t*>(ws + 256 + round_up(((size_t)t->rows + 1) * 4));
  a.table_stride = t->table_stride;
  a.rows = t->rows;
  a.width = t->width;
  a.page_shift = log2_of(t->page_size);
  a.ring_size = t->ring_size;
  a.num_tokens = t->num_tokens;
  a.base_held = t->d_base == t->d_held_out;
  const hipError_t e = kvr::launch_tables(a, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? KVR_OK : hip_failed(e, "table kernels launch");
}

kvr_status kvr_cache_store(const kvr_cache* c, const kvr_store* s, void* hip_stream) {
  kvr_status st = check(c);
  if (st != KVR_OK) return st;
  if (!s) return invalid("store is NULL");
  if (s->struct_size != sizeof(kvr_store)) return invalid("struct_size mismatch (kvr_store)");
  if (s->dtype != KVR_BF16 && s->dtype != KVR_FP16) return invalid("keys and values must be KVR_BF16 or KVR_FP16");
  if (c->dtype != KVR_FP8 && c->dtype != s->dtype) return invalid("a 16-bit cache holds the type that is stored");
  const int64_t chunks = (int64_t)c->kv_heads * c->dim / 8;
  if (s->num_tokens < 0 || s->num_tokens * chunks > kInt - 256)
    return invalid("num_tokens must be >= 0, num_tokens * kv_heads * dim / 8 at most 2^31 - 257");
  if (s->num_tokens == 0) return KVR_OK;
  CacheSteps kc, vc;
  st = check_buffers(c, &kc, &vc);
  if (st != KVR_OK) return st;
  if (!s->d_k || !s->d_v || !s->d_slots) return invalid("d_k, d_v and d_slots are required");
  kvr::StoreArgs a;
  a.k_tok = step(s->k_token, s->num_tokens, 2);
  a.k_head = step(s->k_head, c->kv_heads, 2);
  a.v_tok = step(s->v_token, s->num_tokens, 2);
  a.v_head = step(s->v_head, c->kv_heads, 2);
  if (!aligned(s->d_k, 16) || !aligned(s->d_v, 16) || !on_chunks(a.k_tok, a.k_head) || !on_chunks(a.v_tok, a.v_head))
    return invalid("every head of the keys and values must start on a 16-byte boundary");
  a.k = static_cast<const char*>(s->d_k);
  a.v = static_cast<const char*>(s->d_v);
  a.kc = static_cast<char*>(c->d_k);
  a.vc = static_cast<char*>(c->d_v);
  a.ks = c->d_k_scale;
  a.vs = c->d_v_scale;
  a.slots = s->d_slots;
  a.status = s->d_status;
  a.kc_page = kc.page;
  a.kc_slot = kc.slot;
  a.kc_head = kc.head;
  a.vc_page = vc.page;
  a.vc_slot = vc.slot;
  a.vc_head = vc.head;
  a.chunks = kvr::make_divisor((uint32_t)chunks);
  a.tokens = s->num_tokens;
  a.dim_shift = log2_of(c->dim);
  a.page_shift = log2_of(c->page_size);
  a.slots_limit = c->num_pages * c->page_size;
  a.fp8 = c->dtype == KVR_FP8;
  a.fp16 = s->dtype == KVR_FP16;
  const hipError_t e = kvr::launch_store(a, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? KVR_OK : hip_failed(e, "store kernel launch");
}

kvr_status kvr_attention_workspace(const kvr_cache* c, const kvr_attention* a, size_t* bytes) {
  kvr_status st = check(c, a);
  if (st != KVR_OK) return st;
  if (!bytes) return invalid("bytes is NULL");
  AttendLayout l;
  st = lay_out(c, a, &l);
  if (st != KVR_OK) return st;
  *bytes = l.bytes;
  return KVR_OK;
}

kvr_status kvr_shared_attention(const kvr_cache* c, const kvr_attention* s, void* d_workspace, size_t bytes,
                                void* hip_stream) {
  kvr_status st = check(c, s);
  if (st != KVR_OK) return st;
  AttendLayout l;
  st = lay_out(c, s, &l);
  if (st != KVR_OK) return st;
  if (s->num_tokens == 0) return KVR_OK;
  CacheSteps kc, vc;
  st = check_buffers(c, &kc, &vc);
  if (st != KVR_OK) return st;
  if (!s->d_q || !s->d_out || !s->d_length || (s->width && !s->d_table))
    return invalid("d_q, d_out, d_table and d_length are required");
  if (s->num_groups && (!s->d_group_start || !s->d_prefix_length || (s->prefix_width && !s->d_prefix_table)))
    return invalid("groups need d_group_start, d_prefix_table and d_prefix_length");
  if (s->table_stride < s->width || s->prefix_stride < s->prefix_width)
    return invalid("a table's stride must be at least its width");
  kvr::AttendArgs a;
  a.q_tok = step(s->q_token, s->num_tokens, 2);
  a.q_head = step(s->q_head, s->heads, 2);
  a.o_tok = step(s->out_token, s->num_tokens, 2);
  a.o_head = step(s->out_head, s->heads, 2);
  if (!aligned(s->d_q, 16) || !aligned(s->d_out, 8) || !on_chunks(a.q_tok, a.q_head) || ((a.o_tok | a.o_head) & 7))
    return invalid("every head of the queries must start on a 16-byte boundary, of the results on an 8-byte one");
  if (!d_workspace || !aligned(d_workspace, 256)) return invalid("the workspace must be on a 256-byte boundary");
  if (bytes < l.bytes) return set_error(KVR_ENOMEM, "workspace too small (kvr_attention_workspace)");
  char* ws = static_cast<char*>(d_workspace);
  a.q = static_cast<const char*>(s->d_q);
  a.out = static_cast<char*>(s->d_out);
  a.lse = s->d_lse;
  a.kc = static_cast<const char*>(c->d_k);
  a.vc = static_cast<const char*>(c->d_v);
  a.ks = c->d_k_scale;
  a.vs = c->d_v_scale;
  a.kc_page = (uint32_t)kc.page;
  a.kc_slot = (uint32_t)kc.slot;
  a.kc_head = kc.head;
  a.vc_page = (uint32_t)vc.page;
  a.vc_slot = (uint32_t)vc.slot;
  a.vc_head = vc.head;
  a.row_start = s->d_row_start;
  a.length = s->d_length;
  a.table = s->d_table;
  a.group_start = s->d_group_start;
  a.prefix_table = s->d_prefix_table;
  a.prefix_length = s->d_prefix_length;
  a.table_stride = s->table_stride;
  a.prefix_stride = s->prefix_stride;
  a.status = s->d_status;
  a.hdr = reinterpret_cast<kvr::PlanHdr*>(ws);
  a.bounds = reinterpret_cast<int32_t*>(ws + l.bounds);
  a.group_of = reinterpret_cast<int32_t*>(ws + l.group_of);
  a.waves = reinterpret_cast<int32_t*>(ws + l.waves);
  a.units = reinterpret_cast<kvr::Unit*>(ws + l.units);
  a.joins = reinterpret_cast<int2*>(ws + l.joins);
  a.items = reinterpret_cast<kvr::Item*>(ws + l.items);
  a.ml = reinterpret_cast<float2*>(ws + l.ml);
  a.acc = reinterpret_cast<float*>(ws + l.acc);
  a.share = kvr::make_divisor((uint32_t)(s->heads / c->kv_heads));
  a.scale_log2 = s->scale * 1.44269504088896340736f;
  a.tokens = s->num_tokens;
  a.requests = s->num_requests;
  a.groups = s->num_groups;
  a.heads = s->heads;
  a.kv_heads = c->kv_heads;
  a.dim = c->dim;
  a.page_shift = log2_of(c->page_size);
  a.page_mask = c->page_size - 1;
  a.num_pages = c->num_pages;
  a.own_room = room(s->width, c->page_size);
  a.prefix_room = room(s->prefix_width, c->page_size);
  a.unit_cap = l.unit_cap;
  a.item_cap = l.item_cap;
  a.join_cap = l.join_cap;
  a.split_slots = l.split_slots;
  a.few_waves = c->dtype == KVR_FP8 && c->dim == 256 ? 4 : 1;
  a.one_base = c->page_size >= 512 / c->dim && kvr::lanes_reach(c->dim, a.kc_slot) && kvr::lanes_reach(c->dim, a.vc_slot);
  a.fused = kvr::attend_fused(a);
  a.direct = kvr::attend_direct(a);
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const bool fp16 = s->dtype == KVR_FP16, fp8 = c->dtype == KVR_FP8;
  hipError_t e = kvr::launch_attend_plan(a, stream);
  if (e == hipSuccess)
    e = c->dim == 64    ? kvr::launch_attend_64(a, fp16, fp8, stream)
        : c->dim == 128 ? kvr::launch_attend_128(a, fp16, fp8, stream)
                        : kvr::launch_attend_256(a, fp16, fp8, stream);
  if (e == hipSuccess) e = kvr::launch_attend_join(a, fp16, stream);
  return e == hipSuccess ? KVR_OK : hip_failed(e, "attention kernels launch");
}

}  // extern "C"
