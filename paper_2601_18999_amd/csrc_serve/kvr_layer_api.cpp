// kvr_layer_api.cpp - host side of the norms, the 8-bit products and linear
// attention of include/kvr.h: checks of the arguments, layout of the
// workspaces, launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "kvr_checks.h"
#include "kvr_layer.h"

namespace {

using kvr::aligned;
using kvr::hip_failed;
using kvr::invalid;
using kvr::kInt;
using kvr::on_chunks;
using kvr::round_up;
using kvr::set_error;
using kvr::step;

bool halves(int32_t dtype) { return dtype == KVR_BF16 || dtype == KVR_FP16; }

kvr_status check(const kvr_norm* n) {
  if (!n) return invalid("norm is NULL");
  if (n->struct_size != sizeof(kvr_norm)) return invalid("struct_size mismatch (kvr_norm)");
  if (!halves(n->dtype)) return invalid("dtype must be KVR_BF16 or KVR_FP16");
  if (n->out_dtype != n->dtype && n->out_dtype != KVR_INT8) return invalid("out_dtype must be dtype or KVR_INT8");
  if (n->num_tokens < 0) return invalid("num_tokens must be >= 0");
  if (n->dim < 1 || n->dim > 65536) return invalid("dim must be in 1..65536");
  if (n->activation < KVR_ACT_NONE || n->activation > KVR_ACT_SILU) return invalid("unknown activation");
  if (!(n->eps > 0.0f) || !std::isfinite(n->eps)) return invalid("eps must be finite and > 0");
  if (!std::isfinite(n->residual_scale)) return invalid("residual_scale must be finite");
  if ((n->d_residual != nullptr) != (n->d_residual_out != nullptr))
    return invalid("d_residual and d_residual_out go together");
  if (n->d_residual && n->residual_dtype != n->dtype && n->residual_dtype != KVR_FP32)
    return invalid("residual_dtype must be dtype or KVR_FP32");
  if ((n->out_dtype == KVR_INT8) != (n->d_out_scale != nullptr))
    return invalid("d_out_scale goes with an 8-bit result");
  return KVR_OK;
}

kvr_status check(const kvr_product* p) {
  if (!p) return invalid("product is NULL");
  if (p->struct_size != sizeof(kvr_product)) return invalid("struct_size mismatch (kvr_product)");
  if (p->dtype != KVR_INT8 && !halves(p->dtype)) return invalid("dtype must be KVR_INT8, KVR_BF16 or KVR_FP16");
  if (p->out_dtype != KVR_FP32 && !halves(p->out_dtype))
    return invalid("out_dtype must be KVR_BF16, KVR_FP16 or KVR_FP32");
  if (p->num_tokens < 0) return invalid("num_tokens must be >= 0");
  // (sums of 65,536 products of 8-bit integers are below 2^31)
  if (p->dim < 16 || p->dim > 65536 || p->dim % 16) return invalid("dim must be a multiple of 16 in 16..65536");
  if (p->channels < 1 || p->channels > (1 << 24)) return invalid("channels must be in 1..2^24");
  // (a launch has fewer than 2^32 threads, a tile up to 512; product_tile takes none of which there are more)
  if ((int64_t)(p->num_tokens / 128 + 1) * (p->channels / 128 + 1) >= 1 << 23)
    return invalid("too many tokens and channels for one call: (num_tokens / 128 + 1) * (channels / 128 + 1) must be "
                   "below 2^23");
  if ((p->dtype == KVR_INT8) != (p->d_x_scale != nullptr)) return invalid("d_x_scale goes with 8-bit tokens");
  return KVR_OK;
}

// Whether 16-bit tokens go through the workspace, as integers.
bool quantised_first(const kvr_product* p) {
  return p->dtype != KVR_INT8 && !kvr::quantised_within(p->num_tokens, p->dim, p->channels);
}

size_t product_bytes(const kvr_product* p) {
  return !quantised_first(p) ? 0 : round_up((size_t)p->num_tokens * 4) + round_up((size_t)p->num_tokens * p->dim);
}

kvr_status check(const kvr_linear* l) {
  if (!l) return invalid("linear is NULL");
  if (l->struct_size != sizeof(kvr_linear)) return invalid("struct_size mismatch (kvr_linear)");
  if (!halves(l->dtype)) return invalid("dtype must be KVR_BF16 or KVR_FP16");
  if (l->num_tokens < 0) return invalid("num_tokens must be >= 0");
  if (l->num_requests < 1 || l->num_requests > (1 << 20)) return invalid("num_requests must be in 1..2^20");
  if (l->kv_heads < 1 || l->kv_heads > 1024) return invalid("kv_heads must be in 1..1024");
  if (l->heads < 1 || l->heads % l->kv_heads) return invalid("heads must be a positive multiple of kv_heads");
  if (l->dim != 64 && l->dim != 128) return invalid("dim must be 64 or 128");
  if ((int64_t)l->num_tokens * l->heads > kInt) return invalid("num_tokens * heads must be below 2^31");
  if (l->num_slots < 1) return invalid("num_slots must be >= 1");
  if (!std::isfinite(l->scale)) return invalid("scale must be finite");
  if (!l->d_row_start && l->num_tokens != l->num_requests)
    return invalid("without d_row_start there is one token a request");
  return KVR_OK;
}

struct LinearLayout {
  size_t segments, added, bytes;
  int32_t segment, segment_cap;
  bool planned;
};

// Segments of equal length, as many as the device holds workgroups (one takes
// a segment's key head), but hardly of fewer than 256 tokens.  Where there are
// that many requests, half as many: most are not cut then, which takes no
// second pass (16 requests of 128 to 1,024 tokens, 32 heads: 136 -> 120 us;
// one request of 9,216 tokens 132 -> 153 us).
kvr_status lay_out(const kvr_linear* l, LinearLayout* o) {
  const int64_t tokens = l->num_tokens;
  const bool many = (int64_t)l->num_requests * l->kv_heads >= kvr::kLinearSlots;
  const int64_t slots = many ? kvr::kLinearSlots / 2 : kvr::kLinearSlots;
  const int64_t even = (tokens * l->kv_heads + slots - 1) / slots;
  // Shorter ones where the device would be half empty all the same, and the
  // requests are long enough to be cut; query heads that share a state make the
  // most of it (us, with 256, 128 and 64 tokens a segment: one request of 200
  // tokens, 32 / 8 heads of 128: 58, 27, 21.5; of 1,600: 40, 35, 40; of 3,200: 52,
  // 58, 60; four of 100 tokens, 32 / 32 heads: 22, 22, 29).
  int64_t least = 256;
  for (int64_t n = 128; n >= 64; n /= 2)
    if (tokens * (l->heads + l->kv_heads) <= n * kvr::kLinearSlots &&
        tokens > (l->heads == l->kv_heads ? 2 * n : n) * l->num_requests)
      least = n;
  // A batch of short requests is not cut, though one could be long (100 requests
  // of 4 tokens, 4 / 2 heads: 9.7 instead of 20 us, and 100 of 6, which are more in
  // all, 19; 64 of 8, 32 / 8 heads of 128: 29, with a token more 35).  One long one
  // among single tokens pays for that (of 448 among 63, 32 / 8 heads: 94 instead of
  // 73; of 449 106, of 450 75 again; 32 / 32: 84 instead of 86).
  if (tokens <= 512 && tokens <= 16 * (int64_t)l->num_requests) least = 512;
  const int64_t segment = even > least ? (even + 63) / 64 * 64 : least;
  const bool cut = l->d_row_start && tokens > segment;  // whether there can be a request of several segments
  const int64_t cap = l->num_requests + (cut ? tokens / segment : 0);
  // (a launch has fewer than 2^32 threads)
  if (cap * l->kv_heads >= 1 << 24)
    return invalid("too many requests and heads for one launch: num_requests * kv_heads must be below 2^24 - 512");
  o->segment = (int32_t)(segment < kInt ? segment : kInt);
  o->segment_cap = (int32_t)cap;
  o->segments = 256;
  o->added = 256 + round_up((size_t)cap * sizeof(kvr::Segment));
  // a request of several segments has at most twice as many as full ones
  const size_t states = cut ? 2 * (size_t)(tokens / segment) : 0;
  // (without a plan a request has one segment: as many workgroups for a key head as requests)
  o->planned = cut || (l->d_row_start && l->num_requests > kvr::kUnplanned);
  o->bytes = o->planned ? o->added + states * l->kv_heads * l->dim * l->dim * 4 : 0;
  return KVR_OK;
}

}  // namespace

extern "C" {

kvr_status kvr_block_norm(const kvr_norm* n, void* hip_stream) {
  const kvr_status st = check(n);
  if (st != KVR_OK) return st;
  if (n->num_tokens == 0) return KVR_OK;
  if (!n->d_x || !n->d_out) return invalid("d_x and d_out are required");
  const int res_size = n->residual_dtype == KVR_FP32 ? 4 : 2;
  if (!aligned(n->d_x, 2) || !aligned(n->d_after, 2) || !aligned(n->d_gate, 2) || !aligned(n->d_before, 2) ||
      !aligned(n->d_residual, res_size) || !aligned(n->d_residual_out, res_size) || !aligned(n->d_out_scale, 4) ||
      (n->out_dtype != KVR_INT8 && !aligned(n->d_out, 2)))
    return invalid("a buffer is not aligned to its elements");
  kvr::NormArgs a;
  a.x = static_cast<const char*>(n->d_x);
  a.after = static_cast<const char*>(n->d_after);
  a.gate = static_cast<const char*>(n->d_gate);
  a.residual = static_cast<const char*>(n->d_residual);
  a.before = static_cast<const char*>(n->d_before);
  a.residual_out = static_cast<char*>(n->d_residual_out);
  a.out = static_cast<char*>(n->d_out);
  a.out_scale = n->d_out_scale;
  a.x_tok = step(n->x_token, n->num_tokens, 2);
  a.gate_tok = step(n->gate_token, n->num_tokens, 2);
  a.res_tok = step(n->residual_token, n->num_tokens, res_size);
  a.res_out_tok = step(n->residual_out_token, n->num_tokens, res_size);
  a.out_tok = step(n->out_token, n->num_tokens, n->out_dtype == KVR_INT8 ? 1 : 2);
  a.tokens = n->num_tokens;
  a.dim = n->dim;
  a.activation = n->activation;
  a.res32 = n->residual_dtype == KVR_FP32;
  a.int8 = n->out_dtype == KVR_INT8;
  a.eps = n->eps;
  a.residual_scale = n->residual_scale;
  a.inv_dim = 1.0f / (float)n->dim;
  const hipError_t e = kvr::launch_norm(a, n->dtype == KVR_FP16, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? KVR_OK : hip_failed(e, "norm kernel launch");
}

kvr_status kvr_product_workspace(const kvr_product* p, size_t* bytes) {
  const kvr_status st = check(p);
  if (st != KVR_OK) return st;
  if (!bytes) return invalid("bytes is NULL");
  *bytes = product_bytes(p);
  return KVR_OK;
}

kvr_status kvr_integer_product(const kvr_product* p, void* d_workspace, size_t bytes, void* hip_stream) {
  const kvr_status st = check(p);
  if (st != KVR_OK) return st;
  if (p->num_tokens == 0) return KVR_OK;
  if (!p->d_x || !p->d_w || !p->d_out || !p->d_w_scale) return invalid("d_x, d_w, d_w_scale and d_out are required");
  const bool int8 = p->dtype == KVR_INT8;
  const int out_size = p->out_dtype == KVR_FP32 ? 4 : 2;
  kvr::ProductArgs a;
  a.x_tok = step(p->x_token, p->num_tokens, int8 ? 1 : 2);
  a.w_chan = step(p->w_channel, p->channels, 1);
  a.out_tok = step(p->out_token, p->num_tokens, out_size);
  if (!aligned(p->d_w, 16) || (a.w_chan & 15) || (int8 && (!aligned(p->d_x, 16) || (a.x_tok & 15))))
    return invalid("every row of d_w, and of 8-bit d_x, must start on a 16-byte boundary");
  if (!aligned(p->d_x, int8 ? 1 : 2) || !aligned(p->d_out, out_size) || !aligned(p->d_x_scale, 4) ||
      !aligned(p->d_w_scale, 4) || !aligned(p->d_bias, 4))
    return invalid("a buffer is not aligned to its elements");
  const size_t need = product_bytes(p);
  if (need && (!d_workspace || !aligned(d_workspace, 16)))
    return invalid("the workspace must be on a 16-byte boundary");
  if (bytes < need) return set_error(KVR_ENOMEM, "workspace too small (kvr_product_workspace)");
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  a.x = static_cast<const char*>(p->d_x);
  a.w = static_cast<const char*>(p->d_w);
  a.out = static_cast<char*>(p->d_out);
  a.x_scale = p->d_x_scale;
  a.w_scale = p->d_w_scale;
  a.bias = p->d_bias;
  a.tokens = p->num_tokens;
  a.dim = p->dim;
  a.channels = p->channels;
  a.dtype = p->dtype;
  hipError_t e = hipSuccess;
  if (need) {
    kvr::NormArgs n = {};
    n.x = a.x;
    n.x_tok = a.x_tok;
    n.out_scale = static_cast<float*>(d_workspace);
    n.out = static_cast<char*>(d_workspace) + round_up((size_t)p->num_tokens * 4);
    n.out_tok = p->dim;
    n.tokens = p->num_tokens;
    n.dim = p->dim;
    n.int8 = 1;
    e = kvr::launch_norm(n, p->dtype == KVR_FP16, stream);
    a.x = n.out;
    a.x_tok = n.out_tok;
    a.x_scale = n.out_scale;
    a.dtype = KVR_INT8;
  }
  if (e == hipSuccess) e = kvr::launch_product(a, p->out_dtype, stream);
  return e == hipSuccess ? KVR_OK : hip_failed(e, "product kernels launch");
}

kvr_status kvr_linear_workspace(const kvr_linear* l, size_t* bytes) {
  kvr_status st = check(l);
  if (st != KVR_OK) return st;
  if (!bytes) return invalid("bytes is NULL");
  LinearLayout o;
  st = lay_out(l, &o);
  if (st != KVR_OK) return st;
  *bytes = o.bytes;
  return KVR_OK;
}

kvr_status kvr_linear_attention(const kvr_linear* l, void* d_workspace, size_t bytes, void* hip_stream) {
  kvr_status st = check(l);
  if (st != KVR_OK) return st;
  LinearLayout o;
  st = lay_out(l, &o);
  if (st != KVR_OK) return st;
  if (!l->d_state || !l->d_log_decay || !l->d_read) return invalid("d_state, d_log_decay and d_read are required");
  if (l->num_tokens && (!l->d_q || !l->d_k || !l->d_v || !l->d_out))
    return invalid("d_q, d_k, d_v and d_out are required");
  kvr::LinearArgs a;
  a.q_tok = step(l->q_token, l->num_tokens, 2);
  a.q_head = step(l->q_head, l->heads, 2);
  a.k_tok = step(l->k_token, l->num_tokens, 2);
  a.k_head = step(l->k_head, l->kv_heads, 2);
  a.v_tok = step(l->v_token, l->num_tokens, 2);
  a.v_head = step(l->v_head, l->kv_heads, 2);
  a.o_tok = step(l->out_token, l->num_tokens, 2);
  a.o_head = step(l->out_head, l->heads, 2);
  if (!aligned(l->d_q, 16) || !aligned(l->d_k, 16) || !aligned(l->d_v, 16) || !aligned(l->d_out, 8) ||
      !on_chunks(a.q_tok, a.q_head) || !on_chunks(a.k_tok, a.k_head) || !on_chunks(a.v_tok, a.v_head) ||
      ((a.o_tok | a.o_head) & 7))
    return invalid("every head of q, k and v must start on a 16-byte boundary, of the results on an 8-byte one");
  a.state_slot = step(l->state_slot, l->num_slots, 1);
  a.state_head = step(l->state_head, l->kv_heads, 1);
  if (!aligned(l->d_state, 16) || ((a.state_slot | a.state_head) & 3) || !aligned(l->d_log_decay, 4) ||
      !aligned(l->d_row_start, 4) || !aligned(l->d_read, 4) || !aligned(l->d_write, 4))
    return invalid("every state must start on a 16-byte boundary");
  if (o.bytes && (!d_workspace || !aligned(d_workspace, 256)))
    return invalid("the workspace must be on a 256-byte boundary");
  if (bytes < o.bytes) return set_error(KVR_ENOMEM, "workspace too small (kvr_linear_workspace)");
  char* ws = static_cast<char*>(d_workspace);
  a.q = static_cast<const char*>(l->d_q);
  a.k = static_cast<const char*>(l->d_k);
  a.v = static_cast<const char*>(l->d_v);
  a.out = static_cast<char*>(l->d_out);
  a.state = l->d_state;
  a.log_decay = l->d_log_decay;
  a.row_start = l->d_row_start;
  a.read = l->d_read;
  a.write = l->d_write ? l->d_write : l->d_read;
  a.status = l->d_status;
  a.hdr = reinterpret_cast<kvr::LinearHdr*>(ws);
  a.segments = reinterpret_cast<kvr::Segment*>(ws + o.segments);
  a.added = reinterpret_cast<float*>(ws + o.added);
  a.kv_div = kvr::make_divisor((uint32_t)l->kv_heads);
  a.tokens = l->num_tokens;
  a.requests = l->num_requests;
  a.heads = l->heads;
  a.kv_heads = l->kv_heads;
  a.share = l->heads / l->kv_heads;
  a.dim = l->dim;
  a.slots = l->num_slots;
  a.segment = o.segment;
  a.segment_cap = o.segment_cap;
  a.planned = o.planned;
  // a device that would be half empty takes the queries' heads side by side,
  // though each keeps the state (16 requests of 200 tokens, 32 / 4 heads of 128:
  // 41 instead of 112 us; one that is not, 64 requests, 32 / 8 heads: 153
  // instead of 108 us)
  a.teams = 2ll * o.segment_cap * l->kv_heads <= kvr::kLinearSlots && a.share <= 65535 ? a.share : 1;
  // Requests that the device holds at once all take the chunked form, unless
  // they have a token each: a launch less (16 requests, 32 heads of 64: of 2
  // tokens 10.1 instead of 12.1 us, of 40 18.8 instead of 21.6).  Of more, those
  // of few tokens are done sooner apart (100 requests of one token and 100 of 90:
  // 117 instead of 135 us).
  const bool at_once = (int64_t)l->num_requests * l->kv_heads <= kvr::kLinearSlots;
  a.few = l->d_row_start && l->num_tokens > l->num_requests && at_once ? -1 : kvr::kFewTokens;
  a.scale = l->scale;
  const hipError_t e = kvr::launch_linear(a, l->dtype == KVR_FP16, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? KVR_OK : hip_failed(e, "linear attention kernels launch");
}

}  // extern "C"
