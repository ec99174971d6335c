// kvr_layer.h - arguments of the kernels around the attention of a worker's
// layer (norms, 8-bit products) and of linear attention: what the host side
// fills in and the device side reads.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/kvr.h"
#include "kvr_serve.h"

namespace kvr {

// ---- norms ----
struct NormArgs {
  const char *x, *after, *gate, *residual, *before;
  char *residual_out, *out;
  float* out_scale;
  int64_t x_tok, gate_tok, res_tok, res_out_tok, out_tok;  // bytes
  int32_t tokens, dim, activation;
  int32_t res32, int8;  // 1: 32-bit residual; 8-bit result
  float eps, residual_scale, inv_dim;
};

// ---- 8-bit products ----
struct ProductArgs {
  const char *x, *w;
  char* out;
  const float *x_scale, *w_scale, *bias;
  int64_t x_tok, w_chan, out_tok;  // bytes
  int32_t tokens, dim, channels;
  int32_t dtype;  // of x: KVR_INT8, or of few tokens that are not brought to integers yet
};

// Tiles of so many tokens and channels.
inline int64_t product_tiles(int64_t tokens, int64_t channels, int tile_tokens, int tile_channels) {
  return (tokens + tile_tokens - 1) / tile_tokens * ((channels + tile_channels - 1) / tile_channels);
}

// Tiles that pass through LDS, and the groups of waves that have k in turn.
struct ProductTile {
  int channels, tokens, groups, threads;
};

// Those that are done first, by the time of a round of one workgroup a compute
// unit (0.1 us, k = 4,096; those of 128 x 128 without groups are two a compute
// unit where there are as many; kvr_product.hip has the table).  Tiles 64 wide
// are left to others where they are more than a launch holds (it has fewer than
// 2^32 threads): up to 64 channels of 2^29 tokens.
inline ProductTile product_tile(int64_t tokens, int64_t channels) {
  auto rounds = [&](int c, int t) { return (product_tiles(tokens, channels, t, c) + kComputeUnits - 1) / kComputeUnits; };
  auto time = [&](int64_t round, int c, int t) {
    return product_tiles(tokens, channels, t, c) < 1 << 23 ? round * rounds(c, t) : INT64_MAX;
  };
  const int64_t r128 = rounds(128, 128);
  const int64_t t64 = time(115, 64, 64), t12864 = time(175, 128, 64), t128 = r128 == 1 ? 270 : 245 * r128,
                t256 = 620 * rounds(256, 256);
  if (t64 <= t12864 && t64 <= t128 && t64 <= t256) return {64, 64, 2, 512};
  if (t12864 <= t128 && t12864 <= t256) return {128, 64, 2, 512};
  if (t256 < t128) return {256, 256, 1, 512};
  return r128 == 1 ? ProductTile{128, 128, 2, 512} : ProductTile{128, 128, 1, 256};
}

// Whether tokens of 16 bits are brought to integers by every workgroup of the
// product for itself: where they are few elements, and the product is of one
// round of workgroups or of up to 16 tokens (25 tokens x 128 x 1,408: 12.8 us
// with a launch for that, which the host takes).
inline bool quantised_within(int tokens, int dim, int channels) {
  return (int64_t)tokens * dim <= 1 << 16 && (tokens <= 16 || product_tiles(tokens, channels, 64, 32) <= kComputeUnits);
}

// ---- linear attention ----
// Requests of up to so many tokens take the recurrent form (256 requests, us,
// recurrent and chunked: 32 heads of 64: 1 token 64 and 120, 4 tokens 77 and
// 121, 8 tokens 103 and 121, 12 tokens 130 and 121; 8 heads of 128: 4 tokens 63
// and 70, 8 tokens 74 and 73, 12 tokens 85 and 74).
constexpr int kFewTokens = 8;
// So many requests of which none is cut are not planned for: every workgroup
// checks row_start, an entry a thread (one request of 100 tokens, 16 heads: 10.8
// us, with a plan 13.9; 256 requests of 9 tokens: no difference).
constexpr int kUnplanned = 256;
// Workgroups of the chunked form that the device holds.
constexpr int kLinearSlots = 2 * kComputeUnits;

// A run of up to LinearArgs::segment tokens of one request.
struct alignas(32) Segment {
  int32_t request, row0, rows;
  int32_t index, parts;  // of its request's segments
  int32_t slot;          // of LinearArgs::added, of the request's first segment
};

struct LinearHdr {
  int32_t segments, followed, cut;  // in all, such that another one follows, and the first ones of those
  int32_t rejected;
};

struct LinearArgs {
  const char *q, *k, *v;
  char* out;
  float* state;
  const float* log_decay;
  const int32_t *row_start, *read, *write;
  uint32_t* status;
  LinearHdr* hdr;
  Segment* segments;
  // [slot][kv head][dim][dim], one for each segment of the requests of several:
  // what the segment before adds to the state, then the state before this one
  float* added;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;  // bytes
  int64_t state_slot, state_head;                                     // elements
  Divisor kv_div;                                                     // by kv_heads
  int32_t tokens, requests, heads, kv_heads, share, dim, slots;
  int32_t segment, segment_cap;
  int32_t teams;  // of a segment's key head, which share its queries' heads: 1 or share
  int32_t planned;
  int32_t few;  // requests of up to so many tokens take the recurrent form (-1: none)
  float scale;
};

hipError_t launch_norm(const NormArgs& a, bool fp16, hipStream_t st);
// out: KVR_BF16, KVR_FP16 or KVR_FP32
hipError_t launch_product(const ProductArgs& a, int out, hipStream_t st);
hipError_t launch_linear(const LinearArgs& a, bool fp16, hipStream_t st);

}  // namespace kvr
