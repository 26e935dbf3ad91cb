// Host-side interfaces of the rotary and 8-bit paged cache operators (paged_api.cu and the kernel units it calls).
// Not part of the public ABI.
#pragma once

#include "mkv_rows.h"

namespace mkv {

// A rotation as the kernels take it (rope.cu, paged_append.cu).
struct RopeCall {
  int rot = 0;                     // rotated dims of a head; 0: none
  bool pairs = false;              // MKV_ROPE_PAIRS
  const float2* table = nullptr;   // [T_max][rot / 2]
  int64_t T_max = 0;
};

struct RopeTableCall {
  int half;                        // rot_dim / 2
  int scaling;
  double theta, factor, magnitude;
  double low, high, context;       // BANDS: turns; RAMP: low and high are the pairs between which it mixes
  float2* table;
  int64_t T_max;
};
cudaError_t launch_rope_scaled_table(const RopeTableCall& c, cudaStream_t st);

struct RopeApplyCall {
  RopeCall rope;
  int dtype, D, heads;
  bool transposed;
  const uint16_t* x;
  uint16_t* out;
  int64_t x_stride, out_stride;    // elements
  const int32_t* pos;
  int64_t n;
};
cudaError_t launch_rope_apply(const RopeApplyCall& c, cudaStream_t st);

// What the append and the attention share of a paged cache.
struct PagedShape {
  int dtype, format, B, Hq, Hkv, D, page;
  int64_t n;                       // rows of all entries (fits 32 bits)
  int each;                        // start null: rows of every entry
  const int32_t* start;            // [B + 1] or null: n / B each
  int64_t num_pages, max_pages;
  const int32_t* page_table;
};

struct PagedAppendCall {
  PagedShape s;
  RopeCall rope;
  const int32_t* pos;
  const uint16_t *q, *k_new, *v_new;
  uint16_t* q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  int32_t *T_len, *tickets;
  uint8_t *k, *v;
  float *k_scale, *v_scale;
};
cudaError_t launch_paged_append(const PagedAppendCall& c, cudaStream_t st);

struct PagedAttnCall {
  PagedShape s;
  int64_t max_rows;
  float scale;
  const uint16_t* q;
  uint16_t* out;
  int64_t q_stride, out_stride;
  const int32_t* T_len;
  const uint8_t *k, *v;
  const float *k_scale, *v_scale;
};
// By the query rows of a key head (max_rows x heads of a group): up to kPagedFew, what a narrow product takes, paged_decode.cu,
// up to kPagedBlock, a block of a tcgen05 product, paged_block.cu, more paged_prefill.cu.  Over 8 x 8K tokens, 32 / 8 heads:
// one token 31 us (by paged_block.cu 51), two 31 (42), eight 44 (by paged_prefill.cu 74), sixteen 56 (74), 32 71 (75).
constexpr int kPagedFew = 8, kPagedBlock = 128;
size_t paged_decode_ws_bytes(const PagedAttnCall& c);
cudaError_t launch_paged_decode(const PagedAttnCall& c, void* ws, cudaStream_t st);
size_t paged_block_ws_bytes(const PagedAttnCall& c);
cudaError_t launch_paged_block(const PagedAttnCall& c, void* ws, cudaStream_t st);
size_t paged_prefill_ws_bytes(const PagedAttnCall& c);
cudaError_t launch_paged_prefill(const PagedAttnCall& c, void* ws, cudaStream_t st);

}  // namespace mkv
