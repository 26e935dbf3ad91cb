// C ABI layer of the rotary and 8-bit paged cache operators: argument validation, workspace carve-up, dispatch.
// As in mkv_api.cu, a bad argument launches nothing (see include/mkv.h).
#include <math.h>

#include <algorithm>

#include "mkv_common.cuh"
#include "mkv_paged.h"

using namespace mkv;

namespace {

inline bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

bool positive(float x) { return x > 0.f && isfinite(x); }

mkv_status check_rope(const mkv_rope_config* c) {
  MKV_REQUIRE(c != nullptr, MKV_ERR_INVALID_ARG, "rope config is NULL");
  MKV_REQUIRE(c->abi_version == MKV_ABI_VERSION, MKV_ERR_INVALID_ARG, "abi_version %u != %u", c->abi_version,
              MKV_ABI_VERSION);
  MKV_REQUIRE(c->D >= 2 && c->D % 2 == 0, MKV_ERR_INVALID_ARG, "D = %d must be positive and even", c->D);
  MKV_REQUIRE(c->D <= 256, MKV_ERR_UNSUPPORTED, "D = %d above 256", c->D);
  MKV_REQUIRE(c->rot_dim >= 2 && c->rot_dim % 2 == 0 && c->rot_dim <= c->D, MKV_ERR_INVALID_ARG,
              "rot_dim = %d must be even and within 2..D", c->rot_dim);
  MKV_REQUIRE(c->layout == MKV_ROPE_HALF || c->layout == MKV_ROPE_PAIRS, MKV_ERR_INVALID_ARG, "unknown layout %d",
              c->layout);
  MKV_REQUIRE(c->scaling >= MKV_ROPE_PLAIN && c->scaling <= MKV_ROPE_RAMP, MKV_ERR_INVALID_ARG, "unknown scaling %d",
              c->scaling);
  MKV_REQUIRE(positive(c->theta) && c->theta > 1.f, MKV_ERR_INVALID_ARG, "theta must be above 1");
  MKV_REQUIRE(c->scaling == MKV_ROPE_PLAIN || (positive(c->factor) && c->factor >= 1.f), MKV_ERR_INVALID_ARG,
              "factor must be at least 1");
  if (c->scaling == MKV_ROPE_BANDS || c->scaling == MKV_ROPE_RAMP) {
    MKV_REQUIRE(positive(c->low) && positive(c->high) && c->low < c->high, MKV_ERR_INVALID_ARG,
                "turns must be 0 < low < high");
    MKV_REQUIRE(c->context >= 1, MKV_ERR_INVALID_ARG, "context must be positive");
  }
  MKV_REQUIRE(c->magnitude == 0.f || positive(c->magnitude), MKV_ERR_INVALID_ARG, "magnitude must be >= 0");
  return MKV_OK;
}

// A rotation and the table that a call takes.
mkv_status check_table(const mkv_rope_config* c, const float* table, int64_t T_max) {
  MKV_TRY(check_rope(c));
  MKV_REQUIRE(table != nullptr && T_max >= 1, MKV_ERR_INVALID_ARG, "rope table NULL or empty");
  MKV_REQUIRE(aligned(table, 8), MKV_ERR_INVALID_ARG, "rope table must be 8-byte aligned");
  return MKV_OK;
}

RopeCall rope_of(const mkv_rope_config* c, const float* table, int64_t T_max) {
  RopeCall r;
  r.rot = c->rot_dim;
  r.pairs = c->layout == MKV_ROPE_PAIRS;
  r.table = reinterpret_cast<const float2*>(table);
  r.T_max = T_max;
  return r;
}

mkv_status check_paged(const mkv_paged_config* c) {
  MKV_REQUIRE(c != nullptr, MKV_ERR_INVALID_ARG, "config is NULL");
  MKV_REQUIRE(c->abi_version == MKV_ABI_VERSION, MKV_ERR_INVALID_ARG, "abi_version %u != %u", c->abi_version,
              MKV_ABI_VERSION);
  MKV_REQUIRE(c->dtype == MKV_F16 || c->dtype == MKV_BF16, MKV_ERR_INVALID_ARG, "unknown dtype %d", c->dtype);
  MKV_REQUIRE(c->format == MKV_E4M3 || c->format == MKV_I8, MKV_ERR_INVALID_ARG, "unknown code format %d", c->format);
  MKV_REQUIRE(c->B >= 1 && c->Hq >= 1 && c->Hkv >= 1, MKV_ERR_INVALID_ARG, "B, Hq and Hkv must be positive");
  MKV_REQUIRE(c->Hq % c->Hkv == 0, MKV_ERR_INVALID_ARG, "Hq = %d not a multiple of Hkv = %d", c->Hq, c->Hkv);
  MKV_REQUIRE((int64_t)c->B * c->Hkv <= kMaxUnits, MKV_ERR_UNSUPPORTED, "B * Hkv = %lld above %d",
              (long long)c->B * c->Hkv, kMaxUnits);
  MKV_REQUIRE(c->Hq / c->Hkv <= 32, MKV_ERR_UNSUPPORTED, "%d query heads a key head, above 32", c->Hq / c->Hkv);
  MKV_REQUIRE(c->D == 64 || c->D == 128, MKV_ERR_UNSUPPORTED, "D = %d not built", c->D);
  MKV_REQUIRE(c->page_size == 16 || c->page_size == 32 || c->page_size == 64 || c->page_size == 128,
              MKV_ERR_UNSUPPORTED, "page_size = %d not built", c->page_size);
  MKV_REQUIRE(c->softmax_scale >= 0.f && isfinite(c->softmax_scale), MKV_ERR_INVALID_ARG,
              "softmax_scale must be >= 0");
  return MKV_OK;
}

mkv_status check_paged_cache(const mkv_paged_config* c, const mkv_paged_cache* k) {
  MKV_REQUIRE(k != nullptr, MKV_ERR_INVALID_ARG, "cache is NULL");
  MKV_REQUIRE(k->num_pages >= 1 && k->max_pages >= 1, MKV_ERR_INVALID_ARG, "num_pages and max_pages must be positive");
  MKV_REQUIRE(k->page_table && k->T_len && k->tickets && k->k && k->v && k->k_scale && k->v_scale, MKV_ERR_INVALID_ARG,
              "a field of the cache is NULL");
  MKV_REQUIRE(aligned(k->k, 16) && aligned(k->v, 16), MKV_ERR_INVALID_ARG, "cache k and v must be 16-byte aligned");
  MKV_REQUIRE(aligned(k->page_table, 4) && aligned(k->T_len, 4) && aligned(k->tickets, 4) && aligned(k->k_scale, 4) &&
                  aligned(k->v_scale, 4),
              MKV_ERR_INVALID_ARG, "page_table, T_len, tickets and scales must be 4-byte aligned");
  // (page and head are one 32-bit coordinate of the copies, a token's position a 32-bit number)
  MKV_REQUIRE(k->num_pages <= INT32_MAX / c->Hkv, MKV_ERR_UNSUPPORTED, "num_pages x Hkv too large");
  MKV_REQUIRE(k->max_pages <= (INT32_MAX - 256) / c->page_size, MKV_ERR_UNSUPPORTED, "max_pages x page_size too large");
  return MKV_OK;
}

mkv_status check_start(const mkv_paged_config* c, const int32_t* start, int64_t n) {
  MKV_REQUIRE(n >= 1, MKV_ERR_INVALID_ARG, "n must be positive");
  MKV_REQUIRE(n <= INT32_MAX, MKV_ERR_UNSUPPORTED, "n = %lld too large", (long long)n);
  MKV_REQUIRE(start != nullptr || n % c->B == 0, MKV_ERR_INVALID_ARG, "n = %lld not a multiple of B without start",
              (long long)n);
  MKV_REQUIRE(aligned(start, 4), MKV_ERR_INVALID_ARG, "start must be 4-byte aligned");
  return MKV_OK;
}

// One array of rows: its stride, 0 read as `dims`.
mkv_status check_row(const char* name, const void* p, int64_t dims, int64_t* stride) {
  MKV_REQUIRE(p != nullptr, MKV_ERR_INVALID_ARG, "%s is NULL", name);
  MKV_REQUIRE(aligned(p, 16), MKV_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
  if (*stride == 0) *stride = dims;
  MKV_REQUIRE(*stride >= dims && *stride % 8 == 0, MKV_ERR_INVALID_ARG,
              "%s stride %lld must be a multiple of 8 and at least %lld", name, (long long)*stride, (long long)dims);
  return MKV_OK;
}

PagedShape shape_of(const mkv_paged_config* c, int64_t n, const int32_t* start, const mkv_paged_cache* k) {
  PagedShape s{};
  s.dtype = c->dtype;
  s.format = c->format;
  s.B = c->B;
  s.Hq = c->Hq;
  s.Hkv = c->Hkv;
  s.D = c->D;
  s.page = c->page_size;
  s.n = n;
  s.each = start == nullptr ? (int)(n / c->B) : 0;
  s.start = start;
  if (k != nullptr) {
    s.num_pages = k->num_pages;
    s.max_pages = k->max_pages;
    s.page_table = k->page_table;
  }
  return s;
}

mkv_status check_attention_rows(const mkv_paged_config* c, int64_t n, int64_t max_rows) {
  MKV_REQUIRE(n >= 1 && max_rows >= 1 && max_rows <= n, MKV_ERR_INVALID_ARG, "rows must be 1 <= max_rows <= n");
  MKV_REQUIRE(n <= INT32_MAX, MKV_ERR_UNSUPPORTED, "n = %lld too large", (long long)n);
  // (a row's token is found by a multiplication that is exact up to there)
  MKV_REQUIRE(max_rows * (c->Hq / c->Hkv) <= 1 << 26, MKV_ERR_UNSUPPORTED, "max_rows x query heads a key head above %d", 1 << 26);
  return MKV_OK;
}

int64_t rows_of(const PagedAttnCall& c) { return c.max_rows * (c.s.Hq / c.s.Hkv); }
size_t attention_ws_bytes(const PagedAttnCall& c) {
  return rows_of(c) <= kPagedFew     ? paged_decode_ws_bytes(c)
         : rows_of(c) <= kPagedBlock ? paged_block_ws_bytes(c)
                                     : paged_prefill_ws_bytes(c);
}
cudaError_t launch_attention(const PagedAttnCall& c, void* ws, cudaStream_t st) {
  return rows_of(c) <= kPagedFew     ? launch_paged_decode(c, ws, st)
         : rows_of(c) <= kPagedBlock ? launch_paged_block(c, ws, st)
                                     : launch_paged_prefill(c, ws, st);
}

}  // namespace

extern "C" {

mkv_status mkv_rope_scaled_table(const mkv_rope_config* cfg, int64_t T_max, float* table, void* stream) {
  MKV_TRY(check_table(cfg, table, T_max));
  RopeTableCall c{};
  const double r = cfg->rot_dim, log_theta = log((double)cfg->theta);
  c.half = cfg->rot_dim / 2;
  c.scaling = cfg->scaling;
  c.theta = cfg->theta;
  c.factor = cfg->factor;
  c.magnitude = cfg->magnitude > 0.f ? cfg->magnitude : 1.0;
  c.low = cfg->low;
  c.high = cfg->high;
  c.context = (double)cfg->context;
  if (cfg->scaling == MKV_ROPE_RAMP) {
    if (cfg->magnitude == 0.f) c.magnitude = 0.1 * log((double)cfg->factor) + 1.0;
    // the pair that makes `turns` turns within the context, rounded outwards
    const double two_pi = 6.283185307179586;
    const double first = r * log(c.context / (cfg->high * two_pi)) / (2.0 * log_theta);
    const double last = r * log(c.context / (cfg->low * two_pi)) / (2.0 * log_theta);
    c.low = std::max(floor(first), 0.0);
    c.high = std::min(ceil(last), r - 1.0);
  }
  c.table = reinterpret_cast<float2*>(table);
  c.T_max = T_max;
  MKV_CUDA(launch_rope_scaled_table(c, as_stream(stream)));
  return MKV_OK;
}

mkv_status mkv_rope_apply(const mkv_rope_config* cfg, int32_t dtype, const void* x, int64_t x_stride,
                          const int32_t* pos, int64_t n, int32_t heads, const float* table, int64_t T_max,
                          int32_t transposed, void* out, int64_t out_stride, void* stream) {
  MKV_TRY(check_table(cfg, table, T_max));
  MKV_REQUIRE(dtype == MKV_F16 || dtype == MKV_BF16, MKV_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  MKV_REQUIRE(x && pos && out, MKV_ERR_INVALID_ARG, "x/pos/out NULL");
  MKV_REQUIRE(n >= 1 && heads >= 1, MKV_ERR_INVALID_ARG, "n and heads must be positive");
  MKV_REQUIRE(n <= INT32_MAX && heads <= 65535, MKV_ERR_UNSUPPORTED, "n or heads too large");
  MKV_REQUIRE(aligned(x, 2) && aligned(out, 2) && aligned(pos, 4), MKV_ERR_INVALID_ARG,
              "x and out must be 2-byte and pos 4-byte aligned");
  const int64_t dims = (int64_t)heads * cfg->D;
  RopeApplyCall c{};
  c.x_stride = x_stride == 0 ? dims : x_stride;
  c.out_stride = out_stride == 0 ? dims : out_stride;
  MKV_REQUIRE(c.x_stride >= dims && c.out_stride >= dims, MKV_ERR_INVALID_ARG, "strides must be at least heads * D");
  MKV_REQUIRE(out != x || c.out_stride == c.x_stride, MKV_ERR_INVALID_ARG, "in place, the strides must be the same");
  c.rope = rope_of(cfg, table, T_max);
  c.dtype = dtype;
  c.D = cfg->D;
  c.heads = heads;
  c.transposed = transposed != 0;
  c.x = static_cast<const uint16_t*>(x);
  c.out = static_cast<uint16_t*>(out);
  c.pos = pos;
  c.n = n;
  MKV_CUDA(launch_rope_apply(c, as_stream(stream)));
  return MKV_OK;
}

mkv_status mkv_paged_append(const mkv_paged_config* cfg, const mkv_rope_config* rope, const float* table, int64_t T_max,
                            const mkv_paged_rows* rows, mkv_paged_cache* cache, void* stream) {
  MKV_TRY(check_paged(cfg));
  MKV_TRY(check_paged_cache(cfg, cache));
  MKV_REQUIRE(rows != nullptr, MKV_ERR_INVALID_ARG, "rows is NULL");
  MKV_TRY(check_start(cfg, rows->start, rows->n));
  MKV_REQUIRE(aligned(rows->pos, 4), MKV_ERR_INVALID_ARG, "pos must be 4-byte aligned");
  PagedAppendCall c{};
  c.s = shape_of(cfg, rows->n, rows->start, cache);
  c.q_stride = rows->q_stride;
  c.k_stride = rows->k_stride;
  c.v_stride = rows->v_stride;
  c.q_out_stride = rows->q_out_stride;
  const int64_t kv = (int64_t)cfg->Hkv * cfg->D, qd = (int64_t)cfg->Hq * cfg->D;
  MKV_TRY(check_row("k", rows->k, kv, &c.k_stride));
  MKV_TRY(check_row("v", rows->v, kv, &c.v_stride));
  MKV_REQUIRE((rows->q == nullptr) == (rows->q_out == nullptr), MKV_ERR_INVALID_ARG, "q and q_out go together");
  if (rows->q != nullptr) {
    MKV_TRY(check_row("q", rows->q, qd, &c.q_stride));
    MKV_TRY(check_row("q_out", rows->q_out, qd, &c.q_out_stride));
    MKV_REQUIRE(rows->q != rows->q_out || c.q_stride == c.q_out_stride, MKV_ERR_INVALID_ARG,
                "in place, the strides must be the same");
  }
  if (rope != nullptr) {
    MKV_TRY(check_table(rope, table, T_max));
    MKV_REQUIRE(rope->D == cfg->D, MKV_ERR_INVALID_ARG, "rope D = %d, cache D = %d", rope->D, cfg->D);
    MKV_REQUIRE(rope->rot_dim % 16 == 0, MKV_ERR_UNSUPPORTED, "rot_dim = %d not a multiple of 16", rope->rot_dim);
    MKV_REQUIRE(aligned(table, 16), MKV_ERR_INVALID_ARG, "rope table must be 16-byte aligned");
    c.rope = rope_of(rope, table, T_max);
  }
  c.pos = rows->pos;
  c.q = static_cast<const uint16_t*>(rows->q);
  c.k_new = static_cast<const uint16_t*>(rows->k);
  c.v_new = static_cast<const uint16_t*>(rows->v);
  c.q_out = static_cast<uint16_t*>(rows->q_out);
  c.T_len = cache->T_len;
  c.tickets = cache->tickets;
  c.k = static_cast<uint8_t*>(cache->k);
  c.v = static_cast<uint8_t*>(cache->v);
  c.k_scale = cache->k_scale;
  c.v_scale = cache->v_scale;
  MKV_CUDA(launch_paged_append(c, as_stream(stream)));
  return MKV_OK;
}

mkv_status mkv_paged_workspace_size(const mkv_paged_config* cfg, int64_t n, int64_t max_rows, size_t* bytes) {
  MKV_REQUIRE(bytes != nullptr, MKV_ERR_INVALID_ARG, "bytes is NULL");
  MKV_TRY(check_paged(cfg));
  MKV_TRY(check_attention_rows(cfg, n, max_rows));
  PagedAttnCall c{};
  c.s = shape_of(cfg, n, nullptr, nullptr);
  c.max_rows = max_rows;
  *bytes = attention_ws_bytes(c);
  return MKV_OK;
}

mkv_status mkv_paged_attention(const mkv_paged_config* cfg, const void* q, int64_t q_stride, const int32_t* start,
                               int64_t n, int64_t max_rows, const mkv_paged_cache* cache, void* out,
                               int64_t out_stride, void* ws, size_t ws_bytes, void* stream) {
  MKV_TRY(check_paged(cfg));
  MKV_TRY(check_paged_cache(cfg, cache));
  MKV_TRY(check_start(cfg, start, n));
  MKV_TRY(check_attention_rows(cfg, n, max_rows));
  PagedAttnCall c{};
  const int64_t dims = (int64_t)cfg->Hq * cfg->D;
  c.q_stride = q_stride;
  c.out_stride = out_stride;
  MKV_TRY(check_row("q", q, dims, &c.q_stride));
  MKV_TRY(check_row("out", out, dims, &c.out_stride));
  MKV_REQUIRE(q != out || c.q_stride == c.out_stride, MKV_ERR_INVALID_ARG, "in place, the strides must be the same");
  c.s = shape_of(cfg, n, start, cache);
  c.max_rows = max_rows;
  // (chunks of 128 tokens are counted in 32 bits: 2^29, and one more a unit)
  MKV_REQUIRE(cache->max_pages * cfg->page_size <= (int64_t(1) << 36) / ((int64_t)cfg->B * cfg->Hkv), MKV_ERR_UNSUPPORTED,
              "too many tokens (B x Hkv x max_pages x page_size) for one call");
  const size_t need = attention_ws_bytes(c);
  MKV_REQUIRE(ws != nullptr && ws_bytes >= need, MKV_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, need);
  MKV_REQUIRE(aligned(ws, 256), MKV_ERR_INVALID_ARG, "ws must be 256-byte aligned");
  c.scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale : 1.0f / sqrtf((float)cfg->D);
  c.q = static_cast<const uint16_t*>(q);
  c.out = static_cast<uint16_t*>(out);
  c.T_len = cache->T_len;
  c.k = static_cast<const uint8_t*>(cache->k);
  c.v = static_cast<const uint8_t*>(cache->v);
  c.k_scale = cache->k_scale;
  c.v_scale = cache->v_scale;
  MKV_CUDA(launch_attention(c, ws, as_stream(stream)));
  return MKV_OK;
}

}  // extern "C"
