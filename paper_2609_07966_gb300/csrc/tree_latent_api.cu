// C ABI layer of the tree and latent operators: argument validation, workspace carve-up, dispatch.
// As in mkv_api.cu, a bad argument launches nothing (see include/mkv.h).
#include <math.h>

#include "mkv_common.cuh"
#include "mkv_rows.h"

using namespace mkv;

namespace {

inline bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline bool aligned16(const void* p) { return aligned(p, 16); }

// Slots are 32-bit coordinates of the copies, a tile past the end included.
constexpr int64_t kMaxSlots = (int64_t)INT32_MAX - 256;

mkv_status check_latent(const mkv_latent_config* c) {
  MKV_REQUIRE(c != nullptr, MKV_ERR_INVALID_ARG, "config is NULL");
  MKV_REQUIRE(c->abi_version == MKV_ABI_VERSION, MKV_ERR_INVALID_ARG, "abi_version %u != %u", c->abi_version,
              MKV_ABI_VERSION);
  MKV_REQUIRE(c->dtype == MKV_F16 || c->dtype == MKV_BF16, MKV_ERR_INVALID_ARG, "unknown dtype %d", c->dtype);
  MKV_REQUIRE(c->B >= 1 && c->H >= 1, MKV_ERR_INVALID_ARG, "B and H must be positive");
  MKV_REQUIRE(c->B <= kMaxUnits && c->H <= 256, MKV_ERR_UNSUPPORTED, "B = %d above %d or H = %d above 256", c->B,
              kMaxUnits, c->H);
  MKV_REQUIRE(c->rank == 256 || c->rank == 512, MKV_ERR_UNSUPPORTED, "rank = %d not built", c->rank);
  MKV_REQUIRE(c->rope_dim == 64, MKV_ERR_UNSUPPORTED, "rope_dim = %d not built", c->rope_dim);
  MKV_REQUIRE(c->nope_dim == 64 || c->nope_dim == 128, MKV_ERR_UNSUPPORTED, "nope_dim = %d not built", c->nope_dim);
  MKV_REQUIRE(c->v_dim == 64 || c->v_dim == 128, MKV_ERR_UNSUPPORTED, "v_dim = %d not built", c->v_dim);
  MKV_REQUIRE(c->softmax_scale >= 0.f && isfinite(c->softmax_scale), MKV_ERR_INVALID_ARG,
              "softmax_scale must be >= 0");
  return MKV_OK;
}

mkv_status check_latent_cache(const mkv_latent_cache* k) {
  MKV_REQUIRE(k != nullptr, MKV_ERR_INVALID_ARG, "cache is NULL");
  MKV_REQUIRE(k->T_cap >= 1 && k->T_len && k->rows, MKV_ERR_INVALID_ARG, "cache T_cap/T_len/rows invalid");
  MKV_REQUIRE(k->T_cap < kMaxSlots, MKV_ERR_UNSUPPORTED, "T_cap %lld too large", (long long)k->T_cap);
  MKV_REQUIRE(aligned16(k->rows), MKV_ERR_INVALID_ARG, "cache rows must be 16-byte aligned");
  MKV_REQUIRE(aligned(k->T_len, 4), MKV_ERR_INVALID_ARG, "T_len must be 4-byte aligned");
  return MKV_OK;
}

mkv_status check_path(const int32_t* path, const int32_t* n_path) {
  MKV_REQUIRE(aligned(path, 4) && aligned(n_path, 4), MKV_ERR_INVALID_ARG, "path and n_path must be 4-byte aligned");
  return MKV_OK;
}

mkv_status check_tree_n(int32_t n) {
  MKV_REQUIRE(n >= 1, MKV_ERR_INVALID_ARG, "n = %d must be positive", n);
  MKV_REQUIRE(n <= kMaxTree, MKV_ERR_UNSUPPORTED, "n = %d above %d tokens per entry", n, kMaxTree);
  return MKV_OK;
}

mkv_status check_ws(const void* ws, size_t have, size_t need) {
  MKV_REQUIRE(ws != nullptr && have >= need, MKV_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", have, need);
  MKV_REQUIRE((reinterpret_cast<uintptr_t>(ws) & 255) == 0, MKV_ERR_INVALID_ARG, "ws must be 256-byte aligned");
  return MKV_OK;
}

mkv_status check_rows(const RowsCall& r) {
  MKV_REQUIRE(rows_countable(r), MKV_ERR_UNSUPPORTED, "too many key tiles (T_cap x entries x rows) for one call");
  return MKV_OK;
}

float latent_scale(const mkv_latent_config* c) {
  return c->softmax_scale > 0.f ? c->softmax_scale : 1.0f / sqrtf((float)(c->nope_dim + c->rope_dim));
}

// The sizes of a call; pointers are filled in by the entry point.
RowsCall rows_of_tree(const mkv_config* c, int64_t T_cap, int n) {
  RowsCall r{};
  r.dtype = MKV_F16;
  r.B = c->B;
  r.n = n;
  r.H = c->Hq;
  r.Hkv = c->Hkv;
  r.dk = r.dv = c->D;
  r.scale = c->softmax_scale > 0.f ? c->softmax_scale : 1.0f / sqrtf((float)c->D);
  r.T_cap = T_cap;
  return r;
}

RowsCall rows_of_latent(const mkv_latent_config* c, int64_t T_cap, int n) {
  RowsCall r{};
  r.dtype = c->dtype;
  r.B = c->B;
  r.n = n;
  r.H = c->H;
  r.Hkv = 1;
  r.dk = c->rank + c->rope_dim;
  r.dv = c->rank;
  r.latent = true;
  r.scale = latent_scale(c);
  r.T_cap = T_cap;
  return r;
}

ProductCall product_of(const mkv_latent_config* c, Product kind, int64_t rows, const void* x, const void* w,
                       void* out) {
  ProductCall p{};
  p.kind = kind;
  p.dtype = c->dtype;
  p.B = c->B;
  p.H = c->H;
  p.nope = c->nope_dim;
  p.rope = c->rope_dim;
  p.v_dim = c->v_dim;
  p.rank = c->rank;
  p.rows = rows;
  p.x = x;
  p.w = w;
  p.out = out;
  return p;
}

// Config and sizes of a tree call (the FP16 config check wants pointers: any non-null ones).
mkv_status check_tree_cfg(const mkv_config* cfg, int64_t T_cap, int32_t n) {
  size_t dummy = 0;
  MKV_TRY(mkv_workspace_size(cfg, T_cap, &dummy));
  MKV_REQUIRE(cfg->method == MKV_FP16, MKV_ERR_UNSUPPORTED, "tree calls serve FP16 caches only");
  MKV_REQUIRE(T_cap < kMaxSlots, MKV_ERR_UNSUPPORTED, "T_cap %lld too large", (long long)T_cap);
  return check_tree_n(n);
}

}  // namespace

extern "C" {

mkv_status mkv_tree_workspace_size(const mkv_config* cfg, int64_t T_cap, int32_t n, size_t* bytes) {
  MKV_REQUIRE(bytes != nullptr, MKV_ERR_INVALID_ARG, "bytes is NULL");
  MKV_TRY(check_tree_cfg(cfg, T_cap, n));
  const RowsCall r = rows_of_tree(cfg, T_cap, n);
  MKV_TRY(check_rows(r));
  *bytes = rows_ws_bytes(r);
  return MKV_OK;
}

mkv_status mkv_tree_attention(const mkv_config* cfg, const void* q, const mkv_cache* cache, const void* k_tree,
                              const void* v_tree, const uint64_t* mask, int32_t n, void* out, void* ws,
                              size_t ws_bytes, void* stream) {
  MKV_TRY(check_fp16_decode_args(cfg, cache, q, out));
  MKV_TRY(check_tree_cfg(cfg, cache->T_cap, n));
  MKV_REQUIRE(k_tree && v_tree && mask, MKV_ERR_INVALID_ARG, "k_tree/v_tree/mask NULL");
  MKV_REQUIRE(aligned16(q) && aligned16(out) && aligned16(k_tree) && aligned16(v_tree) && aligned16(cache->k) &&
                  aligned16(cache->v),
              MKV_ERR_INVALID_ARG, "q, out, k_tree, v_tree and the cache must be 16-byte aligned");
  MKV_REQUIRE(aligned(mask, 8), MKV_ERR_INVALID_ARG, "mask must be 8-byte aligned");
  MKV_REQUIRE(aligned(cache->T_len, 4), MKV_ERR_INVALID_ARG, "T_len must be 4-byte aligned");
  RowsCall r = rows_of_tree(cfg, cache->T_cap, n);
  MKV_TRY(check_rows(r));
  MKV_TRY(check_ws(ws, ws_bytes, rows_ws_bytes(r)));
  r.q = q;
  r.k = cache->k;
  r.v = cache->v;
  r.T_len = cache->T_len;
  r.k_tree = k_tree;
  r.v_tree = v_tree;
  r.mask = mask;
  r.out = out;
  MKV_CUDA(launch_rows_attention(r, ws, as_stream(stream)));
  return MKV_OK;
}

mkv_status mkv_tree_commit(const mkv_config* cfg, const void* k_tree, const void* v_tree, const int32_t* path,
                           const int32_t* n_path, int32_t n, mkv_cache* cache, void* stream) {
  MKV_TRY(check_fp16_decode_args(cfg, cache, k_tree, v_tree));
  MKV_REQUIRE(n >= 1, MKV_ERR_INVALID_ARG, "n = %d must be positive", n);
  MKV_REQUIRE(aligned16(k_tree) && aligned16(v_tree) && aligned16(cache->k) && aligned16(cache->v),
              MKV_ERR_INVALID_ARG, "k_tree, v_tree and the cache must be 16-byte aligned");
  MKV_REQUIRE(aligned(cache->T_len, 4), MKV_ERR_INVALID_ARG, "T_len must be 4-byte aligned");
  MKV_TRY(check_path(path, n_path));
  CommitCall c{};
  c.B = cfg->B;
  c.n = n;
  c.heads = cfg->Hkv;
  c.row_bytes = cfg->D * 2;
  c.src0 = k_tree;
  c.src1 = v_tree;
  c.dst0 = cache->k;
  c.dst1 = cache->v;
  c.path = path;
  c.n_path = n_path;
  c.T_cap = cache->T_cap;
  c.T_len = cache->T_len;
  MKV_CUDA(launch_commit(c, as_stream(stream)));
  return MKV_OK;
}

mkv_status mkv_latent_workspace_size(const mkv_latent_config* cfg, int64_t T_cap, int32_t n, size_t* bytes) {
  MKV_TRY(check_latent(cfg));
  MKV_REQUIRE(bytes != nullptr && T_cap >= 1, MKV_ERR_INVALID_ARG, "bytes NULL or T_cap < 1");
  MKV_REQUIRE(T_cap < kMaxSlots, MKV_ERR_UNSUPPORTED, "T_cap %lld too large", (long long)T_cap);
  MKV_TRY(check_tree_n(n));
  const RowsCall r = rows_of_latent(cfg, T_cap, n);
  MKV_TRY(check_rows(r));
  *bytes = rows_ws_bytes(r);
  return MKV_OK;
}

mkv_status mkv_latent_absorb(const mkv_latent_config* cfg, const void* q, const void* w_kv, int32_t n, void* q_abs,
                             void* stream) {
  MKV_TRY(check_latent(cfg));
  MKV_REQUIRE(q && w_kv && q_abs && n >= 1, MKV_ERR_INVALID_ARG, "q/w_kv/q_abs NULL or n < 1");
  MKV_REQUIRE(aligned16(q) && aligned16(w_kv) && aligned16(q_abs), MKV_ERR_INVALID_ARG,
              "q, w_kv and q_abs must be 16-byte aligned");
  MKV_REQUIRE((int64_t)cfg->B * n < kMaxSlots, MKV_ERR_UNSUPPORTED, "B * n too large");
  MKV_CUDA(launch_latent_product(product_of(cfg, Product::kAbsorb, n, q, w_kv, q_abs), as_stream(stream)));
  return MKV_OK;
}

mkv_status mkv_latent_project(const mkv_latent_config* cfg, const void* o_lat, const void* w_kv, int32_t n, void* out,
                              void* stream) {
  MKV_TRY(check_latent(cfg));
  MKV_REQUIRE(o_lat && w_kv && out && n >= 1, MKV_ERR_INVALID_ARG, "o_lat/w_kv/out NULL or n < 1");
  MKV_REQUIRE(aligned16(o_lat) && aligned16(w_kv) && aligned16(out), MKV_ERR_INVALID_ARG,
              "o_lat, w_kv and out must be 16-byte aligned");
  MKV_REQUIRE((int64_t)cfg->B * n < kMaxSlots, MKV_ERR_UNSUPPORTED, "B * n too large");
  MKV_CUDA(launch_latent_product(product_of(cfg, Product::kProject, n, o_lat, w_kv, out), as_stream(stream)));
  return MKV_OK;
}

mkv_status mkv_latent_expand(const mkv_latent_config* cfg, const mkv_latent_cache* cache, const void* w_kv,
                             int64_t T_max, void* kv, void* stream) {
  MKV_TRY(check_latent(cfg));
  MKV_TRY(check_latent_cache(cache));
  MKV_REQUIRE(w_kv && kv, MKV_ERR_INVALID_ARG, "w_kv/kv NULL");
  MKV_REQUIRE(T_max >= 1 && T_max <= cache->T_cap, MKV_ERR_INVALID_ARG, "T_max %lld outside [1, T_cap]",
              (long long)T_max);
  MKV_REQUIRE(aligned16(w_kv) && aligned16(kv), MKV_ERR_INVALID_ARG, "w_kv and kv must be 16-byte aligned");
  ProductCall p = product_of(cfg, Product::kExpand, T_max, cache->rows, w_kv, kv);
  p.T_cap = cache->T_cap;
  p.T_len = cache->T_len;
  MKV_CUDA(launch_latent_product(p, as_stream(stream)));
  return MKV_OK;
}

mkv_status mkv_latent_attention(const mkv_latent_config* cfg, const void* q_abs, const mkv_latent_cache* cache,
                                const void* rows_tree, const uint64_t* mask, int32_t n, void* o_lat, void* ws,
                                size_t ws_bytes, void* stream) {
  MKV_TRY(check_latent(cfg));
  MKV_TRY(check_latent_cache(cache));
  MKV_TRY(check_tree_n(n));
  MKV_REQUIRE(q_abs && o_lat, MKV_ERR_INVALID_ARG, "q_abs/o_lat NULL");
  MKV_REQUIRE(rows_tree == nullptr || mask != nullptr, MKV_ERR_INVALID_ARG, "rows_tree needs a mask");
  MKV_REQUIRE(aligned16(q_abs) && aligned16(o_lat) && aligned16(rows_tree), MKV_ERR_INVALID_ARG,
              "q_abs, o_lat and rows_tree must be 16-byte aligned");
  MKV_REQUIRE(rows_tree == nullptr || aligned(mask, 8), MKV_ERR_INVALID_ARG, "mask must be 8-byte aligned");
  RowsCall r = rows_of_latent(cfg, cache->T_cap, n);
  MKV_TRY(check_rows(r));
  MKV_TRY(check_ws(ws, ws_bytes, rows_ws_bytes(r)));
  r.q = q_abs;
  r.k = r.v = cache->rows;
  r.T_len = cache->T_len;
  r.k_tree = rows_tree;
  r.mask = mask;
  r.out = o_lat;
  MKV_CUDA(launch_rows_attention(r, ws, as_stream(stream)));
  return MKV_OK;
}

mkv_status mkv_latent_prefill(const mkv_latent_config* cfg, const void* q, const void* kv, int64_t T_max,
                              const mkv_latent_cache* cache, const int32_t* q_len, int32_t n, void* out,
                              void* stream) {
  MKV_TRY(check_latent(cfg));
  MKV_TRY(check_latent_cache(cache));
  MKV_REQUIRE(q && kv && out && n >= 1, MKV_ERR_INVALID_ARG, "q/kv/out NULL or n < 1");
  MKV_REQUIRE(T_max >= 1 && T_max <= cache->T_cap, MKV_ERR_INVALID_ARG, "T_max %lld outside [1, T_cap]",
              (long long)T_max);
  MKV_REQUIRE(aligned16(q) && aligned16(kv) && aligned16(out), MKV_ERR_INVALID_ARG,
              "q, kv and out must be 16-byte aligned");
  MKV_REQUIRE(aligned(q_len, 4), MKV_ERR_INVALID_ARG, "q_len must be 4-byte aligned");
  MKV_REQUIRE((int64_t)cfg->B * cfg->H <= 65535, MKV_ERR_UNSUPPORTED, "B * H above 65535");
  PrefillCall p{};
  p.dtype = cfg->dtype;
  p.B = cfg->B;
  p.n = n;
  p.H = cfg->H;
  p.nope = cfg->nope_dim;
  p.rope = cfg->rope_dim;
  p.v_dim = cfg->v_dim;
  p.rank = cfg->rank;
  p.scale = latent_scale(cfg);
  p.q = q;
  p.kv = kv;
  p.rows = cache->rows;
  p.T_max = T_max;
  p.T_cap = cache->T_cap;
  p.T_len = cache->T_len;
  p.q_len = q_len;
  p.out = out;
  MKV_CUDA(launch_latent_prefill(p, as_stream(stream)));
  return MKV_OK;
}

mkv_status mkv_latent_commit(const mkv_latent_config* cfg, const void* rows_new, const int32_t* path,
                             const int32_t* n_path, int32_t n, mkv_latent_cache* cache, void* stream) {
  MKV_TRY(check_latent(cfg));
  MKV_TRY(check_latent_cache(cache));
  MKV_REQUIRE(rows_new && n >= 1, MKV_ERR_INVALID_ARG, "rows_new NULL or n < 1");
  MKV_REQUIRE(aligned16(rows_new), MKV_ERR_INVALID_ARG, "rows_new must be 16-byte aligned");
  MKV_TRY(check_path(path, n_path));
  CommitCall c{};
  c.B = cfg->B;
  c.n = n;
  c.heads = 1;
  c.row_bytes = (cfg->rank + cfg->rope_dim) * 2;
  c.src0 = rows_new;
  c.dst0 = cache->rows;
  c.path = path;
  c.n_path = n_path;
  c.T_cap = cache->T_cap;
  c.T_len = cache->T_len;
  MKV_CUDA(launch_commit(c, as_stream(stream)));
  return MKV_OK;
}

}  // extern "C"
