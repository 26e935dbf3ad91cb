// Host-side interfaces of the tree and latent operators (tree_latent_api.cu and the kernel units it
// calls), and the error plumbing of the entry points.  Not part of the public ABI.
#pragma once

#include "mkv_internal.h"

// A failed check or CUDA call sets the thread's error text and returns its status.
#define MKV_CUDA(expr)                                                          \
  do {                                                                          \
    cudaError_t e_ = (expr);                                                    \
    if (e_ != cudaSuccess) {                                                    \
      set_error("%s: %s", #expr, cudaGetErrorString(e_));                       \
      return MKV_ERR_CUDA;                                                      \
    }                                                                           \
  } while (0)

#define MKV_REQUIRE(cond, code, ...) \
  do {                               \
    if (!(cond)) {                   \
      set_error(__VA_ARGS__);        \
      return code;                   \
    }                                \
  } while (0)

#define MKV_TRY(expr)              \
  do {                             \
    mkv_status s_ = (expr);        \
    if (s_ != MKV_OK) return s_;   \
  } while (0)

namespace mkv {

inline cudaStream_t as_stream(void* s) { return static_cast<cudaStream_t>(s); }

constexpr int kMaxTree = 64;     // drafted tokens per entry: one mask bit each

// Attention of n tokens' query rows over a cache and the drafted tokens (rows_attn.cu).
struct RowsCall {
  int dtype;                       // mkv_dtype
  int B, n, H, Hkv;                // entries, tokens per entry, query heads, key heads (latent: 1)
  int dk, dv;                      // dims of a query/key and of a value (latent: rank + rope, rank)
  bool latent;                     // values are the keys' first dv dims
  float scale;
  const void *q, *k, *v;           // queries [B][n][H][dk]; cache [B][Hkv][T_cap][.]
  int64_t T_cap;
  const int32_t* T_len;
  const void *k_tree, *v_tree;     // [B][n][Hkv][.] or null (latent: v_tree null)
  const uint64_t* mask;
  void* out;                       // [B][n][H][dv]
};
size_t rows_ws_bytes(const RowsCall& c);
bool rows_countable(const RowsCall& c);   // its key tiles fit the kernel's 32-bit counts
cudaError_t launch_rows_attention(const RowsCall& c, void* ws, cudaStream_t st);

// Causal attention over expanded keys and values (latent_prefill.cu).
struct PrefillCall {
  int dtype, B, n, H, nope, rope, v_dim, rank;
  float scale;
  const void *q, *kv, *rows;
  int64_t T_max, T_cap;
  const int32_t *T_len, *q_len;
  void* out;
};
cudaError_t launch_latent_prefill(const PrefillCall& c, cudaStream_t st);

// The per-head products around latent attention (latent_product.cu).
enum class Product { kAbsorb, kProject, kExpand };
struct ProductCall {
  Product kind;
  int dtype, B, H, nope, rope, v_dim, rank;
  int64_t rows;                    // tokens per entry (expand: T_max)
  const void *x, *w;
  int64_t T_cap;                   // expand: slots of the cache rows x
  const int32_t* T_len;
  void* out;
};
cudaError_t launch_latent_product(const ProductCall& c, cudaStream_t st);

// Rows of the accepted path into one or two caches (commit.cu).
struct CommitCall {
  int B, n, heads;                 // heads: Hkv, or 1 for latent rows
  int row_bytes;                   // bytes of one (token, head) row, a multiple of 16
  const void *src0, *src1;         // [B][n][heads][row]; src1 null: one cache
  void *dst0, *dst1;               // [B][heads][T_cap][row]
  const int32_t *path, *n_path;
  int64_t T_cap;
  int32_t* T_len;
  uint32_t* status;                // MKV_FLAG_* bits (filled in by the launch)
};
cudaError_t launch_commit(const CommitCall& c, cudaStream_t st);

// The word (on the current device) that these units' kernels raise MKV_FLAG_* bits in.  It is append.cu's, which
// mkv_get_status reads anyway: a word of each unit would cost its callers a round trip each.
cudaError_t status_word(uint32_t** word);

// One CTA whose roles' waits run out after ms (mkv_roles.cu).
cudaError_t launch_role_wait_selftest(int ms, cudaStream_t st);

}  // namespace mkv
