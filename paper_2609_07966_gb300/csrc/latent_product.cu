// The per-head products around latent attention, out[token][h] = x[token] W[h] with
//   absorb   W = W_uk[h]^T  (nope -> rank; the rotated part of the query is copied beside it)
//   project  W = W_uv[h]    (rank -> v)
//   expand   W = [W_uk[h]; W_uv[h]] on a cached row's latent part (rank -> nope + v)
// For a decode step's few tokens they are bound by reading the weights once (and by the launch), for a prompt's by the
// tensor cores.  One kernel: a CTA holds a tile of one head's weights (NT output dims x all of K) in shared memory and
// streams 128-token blocks past it,
//   D [128 tokens x NT] = X [128 x K] W [K x NT]
// with the accumulator in tensor memory twice, so a block's stores run under the next one's products.  CTAs take
// equal runs of the (weight tile, token block) pairs, token blocks fastest, so a weight tile is loaded once or twice.
// W is used as it is stored: along K for project and expand, along the output dims for absorb.
#include <algorithm>

#include "mkv_roles.cuh"
#include "mkv_rows.h"

namespace mkv {

__device__ uint32_t g_status_product;   // MKV_FLAG_* bits raised here

cudaError_t take_status_product(uint32_t* flags, cudaStream_t st) {
  uint32_t v = 0, zero = 0;
  cudaError_t e = cudaMemcpyFromSymbolAsync(&v, g_status_product, sizeof(v), 0, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess)
    e = cudaMemcpyToSymbolAsync(g_status_product, &zero, sizeof(zero), 0, cudaMemcpyHostToDevice, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  *flags |= v;
  return e;
}

namespace {

struct ProductArgs {
  int B, H, K;                 // K: length of the sums
  int w_row;                   // first row of a head's weights used (project: nope)
  int n_dim;                   // output dims per head, dims per output row
  int out_row;
  int64_t rows;                // tokens (expand: of each entry)
  int64_t blocks;              // 128-token blocks (expand: of each entry)
  int64_t items;               // H x dim tiles x blocks (x B)
  int dim_tiles;
  const int32_t* T_len;        // expand
  const uint16_t* x;           // absorb: the queries, for their rotated part
  int x_row, rope_at;
  uint16_t* out;
};

constexpr int kTok = 128;
constexpr int kPrThreads = 192;    // four warps of stores, one of loads, one of products
constexpr int kStagesA = 5;
constexpr int kAtomA = kTok * 128;

template <bool BF16_, Product KIND_, int NT_>
struct PrShape {
  static constexpr bool BF16 = BF16_;
  static constexpr Product KIND = KIND_;
  static constexpr int NT = NT_;
  static constexpr bool W_MN = KIND == Product::kAbsorb;   // weights contiguous along the output dims
  static constexpr int TMEM = 2 * NT;
};

struct PrCtl {
  uint64_t wfull, wempty, afull[kStagesA], aempty[kStagesA], tfull[2], tempty[2];
  uint32_t tslot;
  int fail, loaded, weights, issued;
};
static_assert(sizeof(PrCtl) <= 256, "control block");

__host__ __device__ inline int weight_bytes(bool w_mn, int NT, int K) { return (w_mn ? NT / 64 * K : K / 64 * NT) * 128; }

template <class S>
__global__ void __launch_bounds__(kPrThreads, 1)
    product_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap,
                   const ProductArgs a) {
  constexpr int NT = S::NT;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  const int wbytes = weight_bytes(S::W_MN, NT, a.K);
  uint8_t* sa = sm + wbytes;                              // [kStagesA] 128 tokens x 64 of K
  PrCtl* ctl = reinterpret_cast<PrCtl*>(sa + kStagesA * kAtomA);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t first = a.items * blockIdx.x / gridDim.x, last = a.items * (blockIdx.x + 1) / gridDim.x;
  const int kc = a.K / 64;

  struct Item {
    int64_t wt, b, t0;          // weight tile (h, dims), entry, first token of the block
    int limit;                  // tokens of the block that exist
  };
  const int64_t per_wt = S::KIND == Product::kExpand ? a.B * a.blocks : a.blocks;
  auto item = [&](int64_t i) {
    Item x;
    x.wt = i / per_wt;
    const int64_t r = i % per_wt;
    x.b = S::KIND == Product::kExpand ? r / a.blocks : 0;
    x.t0 = (S::KIND == Product::kExpand ? r % a.blocks : r) * kTok;
    int64_t n = a.rows;
    if (S::KIND == Product::kExpand) n = std::min<int64_t>(n, a.T_len[x.b]);
    x.limit = (int)std::max<int64_t>(0, std::min<int64_t>(kTok, n - x.t0));
    return x;
  };

  if (warp == 4) tc_alloc(&ctl->tslot, S::TMEM);
  if (threadIdx.x == 0) {
    tc_mbar_init(&ctl->wfull, 1);
    tc_mbar_init(&ctl->wempty, 1);
    for (int s = 0; s < kStagesA; ++s) {
      tc_mbar_init(&ctl->afull[s], 1);
      tc_mbar_init(&ctl->aempty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      tc_mbar_init(&ctl->tfull[s], 1);
      tc_mbar_init(&ctl->tempty[s], 4);
    }
    tc_fence_mbar_init();
    ctl->fail = ctl->loaded = ctl->weights = ctl->issued = 0;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = ctl->tslot;
  volatile int* fail = &ctl->fail;
  uint32_t* status = &g_status_product;

  if (warp == 4) {
    if (elect_one()) {
      int64_t held = -1;
      int c = 0, w = 0;
      for (int64_t i = first; i < last; ++i) {
        const Item x = item(i);
        if (x.limit == 0) continue;
        const int h = (int)(x.wt / a.dim_tiles), d0 = (int)(x.wt % a.dim_tiles) * NT;
        if (x.wt != held) {
          if (w > 0 && !wait_or_fail(&ctl->wempty, (uint32_t)((w - 1) & 1), fail, status)) break;
          tc_mbar_expect_tx(&ctl->wfull, wbytes);
          if (S::W_MN) {
            for (int j = 0; j < NT / 64; ++j)
              tma_load_4d(sm + j * a.K * 128, &wmap, d0 + j * 64, a.w_row, h, 0, &ctl->wfull);
          } else {
            for (int j = 0; j < kc; ++j) tma_load_4d(sm + j * NT * 128, &wmap, j * 64, a.w_row + d0, h, 0, &ctl->wfull);
          }
          held = x.wt;
          ctl->weights = ++w;
        }
        bool ok = true;
        for (int j = 0; j < kc; ++j, ++c) {
          const int s = c % kStagesA, u = c / kStagesA;
          if (u > 0 && !wait_or_fail(&ctl->aempty[s], (uint32_t)((u - 1) & 1), fail, status)) {
            ok = false;
            break;
          }
          tc_mbar_expect_tx(&ctl->afull[s], kAtomA);
          if (S::KIND == Product::kExpand)
            tma_load_4d(sa + s * kAtomA, &xmap, j * 64, (int)x.t0, (int)x.b, 0, &ctl->afull[s]);
          else
            tma_load_4d(sa + s * kAtomA, &xmap, j * 64, h, (int)x.t0, 0, &ctl->afull[s]);
          ctl->loaded = c + 1;
        }
        if (!ok) break;
      }
    }
  } else if (warp == 5) {
    if (elect_one()) {
      constexpr uint32_t id = tc_idesc(S::BF16, kTok, NT, false, S::W_MN);
      const Desc ad = tc_desc_sw128(smem_addr(sa));
      const Desc wd = S::W_MN ? tc_desc_mn<64>(smem_addr(sm), (uint32_t)a.K * 128) : tc_desc_sw128(smem_addr(sm));
      int64_t held = -1;
      int c = 0, w = 0, n = 0;
      bool ok = true;
      for (int64_t i = first; ok && i < last; ++i) {
        const Item x = item(i);
        if (x.limit == 0) continue;
        if (x.wt != held) {
          if (w > 0) tc_commit(&ctl->wempty);             // the products with the old weights
          ok = wait_or_fail(&ctl->wfull, (uint32_t)(w & 1), fail, status);
          held = x.wt;
          ++w;
        }
        const int buf = n & 1;
        if (ok && n >= 2) ok = wait_or_fail(&ctl->tempty[buf], (uint32_t)((n / 2 - 1) & 1), fail, status);
        for (int j = 0; ok && j < kc; ++j, ++c) {
          const int s = c % kStagesA;
          ok = wait_or_fail(&ctl->afull[s], (uint32_t)((c / kStagesA) & 1), fail, status);
          if (!ok) break;
          tc_fence_after();
          const Desc as = ad.at(s * kAtomA), ws = wd.at(S::W_MN ? j * 64 * 128 : j * NT * 128);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            tc_mma_ss(tbase + (uint32_t)(buf * NT), as.at(kk * 32), ws.at(S::W_MN ? kk * 2048 : kk * 32), id,
                      j > 0 || kk > 0 ? 1u : 0u);
          tc_commit(&ctl->aempty[s]);
        }
        if (!ok) break;
        tc_commit(&ctl->tfull[buf]);
        ctl->issued = ++n;
      }
    }
  } else {
    // stores: thread = token of the block
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    int n = 0;
    for (int64_t i = first; i < last; ++i) {
      const Item x = item(i);
      if (x.limit == 0) continue;
      const int h = (int)(x.wt / a.dim_tiles), d0 = (int)(x.wt % a.dim_tiles) * NT, buf = n & 1;
      const bool ok = wait_or_fail(&ctl->tfull[buf], (uint32_t)((n / 2) & 1), fail, status);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after();
      const int r = warp * 32 + lane;
      const bool live = r < x.limit;
      const int64_t orow = S::KIND == Product::kExpand ? (x.b * a.H + h) * a.rows + x.t0 + r : (x.t0 + r) * a.H + h;
      uint4* dst = reinterpret_cast<uint4*>(a.out + orow * a.out_row + d0);
#pragma unroll
      for (int c = 0; c < NT / 32; ++c) {
        float v[32];
        tm_load<32>(tbase + lanes + (uint32_t)(buf * NT + c * 32), v);
        if (live) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            dst[c * 4 + e] = make_uint4(pack2<S::BF16>(v[8 * e], v[8 * e + 1]), pack2<S::BF16>(v[8 * e + 2], v[8 * e + 3]),
                                        pack2<S::BF16>(v[8 * e + 4], v[8 * e + 5]), pack2<S::BF16>(v[8 * e + 6], v[8 * e + 7]));
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) tc_mbar_arrive(&ctl->tempty[buf]);
      if (S::KIND == Product::kAbsorb && d0 == 0 && live) {     // the rotated part of the query, as it is
        const uint4* src = reinterpret_cast<const uint4*>(a.x + ((x.t0 + r) * a.H + h) * a.x_row + a.rope_at);
#pragma unroll
        for (int e = 0; e < 8; ++e) dst[a.n_dim / 8 + e] = src[e];
      }
      ++n;
    }
  }
  // teardown: on a failure wait (bounded) for the copies and products already issued
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && ctl->fail) {
    if (ctl->weights > 0) tc_mbar_wait(&ctl->wfull, (uint32_t)((ctl->weights - 1) & 1), kRoleWaitNs);
    for (int c = std::max(0, ctl->loaded - kStagesA); c < ctl->loaded; ++c)
      tc_mbar_wait(&ctl->afull[c % kStagesA], (uint32_t)((c / kStagesA) & 1), kRoleWaitNs);
    if (ctl->issued > 0) tc_mbar_wait(&ctl->tfull[(ctl->issued - 1) & 1], (uint32_t)(((ctl->issued - 1) / 2) & 1), kRoleWaitNs);
  }
  __syncthreads();
  tc_fence_after();
  if (warp == 4) tc_dealloc(tbase, S::TMEM);
}

template <class S>
cudaError_t launch_shape(const ProductCall& c, ProductArgs a, cudaStream_t st) {
  const int64_t H = c.H, d = c.nope + c.v_dim, r = c.rank;
  a.dim_tiles = a.n_dim / S::NT;
  a.items = H * a.dim_tiles * a.blocks * (S::KIND == Product::kExpand ? c.B : 1);
  CUtensorMap xm, wm;
  cudaError_t e;
  if (S::KIND == Product::kExpand) {
    const int64_t row = r + c.rope;
    e = encode_map(&xm, c.x, {row, c.T_cap, c.B, 1}, {row, c.T_cap * row, c.B * c.T_cap * row}, kTok, 1);
  } else {
    const int64_t row = a.x_row;
    e = encode_map(&xm, c.x, {row, H, a.rows, 1}, {row, H * row, a.rows * H * row}, 1, kTok);
  }
  if (e == cudaSuccess)
    e = encode_map(&wm, c.w, {r, d, H, 1}, {r, d * r, H * d * r}, S::W_MN ? a.K : S::NT, 1);
  if (e != cudaSuccess) return e;
  // one CTA an SM: it may then take tensor memory without waiting for another's
  const int smem = std::max(weight_bytes(S::W_MN, S::NT, a.K) + kStagesA * kAtomA + 256 + 1024, 116 * 1024);
  e = cudaFuncSetAttribute(product_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
  if (e != cudaSuccess) return e;
  product_kernel<S><<<(unsigned)std::min<int64_t>(a.items, kNumSMs), kPrThreads, smem, st>>>(xm, wm, a);
  return cudaPeekAtLastError();
}

template <bool BF16, Product KIND>
cudaError_t launch_kind(const ProductCall& c, const ProductArgs& a, cudaStream_t st) {
  // 64-dim tiles where 128 would not divide the dims, or would leave SMs without work
  const int64_t wide = (int64_t)c.H * (a.n_dim / 128) * a.blocks * (KIND == Product::kExpand ? c.B : 1);
  if (a.n_dim % 128 != 0 || wide < kNumSMs) return launch_shape<PrShape<BF16, KIND, 64>>(c, a, st);
  return launch_shape<PrShape<BF16, KIND, 128>>(c, a, st);
}

template <bool BF16>
cudaError_t launch_t(const ProductCall& c, cudaStream_t st) {
  ProductArgs a{};
  a.B = c.B;
  a.H = c.H;
  a.T_len = c.T_len;
  a.x = static_cast<const uint16_t*>(c.x);
  a.out = static_cast<uint16_t*>(c.out);
  a.rows = c.kind == Product::kExpand ? c.rows : c.rows * c.B;
  a.blocks = ceil_div(a.rows, kTok);
  switch (c.kind) {
    case Product::kAbsorb:
      a.K = c.nope;
      a.n_dim = c.rank;
      a.out_row = c.rank + c.rope;
      a.x_row = c.nope + c.rope;
      a.rope_at = c.nope;
      return launch_kind<BF16, Product::kAbsorb>(c, a, st);
    case Product::kProject:
      a.K = c.rank;
      a.w_row = c.nope;
      a.n_dim = a.out_row = c.v_dim;
      a.x_row = c.rank;
      return launch_kind<BF16, Product::kProject>(c, a, st);
    case Product::kExpand:
      a.K = c.rank;
      a.n_dim = a.out_row = c.nope + c.v_dim;
      return launch_kind<BF16, Product::kExpand>(c, a, st);
  }
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_latent_product(const ProductCall& c, cudaStream_t st) {
  return c.dtype == MKV_BF16 ? launch_t<true>(c, st) : launch_t<false>(c, st);
}

}  // namespace mkv
