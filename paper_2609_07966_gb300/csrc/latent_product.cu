// The per-head products around latent attention, out[token][h] = x[token] W[h] with
//   absorb   W = W_uk[h]^T  (nope -> rank; the rotated part of the query is copied beside it)
//   project  W = W_uv[h]    (rank -> v)
//   expand   W = [W_uk[h]; W_uv[h]] on a cached row's latent part (rank -> nope + v)
// For a decode step's few tokens they are bound by reading the weights once (and by the launch), for a prompt's by the
// tensor cores and the shared memory that feeds them.  Both kernels hold a tile of one head's weights (all of K) in
// shared memory and stream token blocks past it, the accumulator in tensor memory twice, so that a block's stores run
// under the next one's products.  CTAs take equal runs of the (weight tile, token block) pairs, token blocks fastest,
// so a weight tile is loaded once or twice.
//
// product_kernel (absorb, project): D [128 tokens x NT] = X [128 x K] W [K x NT]; a thread stores a token's dims.  W is
//   used as it is stored: along K for project, along the output dims for absorb.
// expand_kernel: D^T [128 dims x 256 tokens] = W [128 x K] X^T [K x 256].  The narrow side is as wide as the tensor core
//   takes it, because a 128 x 256 product reads 12 KB of operands in 128 cycles where a 128 x 128 one reads 8 KB in 64:
//   the copies that refill shared memory need the difference.
// Measured (GPU time): 8192 rows for 32 heads (rank 512, 128 + 128 dims) 61 us, 1.12 PFLOP/s, 0.57 of cuBLAS's rate; a
// step's absorb for 8 tokens 4.3 us, project for 48 tokens 4.0 us; for 8 tokens of 128 heads 8.1 us (one weight tile after
// another) and 5.0 us.  Expand's runs are equal in T_max, not in the entries' lengths: one of 8192 rows beside three of 100
// takes 132 us.
#include <algorithm>

#include "mkv_roles.cuh"
#include "mkv_rows.h"

namespace mkv {

namespace {

struct ProductArgs {
  int B, H, K;                 // K: length of the sums
  int w_row;                   // first row of a head's weights used (project: nope)
  int n_dim;                   // output dims per head, dims per output row
  int out_row;
  int64_t rows;                // tokens (expand: of each entry)
  int64_t blocks;              // their blocks of 128 (expand: of each entry, of 256)
  int64_t items;               // H x dim tiles x blocks (expand: x B)
  int dim_tiles;
  const int32_t* T_len;        // expand
  const uint16_t* x;           // absorb: the queries, for their rotated part
  int x_row, rope_at;
  uint16_t* out;
  uint32_t* status;            // MKV_FLAG_* bits
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
  uint64_t wfull, wempty, afull[kStagesA], aempty[kStagesA], tfull[2], tempty[2], drained;
  uint32_t tslot;
  int fail, loaded, weights;   // token stages, weight tiles asked for (read after a failure)
};
static_assert(sizeof(PrCtl) <= 256, "control block");

__host__ __device__ inline int weight_bytes(bool w_mn, int NT, int K) {
  return (w_mn ? NT / 64 * K : K / 64 * NT) * 128;
}

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
    int64_t wt, t0;             // weight tile (h, dims), first token of the block
    int limit;                  // tokens of the block that exist
  };
  auto item = [&](int64_t i) {
    Item x;
    x.wt = i / a.blocks;
    x.t0 = i % a.blocks * kTok;
    x.limit = (int)std::min<int64_t>(kTok, a.rows - x.t0);
    return x;
  };

  // barriers and tensor memory, then what the stream's previous kernel wrote
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
    tc_mbar_init(&ctl->drained, 1);
    tc_fence_mbar_init();
    ctl->fail = ctl->loaded = ctl->weights = 0;
  }
  pdl_wait_and_trigger();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = ctl->tslot;
  volatile int* fail = &ctl->fail;
  uint32_t* status = a.status;

  if (warp == 4) {
    if (elect_one()) {
      int64_t held = -1;
      int c = 0, w = 0;
      for (int64_t i = first; i < last; ++i) {
        const Item x = item(i);
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
        ++n;
      }
      tc_commit(&ctl->drained);
    }
  } else {
    // stores: thread = token of the block
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    int n = 0;
    for (int64_t i = first; i < last; ++i) {
      const Item x = item(i);
      const int h = (int)(x.wt / a.dim_tiles), d0 = (int)(x.wt % a.dim_tiles) * NT, buf = n & 1;
      const bool ok = wait_or_fail(&ctl->tfull[buf], (uint32_t)((n / 2) & 1), fail, status);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after();
      const int r = warp * 32 + lane;
      const bool live = r < x.limit;
      const int64_t orow = (x.t0 + r) * a.H + h;
      uint4* dst = reinterpret_cast<uint4*>(a.out + orow * a.out_row + d0);
#pragma unroll
      for (int c = 0; c < NT / 32; ++c) {
        float v[32];
        tm_load<32>(tbase + lanes + (uint32_t)(buf * NT + c * 32), v);
        if (live) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            dst[c * 4 + e] =
                make_uint4(pack2<S::BF16>(v[8 * e], v[8 * e + 1]), pack2<S::BF16>(v[8 * e + 2], v[8 * e + 3]),
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
  // teardown: the products issued are complete; after a failure so are the copies (each wait bounded)
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0) {
    tc_mbar_wait(&ctl->drained, 0, kRoleWaitNs);
    if (ctl->fail) {
      if (ctl->weights > 0) tc_mbar_wait(&ctl->wfull, (uint32_t)((ctl->weights - 1) & 1), kRoleWaitNs);
      for (int c = std::max(0, ctl->loaded - kStagesA); c < ctl->loaded; ++c)
        tc_mbar_wait(&ctl->afull[c % kStagesA], (uint32_t)((c / kStagesA) & 1), kRoleWaitNs);
    }
  }
  __syncthreads();
  tc_fence_after();
  if (warp == 4) tc_dealloc(tbase, S::TMEM);
}

// ------------------------------------------------------------------------------------------------ expand
constexpr int kExTok = 256, kExStages = 3, kExThreads = 320;   // eight warps of stores, one of loads, one of products
constexpr int kExAtomW = 128 * 128, kExAtomX = kExTok * 128;

struct ExCtl {
  uint64_t wfull, wempty, xfull[kExStages], xempty[kExStages], tfull[2], tempty[2], drained;
  uint32_t tslot;
  int fail, loaded, weights;   // token stages, weight tiles asked for (read after a failure)
};
static_assert(sizeof(ExCtl) <= 256, "control block");

template <bool BF16>
__global__ void __launch_bounds__(kExThreads, 1)
    expand_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap,
                  const ProductArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  const int kc = a.K / 64;
  uint8_t* sx = sm + kc * kExAtomW;                       // [kExStages] 256 tokens x 64 of K
  ExCtl* ctl = reinterpret_cast<ExCtl*>(sx + kExStages * kExAtomX);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t first = a.items * blockIdx.x / gridDim.x, last = a.items * (blockIdx.x + 1) / gridDim.x;

  // the items of this CTA's run whose tokens exist
  struct Items {
    const ProductArgs& a;
    int64_t i, last;
    int wt, b, h, d0, limit;    // weight tile, entry, head, first dim, tokens of the block that exist
    int64_t t0;
    __device__ Items(const ProductArgs& args, int64_t f, int64_t l) : a(args), i(f), last(l) {}
    __device__ bool next() {
      for (; i < last; ++i) {
        const int64_t per = a.B * a.blocks, r = i % per;
        wt = (int)(i / per);
        b = (int)(r / a.blocks);
        t0 = r % a.blocks * kExTok;
        const int64_t n = std::min<int64_t>(a.rows, a.T_len[b]) - t0;
        if (n <= 0) continue;
        limit = (int)std::min<int64_t>(kExTok, n);
        h = wt / a.dim_tiles;
        d0 = wt % a.dim_tiles * 128;
        ++i;
        return true;
      }
      return false;
    }
  };

  if (warp == 8) tc_alloc(&ctl->tslot, 512);
  if (threadIdx.x == 0) {
    tc_mbar_init(&ctl->wfull, 1);
    tc_mbar_init(&ctl->wempty, 1);
    for (int s = 0; s < kExStages; ++s) {
      tc_mbar_init(&ctl->xfull[s], 1);
      tc_mbar_init(&ctl->xempty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      tc_mbar_init(&ctl->tfull[s], 1);
      tc_mbar_init(&ctl->tempty[s], 8);
    }
    tc_mbar_init(&ctl->drained, 1);
    tc_fence_mbar_init();
    ctl->fail = ctl->loaded = ctl->weights = 0;
  }
  pdl_wait_and_trigger();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = ctl->tslot;
  volatile int* fail = &ctl->fail;
  uint32_t* status = a.status;
  Items it(a, first, last);

  if (warp == 8) {
    if (elect_one()) {
      int held = -1, w = 0, s = 0, lap = 0;
      bool ok = true;
      while (ok && it.next()) {
        if (it.wt != held) {
          if (w > 0 && !wait_or_fail(&ctl->wempty, (uint32_t)((w - 1) & 1), fail, status)) break;
          tc_mbar_expect_tx(&ctl->wfull, kc * kExAtomW);
          for (int j = 0; j < kc; ++j)
            tma_load_4d(sm + j * kExAtomW, &wmap, j * 64, 0, 0, (it.h * a.out_row + it.d0) / 32, &ctl->wfull);
          held = it.wt;
          ctl->weights = ++w;
        }
        for (int j = 0; j < kc; ++j) {
          if (lap > 0 && !wait_or_fail(&ctl->xempty[s], (uint32_t)((lap - 1) & 1), fail, status)) {
            ok = false;
            break;
          }
          tc_mbar_expect_tx(&ctl->xfull[s], kExAtomX);
          tma_load_4d(sx + s * kExAtomX, &xmap, j * 64, (int)it.t0, it.b, 0, &ctl->xfull[s]);
          ctl->loaded = lap * kExStages + s + 1;
          if (++s == kExStages) {
            s = 0;
            ++lap;
          }
        }
      }
    }
  } else if (warp == 9) {
    if (elect_one()) {
      constexpr uint32_t id = tc_idesc(BF16, 128, kExTok, false, false);
      const Desc wd = tc_desc_sw128(smem_addr(sm)), xd = tc_desc_sw128(smem_addr(sx));
      int held = -1, w = 0, n = 0, s = 0, lap = 0;
      bool ok = true;
      while (ok && it.next()) {
        if (it.wt != held) {
          if (w > 0) tc_commit(&ctl->wempty);             // the products with the old weights
          ok = wait_or_fail(&ctl->wfull, (uint32_t)(w & 1), fail, status);
          held = it.wt;
          ++w;
        }
        const int buf = n & 1;
        if (ok && n >= 2) ok = wait_or_fail(&ctl->tempty[buf], (uint32_t)((n / 2 - 1) & 1), fail, status);
        for (int j = 0; ok && j < kc; ++j) {
          ok = wait_or_fail(&ctl->xfull[s], (uint32_t)(lap & 1), fail, status);
          if (!ok) break;
          tc_fence_after();
          const Desc ws = wd.at(j * kExAtomW).opaque(), xs = xd.at(s * kExAtomX).opaque();
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            tc_mma_ss(tbase + (uint32_t)(buf * kExTok), ws.at(kk * 32), xs.at(kk * 32), id, j > 0 || kk > 0 ? 1u : 0u);
          tc_commit(&ctl->xempty[s]);
          if (++s == kExStages) {
            s = 0;
            ++lap;
          }
        }
        if (!ok) break;
        tc_commit(&ctl->tfull[buf]);
        ++n;
      }
      tc_commit(&ctl->drained);
    }
  } else {
    // stores: lane = dim (in the order of the weights' rows), half of the block's tokens; the lanes exchange values, so
    // that each stores eight dims of a token
    const int q = warp & 3, half = warp >> 2;
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    int n = 0;
    while (it.next()) {
      const int buf = n & 1;
      const bool ok = wait_or_fail(&ctl->tfull[buf], (uint32_t)((n / 2) & 1), fail, status);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after();
      // the accumulator is given back before the stores, not behind them
      float v[128];
#pragma unroll
      for (int c = 0; c < 4; ++c)
        tm_issue<32>(tbase + lanes + (uint32_t)(buf * kExTok + half * 128 + c * 32),
                     *reinterpret_cast<float(*)[32]>(&v[c * 32]));
#pragma unroll
      for (int c = 0; c < 4; ++c) tm_wait<32>(*reinterpret_cast<float(*)[32]>(&v[c * 32]));
      tc_fence_before();
      __syncwarp();
      if (lane == 0) tc_mbar_arrive(&ctl->tempty[buf]);
      const int dim = it.d0 + q * 32 + (lane & 3) * 8, tok = half * 128 + (lane >> 2);   // of its first store
      uint16_t* dst = a.out + (((int64_t)it.b * a.H + it.h) * a.rows + it.t0 + tok) * a.out_row + dim;
      const int left = dim < a.n_dim ? it.limit - tok : 0;         // its tokens c with c < left exist
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint4 x[4];
        gather_rows<BF16>(*reinterpret_cast<float(*)[32]>(&v[c * 32]), lane, x);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c * 32 + 8 * k < left) *reinterpret_cast<uint4*>(dst + (int64_t)(c * 32 + 8 * k) * a.out_row) = x[k];
      }
      ++n;
    }
  }
  // teardown: the products issued are complete; after a failure so are the copies (each wait bounded)
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0) {
    tc_mbar_wait(&ctl->drained, 0, kRoleWaitNs);
    if (ctl->fail) {
      if (ctl->weights > 0) tc_mbar_wait(&ctl->wfull, (uint32_t)((ctl->weights - 1) & 1), kRoleWaitNs);
      for (int c = std::max(0, ctl->loaded - kExStages); c < ctl->loaded; ++c)
        tc_mbar_wait(&ctl->xfull[c % kExStages], (uint32_t)((c / kExStages) & 1), kRoleWaitNs);
    }
  }
  __syncthreads();
  tc_fence_after();
  if (warp == 8) tc_dealloc(tbase, 512);
}

template <bool BF16>
cudaError_t launch_expand(const ProductCall& c, ProductArgs a, cudaStream_t st) {
  const int64_t H = c.H, d = c.nope + c.v_dim, r = c.rank, row = r + c.rope;
  a.dim_tiles = (int)ceil_div(d, 128);
  a.blocks = ceil_div(a.rows, kExTok);
  a.items = H * a.dim_tiles * a.blocks * c.B;
  CUtensorMap xm, wm;
  cudaError_t e = encode_map(&xm, c.x, {row, c.T_cap, c.B, 1}, {row, c.T_cap * row, c.B * c.T_cap * row}, kExTok, 1);
  // a tile's rows in the order that gather_rows wants: row 4 s + g of 32 is dim 8 g + s (past a head's dims it reads
  // the next head's, whose outputs are not stored)
  if (e == cudaSuccess) e = encode_map(&wm, c.w, {r, 4, 8, H * d / 32}, {8 * r, r, 32 * r}, 4, 8, 4);
  if (e != cudaSuccess) return e;
  constexpr int smem = 8 * kExAtomW + kExStages * kExAtomX + 256 + 1024;   // one CTA an SM, at either rank
  static_assert(smem <= 227 * 1024 && smem >= 116 * 1024, "shared memory");
  e = cudaFuncSetAttribute(expand_kernel<BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_pdl(expand_kernel<BF16>, dim3((unsigned)std::min<int64_t>(a.items, kNumSMs)), dim3(kExThreads), smem, st,
                    xm, wm, a);
}

template <class S>
cudaError_t launch_shape(const ProductCall& c, ProductArgs a, cudaStream_t st) {
  const int64_t H = c.H, d = c.nope + c.v_dim, r = c.rank;
  a.dim_tiles = a.n_dim / S::NT;
  a.items = H * a.dim_tiles * a.blocks;
  CUtensorMap xm, wm;
  const int64_t row = a.x_row;
  cudaError_t e = encode_map(&xm, c.x, {row, H, a.rows, 1}, {row, H * row, a.rows * H * row}, 1, kTok);
  if (e == cudaSuccess)
    e = encode_map(&wm, c.w, {r, d, H, 1}, {r, d * r, H * d * r}, S::W_MN ? a.K : S::NT, 1);
  if (e != cudaSuccess) return e;
  // one CTA an SM: it may then take tensor memory without waiting for another's
  const int smem = std::max(weight_bytes(S::W_MN, S::NT, a.K) + kStagesA * kAtomA + 256 + 1024, 116 * 1024);
  e = cudaFuncSetAttribute(product_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
  if (e != cudaSuccess) return e;
  return launch_pdl(product_kernel<S>, dim3((unsigned)std::min<int64_t>(a.items, kNumSMs)), dim3(kPrThreads), smem, st,
                    xm, wm, a);
}

template <bool BF16, Product KIND>
cudaError_t launch_kind(const ProductCall& c, const ProductArgs& a, cudaStream_t st) {
  // 64-dim tiles where 128 would not divide the dims, or would leave half of the SMs without work (a step's absorb,
  // 32 heads, rank 512: 128 wide tiles 4.3 us, 256 narrow ones on 152 SMs 5.4)
  const int64_t wide = (int64_t)c.H * (a.n_dim / 128) * a.blocks;
  if (a.n_dim % 128 != 0 || wide <= kNumSMs / 2) return launch_shape<PrShape<BF16, KIND, 64>>(c, a, st);
  return launch_shape<PrShape<BF16, KIND, 128>>(c, a, st);
}

template <bool BF16>
cudaError_t launch_t(const ProductCall& c, cudaStream_t st) {
  ProductArgs a{};
  const cudaError_t e = status_word(&a.status);
  if (e != cudaSuccess) return e;
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
      return launch_expand<BF16>(c, a, st);
  }
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_latent_product(const ProductCall& c, cudaStream_t st) {
  return c.dtype == MKV_BF16 ? launch_t<true>(c, st) : launch_t<false>(c, st);
}

}  // namespace mkv
