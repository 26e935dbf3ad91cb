// Attention of a few tokens' query rows over a cache and the drafted tokens behind it: the tree form of an
// FP16 cache's decode step and the absorbed form of latent attention,
//   out_r = sum_t p_rt v_t / sum_t p_rt,  p_rt = 2^(scale log2(e) q_r . k_t - m_r) over the tokens t that r sees.
//
// All query rows that share a key head (n tokens x the group's heads; latent: x all heads) meet every key, so
// a key is loaded once per block of N rows and both products run on the tensor cores with the rows as the
// narrow side:
//   S^T [keys x N]  = K [keys x dk] Q^T           A = the key tile as loaded, B = the query block
//   O^T [dv x N]   += V^T [dv x keys] P^T         A = the value tile read along its other index (no transposed
//                                                  copy), B = the weights
// so no row is padded to the 128 of the wide side, and for a latent cache the value tile is the key tile itself
// (its first dv dims): one load of a row serves both products.  Accumulators live in tensor memory: S^T twice
// (tile t + 1's scores are computed under tile t's softmax), O^T as dv / 128 blocks of N columns.
//
// A CTA takes one (batch entry, key head), one block of N rows and a run of key tiles (the drafted tokens are
// one more tile at the end); runs of one block are joined by join_kernel.  Warps 0..4g-1 are the softmax
// (a thread holds one key and N / g rows), then one warp loads tiles by TMA and one issues the products.
//
// The running maximum m is only raised when some score of a tile passes it by 2^8 (weights then stay below
// 2^14 with the offset below), which a group-wide vote finds: after the first tiles almost never, so the O^T
// accumulator is almost never rescaled.  m, the weight sums and O^T are fp32; the weights are rounded once
// to the 16-bit type of the values, as the tensor cores take them.
#include <math.h>

#include <algorithm>

#include "mkv_roles.cuh"
#include "mkv_rows.h"

namespace mkv {

__device__ uint32_t g_status_rows;   // MKV_FLAG_* bits raised here

cudaError_t take_status_rows(uint32_t* flags, cudaStream_t st) {
  uint32_t v = 0, zero = 0;
  cudaError_t e = cudaMemcpyFromSymbolAsync(&v, g_status_rows, sizeof(v), 0, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaMemcpyToSymbolAsync(g_status_rows, &zero, sizeof(zero), 0, cudaMemcpyHostToDevice, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  *flags |= v;
  return e;
}

namespace {

constexpr float kRaise = 8.f;       // a score may pass the running maximum by this (log2) before it is raised
// Weights carry 2^kOffset, so that those far below the maximum keep full precision in fp16 (normal down to
// 2^-20 of the maximum); it cancels in the division by their sum.
constexpr float kOffset = 6.f;
constexpr float kNoMax = -1e30f;    // running maximum of a row that has seen nothing

struct RowsArgs {
  int B, n, H, Hkv, G;              // G: query heads per key head (latent: H)
  int R;                            // rows per unit: n G
  int n_split;
  bool tree;
  int64_t T_cap;
  float scale_log2;
  const int32_t* T_len;
  const uint64_t* mask;             // [B][n]
  const uint16_t* v_tree;           // values of the drafted tokens (for non-finite ones)
  int64_t v_tok, v_head;            // their strides: token, key head
  void* out;
  float* part_o;                    // [units][R][n_split][DV]
  float2* part_ml;                  // [units][R][n_split]
};

// KA / VA: 64-dim atoms of a key / value; SHARED: values are the keys' first atoms; KT keys a tile, N rows a
// block, NS stages, NP weight buffers.
template <bool BF16_, int KA_, int VA_, bool SHARED_, int KT_, int N_, int NS_, int NP_>
struct Shape {
  static constexpr bool BF16 = BF16_, SHARED = SHARED_;
  static constexpr int KA = KA_, VA = VA_, KT = KT_, N = N_, NS = NS_, NP = NP_;
  static constexpr int DV = VA * 64;
  static constexpr int MV = DV >= 128 ? 128 : 64;          // value dims per product (its M)
  static constexpr int NB = DV / MV;                       // O^T blocks
  static constexpr int NG = N > 64 ? 4 : 2;                // softmax groups of 128 threads
  static constexpr int C = N / NG;                         // rows a softmax thread holds
  static constexpr int THREADS = NG * 128 + 128;           // softmax groups; loads, products (and two idle warps)
  // registers a thread: what a launch of THREADS gets, and its split between softmax and the others
  static constexpr int RL = NG == 2 ? 168 : 96, RS = NG == 2 ? 208 : 104, RO = NG == 2 ? 88 : 64;
  static_assert(NG * RS + RO <= (NG + 1) * RL, "register shares");
  static constexpr int PW = N >= 64 ? 64 : N;              // row width of a weight tile (elements)
  static constexpr int ATOM = KT * 128;                    // bytes of 64 dims of a tile
  static constexpr int QATOM = N * 128;
  static constexpr int STAGE = (KA + (SHARED ? 0 : VA)) * ATOM;
  static constexpr int V_OFF = SHARED ? 0 : KA * ATOM;     // of the values within a stage
  static constexpr int PBUF = KT * N * 2;
  static constexpr int Q_OFF = 0;
  static constexpr int KV_OFF = KA * QATOM;
  static constexpr int P_OFF = KV_OFF + NS * STAGE;
  static constexpr int CTL_OFF = P_OFF + NP * PBUF;
  static constexpr int RED_OFF = CTL_OFF + 768;            // [4][N] floats
  static constexpr int BYTES = RED_OFF + 4 * N * 4;
  static constexpr int ALLOC = BYTES + 1024;               // slack to align the base to 1024 B
  static constexpr int COLS = (2 + NB) * N;
  static constexpr int TMEM = COLS <= 32 ? 32 : COLS <= 64 ? 64 : COLS <= 128 ? 128 : COLS <= 256 ? 256 : 512;
  static_assert(COLS <= 512 && ALLOC <= 227 * 1024, "does not fit an SM");
};

struct RowsCtl {
  uint64_t qfull, kfull[4], kempty[4], sfull[2], pfull[2], pvdone[2];
  uint64_t nonfinite;     // drafted tokens that hold a non-finite value
  uint32_t tslot;
  int fail, loaded, issued;
  uint64_t mask[kMaxTree];
};
static_assert(sizeof(RowsCtl) <= 768, "control block");

template <class S>
__global__ void __launch_bounds__(S::THREADS, 1)
    rows_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CUtensorMap ktmap,
                const __grid_constant__ CUtensorMap vtmap, const RowsArgs a) {
  constexpr int KT = S::KT, N = S::N, C = S::C;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  RowsCtl* ctl = reinterpret_cast<RowsCtl*>(sm + S::CTL_OFF);
  float* red = reinterpret_cast<float*>(sm + S::RED_OFF);
  const int split = blockIdx.x, rb = blockIdx.y, unit = blockIdx.z;
  const int b = unit / a.Hkv, kvh = unit % a.Hkv;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // this CTA's tiles: the entry's cached tiles, then the drafted tokens' tile
  const int len = (int)std::min<int64_t>(std::max(a.T_len[b], 0), a.T_cap);
  const int ctiles = (len + KT - 1) / KT, tiles = ctiles + (a.tree ? 1 : 0);
  const int t_begin = (int)((int64_t)tiles * split / a.n_split);
  const int t_end = (int)((int64_t)tiles * (split + 1) / a.n_split);
  const int nt = t_end - t_begin;
  const int row0 = rb * N;
  const int rows = std::min(N, a.R - row0);
  if (nt == 0) {
    for (int r = threadIdx.x; r < rows; r += S::THREADS)
      if (a.n_split > 1) a.part_ml[((int64_t)unit * a.R + row0 + r) * a.n_split + split] = make_float2(-INFINITY, 0.f);
    if (a.n_split == 1)
      for (int e = threadIdx.x; e < rows * S::DV; e += S::THREADS) {
        const int r = row0 + e / S::DV;
        const int64_t o = ((int64_t)b * a.n + r / a.G) * a.H + (int64_t)kvh * a.G + r % a.G;
        static_cast<uint16_t*>(a.out)[o * S::DV + e % S::DV] = 0;
      }
    return;
  }

  if (warp == S::NG * 4) tc_alloc(&ctl->tslot, S::TMEM);
  if (threadIdx.x == 0) {
    tc_mbar_init(&ctl->qfull, 1);
    for (int s = 0; s < S::NS; ++s) {
      tc_mbar_init(&ctl->kfull[s], 1);
      tc_mbar_init(&ctl->kempty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      tc_mbar_init(&ctl->sfull[s], 1);
      tc_mbar_init(&ctl->pfull[s], S::NG * 4);
      tc_mbar_init(&ctl->pvdone[s], 1);
    }
    tc_fence_mbar_init();
    ctl->nonfinite = 0;
    ctl->fail = 0;
    ctl->loaded = 0;
    ctl->issued = 0;
  }
  if (a.tree && threadIdx.x < a.n) ctl->mask[threadIdx.x] = a.mask[(int64_t)b * a.n + threadIdx.x];
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = ctl->tslot;
  const uint32_t tO = tbase + 2 * N;
  volatile int* fail = &ctl->fail;

  if (warp >= S::NG * 4) {
    regs_down<S::RO>();
    if (warp == S::NG * 4) {
      // ---------------------------------------------------------------- loads
      if (lane == 0) {
        tc_mbar_expect_tx(&ctl->qfull, S::KA * S::QATOM);
        for (int at = 0; at < S::KA; ++at)
          if (S::SHARED)
            tma_load_4d(sm + S::Q_OFF + at * S::QATOM, &qmap, at * 64, row0, b, 0, &ctl->qfull);
          else
            tma_load_4d(sm + S::Q_OFF + at * S::QATOM, &qmap, at * 64, kvh * a.G, row0 / a.G, b, &ctl->qfull);
        for (int t = 0; t < nt; ++t) {
          const int s = t % S::NS, u = t / S::NS;
          if (u > 0 && !wait_or_fail(&ctl->kempty[s], (uint32_t)((u - 1) & 1), fail, &g_status_rows)) break;
          const bool tr = t_begin + t >= ctiles;
          const int key = tr ? 0 : (t_begin + t) * KT;
          uint8_t* dst = sm + S::KV_OFF + s * S::STAGE;
          tc_mbar_expect_tx(&ctl->kfull[s], S::STAGE);
          for (int at = 0; at < S::KA; ++at)
            tma_load_4d(dst + at * S::ATOM, tr ? &ktmap : &kmap, at * 64, key, S::SHARED ? b : kvh, S::SHARED ? 0 : b,
                        &ctl->kfull[s]);
          if (!S::SHARED)
            for (int at = 0; at < S::VA; ++at)
              tma_load_4d(dst + S::V_OFF + at * S::ATOM, tr ? &vtmap : &vmap, at * 64, key, kvh, b, &ctl->kfull[s]);
          ctl->loaded = t + 1;
        }
      }
    } else if (warp == S::NG * 4 + 1) {
      // ---------------------------------------------------------------- products
      if (lane == 0) {
        constexpr uint32_t idS = tc_idesc(S::BF16, KT, N, false, false);
        constexpr uint32_t idO = tc_idesc(S::BF16, S::MV, N, true, true);
        const Desc qd = tc_desc_sw128(smem_addr(sm + S::Q_OFF));
        const Desc kd = tc_desc_sw128(smem_addr(sm + S::KV_OFF));
        const Desc vd = tc_desc_mn<64>(smem_addr(sm + S::KV_OFF + S::V_OFF), S::ATOM);
        const Desc pd = tc_desc_mn<S::PW>(smem_addr(sm + S::P_OFF), KT * S::PW * 2);
        auto scores = [&](int t) {        // S^T of tile t
          const int s = t % S::NS;
          if (!wait_or_fail(&ctl->kfull[s], (uint32_t)((t / S::NS) & 1), fail, &g_status_rows)) return false;
          tc_fence_after();
          const Desc ks = kd.at(s * S::STAGE).opaque(), qs = qd.opaque();
  #pragma unroll
          for (int kk = 0; kk < S::KA * 4; ++kk)
            tc_mma_ss(tbase + (uint32_t)((t & 1) * N), ks.at((kk >> 2) * S::ATOM + (kk & 3) * 32),
                      qs.at((kk >> 2) * S::QATOM + (kk & 3) * 32), idS, kk > 0 ? 1u : 0u);
          tc_commit(&ctl->sfull[t & 1]);
          return true;
        };
        bool ok = wait_or_fail(&ctl->qfull, 0, fail, &g_status_rows) && scores(0);
        for (int t = 0; ok && t < nt; ++t) {
          if (t + 1 < nt && !scores(t + 1)) break;
          const int s = t % S::NS, pb = t % S::NP;
          if (!wait_or_fail(&ctl->pfull[pb], (uint32_t)((t / S::NP) & 1), fail, &g_status_rows)) break;
          tc_fence_after();
          const Desc vs = vd.at(s * S::STAGE).opaque(), ps = pd.at(pb * S::PBUF).opaque();
  #pragma unroll
          for (int mb = 0; mb < S::NB; ++mb)
  #pragma unroll
            for (int kk = 0; kk < KT / 16; ++kk)
              tc_mma_ss(tO + (uint32_t)(mb * N), vs.at(mb * (S::MV / 64) * S::ATOM + kk * 2048),
                        ps.at(kk * 16 * S::PW * 2), idO, t > 0 || kk > 0 ? 1u : 0u);
          tc_commit(&ctl->kempty[s]);
          tc_commit(&ctl->pvdone[pb]);
          ctl->issued = t + 1;
        }
      }
    }
  } else {
    regs_up<S::RS>();
    // ---------------------------------------------------------------- softmax
    const int q = warp & 3, grp = warp >> 2;             // lane quarter (keys), rows grp C .. + C - 1
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    // a tile of 64 keys takes lanes 0..15 of each quarter, one of 128 all of them
    const bool live = KT == 128 || lane < 16;
    const int key = KT == 128 ? q * 32 + lane : q * 16 + (lane & 15);
    float m[C], l[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      m[c] = kNoMax;
      l[c] = 0.f;
    }
    // A warp whose wait ran out stops waiting but still meets its group's barriers, so none is left waiting.
    bool dead = false;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (!dead) dead = !__all_sync(0xffffffffu, wait_or_fail(bar, parity, fail, &g_status_rows));
      tc_fence_after();
    };
    for (int t = 0; t < nt; ++t) {
      const int s = t % S::NS, pb = t % S::NP;
      const bool tr = t_begin + t >= ctiles;
      const int valid = tr ? a.n : std::min(KT, len - (t_begin + t) * KT);   // keys of the tile that exist
      wait(&ctl->sfull[t & 1], (uint32_t)((t >> 1) & 1));
      float v[C];
      tm_load<C>(tbase + lanes + (uint32_t)((t & 1) * N + grp * C), v);
      const bool exists = live && key < valid;
      bool over = false;
      if (tr) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int tok = (row0 + grp * C + c) / a.G;
          const bool see = exists && tok < a.n && (ctl->mask[tok] >> key & 1);
          v[c] = see ? v[c] * a.scale_log2 : -INFINITY;
          over |= v[c] > m[c] + kRaise;
        }
      } else {
#pragma unroll
        for (int c = 0; c < C; ++c) {
          v[c] = exists ? v[c] * a.scale_log2 : -INFINITY;
          over |= v[c] > m[c] + kRaise;
        }
      }
      if (bar_or(1 + grp, 128, over)) {
        // some score passed its row's maximum: raise the maxima to the tile's, rescale sums and outputs
        float w[C];
#pragma unroll
        for (int c = 0; c < C; ++c) w[c] = v[c];
        reduce_columns<C>(w, lane, [](float x, float y) { return fmaxf(x, y); });
        if ((lane & (32 / C - 1)) == 0) red[q * N + grp * C + lane / (32 / C)] = w[0];
        bar_sync(1 + grp, 128);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int x = grp * C + c;
          const float mx = fmaxf(fmaxf(red[x], red[N + x]), fmaxf(red[2 * N + x], red[3 * N + x]));
          const float nm = fmaxf(m[c], mx);
          w[c] = ex2_approx(m[c] - nm);
          m[c] = nm;
          l[c] *= w[c];
        }
        if (t > 0) {
          wait(&ctl->pvdone[(t - 1) % S::NP], (uint32_t)(((t - 1) / S::NP) & 1));
#pragma unroll 1
          for (int mb = 0; mb < S::NB; ++mb) {
            float o[C];
            tm_load<C>(tO + lanes + (uint32_t)(mb * N + grp * C), o);
#pragma unroll
            for (int c = 0; c < C; ++c) o[c] *= w[c];
            tm_store<C>(tO + lanes + (uint32_t)(mb * N + grp * C), o);
          }
          tm_store_wait();
        }
      }
      // weights, their sums, and the rounded weights for the second product
      uint32_t pk[C / 2];
#pragma unroll
      for (int c = 0; c < C; c += 2) {
        const float p0 = ex2_approx(v[c] - m[c] + kOffset), p1 = ex2_approx(v[c + 1] - m[c + 1] + kOffset);
        l[c] += p0;
        l[c + 1] += p1;
        pk[c / 2] = pack2<S::BF16>(p0, p1);
      }
      if (t >= S::NP) wait(&ctl->pvdone[pb], (uint32_t)((t / S::NP - 1) & 1));
      if (live) {
        const int col = grp * C;
        uint8_t* pt = sm + S::P_OFF + pb * S::PBUF + (col / S::PW) * (KT * S::PW * 2);
#pragma unroll
        for (int i = 0; i < C / 8; ++i)
          *reinterpret_cast<uint4*>(pt + mn_offset<S::PW>(key, (col % S::PW) / 8 + i)) =
              make_uint4(pk[4 * i], pk[4 * i + 1], pk[4 * i + 2], pk[4 * i + 3]);
      }
      // Values that no row may meet must not meet a zero weight either (0 x NaN): slots past the length become
      // zeros; a drafted token's non-finite values become zeros here and are added to the rows that see it at
      // the end.  (Latent: the scores of this tile are complete, so its keys may be overwritten.)
      if (valid < KT && !tr) {
        uint8_t* vt = sm + S::KV_OFF + s * S::STAGE + S::V_OFF;
        for (int e = threadIdx.x; e < (KT - valid) * 8 * S::VA; e += S::NG * 128) {
          const int r = valid + e / (8 * S::VA), x = e % (8 * S::VA);
          *reinterpret_cast<uint4*>(vt + (x >> 3) * S::ATOM + r * 128 + ((x & 7) << 4)) = make_uint4(0, 0, 0, 0);
        }
      }
      if (tr) {
        uint8_t* vt = sm + S::KV_OFF + s * S::STAGE + S::V_OFF;
        for (int e = threadIdx.x; e < valid * 8 * S::VA; e += S::NG * 128) {
          const int r = e / (8 * S::VA), x = e % (8 * S::VA);
          uint4* p8 = reinterpret_cast<uint4*>(vt + (x >> 3) * S::ATOM + r * 128 + ((x & 7) << 4));
          uint4 raw = *p8;
          if (bad_pairs<S::BF16>(raw)) {
            *p8 = raw;
            atomicOr(reinterpret_cast<unsigned long long*>(&ctl->nonfinite), 1ull << r);
          }
        }
      }
      fence_async_smem();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) tc_mbar_arrive(&ctl->pfull[pb]);
    }
    // ---------------------------------------------------------------- outputs of this run of tiles
    wait(&ctl->pvdone[(nt - 1) % S::NP], (uint32_t)(((nt - 1) / S::NP) & 1));
    if (!bar_or(1 + grp, 128, dead)) {                   // (the group's earlier reads of `red` are done)
      float w[C];
#pragma unroll
      for (int c = 0; c < C; ++c) w[c] = live ? l[c] : 0.f;
      reduce_columns<C>(w, lane, [](float x, float y) { return x + y; });
      if ((lane & (32 / C - 1)) == 0) red[q * N + grp * C + lane / (32 / C)] = w[0];
      bar_sync(1 + grp, 128);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int x = grp * C + c;
        l[c] = (red[x] + red[N + x]) + (red[2 * N + x] + red[3 * N + x]);
      }
      if (a.n_split > 1 && q == 0 && lane == 0) {
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (grp * C + c < rows)
            a.part_ml[((int64_t)unit * a.R + row0 + grp * C + c) * a.n_split + split] =
                make_float2(l[c] == 0.f ? -INFINITY : m[c], l[c]);
      }
      const uint64_t nf = ctl->nonfinite;
      const bool dlive = S::MV == 128 || lane < 16;
#pragma unroll 1
      for (int mb = 0; mb < S::NB; ++mb) {
        const int d = mb * S::MV + (S::MV == 128 ? q * 32 + lane : q * 16 + (lane & 15));
        float o[C];
        tm_load<C>(tO + lanes + (uint32_t)(mb * N + grp * C), o);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int r = grp * C + c;
          if (r >= rows || !dlive) continue;
          const int tok = (row0 + r) / a.G, g = (row0 + r) % a.G;
          float x = o[c];
          if (nf != 0) {                                 // the non-finite values that this row sees
            for (uint64_t bits = nf & ctl->mask[tok]; bits; bits &= bits - 1) {
              const int j = __ffsll((long long)bits) - 1;
              const uint16_t y = a.v_tree[((int64_t)b * a.n + j) * a.v_tok + kvh * a.v_head + d];
              if (non_finite<S::BF16>(y)) x += widen<S::BF16>(y);
            }
          }
          if (a.n_split > 1) {
            a.part_o[(((int64_t)unit * a.R + row0 + r) * a.n_split + split) * S::DV + d] = x;
          } else {
            const int64_t at = (((int64_t)b * a.n + tok) * a.H + (int64_t)kvh * a.G + g) * S::DV + d;
            static_cast<uint16_t*>(a.out)[at] = (uint16_t)pack2<S::BF16>(l[c] == 0.f ? 0.f : x / l[c], 0.f);
          }
        }
      }
    }
  }
  // teardown: on a failure wait (bounded) for the copies and products already issued
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && ctl->fail) {
    tc_mbar_wait(&ctl->qfull, 0, kRoleWaitNs);
    for (int t = std::max(0, ctl->loaded - S::NS); t < ctl->loaded; ++t)
      tc_mbar_wait(&ctl->kfull[t % S::NS], (uint32_t)((t / S::NS) & 1), kRoleWaitNs);
    if (ctl->issued > 0) {
      const int t = ctl->issued - 1;
      tc_mbar_wait(&ctl->pvdone[t % S::NP], (uint32_t)((t / S::NP) & 1), kRoleWaitNs);
    }
  }
  __syncthreads();
  tc_fence_after();
  if (warp == S::NG * 4) tc_dealloc(tbase, S::TMEM);
}

// out = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s over the splits of one row.  A thread takes four dims.
template <bool BF16>
__global__ void __launch_bounds__(128) join_kernel(const RowsArgs a, int DV) {
  pdl_wait_and_trigger();
  const int64_t row = blockIdx.x;                        // unit R + r
  const int64_t unit = row / a.R;
  const int r = (int)(row % a.R), b = (int)(unit / a.Hkv), kvh = (int)(unit % a.Hkv);
  const float2* ml = a.part_ml + row * a.n_split;
  float M = -INFINITY;
  for (int s = 0; s < a.n_split; ++s) M = fmaxf(M, ml[s].x);
  const int64_t at = (((int64_t)b * a.n + r / a.G) * a.H + (int64_t)kvh * a.G + r % a.G) * DV;
  for (int d = threadIdx.x * 4; d < DV; d += 512) {
    float L = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < a.n_split; ++s) {
      const float2 x = ml[s];
      if (x.x == -INFINITY) continue;                    // nothing seen: its output was not written
      const float w = ex2_approx(x.x - M);
      const float4 y = *reinterpret_cast<const float4*>(a.part_o + (row * a.n_split + s) * DV + d);
      L += w * x.y;
      o.x += w * y.x;
      o.y += w * y.y;
      o.z += w * y.z;
      o.w += w * y.w;
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    uint2 h;
    h.x = pack2<BF16>(o.x * inv, o.y * inv);
    h.y = pack2<BF16>(o.z * inv, o.w * inv);
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at + d) = h;
  }
}

// ---------------------------------------------------------------- host side
struct Plan {
  int N, KT, R, row_blocks, n_split;
  size_t ml_off, o_off, bytes;
};

Plan plan_rows(const RowsCall& c) {
  Plan p{};
  p.R = c.n * (c.H / c.Hkv);
  p.N = 64;
  p.KT = c.latent ? 64 : 128;
  p.row_blocks = (int)ceil_div(p.R, p.N);
  // the run length that leaves the busiest SM least to do; a run costs a few tiles' time by itself
  const int64_t tiles = ceil_div(c.T_cap, p.KT) + 1, blocks = (int64_t)c.B * c.Hkv * p.row_blocks;
  int64_t best = 1, cost = INT64_MAX;
  for (int64_t n = 1; n <= std::min<int64_t>(tiles, kNumSMs); ++n) {
    const int64_t x = ceil_div(blocks * n, kNumSMs) * (ceil_div(tiles, n) + 4);
    if (x < cost) {
      cost = x;
      best = n;
    }
  }
  p.n_split = (int)best;
  const size_t parts = (size_t)c.B * c.Hkv * p.R * p.n_split;
  p.ml_off = kCounterBytes;
  p.o_off = p.ml_off + align256(parts * sizeof(float2));
  p.bytes = p.n_split > 1 ? p.o_off + align256(parts * c.dv * sizeof(float)) : kCounterBytes;
  return p;
}

template <class S>
cudaError_t launch_shape(const RowsCall& c, const Plan& p, RowsArgs a, cudaStream_t st) {
  CUtensorMap qm, km, vm, ktm, vtm;
  const int64_t dk = c.dk, T = c.T_cap, n = c.n, B = c.B, Hkv = c.Hkv, H = c.H, G = H / Hkv;
  cudaError_t e;
  if (S::SHARED) {
    e = encode_map(&qm, c.q, {dk, n * H, B, 1}, {dk, n * H * dk, B * n * H * dk}, S::N, 1);
    if (e == cudaSuccess) e = encode_map(&km, c.k, {dk, T, B, 1}, {dk, T * dk, B * T * dk}, S::KT, 1);
    ktm = km;
    if (e == cudaSuccess && c.k_tree != nullptr)
      e = encode_map(&ktm, c.k_tree, {dk, n, B, 1}, {dk, n * dk, B * n * dk}, S::KT, 1);
    vm = km;
    vtm = ktm;
  } else {
    e = encode_map(&qm, c.q, {dk, H, n, B}, {dk, H * dk, n * H * dk}, (int)G, (int)(S::N / G));
    if (e == cudaSuccess) e = encode_map(&km, c.k, {dk, T, Hkv, B}, {dk, T * dk, Hkv * T * dk}, S::KT, 1);
    if (e == cudaSuccess) e = encode_map(&vm, c.v, {dk, T, Hkv, B}, {dk, T * dk, Hkv * T * dk}, S::KT, 1);
    if (e == cudaSuccess) e = encode_map(&ktm, c.k_tree, {dk, n, Hkv, B}, {Hkv * dk, dk, n * Hkv * dk}, S::KT, 1);
    if (e == cudaSuccess) e = encode_map(&vtm, c.v_tree, {dk, n, Hkv, B}, {Hkv * dk, dk, n * Hkv * dk}, S::KT, 1);
  }
  if (e != cudaSuccess) return e;
  // one CTA an SM: it may then take tensor memory without waiting for another's
  constexpr int smem = std::max(S::ALLOC, 116 * 1024);
  e = cudaFuncSetAttribute(rows_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  rows_kernel<S><<<dim3(p.n_split, p.row_blocks, (unsigned)(B * Hkv)), S::THREADS, smem, st>>>(qm, km, vm, ktm, vtm, a);
  e = cudaPeekAtLastError();
  if (e != cudaSuccess || p.n_split == 1) return e;
  return launch_pdl(join_kernel<S::BF16>, dim3((unsigned)(B * Hkv * p.R)), dim3(std::min(128, S::DV / 4)), 0, st, a,
                    (int)S::DV);
}

template <bool BF16>
cudaError_t launch_latent(const RowsCall& c, const Plan& p, const RowsArgs& a, cudaStream_t st) {
  if (c.dv == 512) return launch_shape<Shape<BF16, 9, 8, true, 64, 64, 2, 1>>(c, p, a, st);
  return launch_shape<Shape<BF16, 5, 4, true, 64, 64, 3, 2>>(c, p, a, st);
}

}  // namespace

size_t rows_ws_bytes(const RowsCall& c) { return plan_rows(c).bytes; }

cudaError_t launch_rows_attention(const RowsCall& c, void* ws, cudaStream_t st) {
  const Plan p = plan_rows(c);
  RowsArgs a{};
  a.B = c.B;
  a.n = c.n;
  a.H = c.H;
  a.Hkv = c.Hkv;
  a.G = c.H / c.Hkv;
  a.R = p.R;
  a.n_split = p.n_split;
  a.tree = c.k_tree != nullptr;
  a.T_cap = c.T_cap;
  a.scale_log2 = c.scale * kLog2e;
  a.T_len = c.T_len;
  a.mask = c.mask;
  a.v_tree = static_cast<const uint16_t*>(c.latent ? c.k_tree : c.v_tree);
  a.v_tok = c.latent ? c.dk : (int64_t)c.Hkv * c.dv;
  a.v_head = c.latent ? 0 : c.dv;
  a.out = c.out;
  a.part_ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(ws) + p.ml_off);
  a.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + p.o_off);
  if (c.latent) return c.dtype == MKV_BF16 ? launch_latent<true>(c, p, a, st) : launch_latent<false>(c, p, a, st);
  if (c.dv == 128) return launch_shape<Shape<false, 2, 2, false, 128, 64, 2, 2>>(c, p, a, st);
  return launch_shape<Shape<false, 1, 1, false, 128, 64, 3, 2>>(c, p, a, st);
}

}  // namespace mkv
