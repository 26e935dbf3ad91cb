// Causal attention of a prompt's queries over expanded latent keys and values:
//   out_i = sum_{j <= pos_i} p_ij v_j / sum p_ij,  p_ij = 2^(scale log2(e) (q_i[:nope] . k_j + q_i[nope:] . r_j) - m_i)
// with a head's own key part k_j and value v_j (mkv_latent_expand) and the rotated part r_j that all heads share,
// which is read from the cache's rows: a key tile is assembled in shared memory from the two.
//
// Bound by the tensor cores (640 flops a pair at 192 / 128 dims against 2 exponentials' worth of special-function
// time).  A CTA takes 256 queries of one head as two blocks of 128 rows and streams 128-key tiles past both, so the
// tensor cores work on one block while the other is in its softmax:
//   S_i [128 x 128] = Q_i K^T    operands in shared memory, accumulator in tensor memory
//   O_i [128 x dv] += P_i V      P_i from tensor memory (it overwrites the S_i it came from), V from shared memory,
//                                read along its other index
// Measured: the second half of an 8K prompt, 32 heads, fp16: 336 to 348 us GPU time, 1.5 PFLOP/s, 0.76 of cuBLAS's
// rate (the tensor pipe is busy 77 % of the time); three prompts of up to 333 tokens, bf16: 21 us (masked
// tiles' latency).  A short chunk over a long history leaves SMs idle, as a block's keys are not shared out: 256 queries
// at the end of 4096 tokens, 32 heads, 60 us (a floor of 11), 8 heads 55.
// Tensor memory is full: 2 x (128 columns S / P + 128 columns O).  Warps 0..3 and 4..7 are the two softmax groups (a
// thread holds one row: its maximum and sum need no exchange), then one warp loads tiles by TMA and one issues the
// products in the order PV_0(t), QK_0(t + 1), PV_1(t), QK_1(t + 1).
//
// As in rows_attn.cu a row's maximum is raised only when a score passes it by 2^8, so O is almost never rescaled;
// statistics and accumulators are fp32, the weights are rounded once to the type the tensor cores take.
#include <algorithm>

#include "mkv_roles.cuh"
#include "mkv_rows.h"

namespace mkv {

namespace {

constexpr int kBR = 128;            // rows a block, keys a tile
constexpr float kRaise = 8.f;       // a score may pass the running maximum by this (log2) before it is raised
constexpr float kOffset = 6.f;      // weights carry 2^kOffset (fp16: full precision down to 2^-20 of the maximum)
constexpr float kNoMax = -3.402823466e+38f;   // running maximum of a row that has seen nothing: no score is below it
// Up to this maximum (log2) an unrounded product of score and scale is within a half of the rounded one.
constexpr float kFused = 16777216.f;

struct PrefillArgs {
  int n, H;
  int64_t T_max;
  float scale_log2;
  const int32_t *T_len, *q_len;
  const uint16_t* kv;               // values, for non-finite ones
  uint16_t* out;
  int rank;
  int units, group;                 // (entry, head) pairs; how many of them are worked on together
  uint32_t* status;                 // MKV_FLAG_* bits
};

template <bool BF16_, int DN_, int DV_>
struct PShape {
  static constexpr bool BF16 = BF16_;
  static constexpr int DN = DN_, DV = DV_, DK = DN + 64;
  static constexpr int KA = DK / 64, VA = DV / 64;
  static constexpr int ATOM = kBR * 128;                    // 128 rows of 64 dims
  static constexpr int QBLK = KA * ATOM;
  // Key and value atoms pass through one ring in the order K0 V0 K1 V1 .., which is the order they are done with.  What
  // shared memory holds beside the queries (8 atoms of 16 KB at 192 / 128 dims) is a tile's keys, the values of the
  // tile before it, and the next values: with a fixed pair of key stages the single value stage left was waited for
  // (a fifth of the tile time).
  static constexpr int TA = KA + VA;                        // atoms of a tile
  static constexpr int RING = (227 * 1024 - 1536 - 2 * QBLK) / ATOM;
  static_assert(RING >= TA + VA, "shared memory");
  static constexpr int Q_OFF = 0, R_OFF = 2 * QBLK;
  static constexpr int CTL_OFF = R_OFF + RING * ATOM;
  static constexpr int ALLOC = CTL_OFF + 512 + 1024;
  static_assert(ALLOC <= 227 * 1024, "shared memory");
};
// Of keys and values worked on together, so that they stay in L2 (4096 of 8192 queries, 32 heads of 4 MB each: 348 us;
// 16 MB 360, 48 MB 353, all heads at once 374)
constexpr int64_t kGroupBytes = 32 << 20;
constexpr int kBars = 4;            // tiles whose barriers are told apart: more than the ring holds
// Two softmax warpgroups, loads and products (and two idle warps); registers a thread at launch (168, what 384
// threads get) split 2 x 208 + 88.
constexpr int kPThreads = 384, kPRegsSoftmax = 208, kPRegsOther = 88;
static_assert(2 * kPRegsSoftmax + kPRegsOther <= 3 * 168, "register shares");
constexpr int kFixWords = 16;       // flags of the keys of the tiles that some row sees only in part

struct PCtl {
  uint64_t drained, qfull[2], kfull[kBars], kempty[kBars], vfull[kBars], vempty[kBars], sfull[2], pfull[2][2], pvdone[2];
  uint32_t tslot;
  int fail, k_loads, v_loads;       // tiles whose keys or values were asked for (read after a failure)
  uint32_t nonfinite[kFixWords];    // keys (from the first partial tile) whose value holds a non-finite number
};
static_assert(sizeof(PCtl) <= 512, "control block");

template <class S>
__global__ void __launch_bounds__(kPThreads, 1)
    latent_prefill_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kvmap,
                          const __grid_constant__ CUtensorMap rmap, const PrefillArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  PCtl* ctl = reinterpret_cast<PCtl*>(sm + S::CTL_OFF);
  // Launch order: groups of a.group (entry, head) units whose keys and values fit L2 together; within a group the
  // query blocks with the most keys first, so that the last blocks to start are short.
  const int nblk = (a.n + 2 * kBR - 1) / (2 * kBR);
  const int grp = (int)(blockIdx.x / ((unsigned)a.group * nblk));
  const int in = (int)(blockIdx.x - (unsigned)grp * a.group * nblk);
  const int size = std::min(a.group, a.units - grp * a.group), unit = grp * a.group + in % size;
  const int h = unit % a.H, b = unit / a.H;
  const int i0 = (nblk - 1 - in / size) * 2 * kBR;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  pdl_wait_and_trigger();                                // (from here on memory that the stream's previous kernel wrote)
  const int tl = a.T_len[b];
  const int len = (int)std::min<int64_t>(std::max(tl, 0), a.T_max);
  const int ql = a.q_len != nullptr ? std::min(std::max(a.q_len[b], 0), a.n) : a.n;
  // tokens that query i sees
  auto seen_by = [&](int i) {
    return i < ql ? (int)std::min<int64_t>(len, std::max<int64_t>(0, (int64_t)tl - ql + i + 1)) : 0;
  };
  int nt[2];                                             // tiles of each block
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int first = i0 + k * kBR, last = std::min(first + kBR, ql) - 1;
    nt[k] = last >= first ? (seen_by(last) + kBR - 1) / kBR : 0;
  }
  const int ntiles = std::max(nt[0], nt[1]);
  if (ntiles == 0) {
    const int rows = std::min(2 * kBR, a.n - i0);
    for (int e = threadIdx.x; e < rows * (S::DV / 8); e += kPThreads)
      reinterpret_cast<uint4*>(a.out + (((int64_t)b * a.n + i0 + e / (S::DV / 8)) * a.H + h) * S::DV)[e % (S::DV / 8)] =
          make_uint4(0, 0, 0, 0);
    return;
  }
  const int td = seen_by(i0) / kBR;                      // first tile that the first row does not see whole

  if (warp == 8) tc_alloc(&ctl->tslot, 512);
  if (threadIdx.x == 0) {
    for (int s = 0; s < kBars; ++s) {
      tc_mbar_init(&ctl->kfull[s], S::KA);
      tc_mbar_init(&ctl->kempty[s], 1);
      tc_mbar_init(&ctl->vfull[s], S::VA);
      tc_mbar_init(&ctl->vempty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      tc_mbar_init(&ctl->qfull[s], 1);
      tc_mbar_init(&ctl->sfull[s], 1);
      tc_mbar_init(&ctl->pfull[s][0], 4);
      tc_mbar_init(&ctl->pfull[s][1], 4);
      tc_mbar_init(&ctl->pvdone[s], 1);
    }
    tc_mbar_init(&ctl->drained, 1);
    tc_fence_mbar_init();
    ctl->fail = ctl->k_loads = ctl->v_loads = 0;
    for (int w = 0; w < kFixWords; ++w) ctl->nonfinite[w] = 0;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = ctl->tslot;
  volatile int* fail = &ctl->fail;
  uint32_t* status = a.status;

  if (warp >= 8) {
    regs_down<kPRegsOther>();
    if (warp == 8) {
      // ---------------------------------------------------------------- loads: Q0 K0 Q1 V0 K1 V1 ..
      if (elect_one()) {
        auto load_q = [&](int k) {
          tc_mbar_expect_tx(&ctl->qfull[k], S::QBLK);
          for (int at = 0; at < S::KA; ++at)
            tma_load_4d(sm + S::Q_OFF + k * S::QBLK + at * S::ATOM, &qmap, at * 64, i0 + k * kBR, h, b, &ctl->qfull[k]);
        };
        // the ring slot of atom j of tile t, free once its last atom is done with
        auto slot_for = [&](int t, int j, uint8_t*& dst) {
          const int x = t * S::TA + j, was = x - S::RING;
          dst = sm + S::R_OFF + x % S::RING * S::ATOM;
          if (was < 0) return true;
          const int pt = was / S::TA;
          return wait_or_fail(was % S::TA < S::KA ? &ctl->kempty[pt % kBars] : &ctl->vempty[pt % kBars],
                              (uint32_t)((pt / kBars) & 1), fail, status);
        };
        auto load_k = [&](int t) {
          uint64_t* bar = &ctl->kfull[t % kBars];
          for (int j = 0; j < S::KA; ++j) {
            uint8_t* dst;
            if (!slot_for(t, j, dst)) {
              if (j > 0) give_up(bar, S::KA - j);
              return false;
            }
            tc_mbar_expect_tx(bar, S::ATOM);
            if (j < S::DN / 64)
              tma_load_4d(dst, &kvmap, j * 64, t * kBR, h, b, bar);
            else
              tma_load_4d(dst, &rmap, a.rank, t * kBR, b, 0, bar);
            ctl->k_loads = t + 1;
          }
          return true;
        };
        auto load_v = [&](int t) {
          uint64_t* bar = &ctl->vfull[t % kBars];
          for (int j = 0; j < S::VA; ++j) {
            uint8_t* dst;
            if (!slot_for(t, S::KA + j, dst)) {
              if (j > 0) give_up(bar, S::VA - j);
              return false;
            }
            tc_mbar_expect_tx(bar, S::ATOM);
            tma_load_4d(dst, &kvmap, S::DN + j * 64, t * kBR, h, b, bar);
            ctl->v_loads = t + 1;
          }
          return true;
        };
        load_q(0);
        bool ok = load_k(0);
        load_q(1);
        for (int t = 0; ok && t < ntiles; ++t) {
          ok = load_v(t);
          if (ok && t + 1 < ntiles) ok = load_k(t + 1);
        }
      }
    } else if (warp == 9) {
      // ---------------------------------------------------------------- products
      if (elect_one()) {
        constexpr uint32_t idS = tc_idesc(S::BF16, kBR, kBR, false, false);
        constexpr uint32_t idO = tc_idesc(S::BF16, kBR, 64, false, true);
        const Desc qd = tc_desc_sw128(smem_addr(sm + S::Q_OFF));
        const Desc kd = tc_desc_sw128(smem_addr(sm + S::R_OFF));
        const Desc vd = tc_desc_mn<64>(smem_addr(sm + S::R_OFF), S::ATOM);
        auto wait = [&](uint64_t* bar, uint32_t parity) {
          const bool ok = wait_or_fail(bar, parity, fail, status);
          tc_fence_after();
          return ok;
        };
        auto scores = [&](int k, int t) {     // S_k of tile t
          int slot = t * S::TA % S::RING;
#pragma unroll
          for (int j = 0; j < S::KA; ++j) {
            const Desc q0 = qd.at(k * S::QBLK + j * S::ATOM).opaque(), k0 = kd.at(slot * S::ATOM).opaque();
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              tc_mma_ss(tbase + (uint32_t)(k * kBR), q0.at(kk * 32), k0.at(kk * 32), idS, j > 0 || kk > 0 ? 1u : 0u);
            if (++slot == S::RING) slot = 0;
          }
          tc_commit(&ctl->sfull[k]);
        };
        auto values = [&](int k, int t, int half) {     // O_k += P_k V over half of tile t's keys
          int slot = (t * S::TA + S::KA) % S::RING;   // (64 dims a product: a tile's value atoms need not be neighbours)
#pragma unroll
          for (int j = 0; j < S::VA; ++j) {
            const Desc v0 = vd.at(slot * S::ATOM + half * (kBR / 2) * 128).opaque();
            const uint32_t p0 = tbase + (uint32_t)(k * kBR + half * (kBR / 4));
#pragma unroll
            for (int kk = 0; kk < kBR / 32; ++kk)
              tc_mma_ts(tbase + (uint32_t)(2 * kBR + k * kBR + j * 64), p0 + (uint32_t)(kk * 8), v0.at(kk * 2048), idO,
                        t > 0 || half > 0 || kk > 0 ? 1u : 0u);
            if (++slot == S::RING) slot = 0;
          }
        };
        bool ok = wait(&ctl->kfull[0], 0);
        for (int k = 0; ok && k < 2; ++k) {
          ok = wait(&ctl->qfull[k], 0);
          if (ok && nt[k] > 0) scores(k, 0);
        }
        if (ok) tc_commit(&ctl->kempty[0]);
        for (int t = 0; ok && t < ntiles; ++t) {
          ok = wait(&ctl->vfull[t % kBars], (uint32_t)((t / kBars) & 1));
          for (int k = 0; ok && k < 2; ++k) {
            if (t < nt[k]) {
              // (the first half's weights arrive while the softmax works on the second)
              ok = wait(&ctl->pfull[k][0], (uint32_t)(t & 1));
              if (!ok) break;
              values(k, t, 0);
              ok = wait(&ctl->pfull[k][1], (uint32_t)(t & 1));
              if (!ok) break;
              values(k, t, 1);
              tc_commit(&ctl->pvdone[k]);
            }
            if (k == 1) tc_commit(&ctl->vempty[t % kBars]);
            if (k == 0 && t + 1 < ntiles) {
              ok = wait(&ctl->kfull[(t + 1) % kBars], (uint32_t)(((t + 1) / kBars) & 1));
              if (!ok) break;
            }
            if (t + 1 < nt[k]) scores(k, t + 1);
            if (k == 1 && t + 1 < ntiles) tc_commit(&ctl->kempty[(t + 1) % kBars]);
          }
        }
        tc_commit(&ctl->drained);
      }
    }
  } else {
    regs_up<kPRegsSoftmax>();
    // ---------------------------------------------------------------- softmax: group k, row 32 (warp % 4) + lane
    const int k = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tbase + lanes + (uint32_t)(k * kBR), tO = tbase + lanes + (uint32_t)(2 * kBR + k * kBR);
    const int row = (warp & 3) * 32 + lane, i = i0 + k * kBR + row;
    const int seen = seen_by(i);
    float m = kNoMax, l = 0.f;
    bool dead = false;      // this warp's waits ran out: no barrier but mbarriers joins warps here, so it just stops
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (!dead) dead = !__all_sync(0xffffffffu, wait_or_fail(bar, parity, fail, status));
      tc_fence_after();
      return !dead;
    };
    for (int t = 0; t < nt[k]; ++t) {
      if (!wait(&ctl->sfull[k], (uint32_t)(t & 1))) break;
      const int lim = t >= td ? seen - t * kBR : kBR;    // columns of the tile that this row sees
      const bool part = t >= td;                         // (a tile that some row sees only in part)
      float v[kBR];
      float mt = -INFINITY;
      auto raw_max = [&](const float(&x)[32]) {
        float a0 = fmax3(x[0], x[1], x[2]), a1 = fmax3(x[3], x[4], x[5]);
#pragma unroll
        for (int e = 6; e < 30; e += 4) {
          a0 = fmax3(a0, x[e], x[e + 1]);
          a1 = fmax3(a1, x[e + 2], x[e + 3]);
        }
        mt = fmax3(mt, fmax3(a0, x[30], x[31]), a1);
      };
#pragma unroll
      for (int c = 0; c < 4; ++c) tm_issue<32>(tS + c * 32, *reinterpret_cast<float(*)[32]>(&v[c * 32]));
#pragma unroll
      for (int c = 0; c < 4; ++c) tm_wait<32>(*reinterpret_cast<float(*)[32]>(&v[c * 32]));
      if (part) {
#pragma unroll
        for (int c = 0; c < kBR; ++c) v[c] = c < lim ? v[c] : -INFINITY;
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) raw_max(*reinterpret_cast<float(*)[32]>(&v[c * 32]));
      mt *= a.scale_log2;                                // (the scale is positive)
      if (__any_sync(0xffffffffu, mt > m + kRaise)) {
        const float nm = fmaxf(m, mt), w = ex2_approx(m - nm);
        m = nm;
        l *= w;
        if (t > 0) {
          if (!wait(&ctl->pvdone[k], (uint32_t)((t - 1) & 1))) break;
#pragma unroll 1
          for (int c = 0; c < S::DV / 32; ++c) {
            float o[32];
            tm_load<32>(tO + c * 32, o);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] *= w;
            tm_store<32>(tO + c * 32, o);
          }
        }
      }
      if (t >= td && (k == 0 || t >= nt[0])) {
        // Values that some row of the CTA does not see must not meet its zero weight (0 x NaN): slots past the
        // length become zeros; a token's non-finite values become zeros here and are added to the rows that see it
        // at the end.  Done by the first block that meets the tile, before its product.
        if (!wait(&ctl->vfull[t % kBars], (uint32_t)((t / kBars) & 1))) break;
        // (a thread's pieces of an atom are 16 rows apart, so the swizzle leaves them 2 KB apart)
        const int r0 = (threadIdx.x & 127) >> 3;
#pragma unroll 1
        for (int j = 0; j < S::VA; ++j) {
          uint8_t* atom = sm + S::R_OFF + (t * S::TA + S::KA + j) % S::RING * S::ATOM;
          uint8_t* piece = atom + mn_offset<64>(r0, threadIdx.x & 7);
          const int tail = len - t * kBR - r0;           // its rows from here on are past the length
#pragma unroll
          for (int x = 0; x < kBR; x += 16) {
            uint4* p8 = reinterpret_cast<uint4*>(piece + x * 128);
            uint4 raw = *p8;
            if (x >= tail) {
              *p8 = make_uint4(0, 0, 0, 0);
            } else if (any_non_finite<S::BF16>(raw)) {
              bad_pairs<S::BF16>(raw);
              *p8 = raw;
              const int key = (t - td) * kBR + r0 + x;
              atomicOr(&ctl->nonfinite[key >> 5], 1u << (key & 31));
            }
          }
        }
        fence_async_smem();
      }
      // A weight's exponent is one fused product and sum, score x scale - m, in which the product is not rounded but the
      // maximum it meets is: a factor that all of a row's weights share, unless the maximum is so large that its
      // rounding alone passes the exponent's range.  Then the product is rounded too, as the maximum was.
      float sc = a.scale_log2, off = kOffset - m;
      if (__any_sync(0xffffffffu, fabsf(m) > kFused && m != kNoMax)) {
#pragma unroll
        for (int c = 0; c < kBR; ++c) v[c] = __fsub_rn(__fmul_rn(v[c], sc), m);
        sc = 1.f;
        off = kOffset;
      }
      const uint64_t sc2 = pk2(sc, sc), off2 = pk2(off, off);
      uint64_t sum2[2] = {0ull, 0ull};
      // 32 scores -> 16 columns of packed weights
      auto weights = [&](const float(&x)[32], float(&pk)[16]) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float2 y = upk2(ffma2(pk2(x[2 * e], x[2 * e + 1]), sc2, off2));
          const float p0 = ex2_approx(y.x), p1 = ex2_approx(y.y);
          sum2[e & 1] = fadd2(sum2[e & 1], pk2(p0, p1));
          pk[e] = __uint_as_float(pack2<S::BF16>(p0, p1));
        }
      };
      auto hand_over = [&](int half) {
        tm_store_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) tc_mbar_arrive(&ctl->pfull[k][half]);
      };
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float pk[16];
        weights(*reinterpret_cast<float(*)[32]>(&v[c * 32]), pk);
        tm_store<16>(tS + c * 16, pk);
        if (c & 1) hand_over(c >> 1);
      }
      const float2 s0 = upk2(sum2[0]), s1 = upk2(sum2[1]);
      l += (s0.x + s0.y) + (s1.x + s1.y);
    }
    // ---------------------------------------------------------------- output
    // the other block's last tile may hold values zeroed for this one: its flags are complete once both are done
    if (nt[k] > 0) wait(&ctl->pvdone[k], (uint32_t)((nt[k] - 1) & 1));
    if (!dead) {
      // zeros for a row that sees nothing; NaN for one whose scores are all minus infinity
      const float inv = seen <= 0 ? 0.f : l == 0.f ? NAN : 1.f / l;
      uint16_t* dst = a.out + (((int64_t)b * a.n + i) * a.H + h) * S::DV;
      uint32_t any = 0;
      for (int w = 0; w < kFixWords; ++w) any |= ctl->nonfinite[w];
#pragma unroll 1
      for (int c = 0; c < S::DV / 32; ++c) {
        float o[32];
        if (nt[k] > 0) {
          tm_load<32>(tO + c * 32, o);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
        }
        if (any != 0) {                      // the non-finite values that this row sees
          for (int key = td * kBR; key < seen; ++key) {
            const int f = key - td * kBR;
            if (!(ctl->nonfinite[f >> 5] >> (f & 31) & 1)) continue;
            const uint16_t* y = a.kv + (((int64_t)b * a.H + h) * a.T_max + key) * (S::DN + S::DV) + S::DN + c * 32;
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] += non_finite<S::BF16>(y[e]) ? widen<S::BF16>(y[e]) : 0.f;
          }
        }
        if (i < a.n) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint4 x;
            x.x = pack2<S::BF16>(inv == 0.f ? 0.f : o[8 * e] * inv, inv == 0.f ? 0.f : o[8 * e + 1] * inv);
            x.y = pack2<S::BF16>(inv == 0.f ? 0.f : o[8 * e + 2] * inv, inv == 0.f ? 0.f : o[8 * e + 3] * inv);
            x.z = pack2<S::BF16>(inv == 0.f ? 0.f : o[8 * e + 4] * inv, inv == 0.f ? 0.f : o[8 * e + 5] * inv);
            x.w = pack2<S::BF16>(inv == 0.f ? 0.f : o[8 * e + 6] * inv, inv == 0.f ? 0.f : o[8 * e + 7] * inv);
            reinterpret_cast<uint4*>(dst + c * 32)[e] = x;
          }
        }
      }
    }
  }
  // teardown: the products issued are complete; after a failure so are the copies (each wait bounded)
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0) {
    tc_mbar_wait(&ctl->drained, 0, kRoleWaitNs);
    if (ctl->fail) {
      tc_mbar_wait(&ctl->qfull[0], 0, kRoleWaitNs);
      tc_mbar_wait(&ctl->qfull[1], 0, kRoleWaitNs);
      for (int t = std::max(0, ctl->k_loads - kBars); t < ctl->k_loads; ++t)
        tc_mbar_wait(&ctl->kfull[t % kBars], (uint32_t)((t / kBars) & 1), kRoleWaitNs);
      for (int t = std::max(0, ctl->v_loads - kBars); t < ctl->v_loads; ++t)
        tc_mbar_wait(&ctl->vfull[t % kBars], (uint32_t)((t / kBars) & 1), kRoleWaitNs);
    }
  }
  __syncthreads();
  tc_fence_after();
  if (warp == 8) tc_dealloc(tbase, 512);
}

template <class S>
cudaError_t launch_shape(const PrefillCall& c, PrefillArgs a, cudaStream_t st) {
  CUtensorMap qm, kvm, rm;
  const int64_t dk = S::DK, n = c.n, H = c.H, B = c.B, d = S::DN + S::DV, T = c.T_max, row = c.rank + c.rope;
  cudaError_t e = encode_map(&qm, c.q, {dk, n, H, B}, {H * dk, dk, n * H * dk}, kBR, 1);
  if (e == cudaSuccess) e = encode_map(&kvm, c.kv, {d, T, H, B}, {d, T * d, H * T * d}, kBR, 1);
  if (e == cudaSuccess)
    e = encode_map(&rm, c.rows, {row, c.T_cap, B, 1}, {row, c.T_cap * row, B * c.T_cap * row}, kBR, 1);
  if (e != cudaSuccess) return e;
  a.units = c.B * c.H;
  a.group = (int)std::max<int64_t>(1, std::min<int64_t>(a.units, kGroupBytes / (T * d * 2)));
  const int64_t grid = ceil_div(n, 2 * kBR) * a.units;
  if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
  constexpr int smem = std::max(S::ALLOC, 116 * 1024);      // one CTA an SM: it takes all of the tensor memory
  e = cudaFuncSetAttribute(latent_prefill_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_pdl(latent_prefill_kernel<S>, dim3((unsigned)grid), dim3(kPThreads), smem, st, qm, kvm, rm, a);
}

template <bool BF16>
cudaError_t launch_t(const PrefillCall& c, const PrefillArgs& a, cudaStream_t st) {
  if (c.nope == 128 && c.v_dim == 128) return launch_shape<PShape<BF16, 128, 128>>(c, a, st);
  if (c.nope == 128) return launch_shape<PShape<BF16, 128, 64>>(c, a, st);
  if (c.v_dim == 128) return launch_shape<PShape<BF16, 64, 128>>(c, a, st);
  return launch_shape<PShape<BF16, 64, 64>>(c, a, st);
}

}  // namespace

cudaError_t launch_latent_prefill(const PrefillCall& c, cudaStream_t st) {
  PrefillArgs a{};
  const cudaError_t e = status_word(&a.status);
  if (e != cudaSuccess) return e;
  a.n = c.n;
  a.H = c.H;
  a.T_max = c.T_max;
  a.scale_log2 = c.scale * kLog2e;
  a.T_len = c.T_len;
  a.q_len = c.q_len;
  a.kv = static_cast<const uint16_t*>(c.kv);
  a.out = static_cast<uint16_t*>(c.out);
  a.rank = c.rank;
  return c.dtype == MKV_BF16 ? launch_t<true>(c, a, st) : launch_t<false>(c, a, st);
}

}  // namespace mkv
