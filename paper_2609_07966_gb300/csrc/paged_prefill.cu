// Attention of an entry's newest tokens over its 8-bit pages where more than 32 query rows share a key head: prompts, their
// next chunks, many drafted tokens.  The formula, and the two running maxima, are those of paged_decode.cu.
//
// Bound by the tensor cores.  A CTA takes 256 rows of a key head (tokens x heads of the group, so that grouped heads share
// every converted key) as two blocks of 128 and streams 128-token tiles past both: the tensor cores work on one block while
// the other is in its softmax.
//   S_i [128 x 128] = Q_i K^T    fp16 operands in shared memory, accumulator in tensor memory
//   O_i [128 x D]  += W_i V      W_i (the weights, fp16) from tensor memory, over the S_i they came from
// The tensor cores have no product of 16-bit queries with 8-bit codes, so one warpgroup widens every tile's codes to fp16
// (exactly) on their way into shared memory: plain 16-byte loads, eight of the next operand always under way, then the
// swizzled layout that the products read.  Once a tile serves 256 rows its conversion is an eighth of the products' time.
//
// A tile's pages have scales of their own: within 16 columns both are constant, so a score's is part of the factor of its
// exponent, the maxima are kept per 16 columns until they are scaled, and a weight is p vs 2^(m - m2 + 6).
//
// With fewer units (256 rows of a key head) than SMs, the tokens of each are shared out too and join_kernel adds the parts up.
#include <math.h>

#include <algorithm>

#include "mkv_paged.cuh"

namespace mkv {

namespace {

constexpr int kBR = 128;            // rows a block, tokens a tile
constexpr int kRows = 2 * kBR;      // rows a unit
// Up to this maximum (log2) an unrounded product of score and scale is within a half of the rounded one.
constexpr float kFused = 16777216.f;
constexpr int kThreads = 512;       // two softmax warpgroups, one that converts, one whose first warp issues products
constexpr int kRegsSoftmax = 192, kRegsConvert = 80, kRegsIssue = 48;
static_assert(2 * kRegsSoftmax + kRegsConvert + kRegsIssue <= 4 * 128, "register shares");
constexpr int kScales = 4;          // tiles whose scales are held

struct PrefillArgs {
  PagedAttnCall c;
  uint32_t* status;
  int G;
  float scale_log2;
  int64_t slots;                    // units of all entries, a key head's
  int per;                          // start null: units of an entry
  int splits;                       // parts of a unit's tokens
  float* part_o;                    // [slot][Hkv][splits][256][D]
  float4* part_st;                  // the same without D: m, sum, m2
};

template <int FMT_, int D_>
struct PShape {
  static constexpr int FMT = FMT_, D = D_, KA = D / 64;
  static constexpr int ATOM = kBR * 128, TILE = KA * ATOM, QBLK = TILE;
  static constexpr int Q_OFF = 0, R_OFF = 2 * QBLK;        // ring: K, V of even tiles, then of odd ones
  static constexpr int SC_OFF = R_OFF + 4 * TILE;          // [kScales][8] float4: key factor, vs mantissa, exponent, seen
  static constexpr int QS_OFF = SC_OFF + kScales * 8 * 16; // [256] floats
  static constexpr int CTL_OFF = QS_OFF + kRows * 4;
  static constexpr int ALLOC = CTL_OFF + 256 + 1024;
  static_assert(ALLOC <= 227 * 1024, "shared memory");
};

struct PCtl {
  uint64_t qfull, drained, kfull[2], kempty[2], vfull[2], vempty[2], sfull[2], pfull[2][2], pvdone[2];
  uint32_t tslot;
  int fail;
};
static_assert(sizeof(PCtl) <= 256, "control block");

// Units lie entry after entry, enough of them for each entry's rows.
__device__ __forceinline__ int64_t unit_base(const PrefillArgs& a, int b) {
  if (a.c.s.start == nullptr) return (int64_t)b * a.per;
  return (min(max((int64_t)a.c.s.start[b], (int64_t)0), a.c.s.n) * a.G + (int64_t)b * (kRows - 1)) / kRows;
}
struct Unit {
  int b, kvh, rb, rows, G, len;    // rows of the entry (tokens x G)
  int64_t row0;                    // its first token's row
  bool live;
  __device__ __forceinline__ int pos(int row) const { return len - rows / G + row / G; }   // a row's position
  // tokens that a row sees
  __device__ __forceinline__ int seen(int row) const { return row < rows ? max(0, min(len, pos(row) + 1)) : 0; }
  // tiles of block k: at least one where it has rows, so that they are written
  __device__ __forceinline__ int tiles(int k) const {
    const int first = rb * kRows + k * kBR, last = min(first + kBR, rows) - 1;
    return last >= first ? max(1, (seen(last) + kBR - 1) / kBR) : 0;
  }
};
__device__ __forceinline__ Unit unit_of(const PrefillArgs& a, int64_t slot, int kvh, int lane, bool report) {
  Unit u;
  u.b = a.c.s.start == nullptr ? (int)(slot / a.per)
                               : find_entry(a.c.s.B, lane, [&](int b) { return unit_base(a, b) <= slot; });
  u.kvh = kvh;
  u.G = a.G;
  u.rb = (int)(slot - unit_base(a, u.b));
  const EntryRows r = entry_rows(a.c.s, u.b);
  u.row0 = r.first;
  u.live = r.count <= a.c.max_rows;
  if (!u.live && report && u.rb == 0 && kvh == 0) atomicOr(a.status, MKV_FLAG_BAD_INDEX);
  u.rows = (int)min(r.count, a.c.max_rows) * a.G;
  u.live = u.live && u.rb >= 0 && (int64_t)u.rb * kRows < u.rows;
  u.len = (int)min((int64_t)max(a.c.T_len[u.b], 0), a.c.s.max_pages * a.c.s.page);
  return u;
}

__device__ __forceinline__ uint64_t fmul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

template <class S, bool BF16>
__global__ void __launch_bounds__(kThreads, 1) prefill_kernel(const PrefillArgs a) {
  constexpr int D = S::D;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  PCtl* ctl = reinterpret_cast<PCtl*>(sm + S::CTL_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PagedAttnCall& c = a.c;
  const int Hkv = c.s.Hkv, page = c.s.page;

  pdl_wait_and_trigger();
  // Launch order: the last rows of the entries first (they see the most), all key heads and parts of a slot together.
  const int64_t each = (int64_t)Hkv * a.splits, at = blockIdx.x / each;
  const int in = (int)(blockIdx.x - at * each), split = in / Hkv;
  const int64_t slot = a.slots - 1 - at;
  const Unit u = unit_of(a, slot, in % Hkv, lane, true);
  if (!u.live) return;
  const int all0 = u.tiles(0), all1 = u.tiles(1), all = max(all0, all1);
  const int c0 = (int)((int64_t)all * split / a.splits), c1 = (int)((int64_t)all * (split + 1) / a.splits);
  const int nt[2] = {max(0, min(all0, c1) - c0), max(0, min(all1, c1) - c0)};   // tiles of each block here
  const int ntiles = c1 - c0;
  const int base_row = u.rb * kRows;
  const int64_t part = ((slot * Hkv + u.kvh) * a.splits + split) * kRows;
  if (ntiles == 0) {                                       // (fewer tiles than parts)
    for (int r = threadIdx.x; r < kRows; r += kThreads) a.part_st[part + r] = make_float4(kNoMax, 0.f, kNoMax, 0.f);
    return;
  }

  if (warp == 12) tc_alloc(&ctl->tslot, 512);
  if (threadIdx.x == 0) {
    tc_mbar_init(&ctl->qfull, 8);
    tc_mbar_init(&ctl->drained, 1);
    for (int s = 0; s < 2; ++s) {
      tc_mbar_init(&ctl->kfull[s], 4);
      tc_mbar_init(&ctl->vfull[s], 4);
      tc_mbar_init(&ctl->kempty[s], 1);
      tc_mbar_init(&ctl->vempty[s], 1);
      tc_mbar_init(&ctl->sfull[s], 1);
      tc_mbar_init(&ctl->pfull[s][0], 4);
      tc_mbar_init(&ctl->pfull[s][1], 4);
      tc_mbar_init(&ctl->pvdone[s], 1);
    }
    tc_fence_mbar_init();
    ctl->fail = 0;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = ctl->tslot;
  volatile int* fail = &ctl->fail;
  uint32_t* status = a.status;

  if (warp >= 12) {
    regs_down<kRegsIssue>();
    if (warp == 12 && elect_one()) {
      // ---------------------------------------------------------------- products
      constexpr uint32_t idS = tc_idesc(false, kBR, kBR, false, false);
      constexpr uint32_t idO = tc_idesc(false, kBR, D, false, true);
      const Desc qd = tc_desc_sw128(smem_addr(sm + S::Q_OFF));
      const Desc kd = tc_desc_sw128(smem_addr(sm + S::R_OFF));
      const Desc vd = tc_desc_mn<64>(smem_addr(sm + S::R_OFF), S::ATOM);
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        const bool ok = wait_or_fail(bar, parity, fail, status);
        tc_fence_after();
        return ok;
      };
      auto scores = [&](int k, int t) {
        const Desc q0 = qd.at(k * S::QBLK).opaque(), k0 = kd.at((t & 1) * 2 * S::TILE).opaque();
#pragma unroll
        for (int j = 0; j < S::KA * 4; ++j)
          tc_mma_ss(tbase + (uint32_t)(k * kBR), q0.at((j >> 2) * S::ATOM + (j & 3) * 32),
                    k0.at((j >> 2) * S::ATOM + (j & 3) * 32), idS, j > 0 ? 1u : 0u);
        tc_commit(&ctl->sfull[k]);
      };
      auto values = [&](int k, int t, int half) {           // over half of tile t's tokens
        const Desc v0 = vd.at(((t & 1) * 2 + 1) * S::TILE + half * (kBR / 2) * 128).opaque();
        const uint32_t p0 = tbase + (uint32_t)(k * kBR + half * (kBR / 4));
#pragma unroll
        for (int kk = 0; kk < kBR / 32; ++kk)
          tc_mma_ts(tbase + (uint32_t)(2 * kBR + k * kBR), p0 + (uint32_t)(kk * 8), v0.at(kk * 2048), idO,
                    t > 0 || half > 0 || kk > 0 ? 1u : 0u);
      };
      bool ok = wait(&ctl->qfull, 0) && wait(&ctl->kfull[0], 0);
      if (ok) {
        for (int k = 0; k < 2; ++k)
          if (nt[k] > 0) scores(k, 0);
        tc_commit(&ctl->kempty[0]);
      }
      for (int t = 0; ok && t < ntiles; ++t) {
        ok = wait(&ctl->vfull[t & 1], (uint32_t)((t >> 1) & 1));
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
          if (k == 1) tc_commit(&ctl->vempty[t & 1]);
          if (k == 0 && t + 1 < ntiles) {
            ok = wait(&ctl->kfull[(t + 1) & 1], (uint32_t)(((t + 1) >> 1) & 1));
            if (!ok) break;
          }
          if (t + 1 < nt[k]) scores(k, t + 1);
          if (k == 1 && t + 1 < ntiles) tc_commit(&ctl->kempty[(t + 1) & 1]);
        }
      }
      tc_commit(&ctl->drained);
    }
  } else if (warp >= 8) {
    regs_down<kRegsConvert>();
    // ---------------------------------------------------------------- codes to fp16
    // A thread takes one 16-byte piece of STEP rows a tile, rows ROWS apart; eight neighbouring threads two rows of four
    // pieces, so that their stores meet different banks.
    constexpr int ROWS = D == 128 ? 16 : 32, STEP = kBR / ROWS;
    const int tid = threadIdx.x - 256;
    const int piece = D == 128 ? (tid & 3) | (tid >> 3 & 1) << 2 : tid & 3;
    const int row = D == 128 ? (tid >> 4) * 2 + (tid >> 2 & 1) : tid >> 2;
    const int32_t* table = c.s.page_table + (int64_t)u.b * c.s.max_pages;
    // lane g < 8: page of tokens 16 g .. of a tile, -1 where there is none
    auto fetch = [&](int t) {
      const int64_t tok = (int64_t)(c0 + t) * kBR + 16 * lane;
      return lane < 8 && t < ntiles && tok < u.len ? table[tok / page] : -1;
    };
    auto check = [&](int t, int pid) {
      const int64_t tok = (int64_t)(c0 + t) * kBR + 16 * lane;
      if (!(lane < 8 && t < ntiles && tok < u.len)) return -1;
      if (pid >= 0 && pid < c.s.num_pages) return pid;
      atomicOr(status, MKV_FLAG_BAD_INDEX);
      return -1;
    };
    // its codes' offset (page and head; -1: none)
    auto offset = [&](int t, int pid) {
      const int64_t tok = (int64_t)(c0 + t) * kBR + 16 * lane;
      return pid < 0 ? (int64_t)-1 : (((int64_t)pid * Hkv + u.kvh) * page + tok % page) * D;
    };
    uint4 x[STEP];
    auto load = [&](int i, int64_t off, const uint8_t* codes) {
      const int64_t o = __shfl_sync(0xffffffffu, off, D == 128 ? i : 2 * i + (row >> 4));
      x[i] = o < 0 ? make_uint4(0, 0, 0, 0)
                   : __ldg(reinterpret_cast<const uint4*>(codes + o + (row & 15) * D + piece * 16));
    };
    auto store = [&](int i, uint8_t* tile, bool zero) {
      const uint32_t w[4] = {zero ? 0u : x[i].x, zero ? 0u : x[i].y, zero ? 0u : x[i].z, zero ? 0u : x[i].w};
      uint32_t e[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) widen_codes<S::FMT>(w[k], e[2 * k], e[2 * k + 1]);
      const int r = i * ROWS + row;
      uint8_t* atom = tile + (piece >> 2) * S::ATOM;
      *reinterpret_cast<uint4*>(atom + mn_offset<64>(r, 2 * (piece & 3))) = make_uint4(e[0], e[1], e[2], e[3]);
      *reinterpret_cast<uint4*>(atom + mn_offset<64>(r, 2 * (piece & 3) + 1)) = make_uint4(e[4], e[5], e[6], e[7]);
    };
    auto hand_over = [&](uint64_t* bar) {
      fence_async_smem();
      __syncwarp();
      if (lane == 0) tc_mbar_arrive(bar);
    };
    int pid = check(0, fetch(0));
    int64_t off = offset(0, pid);
#pragma unroll
    for (int i = 0; i < STEP; ++i) load(i, off, c.k);
    bool ok = true;
    for (int t = 0; ok && t < ntiles; ++t) {
      const int s = t & 1;
      uint8_t* tile = sm + S::R_OFF + s * 2 * S::TILE;
      float ks = 0.f, vs = 1.f;
      if (warp == 8 && pid >= 0) {
        ks = c.k_scale[(int64_t)pid * Hkv + u.kvh];
        vs = c.v_scale[(int64_t)pid * Hkv + u.kvh];
      }
      const int next = fetch(t + 1);
      if (t > 1) ok = __all_sync(0xffffffffu, wait_or_fail(&ctl->kempty[s], (uint32_t)(((t >> 1) - 1) & 1), fail, status));
      if (!ok) break;
#pragma unroll
      for (int i = 0; i < STEP; ++i) {
        store(i, tile, false);
        load(i, off, c.v);
      }
      if (warp == 8 && lane < 8) {
        int e;
        const float m = frexpf(vs, &e);
        reinterpret_cast<float4*>(sm + S::SC_OFF)[(t % kScales) * 8 + lane] =
            make_float4(ks * a.scale_log2, m, (float)e, pid >= 0 ? 1.f : 0.f);
      }
      hand_over(&ctl->kfull[s]);
      pid = check(t + 1, next);
      off = offset(t + 1, pid);
      const int tail = u.len - (c0 + t) * kBR;             // rows of the tile that exist
      if (t > 1) ok = __all_sync(0xffffffffu, wait_or_fail(&ctl->vempty[s], (uint32_t)(((t >> 1) - 1) & 1), fail, status));
      if (!ok) break;
#pragma unroll
      for (int i = 0; i < STEP; ++i) {
        // (what lies behind the length, whatever it is, must not meet a zero weight as NaN)
        store(i, tile + S::TILE, i * ROWS + row >= tail);
        load(i, off, c.k);
      }
      hand_over(&ctl->vfull[s]);
    }
  } else {
    regs_up<kRegsSoftmax>();
    const int k = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tbase + lanes + (uint32_t)(k * kBR), tO = tbase + lanes + (uint32_t)(2 * kBR + k * kBR);
    float* qs = reinterpret_cast<float*>(sm + S::QS_OFF);
    // ---------------------------------------------------------------- queries, D / 8 lanes a row
    {
      constexpr int LN = D / 8, PER = 32 / LN, U = 4;
      const int ch = lane % LN;
#pragma unroll 1
      for (int r0 = warp * PER + lane / LN; r0 < kRows; r0 += 8 * PER * U) {
        uint4 y[U];
#pragma unroll
        for (int q = 0; q < U; ++q) {
          const int row = base_row + r0 + q * 8 * PER;
          y[q] = make_uint4(0, 0, 0, 0);
          if (row < u.rows)
            y[q] = *reinterpret_cast<const uint4*>(c.q + (u.row0 + row / u.G) * c.q_stride +
                                                   (int64_t)(u.kvh * u.G + row % u.G) * D + ch * 8);
        }
#pragma unroll
        for (int q = 0; q < U; ++q) {
          const int r = r0 + q * 8 * PER;
          if (BF16) {                                      // a power of two a row (paged_decode.cu)
            float v[8], most = 0.f;
            widen8<true>(y[q], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(v[i]) < INFINITY ? fabsf(v[i]) : 0.f);
#pragma unroll
            for (int d = 1; d < LN; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
            const int e = row_exponent(most);
            const float f = power_of_two(e);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= f;
            y[q] = narrow8<false>(v);
            if (ch == 0) qs[r] = power_of_two(-e);
          }
          *reinterpret_cast<uint4*>(sm + S::Q_OFF + (r / kBR) * S::QBLK + (ch >> 3) * S::ATOM + mn_offset<64>(r % kBR, ch & 7)) =
              y[q];
        }
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) tc_mbar_arrive(&ctl->qfull);
    }
    bool dead = false;      // this warp's waits ran out: no barrier but mbarriers joins warps here, so it just stops
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (!dead) dead = !__all_sync(0xffffffffu, wait_or_fail(bar, parity, fail, status));
      tc_fence_after();
      return !dead;
    };
    // ---------------------------------------------------------------- softmax: row 32 (warp % 4) + lane of block k
    const int rin = k * kBR + (warp & 3) * 32 + lane, row = base_row + rin, seen = u.seen(row);
    const int td = u.seen(base_row) / kBR;                 // first tile that the unit's first row does not see whole
    float back = 1.f;
    if (BF16) {                                            // (all warps' queries are in place)
      wait(&ctl->qfull, 0);
      back = qs[rin];
    }
    float m = kNoMax, m2 = kNoMax, l = 0.f;
    for (int t = 0; t < nt[k]; ++t) {
      if (!wait(&ctl->sfull[k], (uint32_t)(t & 1))) break;
      const float4* sc = reinterpret_cast<const float4*>(sm + S::SC_OFF) + (t % kScales) * 8;
      float v[kBR];
#pragma unroll
      for (int i = 0; i < 4; ++i) tm_issue<32>(tS + i * 32, *reinterpret_cast<float(*)[32]>(&v[i * 32]));
#pragma unroll
      for (int i = 0; i < 4; ++i) tm_wait<32>(*reinterpret_cast<float(*)[32]>(&v[i * 32]));
      const bool holes = __any_sync(0xffffffffu, sc[lane & 7].w == 0.f);     // a page outside the pool or past the length
      if (c0 + t >= td || holes) {
        const int lim = seen - (c0 + t) * kBR;             // columns of the tile that this row sees
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const int upto = sc[g].w != 0.f ? lim : 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) v[16 * g + i] = 16 * g + i < upto ? v[16 * g + i] : -INFINITY;
        }
      }
      float mt = -INFINITY, mt2 = -INFINITY;
#pragma unroll
      for (int g = 0; g < 8; ++g) {
        const float* y = v + 16 * g;
        float x0 = fmax3(y[0], y[1], y[2]), x1 = fmax3(y[3], y[4], y[5]);
        x0 = fmax3(x0, y[6], y[7]);
        x1 = fmax3(x1, y[8], y[9]);
        x0 = fmax3(x0, y[10], y[11]);
        x1 = fmax3(x1, y[12], y[13]);
        x0 = fmax3(fmaxf(x0, x1), y[14], y[15]);
        const float4 s4 = sc[g];
        x0 *= fmaxf(s4.x * back, 1.17549435e-38f);         // (a factor of zero would make NaN of a masked score)
        mt = fmaxf(mt, x0);
        mt2 = fmaxf(mt2, x0 + s4.z);
      }
      if (__any_sync(0xffffffffu, mt > m + kRaise || mt2 > m2 + kRaise)) {
        const float nm = fmaxf(m, mt), nm2 = fmaxf(m2, mt2);
        l *= ex2_approx(m - nm);
        const float w = ex2_approx(m2 - nm2);
        m = nm;
        m2 = nm2;
        if (t > 0) {
          if (!wait(&ctl->pvdone[k], (uint32_t)((t - 1) & 1))) break;
#pragma unroll 1
          for (int i = 0; i < D / 32; ++i) {
            float o[32];
            tm_load<32>(tO + i * 32, o);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] *= w;
            tm_store<32>(tO + i * 32, o);
          }
        }
      }
      // (a maximum so large that its rounding alone passes the exponent's range: the products are rounded as it was)
      const bool plain = __any_sync(0xffffffffu, fabsf(m) > kFused && m != kNoMax);
      if (plain) {
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const float f = fmaxf(sc[g].x * back, 1.17549435e-38f);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[16 * g + i] = __fsub_rn(__fmul_rn(v[16 * g + i], f), m);
        }
      }
      const float off = plain ? 0.f : -m, up = m - m2 + kOffset;
      const uint64_t off2 = pk2(off, off);
      uint64_t sum2[2] = {0ull, 0ull};
#pragma unroll
      for (int h = 0; h < 4; ++h) {                        // 32 columns: two groups
        float pk[16];
#pragma unroll
        for (int g = 2 * h; g < 2 * h + 2; ++g) {
          const float4 s4 = sc[g];
          const float f = plain ? 1.f : fmaxf(s4.x * back, 1.17549435e-38f), w = ex2_approx(up + s4.z) * s4.y;
          const uint64_t f2 = pk2(f, f), w2 = pk2(w, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float2 y = upk2(ffma2(pk2(v[16 * g + 2 * i], v[16 * g + 2 * i + 1]), f2, off2));
            const uint64_t p = pk2(ex2_approx(y.x), ex2_approx(y.y));
            sum2[i & 1] = fadd2(sum2[i & 1], p);
            const float2 z = upk2(fmul2(p, w2));
            pk[(g & 1) * 8 + i] = __uint_as_float(pack2<false>(z.x, z.y));
          }
        }
        tm_store<16>(tS + h * 16, pk);
        if (h & 1) {
          tm_store_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) tc_mbar_arrive(&ctl->pfull[k][h >> 1]);
        }
      }
      const float2 s0 = upk2(sum2[0]), s1 = upk2(sum2[1]);
      l += (s0.x + s0.y) + (s1.x + s1.y);
    }
    // ---------------------------------------------------------------- output
    if (nt[k] > 0) wait(&ctl->pvdone[k], (uint32_t)((nt[k] - 1) & 1));
    if (!dead) {
      const bool whole = a.splits == 1;
      // zeros for a row that sees nothing; NaN for one whose scores are all minus infinity
      const float inv = seen <= 0 ? 0.f : l == 0.f ? NAN : 1.f / l, hp = half_power(m, m2);
      if (!whole) a.part_st[part + rin] = make_float4(m, l, m2, 0.f);
      uint16_t* dst = c.out + (u.row0 + row / u.G) * c.out_stride + (int64_t)(u.kvh * u.G + row % u.G) * D;
      float* po = a.part_o + (part + rin) * D;
      if (nt[k] > 0) {
#pragma unroll 1
        for (int i = 0; i < D / 32; ++i) {
          float o[32];
          tm_load<32>(tO + i * 32, o);
          if (row >= u.rows) continue;
          if (whole) {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = inv == 0.f ? 0.f : o[e] * inv * hp * hp;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              reinterpret_cast<uint4*>(dst + i * 32)[e] =
                  make_uint4(pack2<BF16>(o[8 * e], o[8 * e + 1]), pack2<BF16>(o[8 * e + 2], o[8 * e + 3]),
                             pack2<BF16>(o[8 * e + 4], o[8 * e + 5]), pack2<BF16>(o[8 * e + 6], o[8 * e + 7]));
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              reinterpret_cast<float4*>(po + i * 32)[e] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          }
        }
      }
    }
  }
  // teardown: the products issued are complete (a bounded wait)
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0) tc_mbar_wait(&ctl->drained, 0, kRoleWaitNs);
  __syncthreads();
  tc_fence_after();
  if (warp == 12) tc_dealloc(tbase, 512);
}

// out = sum_s 2^(m2_s - M2) o_s / sum_s 2^(m_s - M) l_s, a warp a row.
template <int FMT, int D, bool BF16>
__global__ void __launch_bounds__(256) join_kernel(const PrefillArgs a) {
  pdl_wait_and_trigger();
  const int lane = threadIdx.x & 31, Hkv = a.c.s.Hkv;
  const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), unit = w / kRows;
  const int rin = (int)(w - unit * kRows);
  const int64_t slot = unit / Hkv;
  const Unit u = unit_of(a, slot, (int)(unit - slot * Hkv), lane, false);
  const int row = u.rb * kRows + rin;
  if (!u.live || row >= u.rows) return;
  const int64_t part = unit * a.splits * kRows + rin;
  float mx = kNoMax, mx2 = kNoMax;
  const float4 st = lane < a.splits ? a.part_st[part + (int64_t)lane * kRows] : make_float4(kNoMax, 0.f, kNoMax, 0.f);
  mx = st.x;
  mx2 = st.z;
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    mx2 = fmaxf(mx2, __shfl_xor_sync(0xffffffffu, mx2, d));
  }
  float sum = st.y * ex2_approx(st.x - mx);
  const float w2 = ex2_approx(st.z - mx2);
#pragma unroll
  for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  // (a part that met no tile of the row's block wrote no outputs)
  const unsigned has = __ballot_sync(0xffffffffu, st.z != kNoMax);
  constexpr int VL = D / 32;
  float y[VL];
#pragma unroll
  for (int k = 0; k < VL; ++k) y[k] = 0.f;
#pragma unroll 4
  for (int s = 0; s < a.splits; ++s) {
    const float f = __shfl_sync(0xffffffffu, w2, s);
    if (!(has >> s & 1)) continue;
    const float* po = a.part_o + (part + (int64_t)s * kRows) * D + lane * VL;
#pragma unroll
    for (int k = 0; k < VL; ++k) y[k] += f * po[k];
  }
  const float inv = u.seen(row) <= 0 ? 0.f : sum == 0.f ? NAN : 1.f / sum, hp = half_power(mx, mx2);
#pragma unroll
  for (int k = 0; k < VL; ++k) y[k] = inv == 0.f ? 0.f : y[k] * inv * hp * hp;
  uint16_t* dst = a.c.out + (u.row0 + row / u.G) * a.c.out_stride + (int64_t)(u.kvh * u.G + row % u.G) * D + lane * VL;
  if constexpr (VL == 4)
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack2<BF16>(y[0], y[1]), pack2<BF16>(y[2], y[3]));
  else
    *reinterpret_cast<uint32_t*>(dst) = pack2<BF16>(y[0], y[1]);
}

// ---------------------------------------------------------------- host side
struct Plan {
  int64_t slots;
  int per, splits;
};
Plan plan_of(const PagedAttnCall& c) {
  Plan p{};
  const int64_t G = c.s.Hq / c.s.Hkv, m = ceil_div(c.s.n, c.s.B);
  p.per = (int)ceil_div(m * G, kRows);
  p.slots = c.s.start == nullptr ? (int64_t)c.s.B * p.per : (c.s.n * G + (int64_t)c.s.B * (kRows - 1)) / kRows;
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(32, kNumSMs / std::max<int64_t>(1, p.slots * c.s.Hkv)));
  return p;
}

template <class S, bool BF16>
cudaError_t launch_shape(const PrefillArgs& a, cudaStream_t st) {
  const int64_t units = a.slots * a.c.s.Hkv;
  if (units * a.splits > INT32_MAX) return cudaErrorInvalidConfiguration;
  constexpr int smem = std::max(S::ALLOC, 116 * 1024);      // one CTA an SM: it takes all of the tensor memory
  cudaError_t e = cudaFuncSetAttribute(prefill_kernel<S, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  e = launch_pdl(prefill_kernel<S, BF16>, dim3((unsigned)(units * a.splits)), dim3(kThreads), smem, st, a);
  if (e != cudaSuccess || a.splits == 1) return e;
  return launch_pdl(join_kernel<S::FMT, S::D, BF16>, dim3((unsigned)(units * (kRows / 8))), dim3(256), 0, st, a);
}
template <int FMT>
cudaError_t launch_f(const PrefillArgs& a, cudaStream_t st) {
  const bool bf16 = a.c.s.dtype == MKV_BF16;
  if (a.c.s.D == 128) return bf16 ? launch_shape<PShape<FMT, 128>, true>(a, st) : launch_shape<PShape<FMT, 128>, false>(a, st);
  return bf16 ? launch_shape<PShape<FMT, 64>, true>(a, st) : launch_shape<PShape<FMT, 64>, false>(a, st);
}

}  // namespace

size_t paged_prefill_ws_bytes(const PagedAttnCall& c) {
  // (one part an SM at most, where units have several)
  const size_t parts = kNumSMs;
  return kCounterBytes + align256(parts * kRows * sizeof(float4)) + align256(parts * kRows * c.s.D * sizeof(float));
}

cudaError_t launch_paged_prefill(const PagedAttnCall& c, void* ws, cudaStream_t st) {
  PrefillArgs a{};
  const cudaError_t e = status_word(&a.status);
  if (e != cudaSuccess) return e;
  const Plan p = plan_of(c);
  a.c = c;
  a.G = c.s.Hq / c.s.Hkv;
  a.scale_log2 = c.scale * kLog2e;
  a.slots = p.slots;
  a.per = p.per;
  a.splits = p.splits;
  uint8_t* base = static_cast<uint8_t*>(ws) + kCounterBytes;
  a.part_st = reinterpret_cast<float4*>(base);
  a.part_o = reinterpret_cast<float*>(base + align256((size_t)kNumSMs * kRows * sizeof(float4)));
  return c.s.format == MKV_E4M3 ? launch_f<MKV_E4M3>(a, st) : launch_f<MKV_I8>(a, st);
}

}  // namespace mkv
