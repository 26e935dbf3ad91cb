// Attention of an entry's newest tokens over its 8-bit pages, 9 to 128 query rows of a key head (tokens x heads of a group):
// drafted tokens, short chunks.  The formula, and the two running maxima, are those of paged_decode.cu.
//
// Bound by memory, or by shared memory, which every code passes several times: TMA writes a 128-token tile's codes, a
// warpgroup reads them, widens them to fp16 (exactly) and writes them again in the layout that the tensor cores read:
//   S [128 x 128] = Q K^T     Q from tensor memory, K from shared memory
//   O [128 x D]  += W V       W (the weights, fp16) from tensor memory, V from shared memory
// The products have 128 rows whatever the call has.  With up to 32 (64) rows the queries are there four (two) times, and copy
// c takes the tile's tokens 128 / copies c .. alone (8 x 8K: 32 rows 44 us, with two copies 53, with one 64; 64 rows 56 against
// 67): all lanes have scores to work on, a thread 32 (64) of them, each copy has
// maxima and sums of its own, its weights for the other copies' tokens are zeros that are written once, and the copies' sums
// are added up at the end of a piece.
//
// Work is shared out in runs of tiles (mkv_paged_work.cuh).  Roles: one warp finds out its CTA's and loads it (a bulk copy a
// page), four convert keys and four values (four for both took 1.4 us a tile, twice what its bytes take), one issues products,
// whichever is ready (a finished tile's second product first), four or eight do the softmax of a tile while the next one's scores are
// computed.
//
// 8 entries of 4-8K tokens, up to eight drafted each, 32 / 8 heads: 42 us, 0.37 of the copy rate (the launch, first loads and
// first tile take 8 us, the join of pieces 4); 8 x 32K, eight drafted: 0.66.  With one copy (128 rows) the softmax warps are as
// busy as shared memory: 71 us over 8 x 8K.
#include <math.h>

#include <algorithm>

#include "mkv_paged_softmax.cuh"
#include "mkv_paged_work.cuh"

namespace mkv {

namespace {

constexpr int kHeads = 8;           // tiles whose heads and scales are held
constexpr int kSlots = 4;           // widened tiles (K0 V0 K1 V1 ..; with three, conversion is part of the products' chain: 50 against 45 us)
constexpr int kGrid = kNumSMs;

struct BlockArgs {
  PagedAttnCall c;
  WorkArgs w;
  uint32_t* status;
  Heads heads;
  int* tickets;                     // [B][Hkv], zero between calls
  float* part_o;                    // [kGrid][2][ROWS][D]
  float4* part_st;                  // [kGrid][2][ROWS]: m, sum, m2
};

template <int FMT_, int D_, int COPIES_>
struct BShape {
  static constexpr int FMT = FMT_, D = D_, COPIES = COPIES_;
  static constexpr int ROWS = 128 / COPIES, COLS = 128 / COPIES;   // of a copy
  // Warpgroups: softmax, conversion of keys, of values, loads + products (two warps idle).  With one copy there are two of
  // softmax, and a row's columns are halved between the threads of two warps (32 drafted over 8 x 8K 88 -> 71 us; with four
  // copies, where a thread has 32 columns anyway, 44 -> 49).
  static constexpr int HALVES = COPIES == 1 ? 2 : 1, SW = 4 * HALVES;      // softmax warps
  static constexpr int THREADS = 32 * (SW + 12), SOFT = 32 * SW;
  // registers a thread: what a launch gets, and its split (with one copy up to 28 bytes are spilled)
  static constexpr int RL = HALVES == 2 ? 96 : 128, RS = HALVES == 2 ? 112 : 208, RC = HALVES == 2 ? 96 : 104,
                       RO = HALVES == 2 ? 64 : 96;
  static_assert(HALVES * RS + 2 * RC + RO <= (HALVES + 3) * RL, "register shares");
  static constexpr int KA = D / 64, ATOM = 128 * 128, TILE = KA * ATOM;
  static constexpr int RAW = kTokens * D, RAWS = D == 128 ? 4 : 8;
  static constexpr int OROW = 20;                          // floats between rows of the join's 16 dims
  static constexpr int T_OFF = 0;                          // [kSlots] widened tiles
  static constexpr int R_OFF = T_OFF + kSlots * TILE;      // [RAWS] codes
  static constexpr int O_OFF = R_OFF + RAWS * RAW;         // [HALVES][128][OROW] floats
  static constexpr int X_OFF = O_OFF + HALVES * 128 * OROW * 4; // [2][2][128] float2: what the halves of a row tell each other
  static constexpr int SC_OFF = X_OFF + 2 * 2 * 128 * 8;    // scales of kBatches batches
  static constexpr int HD_OFF = SC_OFF + scale_bytes(kBatches);
  static constexpr int ST_OFF = HD_OFF + kHeads * 64;      // [128] + [ROWS] float4: the lanes', the piece's
  static constexpr int CTL_OFF = ST_OFF + (128 + ROWS) * 16;
  static constexpr int ALLOC = CTL_OFF + 512 + 1024;       // slack to align the base to 1024 B
  static_assert(kHeads <= kBatches, "scales are kept");
  static_assert(ALLOC <= 227 * 1024, "shared memory");
  // tensor memory columns
  static constexpr int S = 0, O = 256, P = 384, Q = 448;
};

struct BlockCtl {
  uint64_t raw_full[8], raw_empty[8], tile_full[kSlots], tile_empty[kSlots], head[kHeads], sfull[2], pfull, pvdone, qfull, meet,
      pair[4], drained;
  uint32_t tslot;
  int fail, loads, last;
};
static_assert(sizeof(BlockCtl) <= 512, "control block");

template <class S, bool BF16>
__global__ void __launch_bounds__(S::THREADS, 1) block_kernel(const BlockArgs a) {
  constexpr int D = S::D;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  BlockCtl* ctl = reinterpret_cast<BlockCtl*>(sm + S::CTL_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PagedAttnCall& c = a.c;
  const int Hkv = c.s.Hkv;
  volatile int* fail = &ctl->fail;
  uint32_t* status = a.status;
  auto head_at = [&](int g) { return reinterpret_cast<Head*>(sm + S::HD_OFF + g % kHeads * 64); };

  if (warp == S::SW + 9) tc_alloc(&ctl->tslot, 512);
  if (threadIdx.x == S::SOFT + 256) {
    for (int s = 0; s < S::RAWS; ++s) {
      tc_mbar_init(&ctl->raw_full[s], 1);
      tc_mbar_init(&ctl->raw_empty[s], 4);
    }
    for (int s = 0; s < kSlots; ++s) {
      tc_mbar_init(&ctl->tile_full[s], 4);
      tc_mbar_init(&ctl->tile_empty[s], 1);
    }
    for (int s = 0; s < kHeads; ++s) tc_mbar_init(&ctl->head[s], 1);
    for (int s = 0; s < 2; ++s) tc_mbar_init(&ctl->sfull[s], 1);
    tc_mbar_init(&ctl->pfull, S::SW);
    tc_mbar_init(&ctl->pvdone, 1);
    tc_mbar_init(&ctl->qfull, S::SW);
    tc_mbar_init(&ctl->meet, S::SW);
    for (int w = 0; w < 4; ++w) tc_mbar_init(&ctl->pair[w], 2);
    tc_mbar_init(&ctl->drained, 1);
    tc_fence_mbar_init();
    ctl->fail = ctl->loads = 0;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait_and_trigger();
  const uint32_t tbase = ctl->tslot;
  const int all_copies = (1 << (kTokens >> a.w.log_page)) - 1;

  if (warp >= S::SW + 8) regs_down<S::RO>();
  if (warp == S::SW + 8) {
    // ---------------------------------------------------------------- loads
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      return __all_sync(0xffffffffu, wait_or_fail(bar, parity, fail, status)) != 0;
    };
    int g = 0;
    const int log_page = a.w.log_page;
    const bool ok = work_through(
        c, a.w, status, reinterpret_cast<float2*>(sm + S::SC_OFF), lane, [&](const Piece&) { return true; },
        [&](const Chunk& ch, const Piece& p, bool mine, int id, int at) {
          const uint32_t bytes = (uint32_t)(__popc(ch.copies) * D) << log_page;
          const int64_t from = ((int64_t)id * Hkv + p.kvh) * c.s.page * D;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int item = 2 * g + h, s = item % S::RAWS;
            if (item >= S::RAWS && !wait(&ctl->raw_empty[s], (uint32_t)((item / S::RAWS - 1) & 1))) return false;
            if (lane == 0) {
              tc_mbar_expect_tx(&ctl->raw_full[s], bytes);
              ctl->loads = item + 1;
            }
            __syncwarp();
            if (mine)
              bulk_load(sm + S::R_OFF + s * S::RAW + (at << log_page) * D, (h == 0 ? c.k : c.v) + from, (uint32_t)D << log_page,
                        &ctl->raw_full[s]);
          }
          return true;
        },
        [&](const Chunk& ch, const Piece& p) {
          // (its place is free: tile g's codes could only be loaded once tile g - 8 was done with)
          if (lane == 31) head_at(g)->c = ch;
          if (lane == 31) head_at(g)->p = p;
          __syncwarp();
          if (lane == 0) tc_mbar_arrive(&ctl->head[g % kHeads]);
          ++g;
        });
    if (ok) {
      // (the last head's place: the same reasoning with no codes to wait for needs the wait itself)
      const int item = 2 * g, s = item % S::RAWS;
      if ((item < S::RAWS || wait(&ctl->raw_empty[s], (uint32_t)((item / S::RAWS - 1) & 1))) && lane == 0) {
        head_at(g)->c.flags = kEnd;
        tc_mbar_arrive(&ctl->head[g % kHeads]);
      }
    }
  } else if (warp == S::SW + 9) {
    if (elect_one()) {
      // ---------------------------------------------------------------- products
      constexpr uint32_t idS = tc_idesc(false, 128, 128, false, false);
      constexpr uint32_t idO = tc_idesc(false, 128, D, false, true);
      const Desc kd = tc_desc_sw128(smem_addr(sm + S::T_OFF));
      const Desc vd = tc_desc_mn<64>(smem_addr(sm + S::T_OFF), S::ATOM);
      int ts = 0, tv = 0, pieces = 0;                      // next tile's scores, next tile's second product; pieces begun
      int flags = 0, vflags = 0;                           // of tile ts (0: not looked up yet); of tile tv
      uint64_t since = 0;
      int idle = 0;
      bool ok = true;
      while (ok) {
        if (flags == 0 && mbar_test(&ctl->head[ts % kHeads], (uint32_t)((ts / kHeads) & 1))) flags = head_at(ts)->c.flags | 16;
        if ((flags & kEnd) && tv == ts) break;
        const int ki = 2 * ts, vi = 2 * tv + 1;            // their places in the ring of widened tiles
        const bool can_v = tv < ts && mbar_test(&ctl->pfull, (uint32_t)(tv & 1)) &&
                           mbar_test(&ctl->tile_full[vi % kSlots], (uint32_t)((vi / kSlots) & 1));
        const bool can_s = flags != 0 && !(flags & kEnd) && ts <= tv + 1 && (!(flags & kFirst) || tv == ts) &&
                           (!(flags & kFirst) || mbar_test(&ctl->qfull, (uint32_t)(pieces & 1))) &&
                           mbar_test(&ctl->tile_full[ki % kSlots], (uint32_t)((ki / kSlots) & 1));
        if (can_v) {
          tc_fence_after();
          const Desc v0 = vd.at(vi % kSlots * S::TILE).opaque();
#pragma unroll
          for (int kk = 0; kk < 8; ++kk)
            tc_mma_ts(tbase + S::O, tbase + S::P + (uint32_t)(kk * 8), v0.at(kk * 2048), idO,
                      !(vflags & kFirst) || kk > 0 ? 1u : 0u);
          tc_commit(&ctl->tile_empty[vi % kSlots]);
          tc_commit(&ctl->pvdone);
          ++tv;
          vflags = head_at(tv)->c.flags;                     // (of a tile whose scores are under way, or looked up below)
        }
        if (can_s) {
          tc_fence_after();
          const Desc k0 = kd.at(ki % kSlots * S::TILE).opaque();
          const uint32_t d = tbase + S::S + (uint32_t)((ts & 1) * 128);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            tc_mma_ts(d, tbase + S::Q + (uint32_t)(kk * 8), k0.at((kk >> 2) * S::ATOM + (kk & 3) * 32), idS, kk > 0 ? 1u : 0u);
          tc_commit(&ctl->tile_empty[ki % kSlots]);
          tc_commit(&ctl->sfull[ts & 1]);
          if (flags & kFirst) ++pieces;
          if (ts == tv) vflags = flags;
          ++ts;
          flags = 0;
        }
        if (can_s || can_v) {
          idle = 0;
          continue;
        }
        // nothing is ready: a bounded wait for either, its clock read now and then
        if ((++idle & 63) == 0) {
          const uint64_t now = globaltimer_ns();
          if (idle == 64) since = now;
          if (now - since > kRoleWaitNs) {
            *fail = 1;
            atomicOr(status, MKV_FLAG_WAIT_TIMEOUT);
          }
          ok = *fail == 0;
          if (idle > (1 << 30)) idle = 128;
        }
      }
      tc_commit(&ctl->drained);
    }
  } else if (warp >= S::SW && warp < S::SW + 8) {
    if (S::RC < S::RL) regs_down<S::RC>();
    // ---------------------------------------------------------------- codes to fp16: keys (h 0), values (h 1)
    // A thread takes one 16-byte piece of every STEP'th row.  Of eight neighbouring threads four read the first half of one
    // row and four the second half of the next: different banks, and so are those of the pieces that they store, in an atom
    // each (two rows of one atom with 64 dims).
    constexpr int STEP = D == 128 ? 16 : 32;
    const int h = warp >= S::SW + 4 ? 1 : 0, tid = threadIdx.x - S::SOFT - 128 * h;
    const int piece = D == 128 ? tid & 7 : tid & 3;
    const int row = D == 128 ? (tid >> 4) * 2 + ((tid >> 2 ^ tid >> 3) & 1) : tid >> 2;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      return __all_sync(0xffffffffu, wait_or_fail(bar, parity, fail, status)) != 0;
    };
    for (int g = 0;; ++g) {
      if (!wait(&ctl->head[g % kHeads], (uint32_t)((g / kHeads) & 1))) break;
      if (head_at(g)->c.flags & kEnd) break;
      const int copies = head_at(g)->c.copies, tail = head_at(g)->p.len - head_at(g)->c.chunk * kTokens;
      const int item = 2 * g + h, rs = item % S::RAWS, s = item % kSlots;
      if (!wait(&ctl->raw_full[rs], (uint32_t)((item / S::RAWS) & 1))) break;
      if (item >= kSlots && !wait(&ctl->tile_empty[s], (uint32_t)((item / kSlots - 1) & 1))) break;
      const uint8_t* src = sm + S::R_OFF + rs * S::RAW + row * D + piece * 16;
      uint8_t* dst = sm + S::T_OFF + s * S::TILE + (piece >> 2) * S::ATOM + row * 128;
      const uint32_t c0 = (uint32_t)((2 * (piece & 3)) ^ (row & 7)) << 4;
      uint4 x[128 / STEP];
#pragma unroll
      for (int i = 0; i < 128 / STEP; ++i) x[i] = *reinterpret_cast<const uint4*>(src + i * STEP * D);
      if (h == 1 && (copies != all_copies || tail < kTokens))      // what no row sees must not meet a zero weight as NaN
#pragma unroll
        for (int i = 0; i < 128 / STEP; ++i)
          if (row + i * STEP >= tail || !(copies >> ((row + i * STEP) >> a.w.log_page) & 1)) x[i] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int i = 0; i < 128 / STEP; ++i) {
        uint32_t e[8];
        widen_codes<S::FMT>(x[i].x, e[0], e[1]);
        widen_codes<S::FMT>(x[i].y, e[2], e[3]);
        widen_codes<S::FMT>(x[i].z, e[4], e[5]);
        widen_codes<S::FMT>(x[i].w, e[6], e[7]);
        *reinterpret_cast<uint4*>(dst + i * STEP * 128 + c0) = make_uint4(e[0], e[1], e[2], e[3]);
        *reinterpret_cast<uint4*>(dst + i * STEP * 128 + (c0 ^ 16u)) = make_uint4(e[4], e[5], e[6], e[7]);
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        tc_mbar_arrive(&ctl->tile_full[s]);
        tc_mbar_arrive(&ctl->raw_empty[rs]);
      }
    }
  } else if (warp < S::SW) {
    regs_up<S::RS>();
    // ---------------------------------------------------------------- softmax: lane 32 (warp % 4) + lane, row `row` of copy
    // `copy`; a thread has the copy's columns or half of them
    constexpr int HALVES = S::HALVES, HC = S::COLS / HALVES, CW = HALVES == 2 ? 32 : HC;   // its columns; so many at a time
    constexpr int QD = D / HALVES, OD = D / 32 / HALVES;   // its dims of the queries; 32s of dims of the outputs
    const int half = warp >> 2, at = (warp & 3) * 32 + lane, copy = at / S::ROWS, row = at % S::ROWS, G = a.heads.G;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const int col0 = copy * S::COLS + half * HC;           // its first column of a tile
    const uint32_t tO = tbase + lanes + S::O, tP = tbase + lanes + S::P + (uint32_t)(col0 / 2);
    float* ob = reinterpret_cast<float*>(sm + S::O_OFF) + half * 128 * S::OROW;
    float4* stat = reinterpret_cast<float4*>(sm + S::ST_OFF);
    float4* fin = stat + 128;
    bool dead = false;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (!dead) dead = !__all_sync(0xffffffffu, wait_or_fail(bar, parity, fail, status));
      tc_fence_after();
    };
    // (barriers of the softmax warps, and of the two that share rows, whose waits are bounded too)
    uint32_t met = 0, paired = 0;
    auto meet = [&]() {
      __syncwarp();
      if (lane == 0) tc_mbar_arrive(&ctl->meet);
      wait(&ctl->meet, met);
      met ^= 1;
    };
    auto exchange = [&](float2 x) {                        // with the thread that has the row's other columns, if there is one
      if (HALVES == 1) return x;
      float2* tell = reinterpret_cast<float2*>(sm + S::X_OFF) + paired * 256;
      tell[half * 128 + at] = x;
      __syncwarp();
      if (lane == 0) tc_mbar_arrive(&ctl->pair[warp & 3]);
      wait(&ctl->pair[warp & 3], paired);
      paired ^= 1;
      return tell[(1 - half) * 128 + at];
    };
    // An output is o / sum 2^(m2 - m - 6); zeros for a row before position 0, which sees nothing; NaN where no score leaves a
    // weight.
    auto store_out = [&](const Piece& h, int r, int d, float4 x, float mm, float sum, float mm2) {
      const float f = half_power(mm, mm2), inv = sum == 0.f ? NAN : 1.f / sum;
      x = make_float4(x.x * inv * f * f, x.y * inv * f * f, x.z * inv * f * f, x.w * inv * f * f);
      if (h.len - h.tokens + a.heads.token(r) < 0) x = make_float4(0.f, 0.f, 0.f, 0.f);
      uint16_t* dst = c.out + (int64_t)(h.row0 + a.heads.token(r)) * c.out_stride + (int64_t)(h.kvh * G + a.heads.head(r)) * D + d;
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack2<BF16>(x.x, x.y), pack2<BF16>(x.z, x.w));
    };
    // A piece was handed in and the unit's ticket taken (by thread 0, which looks at it only here): the CTA that took the
    // unit's last one adds the pieces up.
    Piece owed;
    owed.count = 0;
    int ticket = 0;
    auto settle = [&]() {
      if (owed.count == 0 || dead) return;
      if (threadIdx.x == 0) {
        ctl->last = ticket == owed.count - 1;
        if (ctl->last) a.tickets[owed.unit] = 0;
      }
      meet();
      if (dead) return;
      if (ctl->last) {
        const int R = owed.tokens * G;
        if (half == 0 && at < R) {                         // a row a thread: what its pieces' statistics come to
          float mx = kNoMax, mx2 = kNoMax, sum = 0.f;
#pragma unroll 4
          for (int i = 0; i < owed.count; ++i) {
            const float4 st = __ldcg(a.part_st + (int64_t)owed.place(i) * S::ROWS + at);
            const float nm = fmaxf(mx, st.x);
            sum = sum * ex2_approx(mx - nm) + st.y * ex2_approx(st.x - nm);
            mx = nm;
            mx2 = fmaxf(mx2, st.z);
          }
          fin[at] = make_float4(mx, sum, mx2, 0.f);
        }
        meet();
        if (dead) return;
        constexpr int U = 8 / S::HALVES;                   // (so many rows' loads under way together)
#pragma unroll 1
        for (int e0 = threadIdx.x; e0 < R * (D / 4); e0 += U * S::SOFT) {   // four dims of a row
          float4 y[U];
#pragma unroll
          for (int k = 0; k < U; ++k) y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
          for (int i = 0; i < owed.count; ++i) {
            float f[U];
            float4 z[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
              const int e = min(e0 + k * S::SOFT, R * (D / 4) - 1);
              const int64_t p = (int64_t)owed.place(i) * S::ROWS + e / (D / 4);
              f[k] = __ldcg(a.part_st + p).z - fin[e / (D / 4)].z;
              z[k] = __ldcg(reinterpret_cast<const float4*>(a.part_o + p * D + e % (D / 4) * 4));
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
              const float w = ex2_approx(f[k]);
              y[k] = make_float4(y[k].x + w * z[k].x, y[k].y + w * z[k].y, y[k].z + w * z[k].z, y[k].w + w * z[k].w);
            }
          }
#pragma unroll
          for (int k = 0; k < U; ++k) {
            const int e = e0 + k * S::SOFT;
            if (e < R * (D / 4)) {
              const float4 all = fin[e / (D / 4)];
              store_out(owed, e / (D / 4), e % (D / 4) * 4, y[k], all.x, all.y, all.z);
            }
          }
        }
      }
      meet();                                              // (before `last` and `fin` are set again)
      owed.count = 0;
    };
    if (S::COPIES > 1) {                                   // the weights that stay zero
      float z[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] = 0.f;
      if (half == 0) {
        for (int i = 0; i < 4; ++i) tm_store<16>(tbase + lanes + S::P + (uint32_t)(16 * i), z);
        tm_store_wait();
      }
      meet();
    }

    const int log_group = a.w.log_page - 4;
    float m = kNoMax, m2 = kNoMax, l = 0.f, back = 1.f;
    int own = 0, pos0 = 0;                                 // this row's own position, the last that it sees; the first row's
    Piece hd;
    hd.tokens = 0;
    for (int g = 0; !dead; ++g) {
      wait(&ctl->head[g % kHeads], (uint32_t)((g / kHeads) & 1));
      if (dead) break;
      const Chunk now = head_at(g)->c;
      if (now.flags & kEnd) break;
      if (now.flags & kFirst) {
        hd = head_at(g)->p;
        // ---------------------------------------------------------- queries to tensor memory (the earlier piece's are read)
        float q[QD / 2];
        const uint4* src = reinterpret_cast<const uint4*>(c.q + (int64_t)(hd.row0 + a.heads.token(row)) * c.q_stride +
                                                          (int64_t)(hd.kvh * G + a.heads.head(row)) * D + half * QD);
#pragma unroll
        for (int i = 0; i < QD / 8; ++i) {
          const uint4 y = row < hd.tokens * G ? src[i] : make_uint4(0u, 0u, 0u, 0u);
          q[4 * i] = __uint_as_float(y.x);
          q[4 * i + 1] = __uint_as_float(y.y);
          q[4 * i + 2] = __uint_as_float(y.z);
          q[4 * i + 3] = __uint_as_float(y.w);
        }
        if (BF16) {
          float most = 0.f;
#pragma unroll
          for (int i = 0; i < QD / 2; ++i) {
            const uint32_t y = __float_as_uint(q[i]);
            const float x0 = fabsf(widen<true>((uint16_t)y)), x1 = fabsf(widen<true>((uint16_t)(y >> 16)));
            most = fmax3(most, x0 < INFINITY ? x0 : 0.f, x1 < INFINITY ? x1 : 0.f);
          }
          most = fmaxf(most, exchange(make_float2(most, 0.f)).x);
          const int e = row_exponent(most);
          const float f = power_of_two(e);
          back = power_of_two(-e);
#pragma unroll
          for (int i = 0; i < QD / 2; ++i) {
            const uint32_t y = __float_as_uint(q[i]);
            q[i] = __uint_as_float(pack2<false>(widen<true>((uint16_t)y) * f, widen<true>((uint16_t)(y >> 16)) * f));
          }
        }
        constexpr int QW = QD / 2 < 32 ? QD / 2 : 32;
#pragma unroll
        for (int i = 0; i < QD / 2 / QW; ++i)
          tm_store<QW>(tbase + lanes + S::Q + (uint32_t)(half * (QD / 2) + QW * i), *reinterpret_cast<float(*)[QW]>(&q[QW * i]));
        tm_store_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) tc_mbar_arrive(&ctl->qfull);
        m = m2 = kNoMax;
        l = 0.f;
        pos0 = hd.len - hd.tokens;
        own = pos0 + a.heads.token(row);
      }
      const float2* scales = reinterpret_cast<const float2*>(sm + S::SC_OFF) + now.scales;
      wait(&ctl->sfull[g & 1], (uint32_t)((g >> 1) & 1));
      if (dead) break;
      const uint32_t tS = tbase + lanes + S::S + (uint32_t)((g & 1) * 128 + col0);
      const bool part = now.copies != all_copies || (now.chunk + 1) * kTokens > pos0 + 1;
      const int lim = own + 1 - now.chunk * kTokens - col0;       // this thread's columns that its row sees
      // CW columns' scores, those that the row does not see minus infinity
      auto load = [&](int i, float (&v)[CW]) {
#pragma unroll
        for (int k = 0; k < CW / 32; ++k) tm_issue<32>(tS + (uint32_t)(CW * i + 32 * k), *reinterpret_cast<float(*)[32]>(&v[32 * k]));
#pragma unroll
        for (int k = 0; k < CW / 32; ++k) tm_wait<32>(*reinterpret_cast<float(*)[32]>(&v[32 * k]));
        if (part) {
#pragma unroll
          for (int g16 = 0; g16 < CW / 16; ++g16) {
            const int upto = now.copies >> ((col0 / 16 + CW / 16 * i + g16) >> log_group) & 1 ? lim - CW * i : 0;
#pragma unroll
            for (int e = 16 * g16; e < 16 * g16 + 16; ++e) v[e] = e < upto ? v[e] : -INFINITY;
          }
        }
      };
      auto scale_of = [&](int i, int g16) { return scales[(col0 / 16 + CW / 16 * i + g16) >> log_group]; };
      float mt = -INFINITY, mt2 = -INFINITY, v[CW];
#pragma unroll 1
      for (int i = 0; i < HC / CW; ++i) {
        load(i, v);
        columns_max<CW, 16, BF16>(v, back, [&](int g16) { return scale_of(i, g16); }, mt, mt2);
      }
      const float2 other = exchange(make_float2(mt, mt2));
      mt = fmaxf(mt, other.x);
      mt2 = fmaxf(mt2, other.y);
      const bool raise = __any_sync(0xffffffffu, mt > m + kRaise || mt2 > m2 + kRaise);
      float w = 1.f;
      if (raise) {
        const float nm = fmaxf(m, mt), nm2 = fmaxf(m2, mt2);
        l *= ex2_approx(m - nm);
        w = ex2_approx(m2 - nm2);
        m = nm;
        m2 = nm2;
      }
      // (columns that fit the registers are still there, and their weights need not wait)
      float pk[CW / 2];
      auto weights = [&](int i) {
        columns_weights<CW, 16, BF16>(v, part, m, m2, back, [&](int g16) { return scale_of(i, g16); }, l, pk);
      };
      if (HC == CW) weights(0);
      // (the tile before this one's weights have been read, and its product added)
      if (g > 0) wait(&ctl->pvdone, (uint32_t)((g - 1) & 1));
      if (dead) break;
      if (raise && !(now.flags & kFirst)) {
#pragma unroll 1
        for (int i = half * OD; i < (half + 1) * OD; ++i) {
          float o[32];
          tm_load<32>(tO + i * 32, o);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] *= w;
          tm_store<32>(tO + i * 32, o);
        }
      }
#pragma unroll 1
      for (int i = 0; i < HC / CW; ++i) {
        if (HC > CW) {
          load(i, v);
          weights(i);
        }
        tm_store<CW / 2>(tP + (uint32_t)(CW / 2 * i), pk);
      }
      tm_store_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) tc_mbar_arrive(&ctl->pfull);
      if (!(now.flags & kLast)) continue;

      // ------------------------------------------------------------ the end of a piece: the copies added up, 16 dims at a time
      settle();                                            // (the piece before this one's unit)
      wait(&ctl->pvdone, (uint32_t)(g & 1));
      const float both = HALVES == 1 ? l : l + exchange(make_float2(l, 0.f)).x;
      if (half == 0) stat[at] = make_float4(m, both, m2, 0.f);
      meet();
      if (dead) break;
      const int R = hd.tokens * G;
      float mx = kNoMax, mx2 = kNoMax, sum = 0.f;
#pragma unroll
      for (int i = 0; i < S::COPIES; ++i) {
        mx = fmaxf(mx, stat[i * S::ROWS + row].x);
        mx2 = fmaxf(mx2, stat[i * S::ROWS + row].z);
      }
#pragma unroll
      for (int i = 0; i < S::COPIES; ++i) sum += stat[i * S::ROWS + row].y * ex2_approx(stat[i * S::ROWS + row].x - mx);
      const float fo = ex2_approx(m2 - mx2);
      const bool whole = now.flags & kWhole;
      const int64_t mine = (int64_t)hd.mine * S::ROWS;
      if (copy == 0 && half == 0) {
        fin[row] = make_float4(mx, sum, mx2, 0.f);
        if (!whole && row < R) __stcg(a.part_st + mine + row, make_float4(mx, sum, mx2, 0.f));
      }
#pragma unroll 1
      for (int i = half * 2 * OD; i < (half + 1) * 2 * OD; ++i) {
        float o[16];
        tm_load<16>(tO + i * 16, o);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<float4*>(ob + at * S::OROW + 4 * e) =
              make_float4(o[4 * e] * fo, o[4 * e + 1] * fo, o[4 * e + 2] * fo, o[4 * e + 3] * fo);
        meet();
        if (dead) break;
#pragma unroll 1
        for (int e = at; e < R * 4; e += 128) {
          const int r = e >> 2, d = (e & 3) * 4;
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int k = 0; k < S::COPIES; ++k) {
            const float4 y = *reinterpret_cast<const float4*>(ob + (k * S::ROWS + r) * S::OROW + d);
            x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
          }
          if (whole) {
            const float4 st = fin[r];
            store_out(hd, r, i * 16 + d, x, st.x, st.y, st.z);
          } else {
            __stcg(reinterpret_cast<float4*>(a.part_o + (mine + r) * D + i * 16 + d), x);
          }
        }
        meet();
        if (dead) break;
      }
      if (dead) break;
      if (!whole) {
        if (threadIdx.x == 0)
          asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(ticket) : "l"(a.tickets + hd.unit) : "memory");
        owed = hd;
      }
    }
    settle();
  }
  // teardown: the products issued are complete; after a failure so are the copies (each wait bounded)
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0) {
    tc_mbar_wait(&ctl->drained, 0, kRoleWaitNs);
    if (ctl->fail)
      for (int x = std::max(0, ctl->loads - S::RAWS); x < ctl->loads; ++x)
        tc_mbar_wait(&ctl->raw_full[x % S::RAWS], (uint32_t)((x / S::RAWS) & 1), kRoleWaitNs);
  }
  __syncthreads();
  tc_fence_after();
  if (warp == S::SW + 9) tc_dealloc(tbase, 512);
}

// ---------------------------------------------------------------- host side
int copies_of(const PagedAttnCall& c) {
  const int64_t R = c.max_rows * (c.s.Hq / c.s.Hkv);
  return R <= 32 ? 4 : R <= 64 ? 2 : 1;
}

template <class S, bool BF16>
cudaError_t launch_shape(const BlockArgs& a, cudaStream_t st) {
  constexpr int smem = std::max(S::ALLOC, 116 * 1024);      // one CTA an SM: it takes all of the tensor memory
  const cudaError_t e = cudaFuncSetAttribute(block_kernel<S, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  return e != cudaSuccess ? e : launch_pdl(block_kernel<S, BF16>, dim3(kGrid), dim3(S::THREADS), smem, st, a);
}
template <int FMT, int D, bool BF16>
cudaError_t launch_c(const BlockArgs& a, cudaStream_t st) {
  const int copies = copies_of(a.c);
  if (copies == 4) return launch_shape<BShape<FMT, D, 4>, BF16>(a, st);
  if (copies == 2) return launch_shape<BShape<FMT, D, 2>, BF16>(a, st);
  return launch_shape<BShape<FMT, D, 1>, BF16>(a, st);
}
template <int FMT>
cudaError_t launch_f(const BlockArgs& a, cudaStream_t st) {
  const bool bf16 = a.c.s.dtype == MKV_BF16;
  if (a.c.s.D == 128) return bf16 ? launch_c<FMT, 128, true>(a, st) : launch_c<FMT, 128, false>(a, st);
  return bf16 ? launch_c<FMT, 64, true>(a, st) : launch_c<FMT, 64, false>(a, st);
}

}  // namespace

size_t paged_block_ws_bytes(const PagedAttnCall& c) {
  const size_t rows = (size_t)kGrid * 2 * (128 / copies_of(c));
  return kCounterBytes + align256(rows * sizeof(float4)) + align256(rows * c.s.D * sizeof(float));
}

cudaError_t launch_paged_block(const PagedAttnCall& c, void* ws, cudaStream_t st) {
  BlockArgs a{};
  const cudaError_t e = status_word(&a.status);
  if (e != cudaSuccess) return e;
  a.c = c;
  a.w = work_args(c, kGrid, 10);
  a.heads = Heads(c.s.Hq / c.s.Hkv);
  uint8_t* base = static_cast<uint8_t*>(ws);
  a.tickets = reinterpret_cast<int*>(base);
  a.part_st = reinterpret_cast<float4*>(base + kCounterBytes);
  a.part_o = reinterpret_cast<float*>(base + kCounterBytes +
                                      align256((size_t)kGrid * 2 * (128 / copies_of(c)) * sizeof(float4)));
  return c.s.format == MKV_E4M3 ? launch_f<MKV_E4M3>(a, st) : launch_f<MKV_I8>(a, st);
}

}  // namespace mkv
