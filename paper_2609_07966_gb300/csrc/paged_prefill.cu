// Attention of an entry's newest tokens over its 8-bit pages where more than 128 query rows share a key head: prompts, their
// next chunks, many drafted tokens.  The formula, and the two running maxima, are those of paged_decode.cu.
//
// Bound by the tensor cores.  A CTA takes 256 rows of a key head (tokens x heads of the group, so that grouped heads share
// every converted key) as two blocks of 128 and streams 128-token tiles past both: the tensor cores work on one block while
// the other is in its softmax.
//   S_i [128 x 128] = Q_i K^T    fp16 operands in shared memory, accumulator in tensor memory
//   O_i [128 x D]  += W_i V      W_i (the weights, fp16) from tensor memory, over the S_i they came from
// The tensor cores have no product of 16-bit queries with 8-bit codes, so every tile's codes are widened to fp16 (exactly) on
// their way: one warp loads them (a bulk copy a page) into a ring, one warpgroup reads them there and writes the swizzled
// layout that the products read, beside the products and the softmax (a tile's conversion left out saves nothing).  (Without
// the ring, codes in the converting threads' registers eight loads ahead, the loads' latency made it the bottleneck: a
// prompt of 4096 tokens 156 us.)
//
// A tile of 128 tokens takes about 3900 cycles for both blocks, of which the products need 2048: a block's scores, softmax and
// second product follow one another, tensor memory holds one tile of scores a block, and the other block's products fill only
// a part of the wait.  A unit takes another 10 us: its queries, the pipeline's start, the last tile's chain and the output.
// 4096 tokens, 32 / 8 heads of 128: 143 us, 0.50 of the measured peak; 511 and 383 over 8K and 6K: 121 us, 0.44.
//
// A tile's pages have scales of their own: within 16 columns both are constant, so a score's is part of the factor of its
// exponent, the maxima are kept per 16 columns until they are scaled, and a weight is p vs 2^(m - m2 + 6).
//
// A unit is 256 rows of a key head.  With few of them, their tiles lie end to end and are cut into equal runs, one an SM; a
// run's tiles of one unit are a piece, and join_kernel adds up the pieces of units that several runs share.  Many units are
// balanced by the order in which they are launched.  Which it is to be is found out on the device, where the lengths are.
#include <math.h>

#include <algorithm>

#include "mkv_paged_softmax.cuh"
#include "mkv_paged_work.cuh"

namespace mkv {

namespace {

constexpr int kBR = 128;            // rows a block, tokens a tile
constexpr int kRows = 2 * kBR;      // rows a unit
// Warpgroups: four of softmax (two a block: a row's columns are halved between the threads of two warps, whose chains of
// instructions then overlap; with one warp a row 156 us for a prompt of 4096 tokens), one that converts, one for products and
// loads (two warps idle).
constexpr int kThreads = 768;
constexpr int kHeads = 8;           // tiles whose heads and scales are held
constexpr int kSlots = 3;           // widened tiles (K0 V0 K1 V1 ..)
constexpr int kHeldBatches = 4;     // (a tile is one of at least four of a batch)
// Up to this many units their tiles may be shared out: where that takes less time by this count, in tiles: a piece beyond its
// tiles 5 (10 us: queries, the pipeline's start and end, sums stored), the join 4.
// (376 units, 64 tiles each: 355 us shared out, 343 not.)
constexpr int kShared = 2 * kNumSMs, kPieceTiles = 5, kJoinTiles = 4;
static_assert(kShared <= kThreads && kShared % 4 == 0, "a slot a thread");
static_assert(kBR == kTokens && kHeads <= (kHeldBatches - 1) * 4, "tiles are chunks; scales are kept");

struct PrefillArgs {
  PagedAttnCall c;
  uint32_t* status;
  Heads heads;
  WorkArgs w;
  int slots;                        // units of all entries, a key head's
  int per;                          // start null: units of an entry
  int runs;                         // CTAs that may share all tiles; 0: a CTA a unit
  float* part_o;                    // [kNumSMs][2][D / 4][256][4]: pieces; of a run the first one's place and the last one's
  float4* part_st;                  // [kNumSMs][2][256]: m, sum, m2
  int4* joins;                      // [slot][Hkv]: the unit's first run, its first piece's place, how many pieces, its entry
};

// GC: tokens that share a page's scales for certain, 16 or (pages of 32 and more) 32: a 4096-token prompt 154 and 143 us.
template <int FMT_, int D_, int GC_>
struct PShape {
  static constexpr int FMT = FMT_, D = D_, GC = GC_, KA = D / 64;
  static constexpr int ATOM = kBR * 128, TILE = KA * ATOM, QBLK = TILE;
  static constexpr int RAW = kBR * D, RAWS = 3;            // codes of a tile's keys or values
  static constexpr int Q_OFF = 0, T_OFF = 2 * QBLK;        // [kSlots] widened tiles
  static constexpr int R_OFF = T_OFF + kSlots * TILE;      // [RAWS] codes
  static constexpr int SC_OFF = R_OFF + RAWS * RAW;        // scales of kHeldBatches batches
  static constexpr int HD_OFF = SC_OFF + scale_bytes(kHeldBatches);   // [kHeads] Chunk
  static constexpr int QS_OFF = HD_OFF + kHeads * 16;      // [256] exponents that bf16 rows are scaled by
  static constexpr int X_OFF = QS_OFF + kRows;             // [2][2][256] float2: what the halves of a row tell each other
  static constexpr int B_OFF = X_OFF + 2 * 2 * kRows * 8;  // [kShared + 1] where the slots' tiles begin
  static constexpr int CTL_OFF = B_OFF + (kShared + 4) * 4;
  static constexpr int ALLOC = CTL_OFF + 768;
  static_assert(ALLOC <= 227 * 1024, "shared memory");
};

struct PCtl {
  uint64_t qfull, drained, raw_full[4], raw_empty[4], tile_full[kSlots], tile_empty[kSlots], head[kHeads], sfull[2], pfull[2][2],
      pvdone[2];
  uint32_t tslot;
  int fail, loads;
  int b, rb, rows, pos0, len, row0, live, c0, c1, nt[2];   // the unit, and what of it is this CTA's
  int kvh, whole, place, shared;
  int cur, end;                    // of the run: the next piece's first tile, the last one's end
  int before, done[2], pieces;     // tiles of earlier pieces, of each block, and how many there were
  int sums[kThreads / 32], most[kThreads / 32], least[kThreads / 32], units[kThreads / 32];
};
static_assert(sizeof(PCtl) <= 768, "control block");

// Units lie entry after entry, enough of them for each entry's rows.
__device__ __forceinline__ int unit_base(const PrefillArgs& a, int b) {
  if (a.c.s.start == nullptr) return b * a.per;
  const int r0 = min(max(a.c.s.start[b], 0), (int)a.c.s.n);
  return (int)(((int64_t)r0 * a.heads.G + (int64_t)b * (kRows - 1)) / kRows);
}
struct Unit {
  int b, kvh, rb, rows, pos0, len; // its block of rows; rows of the entry (tokens x heads of a group), its first new position
  int row0;                        // its first token's row
  bool live;
  // tokens that a row sees
  __device__ __forceinline__ int seen(const Heads& h, int row) const {
    return row < rows ? max(0, min(len, pos0 + h.token(row) + 1)) : 0;
  }
  // tiles of block k: at least one where it has rows, so that they are written
  __device__ __forceinline__ int tiles(const Heads& h, int k) const {
    const int first = rb * kRows + k * kBR, last = min(first + kBR, rows) - 1;
    return last >= first ? max(1, (seen(h, last) + kBR - 1) / kBR) : 0;
  }
};
__device__ __forceinline__ Unit unit_of(const PrefillArgs& a, int b, int slot, int kvh, bool report) {
  Unit u;
  u.b = b;
  u.kvh = kvh;
  u.rb = slot - unit_base(a, u.b);
  const EntryRows r = entry_rows(a.c.s, u.b);
  u.row0 = r.first;
  u.live = r.count <= a.c.max_rows;
  if (!u.live && report && u.rb == 0 && kvh == 0) atomicOr(a.status, MKV_FLAG_BAD_INDEX);
  const int tokens = (int)min((int64_t)r.count, a.c.max_rows);
  u.rows = tokens * a.heads.G;
  u.live = u.live && u.rb >= 0 && (int64_t)u.rb * kRows < u.rows;
  u.len = (int)min((int64_t)max(a.c.T_len[u.b], 0), a.c.s.max_pages * a.c.s.page);
  u.pos0 = u.len - tokens;
  return u;
}
// (a whole warp finds the entry, or every thread its own)
__device__ __forceinline__ int entry_of_slot(const PrefillArgs& a, int slot, int lane) {
  return a.c.s.start == nullptr ? slot / a.per : find_entry(a.c.s.B, lane, [&](int b) { return unit_base(a, b) <= slot; });
}
__device__ __forceinline__ int entry_of_slot(const PrefillArgs& a, int slot) {
  if (a.c.s.start == nullptr) return slot / a.per;
  int lo = 0, hi = a.c.s.B;                                // the last entry that begins at or before the slot
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (unit_base(a, mid) <= slot)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

template <class S, bool BF16, bool SHARED>
__global__ void __launch_bounds__(kThreads, 1) prefill_kernel(const PrefillArgs a) {
  constexpr int D = S::D, GC = S::GC;
  extern __shared__ __align__(1024) uint8_t sm[];
  PCtl* ctl = reinterpret_cast<PCtl*>(sm + S::CTL_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PagedAttnCall& c = a.c;
  const int Hkv = c.s.Hkv;

  pdl_wait_and_trigger();
  // What tiles c0 .. of a unit this CTA takes, told to all threads.
  auto tell = [&](const Unit& u, int c0, int c1) {
    const int all0 = u.tiles(a.heads, 0), all1 = u.tiles(a.heads, 1);
    ctl->b = u.b;
    ctl->kvh = u.kvh;
    ctl->rb = u.rb;
    ctl->rows = u.rows;
    ctl->pos0 = u.pos0;
    ctl->len = u.len;
    ctl->row0 = u.row0;
    ctl->live = u.live;
    ctl->c0 = c0;
    ctl->c1 = c1;
    ctl->nt[0] = max(0, min(all0, c1) - c0);
    ctl->nt[1] = max(0, min(all1, c1) - c0);
  };
  int* base = reinterpret_cast<int*>(sm + S::B_OFF);
  if (!SHARED) {
    // Launch order: the last rows of the entries first (they see the most), all key heads of a slot together.
    const int slot = a.slots - 1 - blockIdx.x / Hkv;
    if (warp == 0) {                                       // (one warp finds it out: twenty-four took 5 us a CTA)
      const Unit u = unit_of(a, entry_of_slot(a, slot, lane), slot, blockIdx.x % Hkv, true);
      if (lane == 0) {
        tell(u, 0, max(u.tiles(a.heads, 0), u.tiles(a.heads, 1)));
        ctl->whole = 1;
        ctl->place = 0;
      }
    }
  } else {
    // The slots' tiles (of all key heads) end to end: a thread a slot.
    int own = 0;                                           // tiles of a unit
    if (threadIdx.x < a.slots) {
      const Unit u = unit_of(a, entry_of_slot(a, threadIdx.x), threadIdx.x, 0, blockIdx.x == 0);
      if (u.live) own = max(u.tiles(a.heads, 0), u.tiles(a.heads, 1));
      if (!u.live && blockIdx.x == 0)
        for (int h = 0; h < Hkv; ++h) a.joins[threadIdx.x * Hkv + h] = make_int4(0, 0, 0, 0);
    }
    int upto = own * Hkv;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += x;
    }
    const int w_most = __reduce_max_sync(0xffffffffu, own), w_least = __reduce_min_sync(0xffffffffu, own > 0 ? own : INT32_MAX);
    const int w_units = __popc(__ballot_sync(0xffffffffu, own > 0)) * Hkv;
    if (lane == 31) {
      ctl->sums[warp] = upto;
      ctl->most[warp] = w_most;
      ctl->least[warp] = w_least;
      ctl->units[warp] = w_units;
    }
    __syncthreads();
    for (int w = 0; w < warp; ++w) upto += ctl->sums[w];
    if (threadIdx.x < a.slots) base[threadIdx.x + 1] = upto;
    if (threadIdx.x == 0) base[0] = 0;
    __syncthreads();
    int cur, end;                                          // of this CTA's run
    int most = 0, least = INT32_MAX, units = 0;
    for (int w = 0; w < (a.slots + 31) / 32; ++w) {
      most = max(most, ctl->most[w]);
      least = min(least, ctl->least[w]);
      units += ctl->units[w];
    }
    // (a run's pieces: no more than its tiles, or than units of the shortest kind in it and two it shares)
    const int len = (base[a.slots] + kNumSMs - 1) / kNumSMs, alone = units <= kNumSMs ? most : len + most / 2;
    const bool shared = len + kPieceTiles * (min(len, len / least + 2) - 1) + kJoinTiles < alone;
    if (shared) {
      const Runs rs(base[a.slots], a.runs);
      if ((int)blockIdx.x >= rs.runs) return;
      cur = rs.start(blockIdx.x);
      end = rs.start(blockIdx.x + 1);
    } else {                                               // a unit, the entries' last rows first
      const int unit = a.slots * Hkv - 1 - (int)blockIdx.x, slot = unit / Hkv;
      if (unit < 0 || base[slot] == base[slot + 1]) return;
      const int all = (base[slot + 1] - base[slot]) / Hkv;
      cur = base[slot] + (unit - slot * Hkv) * all;
      end = cur + all;
    }
    if (threadIdx.x == 0) {
      ctl->shared = shared;
      ctl->cur = cur;
      ctl->end = end;
      ctl->before = ctl->done[0] = ctl->done[1] = ctl->pieces = 0;
    }
    __syncthreads();
  }
  // The thread whose slot holds tile `cur` finds out the run's next piece.
  auto next_piece = [&]() {
    const int slot = threadIdx.x, cur = ctl->cur, end = ctl->end;
    if (slot >= a.slots || cur < base[slot] || cur >= base[slot + 1]) return;
    const int all = (base[slot + 1] - base[slot]) / Hkv, kvh = (cur - base[slot]) / all, unit0 = base[slot] + kvh * all;
    const Unit u = unit_of(a, entry_of_slot(a, slot), slot, kvh, false);
    const int c0 = cur - unit0, c1 = min(all, end - unit0);
    tell(u, c0, c1);
    ctl->whole = c1 - c0 == all;
    if (!ctl->shared) {
      a.joins[slot * Hkv + kvh] = make_int4(0, 0, 0, 0);
      return;
    }
    const Runs rs(base[a.slots], a.runs);
    const Shares sh(rs, unit0, all);
    ctl->place = (int)blockIdx.x == sh.first ? sh.place0 : 2 * (int)blockIdx.x;
    if (c0 == 0) a.joins[slot * Hkv + kvh] = make_int4(sh.first, sh.place0, sh.count, u.b);
  };
  if (SHARED) next_piece();
  if (warp == 20) tc_alloc(&ctl->tslot, 512);
  if (threadIdx.x == 32) {
    tc_mbar_init(&ctl->qfull, 16);
    tc_mbar_init(&ctl->drained, 1);
    for (int s = 0; s < S::RAWS; ++s) {
      tc_mbar_init(&ctl->raw_full[s], 1);
      tc_mbar_init(&ctl->raw_empty[s], 4);
    }
    for (int s = 0; s < kSlots; ++s) {
      tc_mbar_init(&ctl->tile_full[s], 4);
      tc_mbar_init(&ctl->tile_empty[s], 1);
    }
    for (int s = 0; s < kHeads; ++s) tc_mbar_init(&ctl->head[s], 1);
    for (int s = 0; s < 2; ++s) {
      tc_mbar_init(&ctl->sfull[s], 1);
      tc_mbar_init(&ctl->pfull[s][0], 8);                  // (the first half's weights; both halves' outputs are scaled)
      tc_mbar_init(&ctl->pfull[s][1], 4);                  // (the second half's weights)
      tc_mbar_init(&ctl->pvdone[s], 1);
    }
    tc_fence_mbar_init();
    ctl->fail = ctl->loads = 0;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = ctl->tslot;
  if (!ctl->live) {                                        // (no such rows)
    __syncthreads();
    if (warp == 20) tc_dealloc(tbase, 512);
    return;
  }
  volatile int* fail = &ctl->fail;
  Chunk* heads = reinterpret_cast<Chunk*>(sm + S::HD_OFF);
  uint32_t* status = a.status;
  const int all_copies = (1 << (kTokens >> a.w.log_page)) - 1;
  for (;;) {
    Unit u;
    u.b = ctl->b;
    u.kvh = ctl->kvh;
    u.rb = ctl->rb;
    u.rows = ctl->rows;
    u.pos0 = ctl->pos0;
    u.len = ctl->len;
    u.row0 = ctl->row0;
    const int c0 = ctl->c0, ntiles = ctl->c1 - c0, nt[2] = {ctl->nt[0], ctl->nt[1]}, base_row = u.rb * kRows, kvh = u.kvh;
    const bool whole = ctl->whole != 0;
    const int64_t part = (int64_t)ctl->place * kRows;
    const int before = SHARED ? ctl->before : 0, done0 = SHARED ? ctl->done[0] : 0, done1 = SHARED ? ctl->done[1] : 0;
    const int pieces = SHARED ? ctl->pieces : 0;

    if (warp >= 20) {
      if (warp == 20 && elect_one()) {
        // ---------------------------------------------------------------- products
        constexpr uint32_t idS = tc_idesc(false, kBR, kBR, false, false);
        constexpr uint32_t idO = tc_idesc(false, kBR, D, false, true);
        const Desc qd = tc_desc_sw128(smem_addr(sm + S::Q_OFF));
        const Desc kd = tc_desc_sw128(smem_addr(sm + S::T_OFF));
        const Desc vd = tc_desc_mn<64>(smem_addr(sm + S::T_OFF), S::ATOM);
        auto wait = [&](uint64_t* bar, uint32_t parity) {
          const bool ok = wait_or_fail(bar, parity, fail, status);
          tc_fence_after();
          return ok;
        };
        auto scores = [&](int k, int t) {
          const Desc q0 = qd.at(k * S::QBLK).opaque(), k0 = kd.at(2 * (before + t) % kSlots * S::TILE).opaque();
#pragma unroll
          for (int j = 0; j < S::KA * 4; ++j)
            tc_mma_ss(tbase + (uint32_t)(k * kBR), q0.at((j >> 2) * S::ATOM + (j & 3) * 32),
                      k0.at((j >> 2) * S::ATOM + (j & 3) * 32), idS, j > 0 ? 1u : 0u);
          tc_commit(&ctl->sfull[k]);
        };
        auto values = [&](int k, int t, int half) {           // over half of tile t's tokens
          const Desc v0 = vd.at((2 * (before + t) + 1) % kSlots * S::TILE + half * (kBR / 2) * 128).opaque();
          const uint32_t p0 = tbase + (uint32_t)(k * kBR + half * (kBR / 2));
#pragma unroll
          for (int kk = 0; kk < kBR / 32; ++kk)
            tc_mma_ts(tbase + (uint32_t)(2 * kBR + k * kBR), p0 + (uint32_t)(kk * 8), v0.at(kk * 2048), idO,
                      t > 0 || half > 0 || kk > 0 ? 1u : 0u);
        };
        const int first = 2 * before;
        bool ok = wait(&ctl->qfull, (uint32_t)(pieces & 1)) &&
                  wait(&ctl->tile_full[first % kSlots], (uint32_t)((first / kSlots) & 1));
        if (ok) {
          for (int k = 0; k < 2; ++k)
            if (nt[k] > 0) scores(k, 0);
          tc_commit(&ctl->tile_empty[first % kSlots]);
        }
        for (int t = 0; ok && t < ntiles; ++t) {
          const int vi = 2 * (before + t) + 1, ki = vi + 1;          // places of this tile's values, of the next one's keys
          ok = wait(&ctl->tile_full[vi % kSlots], (uint32_t)((vi / kSlots) & 1));
          for (int k = 0; ok && k < 2; ++k) {
            if (t < nt[k]) {
              // (the first half's weights arrive while the softmax works on the second; a product over half of the tokens adds
              // to all dims of the outputs, so both halves of those have been scaled by then)
              ok = wait(&ctl->pfull[k][0], (uint32_t)(((k == 0 ? done0 : done1) + t) & 1));
              if (!ok) break;
              values(k, t, 0);
              ok = wait(&ctl->pfull[k][1], (uint32_t)(((k == 0 ? done0 : done1) + t) & 1));
              if (!ok) break;
              values(k, t, 1);
              tc_commit(&ctl->pvdone[k]);
            }
            if (k == 1) tc_commit(&ctl->tile_empty[vi % kSlots]);
            if (k == 0 && t + 1 < ntiles) {
              ok = wait(&ctl->tile_full[ki % kSlots], (uint32_t)((ki / kSlots) & 1));
              if (!ok) break;
            }
            if (t + 1 < nt[k]) scores(k, t + 1);
            if (k == 1 && t + 1 < ntiles) tc_commit(&ctl->tile_empty[ki % kSlots]);
          }
        }
        tc_commit(&ctl->drained);
      } else if (warp == 21) {
        // ---------------------------------------------------------------- loads
        auto wait = [&](uint64_t* bar, uint32_t parity) {
          return __all_sync(0xffffffffu, wait_or_fail(bar, parity, fail, status)) != 0;
        };
        const int log_page = a.w.log_page;
        int batch = 0;
        load_chunks<kHeldBatches>(
            c, a.w, status, reinterpret_cast<float2*>(sm + S::SC_OFF), lane, batch, u.b, u.kvh, u.len, c0, c0 + ntiles, 0,
            [&]() { return true; },
            [&](const Chunk& ch, bool mine, int id, int at) {
              const uint32_t bytes = (uint32_t)(__popc(ch.copies) * D) << log_page;
              const int64_t from = ((int64_t)id * Hkv + u.kvh) * c.s.page * D;
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int item = 2 * (before + ch.chunk - c0) + h, s = item % S::RAWS;
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
            [&](const Chunk& ch) {
              // (its place is free: tile t's codes could only be loaded once tile t - 8 was done with)
              const int t = before + ch.chunk - c0;
              if (lane == 0) heads[t % kHeads] = ch;
              __syncwarp();
              if (lane == 0) tc_mbar_arrive(&ctl->head[t % kHeads]);
            });
      }
    } else if (warp >= 16) {
      // ---------------------------------------------------------------- codes to fp16
      // A thread takes one 16-byte piece of every STEP'th row.  Of eight neighbouring threads four read the first half of one
      // row and four the second half of the next: different banks, and so are those of the pieces that they store, in an atom
      // each (two rows of one atom with 64 dims).
      constexpr int STEP = D == 128 ? 16 : 32;
      const int tid = threadIdx.x - 512;
      const int piece = D == 128 ? tid & 7 : tid & 3;
      const int row = D == 128 ? (tid >> 4) * 2 + ((tid >> 2 ^ tid >> 3) & 1) : tid >> 2;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        return __all_sync(0xffffffffu, wait_or_fail(bar, parity, fail, status)) != 0;
      };
      const uint32_t at0 = (uint32_t)((2 * (piece & 3)) ^ (row & 7)) << 4;
      for (int item = 2 * before; item < 2 * (before + ntiles); ++item) {
        const int t = item >> 1, rs = item % S::RAWS, s = item % kSlots;
        if (!(item & 1) && !wait(&ctl->head[t % kHeads], (uint32_t)((t / kHeads) & 1))) break;
        if (!wait(&ctl->raw_full[rs], (uint32_t)((item / S::RAWS) & 1))) break;
        if (item >= kSlots && !wait(&ctl->tile_empty[s], (uint32_t)((item / kSlots - 1) & 1))) break;
        const uint8_t* src = sm + S::R_OFF + rs * S::RAW + row * D + piece * 16;
        uint8_t* dst = sm + S::T_OFF + s * S::TILE + (piece >> 2) * S::ATOM + row * 128;
        uint4 x[kBR / STEP];
#pragma unroll
        for (int i = 0; i < kBR / STEP; ++i) x[i] = *reinterpret_cast<const uint4*>(src + i * STEP * D);
        if (item & 1) {                                      // what no row sees must not meet a zero weight as NaN
          const int copies = heads[t % kHeads].copies, tail = u.len - (c0 + t - before) * kBR;
          if (copies != all_copies || tail < kBR)
#pragma unroll
            for (int i = 0; i < kBR / STEP; ++i)
              if (row + i * STEP >= tail || !(copies >> ((row + i * STEP) >> a.w.log_page) & 1)) x[i] = make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int i = 0; i < kBR / STEP; ++i) {
          uint32_t e[8];
          widen_codes<S::FMT>(x[i].x, e[0], e[1]);
          widen_codes<S::FMT>(x[i].y, e[2], e[3]);
          widen_codes<S::FMT>(x[i].z, e[4], e[5]);
          widen_codes<S::FMT>(x[i].w, e[6], e[7]);
          *reinterpret_cast<uint4*>(dst + i * STEP * 128 + at0) = make_uint4(e[0], e[1], e[2], e[3]);
          *reinterpret_cast<uint4*>(dst + i * STEP * 128 + (at0 ^ 16u)) = make_uint4(e[4], e[5], e[6], e[7]);
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          tc_mbar_arrive(&ctl->tile_full[s]);
          tc_mbar_arrive(&ctl->raw_empty[rs]);
        }
      }
    } else {
      const int k = warp >> 3, half = warp >> 2 & 1;         // its block; its columns 64 half ..
      const int ntk = k == 0 ? nt[0] : nt[1], dk = k == 0 ? done0 : done1;
      const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
      const uint32_t tS = tbase + lanes + (uint32_t)(k * kBR), tO = tbase + lanes + (uint32_t)(2 * kBR + k * kBR);
      int8_t* qs = reinterpret_cast<int8_t*>(sm + S::QS_OFF);
      // ---------------------------------------------------------------- queries, D / 8 lanes a row
      // (copied to their places, and there a thread's own pieces scaled: loops of little code, which is cold in every CTA; held
      // in registers between, eight loads unrolled, a unit's queries took 6000 cycles)
      {
        constexpr int LN = D / 8, PER = 32 / LN;
        const int ch = lane % LN, r0 = warp * PER + lane / LN;
        uint8_t* dst0 = sm + S::Q_OFF + (ch >> 3) * S::ATOM;
        auto place = [&](int r) { return dst0 + (r / kBR) * S::QBLK + mn_offset<64>(r % kBR, ch & 7); };
#pragma unroll 2
        for (int r = r0; r < kRows; r += 16 * PER) {
          const int row = min(base_row + r, u.rows - 1);
          const uint16_t* q = c.q + (u.row0 + a.heads.token(row)) * c.q_stride;
          cp_async16(place(r), q + (int64_t)(kvh * a.heads.G + a.heads.head(row)) * D + ch * 8,
                     base_row + r < u.rows ? 16 : 0);
        }
        cp_async_commit();
        cp_async_wait<0>();
        if (BF16) {                                          // a power of two a row (paged_decode.cu)
#pragma unroll 2
          for (int r = r0; r < kRows; r += 16 * PER) {
            uint4* y = reinterpret_cast<uint4*>(place(r));
            float v[8], most = 0.f;
            widen8<true>(*y, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(v[i]) < INFINITY ? fabsf(v[i]) : 0.f);
#pragma unroll
            for (int d = 1; d < LN; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
            const int e = row_exponent(most);
            const float f = power_of_two(e);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= f;
            *y = narrow8<false>(v);
            if (ch == 0) qs[r] = (int8_t)e;
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) tc_mbar_arrive(&ctl->qfull);
      }
      // A warp whose wait ran out stops waiting but still meets its partner, so that neither is left waiting.
      bool dead = false;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (!dead) dead = !__all_sync(0xffffffffu, wait_or_fail(bar, parity, fail, status));
        tc_fence_after();
        return !dead;
      };
      // ---------------------------------------------------------------- softmax: row 32 (warp % 4) + lane of block k
      const int rin = k * kBR + (warp & 3) * 32 + lane, row = base_row + rin, seen = u.seen(a.heads, row);
      const int td = u.seen(a.heads, base_row) / kBR;                 // first tile that the unit's first row does not see whole
      int turn = 0;
      auto exchange = [&](float2 x) {                        // with the warp that has the rows' other columns
        float2* tell = reinterpret_cast<float2*>(sm + S::X_OFF) + turn * 2 * kRows + rin;
        turn ^= 1;                                           // (one place is read until the barrier after the next)
        tell[half * kRows] = x;
        bar_sync(1 + k * 4 + (warp & 3), 64);
        return tell[(1 - half) * kRows];
      };
      float back = 1.f;
      if (BF16) {                                            // (all warps' queries are in place)
        wait(&ctl->qfull, (uint32_t)(pieces & 1));
        back = power_of_two(-(int)qs[rin]);
      }
      constexpr int HC = kBR / 2;                            // columns of a thread
      const uint32_t tH = tS + (uint32_t)(half * HC);
      const int log_group = a.w.log_page - 4;
      float m = kNoMax, m2 = kNoMax, l = 0.f;
      for (int t = 0; t < ntk; ++t) {
        const int at = (before + t) % kHeads;
        wait(&ctl->head[at], (uint32_t)(((before + t) / kHeads) & 1));
        wait(&ctl->sfull[k], (uint32_t)((dk + t) & 1));
        const int copies = heads[at].copies;
        const float2* scales = reinterpret_cast<const float2*>(sm + S::SC_OFF) + heads[at].scales;
        const bool part = c0 + t >= td || copies != all_copies;      // (a page outside the pool or past the length)
        const int lim = seen - (c0 + t) * kBR - half * HC;   // this thread's columns that its row sees
        // 32 columns' scores, those that the row does not see minus infinity
        auto load = [&](int i, float (&v)[32]) {
          tm_read32(tH + (uint32_t)(32 * i), v);
          if (part) {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              const int upto = copies >> ((4 * half + 2 * i + g) >> log_group) & 1 ? lim - 32 * i : 0;
#pragma unroll
              for (int e = 16 * g; e < 16 * g + 16; ++e) v[e] = e < upto ? v[e] : -INFINITY;
            }
          }
        };
        auto scale_of = [&](int i, int g) { return scales[(4 * half + 2 * i + g * (GC / 16)) >> log_group]; };
        float mt = -INFINITY, mt2 = -INFINITY;
#pragma unroll 1
        for (int i = 0; i < HC / 32; ++i) {
          float v[32];
          load(i, v);
          columns_max<32, GC, BF16>(v, back, [&](int g) { return scale_of(i, g); }, mt, mt2);
        }
        const float2 other = exchange(make_float2(mt, mt2));
        mt = fmaxf(mt, other.x);
        mt2 = fmaxf(mt2, other.y);
        if (__any_sync(0xffffffffu, mt > m + kRaise || mt2 > m2 + kRaise)) {
          const float nm = fmaxf(m, mt), nm2 = fmaxf(m2, mt2);
          l *= ex2_approx(m - nm);
          const float w = ex2_approx(m2 - nm2);
          m = nm;
          m2 = nm2;
          if (t > 0) {
            wait(&ctl->pvdone[k], (uint32_t)((dk + t - 1) & 1));
#pragma unroll 1
            for (int i = half * (D / 64); i < (half + 1) * (D / 64); ++i) {
              float o[32];
              tm_load<32>(tO + i * 32, o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] *= w;
              tm_store<32>(tO + i * 32, o);
            }
          }
        }
        if (half == 1) {                                     // (the other half's warps arrive there after their weights)
          tm_store_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) tc_mbar_arrive(&ctl->pfull[k][0]);
        }
#pragma unroll 1
        for (int i = 0; i < HC / 32; ++i) {                  // (weights over scores that were read before)
          float v[32], pk[16];
          load(i, v);
          columns_weights<32, GC, BF16>(v, part, m, m2, back, [&](int g) { return scale_of(i, g); }, l, pk);
          tm_store<16>(tH + (uint32_t)(16 * i), pk);
        }
        tm_store_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) tc_mbar_arrive(&ctl->pfull[k][half]);
      }
      // ---------------------------------------------------------------- output
      if (ntk > 0) wait(&ctl->pvdone[k], (uint32_t)((dk + ntk - 1) & 1));
      l += exchange(make_float2(l, 0.f)).x;
      if (!dead) {
        // zeros for a row that sees nothing; NaN for one whose scores are all minus infinity
        const float inv = seen <= 0 ? 0.f : l == 0.f ? NAN : 1.f / l, hp = half_power(m, m2);
        if (!whole && half == 0) a.part_st[part + rin] = make_float4(m, l, m2, 0.f);
        uint16_t* dst = c.out + (u.row0 + a.heads.token(row)) * c.out_stride + (int64_t)(kvh * a.heads.G + a.heads.head(row)) * D;
        float4* po = reinterpret_cast<float4*>(a.part_o) + part * (D / 4) + rin;
        if (ntk > 0) {
#pragma unroll 1
          for (int i = half * (D / 64); i < (half + 1) * (D / 64); ++i) {
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
                __stcg(po + (8 * i + e) * kRows, make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]));
            }
          }
        }
      }
    }
    // the piece's end: the products issued are complete; after a failure so are the copies (each wait bounded)
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0) {
      tc_mbar_wait(&ctl->drained, (uint32_t)(pieces & 1), kRoleWaitNs);
      if (ctl->fail)
        for (int x = std::max(0, ctl->loads - S::RAWS); x < ctl->loads; ++x)
          tc_mbar_wait(&ctl->raw_full[x % S::RAWS], (uint32_t)((x / S::RAWS) & 1), kRoleWaitNs);
    }
    __syncthreads();
    tc_fence_after();
    if (!SHARED || ctl->fail || ctl->cur + ntiles >= ctl->end) break;
    __syncthreads();
    if (threadIdx.x == 0) {
      ctl->cur += ntiles;
      ctl->before += ntiles;
      ctl->done[0] += nt[0];
      ctl->done[1] += nt[1];
      ++ctl->pieces;
    }
    __syncthreads();
    next_piece();
    __syncthreads();
  }
  if (warp == 20) tc_dealloc(tbase, 512);
}

// out = sum_i 2^(m2_i - M2) o_i / sum_i 2^(m_i - M) l_i over a unit's pieces i, four dims of a row a thread.
template <int D, int TIMES_>
struct JShape {
  static constexpr int ROWS = 1024 / D, TIMES = TIMES_;    // rows side by side of a CTA, and one after another
  static constexpr int CTAS = kRows / (ROWS * TIMES);      // of a unit
};
template <class J, int D, bool BF16>
__global__ void __launch_bounds__(256) join_kernel(const PrefillArgs a) {
  pdl_wait_and_trigger();
  const int Hkv = a.c.s.Hkv, unit = blockIdx.x / J::CTAS, slot = unit / Hkv;
  const int r0 = blockIdx.x % J::CTAS * (J::ROWS * J::TIMES) + threadIdx.x % J::ROWS, d4 = threadIdx.x / J::ROWS;
  const int4 of = a.joins[unit];
  if (of.z <= 1) return;                                   // (a whole unit, or none)
  // (lengths that another stream changes under way leave CTAs at odds: then nothing outside the workspace is read)
  if (of.x < 0 || of.z > kNumSMs - of.x || of.y < 0 || of.y >= 2 * kNumSMs || of.w < 0 || of.w >= a.c.s.B) return;
  const Unit u = unit_of(a, of.w, slot, unit - slot * Hkv, false);
  auto at = [&](int i) { return (int64_t)(i == 0 ? of.y : 2 * (of.x + i)); };
  float mx[J::TIMES], mx2[J::TIMES], sum[J::TIMES];
  float4 y[J::TIMES];
#pragma unroll
  for (int k = 0; k < J::TIMES; ++k) {
    mx[k] = mx2[k] = kNoMax;
    sum[k] = 0.f;
    y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const float4* po = reinterpret_cast<const float4*>(a.part_o);
#pragma unroll(8 / J::TIMES)
  for (int i = 0; i < of.z; ++i) {
#pragma unroll
    for (int k = 0; k < J::TIMES; ++k) {
      const int r = r0 + k * J::ROWS;
      const float4 st = __ldcg(a.part_st + at(i) * kRows + r);
      float4 z = __ldcg(po + (at(i) * (D / 4) + d4) * kRows + r);
      if (st.z == kNoMax) z = make_float4(0.f, 0.f, 0.f, 0.f);       // (no tile of the row's block: no outputs were written)
      const float nm = fmaxf(mx[k], st.x), nm2 = fmaxf(mx2[k], st.z), f = ex2_approx(mx2[k] - nm2), g = ex2_approx(st.z - nm2);
      sum[k] = sum[k] * ex2_approx(mx[k] - nm) + st.y * ex2_approx(st.x - nm);
      y[k] = make_float4(y[k].x * f + z.x * g, y[k].y * f + z.y * g, y[k].z * f + z.z * g, y[k].w * f + z.w * g);
      mx[k] = nm;
      mx2[k] = nm2;
    }
  }
#pragma unroll
  for (int k = 0; k < J::TIMES; ++k) {
    const int row = u.rb * kRows + r0 + k * J::ROWS;
    if (row >= u.rows) continue;
    // zeros for a row that sees nothing; NaN for one whose scores are all minus infinity
    const float inv = u.seen(a.heads, row) <= 0 ? 0.f : sum[k] == 0.f ? NAN : 1.f / sum[k], hp = half_power(mx[k], mx2[k]);
    const float x[4] = {y[k].x * inv * hp * hp, y[k].y * inv * hp * hp, y[k].z * inv * hp * hp, y[k].w * inv * hp * hp};
    uint16_t* dst = a.c.out + (u.row0 + a.heads.token(row)) * a.c.out_stride;
    dst += (int64_t)(u.kvh * a.heads.G + a.heads.head(row)) * D + d4 * 4;
    *reinterpret_cast<uint2*>(dst) =
        inv == 0.f ? make_uint2(0u, 0u) : make_uint2(pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3]));
  }
}

// ---------------------------------------------------------------- host side
struct Plan {
  int64_t slots;
  int per, runs;
};
Plan plan_of(const PagedAttnCall& c) {
  Plan p{};
  const int64_t G = c.s.Hq / c.s.Hkv, m = ceil_div(c.s.n, c.s.B);
  p.per = (int)ceil_div(m * G, kRows);
  p.slots = c.s.start == nullptr ? (int64_t)c.s.B * p.per : (c.s.n * G + (int64_t)c.s.B * (kRows - 1)) / kRows;
  // (not with caches that hold fewer tiles than a piece and the join cost; tiles are counted in 32 bits)
  const int64_t units = p.slots * c.s.Hkv, tiles = c.s.max_pages * c.s.page / kTokens + 1;
  p.runs = units <= kShared && tiles > kPieceTiles + kJoinTiles && units * tiles <= INT32_MAX / 2 ? kNumSMs : 0;
  return p;
}

template <class S, bool BF16>
cudaError_t launch_shape(const PrefillArgs& a, cudaStream_t st) {
  const int64_t units = (int64_t)a.slots * a.c.s.Hkv;
  if (units > INT32_MAX) return cudaErrorInvalidConfiguration;
  constexpr int smem = std::max(S::ALLOC, 116 * 1024);      // one CTA an SM: it takes all of the tensor memory
  auto* kernel = a.runs != 0 ? prefill_kernel<S, BF16, true> : prefill_kernel<S, BF16, false>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  e = launch_pdl(kernel, dim3((unsigned)std::max<int64_t>(units, a.runs)), dim3(kThreads), smem, st, a);
  if (e != cudaSuccess || a.runs == 0) return e;
  // (few units: more threads, each with one row, for their many pieces: 64 rows over 8K, 8 units, 47 -> 39 us)
  using J1 = JShape<S::D, 1>;
  using J4 = JShape<S::D, 4>;
  return units <= kNumSMs / 2 ? launch_pdl(join_kernel<J1, S::D, BF16>, dim3((unsigned)(units * J1::CTAS)), dim3(256), 0, st, a)
                              : launch_pdl(join_kernel<J4, S::D, BF16>, dim3((unsigned)(units * J4::CTAS)), dim3(256), 0, st, a);
}
template <int FMT, int D>
cudaError_t launch_d(const PrefillArgs& a, cudaStream_t st) {
  const bool bf16 = a.c.s.dtype == MKV_BF16;
  if (a.c.s.page == 16)
    return bf16 ? launch_shape<PShape<FMT, D, 16>, true>(a, st) : launch_shape<PShape<FMT, D, 16>, false>(a, st);
  return bf16 ? launch_shape<PShape<FMT, D, 32>, true>(a, st) : launch_shape<PShape<FMT, D, 32>, false>(a, st);
}

}  // namespace

constexpr size_t kJoinBytes = kShared * sizeof(int4), kStatBytes = (size_t)kNumSMs * 2 * kRows * sizeof(float4);
static_assert(kJoinBytes % 256 == 0 && kStatBytes % 256 == 0, "workspace parts are aligned");
size_t paged_prefill_ws_bytes(const PagedAttnCall& c) {
  return kCounterBytes + kJoinBytes + kStatBytes + align256((size_t)kNumSMs * 2 * kRows * c.s.D * sizeof(float));
}

cudaError_t launch_paged_prefill(const PagedAttnCall& c, void* ws, cudaStream_t st) {
  PrefillArgs a{};
  const cudaError_t e = status_word(&a.status);
  if (e != cudaSuccess) return e;
  const Plan p = plan_of(c);
  a.c = c;
  a.heads = Heads(c.s.Hq / c.s.Hkv);
  a.w = work_args(c, kNumSMs, 0);
  if (p.slots > INT32_MAX) return cudaErrorInvalidConfiguration;
  a.slots = (int)p.slots;
  a.per = p.per;
  a.runs = p.runs;
  uint8_t* base = static_cast<uint8_t*>(ws) + kCounterBytes;
  a.joins = reinterpret_cast<int4*>(base);
  a.part_st = reinterpret_cast<float4*>(base + kJoinBytes);
  a.part_o = reinterpret_cast<float*>(base + kJoinBytes + kStatBytes);
  if (c.s.format == MKV_E4M3) return c.s.D == 128 ? launch_d<MKV_E4M3, 128>(a, st) : launch_d<MKV_E4M3, 64>(a, st);
  return c.s.D == 128 ? launch_d<MKV_I8, 128>(a, st) : launch_d<MKV_I8, 64>(a, st);
}

}  // namespace mkv
