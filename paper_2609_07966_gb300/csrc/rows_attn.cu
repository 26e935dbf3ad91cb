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
// Work: a unit is one (entry, key head, row block); its key tiles are the entry's cached ones and, last, the drafted
// tokens'.  The lengths are read on the device.  Two ways to share the units out, chosen by plan_rows:
//   clusters  a cluster of CTAs per unit, each an equal run of its tiles; the pieces are joined through distributed
//             shared memory (each CTA gets every piece's slice of its dims), so one launch does it all;
//   runs      the tiles of all units laid end to end, an equal run for every CTA, whatever the entries' lengths; a unit
//             inside one run is written directly, the pieces of a unit that several runs share go to the workspace
//             and join_kernel adds them up.  With several row blocks a run belongs to as many CTAs, one block each,
//             that meet its keys at the same time and so share them in L2.
//
// Roles: warps 0..4g-1 are the softmax (a thread holds one key and some rows), then one warp loads chunks by TMA
// into a ring of slots and one issues products, taking whichever is ready: a finished tile's second product
// first (it frees slots), else the next chunk of the scores.
//
// Bound by memory while a block's N rows need fewer tensor cycles a tile than its copy takes (64 keys of 576 dims: 3100
// cycles at an SM's share of HBM against 1600 at N = 32, 2000 at N = 64), else by a tile's chain of scores, softmax and
// second product.  Measured (GPU time): 16 drafted tokens over an 8 x 8K FP16 cache (32/8 heads, D 128) 48 us, 5.5
// TB/s; one latent token over 8 x 8K rows (rank 512) 26.6 us at 32 heads, 2.9 TB/s, and 40 us at 128; 12 drafted over 4
// x 32K ragged rows 123 us, 0.73 PFLOP/s; one latent token over 777 rows 10.5 us where the cache's capacity is near the
// length, 11.1 at 32K slots (the plan goes by the capacity).
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

namespace {

constexpr float kRaise = 8.f;       // a score may pass the running maximum by this (log2) before it is raised
// Weights carry 2^kOffset, so that those far below the maximum keep full precision in fp16 (normal down to
// 2^-20 of the maximum); it cancels in the division by their sum.
constexpr float kOffset = 6.f;
constexpr float kNoMax = -3.402823466e+38f;   // running maximum of a row that has seen nothing: no score is below it

struct RowsArgs {
  int B, n, H, Hkv, G;              // G: query heads per key head (latent: H)
  int R, row_blocks;                // rows per (entry, key head): n G; their blocks of N
  int side;                         // CTAs that take a run together, a row block each (or 1)
  int in_run;                       // row blocks within a run (or 1)
  int log_g;                        // FP16 caches: log2 G
  int cluster, log_cluster;         // CTAs a unit, joined in the kernel (a power of two); 0: runs over all units
  bool tree;
  int64_t T_cap;
  float scale_log2;
  const int32_t* T_len;
  const uint64_t* mask;             // [B][n]
  const uint16_t* v_tree;           // values of the drafted tokens (for non-finite ones)
  int64_t v_tok, v_head;            // their strides: token, key head
  uint16_t* out;
  float* part_o;                    // [CTAs][2][N][DV]: a run's pieces of units that other runs share
  float2* part_ml;                  // [CTAs][2][N]
  struct Joint* joint;              // [B][Hkv][row_blocks]
  uint32_t* status;                 // MKV_FLAG_* bits
};

// KA / VA: 64-dim atoms of a key / value; SHARED: values are the keys' first atoms; KT keys a tile, N rows a
// block, SLOTS ring slots, ROPE slots of the last key atom (SHARED), NP weight buffers.
template <bool BF16_, int KA_, int VA_, bool SHARED_, int KT_, int N_, int SLOTS_, int ROPE_, int NP_>
struct Shape {
  static_assert(N_ == 16 || N_ == 32 || N_ == 64, "rows a block (plan_rows)");
  static constexpr bool BF16 = BF16_, SHARED = SHARED_;
  static constexpr int KA = KA_, VA = VA_, KT = KT_, N = N_, SLOTS = SLOTS_, ROPE = ROPE_, NP = NP_;
  static constexpr int DV = VA * 64;
  static constexpr int MV = DV >= 128 ? 128 : 64;          // value dims per product (its M)
  static constexpr int NB = DV / MV;                       // O^T blocks
  static constexpr int NG = 2;                             // softmax groups of 128 threads
  static constexpr int C = N / NG;                         // rows of a softmax group
  // A tile of 64 keys takes 16 tensor-memory lanes of each warp's quarter: the warp's halves then share its rows, so
  // that no lane idles.  L lanes hold one set of CS rows.
  static constexpr int L = KT == 64 ? 16 : 32, CS = C * L / 32;
  static constexpr int SOFT = NG * 128, THREADS = SOFT + 128;   // (two of the last four warps idle)
  // registers a thread: what a launch of THREADS gets, and its split between softmax and the others
  static constexpr int RL = 168, RS = 208, RO = 88;
  static_assert(NG * RS + RO <= (NG + 1) * RL, "register shares");
  static constexpr int PW = N;                             // row width of a weight tile (elements)
  static constexpr int ATOM = KT * 128;                    // bytes of 64 dims of a tile
  static constexpr int QATOM = N * 128;
  // a tile's ring chunks: SHARED: its value blocks (MV dims each, the last key atom apart); else keys, values
  static constexpr int CH = SHARED ? NB : 2;
  static constexpr int SLOT = SHARED ? (MV / 64) * ATOM : KA * ATOM;
  // "Loaded" barriers (a tile's keys; not SHARED: its values apart), one per tile whose loads may be under way: tile
  // g + AHEAD is only begun once tile g's products are issued (SHARED: its last key atom's slot is free; else its
  // ring slots are).
  static constexpr int AHEAD = SHARED ? ROPE : SLOTS / 2 + 1;
  static_assert(SHARED || KA == VA, "keys and values of one size");
  static_assert(!SHARED || KA == VA + 1, "one key atom past the values");
  static constexpr int PBUF = KT * N * 2;
  static constexpr int Q_OFF = 0;
  static constexpr int KV_OFF = KA * QATOM;
  static constexpr int R_OFF = KV_OFF + SLOTS * SLOT;
  static constexpr int P_OFF = R_OFF + ROPE * ATOM;
  static constexpr int VIS_OFF = P_OFF + NP * PBUF;        // [kMaxTree][VW] words: rows that see a drafted token
  static constexpr int VW = (N + 31) / 32;
  static constexpr int RED_OFF = VIS_OFF + kMaxTree * VW * 4;   // [4][N] floats
  static constexpr int CTL_OFF = RED_OFF + 4 * N * 4;
  static constexpr int ALLOC = CTL_OFF + 512 + 1024;       // slack to align the base to 1024 B
  static constexpr int COLS = (2 + NB) * N;
  static constexpr int TMEM = COLS <= 64 ? 64 : COLS <= 128 ? 128 : COLS <= 256 ? 256 : 512;
  static_assert(COLS <= 512 && ALLOC <= 227 * 1024, "does not fit an SM");
};

constexpr int kMaxCluster = 8;      // CTAs of a cluster: the largest portable size
constexpr int kMaxSlotsRing = 12;
struct RowsCtl {
  uint64_t qfull, qempty, ofree, drained, kfull[8], vfull[8], empty[kMaxSlotsRing], rempty[4], sfull[2], pfull[2], pvdone[2];
  uint64_t nonfinite;     // drafted tokens that hold a non-finite value
  uint32_t tslot;
  int runs, run_len, longer;  // (Runs)
  int run0, run1, base, b0, len0;   // this CTA's run of tiles; first tile of entry b0, which holds run0; its length
  int u0;                           // the unit of that entry that holds run0
  int fail;
  int q_loads, k_loads, v_loads;    // pieces' queries, tiles whose keys or values were asked for (read after a failure)
};
static_assert(sizeof(RowsCtl) <= 512, "control block");

__device__ __forceinline__ int entry_len(const RowsArgs& a, int b) {
  return (int)std::min<int64_t>(std::max(a.T_len[b], 0), a.T_cap);
}
// Tiles of one unit of entry b.
template <int KT>
__device__ __forceinline__ int unit_tiles(const RowsArgs& a, int len) {
  return (len + KT - 1) / KT + (a.tree ? 1 : 0);
}
template <int KT>
__device__ __forceinline__ int entry_tiles(const RowsArgs& a, int b) {
  return unit_tiles<KT>(a, entry_len(a, b));
}

// `total` tiles in `runs` runs, the first total % runs of them one tile longer: run i starts at tile run_start(i).
struct Runs {
  int runs, len, longer;
  __device__ __forceinline__ Runs(int total, int ctas) {
    runs = std::max(1, std::min(ctas, total));           // none of them empty
    len = total / runs;
    longer = total - len * runs;
  }
  __device__ __forceinline__ int start(int i) const { return i * len + std::min(i, longer); }
  __device__ __forceinline__ int of(int tile) const {    // the run that holds a tile
    const int split = longer * (len + 1);
    return tile < split ? tile / (len + 1) : longer + (tile - split) / len;
  }
};

// Where the pieces of a unit that several runs share are: run `run` holds the first one, in its slot `slot`
// (0: its first piece, 1: its last), the runs after it the others in slot 0.
struct Joint {
  int run, slot, count;     // count 1: written directly
};

// A run's pieces, one unit at a time.
template <int KT>
struct Pieces {
  const RowsArgs& a;
  int cur, end, base;       // next tile of the run, its end, first tile of entry b
  int b, per;               // units per entry
  // the current piece: unit `u` of entry b, its tiles t0 .. t1 - 1 of `tiles`
  int u, t0, t1, tiles, len, index;
  int kvh, rb;              // its key head and row block
  __device__ __forceinline__ Pieces(const RowsArgs& args, const RowsCtl* c)
      : a(args), cur(c->run0), end(c->run1), base(c->base), b(c->b0), per(args.Hkv * args.in_run), u(c->u0 - 1),
        len(c->len0), index(-1) {}
  __device__ __forceinline__ bool next() {
    if (cur >= end) return false;
    ++u;                    // after a piece that ends its unit, the next one
#pragma unroll 1
    for (;;) {
      tiles = unit_tiles<KT>(a, len);
      if (cur < base + tiles * per) break;
      base += tiles * per;
      u = 0;
      len = entry_len(a, ++b);
    }
    kvh = a.in_run == 1 ? u : u / a.in_run;
    rb = a.side > 1 ? (int)(blockIdx.x % a.side) : u - kvh * a.in_run;
    t0 = cur - base - u * tiles;
    t1 = std::min(tiles, t0 + (end - cur));
    cur += t1 - t0;
    ++index;
    return true;
  }
};

struct MaxOp {
  __device__ __forceinline__ float operator()(float x, float y) const { return fmaxf(x, y); }
};
struct AddOp {
  __device__ __forceinline__ float operator()(float x, float y) const { return x + y; }
};
// A reduction over one warp quarter's keys: its results for the thread's rows in red[0 .. CS - 1], visible to the
// softmax group on return.
template <class S, typename Op>
__device__ __forceinline__ void group_reduce(float (&w)[S::CS], float* red, int lane, int grp, Op op) {
  reduce_columns<S::L>(w, lane, op);
  if ((lane & (S::L / S::CS - 1)) == 0) red[(lane & (S::L - 1)) / (S::L / S::CS)] = w[0];
  bar_sync(1 + grp, 128);
}

// Adds to dim d of each of W rows (the first `rows` of them from row `row` of the unit on) the non-finite values of the
// drafted tokens `nf` that it sees.
template <class S, int W>
__device__ __forceinline__ void add_non_finite(const RowsArgs& a, uint64_t nf, int b, int kvh, int row, int rows, int d,
                                               float (&o)[W]) {
#pragma unroll 1
  for (int c = 0; c < W && c < rows; ++c) {
    float add = 0.f;
    for (uint64_t bits = nf & a.mask[(int64_t)b * a.n + (row + c) / a.G]; bits; bits &= bits - 1) {
      const int j = __ffsll((long long)bits) - 1;
      const uint16_t y = j < a.n ? a.v_tree[((int64_t)b * a.n + j) * a.v_tok + kvh * a.v_head + d] : 0;
      if (non_finite<S::BF16>(y)) add += widen<S::BF16>(y);
    }
#pragma unroll
    for (int e = 0; e < W; ++e) o[e] += e == c ? add : 0.f;
  }
}

// Bit c: row `row + c` of the unit sees nothing (its entry holds no token and none of its drafted bits is set).  Such a
// row gives zeros; a row that does see tokens, but with scores of minus infinity only, has no weights to divide by: NaN.
template <int W>
__device__ __forceinline__ uint32_t blind_rows(const RowsArgs& a, int len, int b, int row) {
  if (len > 0) return 0;
  uint32_t blind = 0;
#pragma unroll 1
  for (int c = 0; c < W; ++c) {
    const int tok = (row + c) / a.G;
    const uint64_t bits = a.tree && tok < a.n ? a.mask[(int64_t)b * a.n + tok] : 0;
    if (bits << (kMaxTree - a.n) == 0) blind |= 1u << c;
  }
  return blind;
}

// First tile of CTA i of the 2^k that share a unit of `tiles`.
__device__ __forceinline__ int cluster_tile(int tiles, int i, int k) { return (int)((int64_t)tiles * i >> k); }

template <class S>
__global__ void __launch_bounds__(S::THREADS, 1)
    rows_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CUtensorMap ktmap,
                const __grid_constant__ CUtensorMap vtmap, const RowsArgs a) {
  constexpr int KT = S::KT, N = S::N, C = S::C, CH = S::CH, CS = S::CS, L = S::L;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  RowsCtl* ctl = reinterpret_cast<RowsCtl*>(sm + S::CTL_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kLoad = S::NG * 4, kMma = kLoad + 1;      // their warps

  // ---- setup: barriers, tensor memory; then (after the stream's previous kernel) this CTA's run of tiles
  if (warp == kMma) tc_alloc(&ctl->tslot, S::TMEM);
  if (warp == kLoad) {
    if (lane == 0) {
      prefetch_map(&qmap);
      prefetch_map(&kmap);
      tc_mbar_init(&ctl->qfull, 1);
      tc_mbar_init(&ctl->qempty, 1);
      tc_mbar_init(&ctl->ofree, S::NG * 4);
      tc_mbar_init(&ctl->drained, 1);
      for (int s = 0; s < S::AHEAD; ++s) {
        tc_mbar_init(&ctl->kfull[s], S::SHARED ? CH + 1 : 1);
        tc_mbar_init(&ctl->vfull[s], 1);
      }
      for (int s = 0; s < S::SLOTS; ++s) tc_mbar_init(&ctl->empty[s], 1);
      for (int s = 0; s < S::ROPE; ++s) tc_mbar_init(&ctl->rempty[s], 1);
      for (int s = 0; s < 2; ++s) {
        tc_mbar_init(&ctl->sfull[s], 1);
        tc_mbar_init(&ctl->pfull[s], S::NG * 4);
        tc_mbar_init(&ctl->pvdone[s], 1);
      }
      tc_fence_mbar_init();
      ctl->fail = ctl->q_loads = ctl->k_loads = ctl->v_loads = 0;
    }
    pdl_wait_and_trigger();
    const int per = a.Hkv * a.in_run;
    if (a.cluster > 0) {
      if (lane == 0) {
        const int unit = blockIdx.x >> a.log_cluster, i = blockIdx.x & (a.cluster - 1);
        const int b = unit / per, u = unit - b * per;
        const int len = entry_len(a, b), tiles = unit_tiles<KT>(a, len);
        ctl->len0 = len;
        ctl->b0 = b;
        ctl->base = 0;
        ctl->u0 = u;
        ctl->run0 = u * tiles + cluster_tile(tiles, i, a.log_cluster);
        ctl->run1 = u * tiles + cluster_tile(tiles, i + 1, a.log_cluster);
      }
    } else {
      const int len_mine = lane < a.B ? entry_len(a, lane) : 0;
      const int mine0 = lane < a.B ? unit_tiles<KT>(a, len_mine) * per : 0;
      int total = mine0;
      for (int b = lane + 32; b < a.B; b += 32) total += entry_tiles<KT>(a, b) * per;
#pragma unroll
      for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
      const Runs rs(total, a.side == 1 ? gridDim.x : gridDim.x / a.side);
      const int i = a.side == 1 ? blockIdx.x : blockIdx.x / a.side, run0 = i < rs.runs ? rs.start(i) : 0;
      const int run1 = i < rs.runs && total > 0 ? rs.start(i + 1) : 0;
      // the entry that holds tile run0
      int base = 0, b0 = 0;
      for (int c = 0; c < a.B && run0 < run1; c += 32) {
        const int mine = c == 0 ? mine0 : c + lane < a.B ? entry_tiles<KT>(a, c + lane) * per : 0;
        int upto = mine;                                    // inclusive prefix within the 32
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int x = __shfl_up_sync(0xffffffffu, upto, d);
          if (lane >= d) upto += x;
        }
        const unsigned past = __ballot_sync(0xffffffffu, c + lane < a.B && base + upto > run0);
        if (past) {
          const int w = __ffs(past) - 1;
          b0 = c + w;
          base += __shfl_sync(0xffffffffu, upto - mine, w);
          break;
        }
        base += __shfl_sync(0xffffffffu, upto, 31);
      }
      const int len0 = b0 < 32 ? __shfl_sync(0xffffffffu, len_mine, b0) : entry_len(a, b0);
      if (lane == 0) {
        const int tiles0 = std::max(1, unit_tiles<KT>(a, len0));
        ctl->u0 = (run0 - base) / tiles0;
        ctl->len0 = len0;
        ctl->runs = rs.runs;
        ctl->run_len = rs.len;
        ctl->longer = rs.longer;
        ctl->run0 = run0;
        ctl->run1 = run1;
        ctl->base = base;
        ctl->b0 = b0;
      }
    }
  } else {
    pdl_wait_and_trigger();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = ctl->tslot;
  const uint32_t tO = tbase + 2 * N;
  volatile int* fail = &ctl->fail;
  uint32_t* status = a.status;

  if (warp >= kLoad) {
    regs_down<S::RO>();
    if (warp == kLoad) {
      if (elect_one()) {
        // ---------------------------------------------------------------- loads
        Pieces<KT> p(a, ctl);
        int g = 0, slot = 0, lap = 0;                       // tiles loaded so far; next ring slot, times around
        bool ok = true;
        while (ok && p.next()) {
          const int kvh = p.kvh, row0 = p.rb * N;
          if (p.index > 0) ok = wait_or_fail(&ctl->qempty, (uint32_t)((p.index - 1) & 1), fail, status);
          if (!ok) break;
          tc_mbar_expect_tx(&ctl->qfull, S::KA * S::QATOM);
          for (int at = 0; at < S::KA; ++at)
            if (S::SHARED)
              tma_load_4d(sm + S::Q_OFF + at * S::QATOM, &qmap, at * 64, row0, p.b, 0, &ctl->qfull);
            else
              tma_load_4d(sm + S::Q_OFF + at * S::QATOM, &qmap, at * 64, kvh * a.G, row0 >> a.log_g, p.b, &ctl->qfull);
          ctl->q_loads = p.index + 1;
          for (int t = p.t0; ok && t < p.t1; ++t, ++g) {
            const bool tr = a.tree && t == p.tiles - 1;
            const int key = tr ? 0 : t * KT;
            const CUtensorMap* km = tr ? &ktmap : &kmap;
            const CUtensorMap* vm = tr ? &vtmap : &vmap;
            if constexpr (S::SHARED) {
              // the last key atom first: its slot bounds the tiles under way, and so the use of kfull
              const int r = g % S::ROPE, w = g / S::ROPE;
              ok = w == 0 || wait_or_fail(&ctl->rempty[r], (uint32_t)((w - 1) & 1), fail, status);
              if (!ok) break;
              tc_mbar_expect_tx(&ctl->kfull[r], S::ATOM);
              tma_load_4d(sm + S::R_OFF + r * S::ATOM, km, S::VA * 64, key, p.b, 0, &ctl->kfull[r]);
              ctl->k_loads = g + 1;
            }
#pragma unroll
            for (int j = 0; j < CH; ++j) {
              uint64_t* bar = S::SHARED || j == 0 ? &ctl->kfull[g % S::AHEAD] : &ctl->vfull[g % S::AHEAD];
              if (lap > 0 && !wait_or_fail(&ctl->empty[slot], (uint32_t)((lap - 1) & 1), fail, status)) {
                ok = false;
                if (S::SHARED) give_up(bar, CH - j);
                break;
              }
              uint8_t* dst = sm + S::KV_OFF + slot * S::SLOT;
              tc_mbar_expect_tx(bar, S::SLOT);
#pragma unroll
              for (int x = 0; x < S::SLOT / S::ATOM; ++x)
                if (S::SHARED)
                  tma_load_4d(dst + x * S::ATOM, km, (j * (S::MV / 64) + x) * 64, key, p.b, 0, bar);
                else
                  tma_load_4d(dst + x * S::ATOM, j == 0 ? km : vm, x * 64, key, kvh, p.b, bar);
              if (!S::SHARED) (j == 0 ? ctl->k_loads : ctl->v_loads) = g + 1;
              if (++slot == S::SLOTS) {
                slot = 0;
                ++lap;
              }
            }
          }
        }
      }
    } else if (warp == kMma + 1) {
      // ---------------------------------------------------------------- for join_kernel: the units that start here
      if (a.cluster == 0 && elect_one()) {
        Pieces<KT> p(a, ctl);
        Runs rs(1, 1);
        rs.runs = ctl->runs;
        rs.len = ctl->run_len;
        rs.longer = ctl->longer;
        while (p.next())
          if (p.t0 == 0) {
            const int u0 = p.base + p.u * p.tiles;
            const int run = a.side == 1 ? blockIdx.x : blockIdx.x / a.side;
            a.joint[((int64_t)p.b * a.Hkv + p.kvh) * a.row_blocks + p.rb] =
                Joint{run, p.index > 0 ? 1 : 0, rs.of(u0 + p.tiles - 1) - run + 1};
          }
      }
    } else if (warp == kMma) {
      if (elect_one()) {
        // ---------------------------------------------------------------- products
        constexpr uint32_t idS = tc_idesc(S::BF16, KT, N, false, false);
        constexpr uint32_t idO = tc_idesc(S::BF16, S::MV, N, true, true);
        const Desc qd = tc_desc_sw128(smem_addr(sm + S::Q_OFF));
        const Desc kd = tc_desc_sw128(smem_addr(sm + S::KV_OFF));
        const Desc rd = tc_desc_sw128(smem_addr(sm + S::R_OFF));
        const Desc vd = tc_desc_mn<64>(smem_addr(sm + S::KV_OFF), S::ATOM);
        const Desc pd = tc_desc_mn<S::PW>(smem_addr(sm + S::P_OFF), KT * S::PW * 2);
        Pieces<KT> p(a, ctl);
        int g0 = 0;                                         // tiles of the earlier pieces
        int kslot = 0, vslot = 0;                           // ring slots of the next scores' and values' tile
        bool ok = true;
        while (ok && p.next()) {
          const int nt = p.t1 - p.t0;
          ok = wait_or_fail(&ctl->qfull, (uint32_t)(p.index & 1), fail, status);
          int ts = 0, tv = 0;                               // next tile's scores, next tile's second product
          uint64_t since = 0;                               // when it last found nothing ready
          int idle = 0;
          while (ok && tv < nt) {
            const int gs = g0 + ts, gv = g0 + tv;
            // what is ready is looked up together: a product should not wait for more than one look
            // (S^T buffer gs & 1 has been read once tile ts - 2 is past its softmax, that is once ts <= tv + 1)
            const bool can_s = ts < nt && ts <= tv + 1 &&
                               mbar_test(&ctl->kfull[gs % S::AHEAD], (uint32_t)((gs / S::AHEAD) & 1));
            bool can_v = tv < ts && mbar_test(&ctl->pfull[gv % S::NP], (uint32_t)((gv / S::NP) & 1));
            if (!S::SHARED)
              can_v = can_v && mbar_test(&ctl->vfull[gv % S::AHEAD], (uint32_t)((gv / S::AHEAD) & 1));
            if (can_v) {
              if (tv == 0 && p.index > 0)                   // the previous piece's outputs have been read
                ok = wait_or_fail(&ctl->ofree, (uint32_t)((p.index - 1) & 1), fail, status);
              if (!ok) break;
              tc_fence_after();
              const Desc ps = pd.at(gv % S::NP * S::PBUF).opaque();
              int s = S::SHARED ? vslot : vslot + 1 == S::SLOTS ? 0 : vslot + 1;
#pragma unroll
              for (int mb = 0; mb < S::NB; ++mb) {
                const Desc vs = vd.at(s * S::SLOT).opaque();
#pragma unroll
                for (int kk = 0; kk < KT / 16; ++kk)
                  tc_mma_ss(tO + (uint32_t)(mb * N), vs.at(kk * 2048), ps.at(kk * 16 * S::PW * 2), idO,
                            tv > 0 || kk > 0 ? 1u : 0u);
                tc_commit(&ctl->empty[s]);
                if (++s == S::SLOTS) s = 0;
              }
              tc_commit(&ctl->pvdone[gv % S::NP]);
              vslot = s;
              ++tv;
              idle = 0;
            }
            if (can_s) {
              tc_fence_after();
              const uint32_t d = tbase + (uint32_t)((gs & 1) * N);
              constexpr int kAtoms = S::SLOT / S::ATOM, kChunks = S::SHARED ? CH : 1;
              int s = kslot;
#pragma unroll
              for (int j = 0; j < kChunks; ++j) {
                const Desc ks = kd.at(s * S::SLOT).opaque(), qs = qd.at(j * kAtoms * S::QATOM).opaque();
#pragma unroll
                for (int kk = 0; kk < kAtoms * 4; ++kk)
                  tc_mma_ss(d, ks.at((kk >> 2) * S::ATOM + (kk & 3) * 32), qs.at((kk >> 2) * S::QATOM + (kk & 3) * 32),
                            idS, j > 0 || kk > 0 ? 1u : 0u);
                if (!S::SHARED) tc_commit(&ctl->empty[s]);
                if (++s == S::SLOTS) s = 0;
              }
              if constexpr (S::SHARED) {
                const int r = gs % S::ROPE;
                const Desc ks = rd.at(r * S::ATOM).opaque(), qs = qd.at(S::VA * S::QATOM).opaque();
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) tc_mma_ss(d, ks.at(kk * 32), qs.at(kk * 32), idS, 1u);
                tc_commit(&ctl->rempty[r]);
                kslot = s;
              } else {
                kslot = s + 1 == S::SLOTS ? 0 : s + 1;      // past the tile's values
              }
              tc_commit(&ctl->sfull[gs & 1]);
              ++ts;
              if (ts == nt) tc_commit(&ctl->qempty);
              idle = 0;
            }
            if (can_s || can_v) continue;
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
          g0 += nt;
        }
        tc_commit(&ctl->drained);
      }
    }
  } else {
    regs_up<S::RS>();
    // ---------------------------------------------------------------- softmax
    float* red = reinterpret_cast<float*>(sm + S::RED_OFF);
    uint32_t* vis = reinterpret_cast<uint32_t*>(sm + S::VIS_OFF);
    const int q = warp & 3, grp = warp >> 2;             // lane quarter (keys), rows grp C .. + C - 1
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    const int key = q * L + (lane & (L - 1));            // this thread's key of a tile, and its first row
    const int col0 = grp * C + (L == 16 ? (lane >> 4) * CS : 0);
    // A warp whose wait ran out stops waiting but still meets the barriers, so none is left waiting.
    bool dead = false;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (!dead) dead = !__all_sync(0xffffffffu, wait_or_fail(bar, parity, fail, status));
      tc_fence_after();
    };
    bool arrived = false;                                 // at the cluster's barrier
    Pieces<KT> p(a, ctl);
    int g = 0;                                            // tiles met by this CTA so far
    while (p.next()) {
      const int nt = p.t1 - p.t0, kvh = p.kvh, row0 = p.rb * N;
      const int rows = std::min(N, a.R - row0);
      const bool has_tree = a.tree && p.t1 == p.tiles;
      if (has_tree) {                                     // for every drafted token, the rows that see it
        bar_sync(5, S::SOFT);                             // (the previous piece's reads are done)
        if (threadIdx.x == 0) ctl->nonfinite = 0;
#pragma unroll
        for (int w = 0; w < S::VW; ++w) {
          const int r = w * 32 + lane, tok = (row0 + r) / a.G;
          const uint64_t bits = r < rows ? a.mask[(int64_t)p.b * a.n + tok] : 0;
          for (int j = warp; j < a.n; j += S::SOFT / 32) {
            const unsigned word = __ballot_sync(0xffffffffu, (bits >> j & 1) != 0);
            if (lane == 0) vis[j * S::VW + w] = word;
          }
        }
        bar_sync(5, S::SOFT);
      }
      float m[CS], l[CS];
#pragma unroll
      for (int c = 0; c < CS; ++c) {
        m[c] = kNoMax;
        l[c] = 0.f;
      }
      const float4* r4 = reinterpret_cast<const float4*>(red + col0);
      for (int t = 0; t < nt; ++t, ++g) {
        const int pb = g % S::NP;
        const bool tr = has_tree && t == nt - 1;
        const int valid = tr ? a.n : std::min(KT, p.len - (p.t0 + t) * KT);   // keys of the tile that exist
        wait(&ctl->sfull[g & 1], (uint32_t)((g >> 1) & 1));
        float v[CS];
        if constexpr (L == 16)
          tm_load_halves<CS>(tbase + lanes + (uint32_t)((g & 1) * N + grp * C), v);
        else
          tm_load<CS>(tbase + lanes + (uint32_t)((g & 1) * N + grp * C), v);
        bool over = false;
        if (valid == KT && !tr) {
#pragma unroll
          for (int c = 0; c < CS; ++c) {
            v[c] *= a.scale_log2;
            over |= v[c] > m[c] + kRaise;
          }
        } else {
          // the rows of this thread that see its key
          uint32_t see = key < valid ? 0xffffffffu : 0u;
          if (tr && key < valid) see = vis[key * S::VW + col0 / 32] >> (col0 % 32);
#pragma unroll
          for (int c = 0; c < CS; ++c) {
            v[c] = see >> c & 1 ? v[c] * a.scale_log2 : -INFINITY;
            over |= v[c] > m[c] + kRaise;
          }
        }
        if (bar_or(1 + grp, 128, over)) {
          // some score passed its row's maximum: raise the maxima to the tile's, rescale sums and outputs
          float w[CS];
#pragma unroll
          for (int c = 0; c < CS; ++c) w[c] = v[c];
          group_reduce<S>(w, red + q * N + col0, lane, grp, MaxOp());
#pragma unroll
          for (int c = 0; c < CS / 4; ++c) {
            const float4 x0 = r4[c], x1 = r4[N / 4 + c], x2 = r4[2 * N / 4 + c], x3 = r4[3 * N / 4 + c];
            const float mx[4] = {fmax3(x0.x, x1.x, fmaxf(x2.x, x3.x)), fmax3(x0.y, x1.y, fmaxf(x2.y, x3.y)),
                                 fmax3(x0.z, x1.z, fmaxf(x2.z, x3.z)), fmax3(x0.w, x1.w, fmaxf(x2.w, x3.w))};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float nm = fmaxf(m[4 * c + e], mx[e]);
              w[4 * c + e] = ex2_approx(m[4 * c + e] - nm);
              m[4 * c + e] = nm;
              l[4 * c + e] *= w[4 * c + e];
            }
          }
          if (t > 0) {
            // every thread needs its whole group's factors here: passed round through `red`
            bar_sync(1 + grp, 128);
            if (q == 0 && (lane & (L - 1)) == 0) {
#pragma unroll
              for (int c = 0; c < CS; ++c) red[col0 + c] = w[c];
            }
            bar_sync(1 + grp, 128);
            wait(&ctl->pvdone[(g - 1) % S::NP], (uint32_t)(((g - 1) / S::NP) & 1));
#pragma unroll 1
            for (int mb = 0; mb < S::NB; ++mb) {
              float o[C];
              tm_load<C>(tO + lanes + (uint32_t)(mb * N + grp * C), o);
#pragma unroll
              for (int c = 0; c < C; ++c) o[c] *= red[grp * C + c];
              tm_store<C>(tO + lanes + (uint32_t)(mb * N + grp * C), o);
            }
            tm_store_wait();
          }
        }
        // weights, their sums, and the rounded weights for the second product
        uint32_t pk[CS / 2];
#pragma unroll
        for (int c = 0; c < CS; c += 2) {
          const float p0 = ex2_approx(v[c] - m[c] + kOffset), p1 = ex2_approx(v[c + 1] - m[c + 1] + kOffset);
          l[c] += p0;
          l[c + 1] += p1;
          pk[c / 2] = pack2<S::BF16>(p0, p1);
        }
        if (g >= S::NP) wait(&ctl->pvdone[pb], (uint32_t)((g / S::NP - 1) & 1));
        uint8_t* pt = sm + S::P_OFF + pb * S::PBUF + (col0 / S::PW) * (KT * S::PW * 2);
        if constexpr (CS >= 8) {
#pragma unroll
          for (int i = 0; i < CS / 8; ++i)
            *reinterpret_cast<uint4*>(pt + mn_offset<S::PW>(key, (col0 % S::PW) / 8 + i)) =
                make_uint4(pk[4 * i], pk[4 * i + 1], pk[4 * i + 2], pk[4 * i + 3]);
        } else {
          *reinterpret_cast<uint2*>(pt + mn_offset<S::PW>(key, (col0 % S::PW) / 8) + (col0 % 8) * 2) =
              make_uint2(pk[0], pk[1]);
        }
        // Values that no row may meet must not meet a zero weight either (0 x NaN): slots past the length become
        // zeros; a drafted token's non-finite values become zeros here and are added to the rows that see it at
        // the end.  (Latent: the scores of this tile are complete, so its keys may be overwritten.)
        if (tr || valid < KT) {
          if (!S::SHARED) wait(&ctl->vfull[g % S::AHEAD], (uint32_t)((g / S::AHEAD) & 1));
          const int r0 = tr ? 0 : valid, r1 = tr ? a.n : KT;
#pragma unroll 1
          for (int e = threadIdx.x; e < (r1 - r0) * 8 * S::VA; e += S::SOFT) {
            const int r = r0 + e / (8 * S::VA), x = e % (8 * S::VA), at = x >> 3;
            const int s = (g * CH + (S::SHARED ? at / (S::MV / 64) : 1)) % S::SLOTS;
            uint4* p8 = reinterpret_cast<uint4*>(sm + S::KV_OFF + s * S::SLOT +
                                                 (S::SHARED ? at % (S::MV / 64) : at) * S::ATOM +
                                                 mn_offset<64>(r, x & 7));
            if (!tr) {
              *p8 = make_uint4(0, 0, 0, 0);
              continue;
            }
            uint4 raw = *p8;
            if (any_non_finite<S::BF16>(raw)) {
              bad_pairs<S::BF16>(raw);
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
      // -------------------------------------------------------------- this piece's outputs
      wait(&ctl->pvdone[(g - 1) % S::NP], (uint32_t)(((g - 1) / S::NP) & 1));
      if (a.cluster > 0) {
        cluster_arrive();                                  // (this warp is done with the ring)
        arrived = true;
      }
      const bool gone = bar_or(1 + grp, 128, dead);        // (the group's earlier reads of `red` are done)
      group_reduce<S>(l, red + q * N + col0, lane, grp, AddOp());
      if (a.cluster > 0) {                                 // its one piece: joined with the other CTAs' below
        if (q == 0 && (lane & (L - 1)) == 0) {
          float2* ml = reinterpret_cast<float2*>(sm + S::VIS_OFF);
#pragma unroll
          for (int c = 0; c < CS; ++c) {
            const int x = col0 + c;
            const float all = (red[x] + red[N + x]) + (red[2 * N + x] + red[3 * N + x]);
            ml[x] = make_float2(all == 0.f ? -INFINITY : m[c], all);
          }
        }
        break;
      }
      float sum[C];
      const float4* s4 = reinterpret_cast<const float4*>(red + grp * C);
#pragma unroll
      for (int c = 0; c < C / 4; ++c) {
        const float4 x0 = s4[c], x1 = s4[N / 4 + c], x2 = s4[2 * N / 4 + c], x3 = s4[3 * N / 4 + c];
        sum[4 * c] = (x0.x + x1.x) + (x2.x + x3.x);
        sum[4 * c + 1] = (x0.y + x1.y) + (x2.y + x3.y);
        sum[4 * c + 2] = (x0.z + x1.z) + (x2.z + x3.z);
        sum[4 * c + 3] = (x0.w + x1.w) + (x2.w + x3.w);
      }
      if (!gone) {
        const bool whole = nt == p.tiles;
        const int64_t slot = (int64_t)blockIdx.x * 2 + (p.index > 0 ? 1 : 0);
        const uint64_t nf = has_tree ? ctl->nonfinite : 0;
        const bool dlive = S::MV == 128 || lane < 16;
        const int dl = S::MV == 128 ? q * 32 + lane : q * 16 + (lane & 15);
        if (!whole && q == 0 && (lane & (L - 1)) == 0) {
#pragma unroll
          for (int c = 0; c < CS; ++c) {
            const int x = col0 + c;
            const float all = (red[x] + red[N + x]) + (red[2 * N + x] + red[3 * N + x]);
            a.part_ml[slot * N + x] = make_float2(all == 0.f ? -INFINITY : m[c], all);
          }
        }
        const uint32_t blind = whole ? blind_rows<C>(a, p.len, p.b, row0 + grp * C) : 0;
        if (whole) {
#pragma unroll
          for (int c = 0; c < C; ++c) sum[c] = blind >> c & 1 ? 0.f : sum[c] == 0.f ? NAN : 1.f / sum[c];
        }
#pragma unroll 1
        for (int mb = 0; mb < S::NB; ++mb) {
          const int d = mb * S::MV + dl;
          float o[C];
          tm_load<C>(tO + lanes + (uint32_t)(mb * N + grp * C), o);
          if (nf != 0) add_non_finite<S>(a, nf, p.b, kvh, row0 + grp * C, rows - grp * C, d, o);
          if (!whole) {
            float* po = a.part_o + (slot * N + grp * C) * S::DV + d;
            if (dlive) {
#pragma unroll
              for (int c = 0; c < C; ++c)
                if (grp * C + c < rows) po[c * S::DV] = o[c];
            }
          } else {
            // neighbouring lanes swap, so that each stores two dims of one row of a pair
            const bool odd = lane & 1;
#pragma unroll
            for (int c = 0; c < C; c += 2) {
              const float x0 = sum[c] == 0.f ? 0.f : o[c] * sum[c];
              const float x1 = sum[c + 1] == 0.f ? 0.f : o[c + 1] * sum[c + 1];
              const float y = __shfl_xor_sync(0xffffffffu, odd ? x0 : x1, 1);
              const uint32_t h = odd ? pack2<S::BF16>(y, x1) : pack2<S::BF16>(x0, y);
              const int r = grp * C + c + (odd ? 1 : 0), row = row0 + r;
              const int64_t at =
                  S::SHARED ? (int64_t)p.b * a.R + row
                            : ((int64_t)p.b * a.n + (row >> a.log_g)) * a.H + kvh * a.G + (row & (a.G - 1));
              if (r < rows && dlive) *reinterpret_cast<uint32_t*>(a.out + at * S::DV + (d & ~1)) = h;
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) tc_mbar_arrive(&ctl->ofree);
    }
    if (a.cluster > 0 && !arrived) cluster_arrive();      // (a CTA without a tile)
  }
  if (a.cluster > 0 && warp >= kLoad) {
    __syncwarp();
    cluster_arrive();
  }
  tc_fence_before();
  __syncthreads();
  if (a.cluster > 0) {
    // ---------------------------------------------------------------- the cluster's pieces joined
    // The ring is idle in every CTA past the barrier's wait.  Each sends slice i of its output's dims, unweighted, to
    // CTA i, its rows' (maximum, sum) to all; each then adds up its own slice.  Loops stay rolled: code that runs once
    // comes from a cold instruction cache, about 14 cycles an instruction (unrolled, the weights alone took 7000).
    const int per = a.Hkv * a.row_blocks, b = ctl->b0, u = (int)(blockIdx.x >> a.log_cluster) - b * per;
    const int kvh = u / a.row_blocks, row0 = u % a.row_blocks * N, rows = std::min(N, a.R - row0);
    const int len = ctl->len0, tiles = unit_tiles<KT>(a, len), rank = (int)cluster_rank();
    unsigned has = 0;                                                       // the CTAs that hold a piece
#pragma unroll 1
    for (int i = 0; i < a.cluster; ++i)
      has |= (cluster_tile(tiles, i, a.log_cluster) < cluster_tile(tiles, i + 1, a.log_cluster) ? 1u : 0u) << i;
    const int slice = S::DV >> a.log_cluster, log_s = 31 - __clz(slice);
    float* pieces = reinterpret_cast<float*>(sm + S::KV_OFF);               // [cluster][N][slice]
    float2* stats = reinterpret_cast<float2*>(pieces + N * S::DV);          // [cluster][N]; then x is the weight
    static_assert(N * S::DV * 4 + kMaxCluster * N * 8 <= S::SLOTS * S::SLOT + S::ROPE * S::ATOM &&
                      N * 8 <= kMaxTree * S::VW * 4,
                  "room for the join");
    tc_fence_after();
    cluster_wait();
    if (warp < kLoad && (has >> rank & 1)) {
      const int q = warp & 3, grp = warp >> 2;
      const float2* ml = reinterpret_cast<const float2*>(sm + S::VIS_OFF);  // [N]
      for (int e = threadIdx.x; e < N << a.log_cluster; e += S::SOFT)
        st_cluster2(cluster_addr(stats + rank * N + e % N, (uint32_t)(e / N)), ml[e % N]);
      const uint64_t nf = a.tree && cluster_tile(tiles, rank + 1, a.log_cluster) == tiles ? ctl->nonfinite : 0;
      constexpr int CJ = C > 16 ? 16 : C;                          // rows at a time (few registers are left here)
#pragma unroll 1
      for (int e = 0; e < S::NB * (C / CJ); ++e) {
        const int mb = e / (C / CJ), col = grp * C + e % (C / CJ) * CJ;
        const int d = mb * S::MV + (S::MV == 128 ? q * 32 + lane : q * 16 + (lane & 15));
        float o[CJ];
        tm_load<CJ>(tO + ((uint32_t)(q * 32) << 16) + (uint32_t)(mb * N + col), o);
        if (nf != 0) add_non_finite<S>(a, nf, b, kvh, row0 + col, rows - col, d, o);
        const uint32_t to =
            cluster_addr(pieces + ((rank * N + col) << log_s) + (d & (slice - 1)), (uint32_t)(d >> log_s));
        if (S::MV == 128 || lane < 16) {
#pragma unroll
          for (int c = 0; c < CJ; ++c)
            if (col + c < rows) st_cluster(to + ((uint32_t)c << (log_s + 2)), o[c]);
        }
      }
    }
    __syncwarp();
    cluster_sync();                                                // all pieces are here; none is sent any more
    if (warp < kLoad) {
      // eight lanes a row, one piece each
#pragma unroll 1
      for (int e = threadIdx.x; e < N * kMaxCluster; e += S::SOFT) {
        const int i = e % kMaxCluster;
        float2* x = stats + i * N + e / kMaxCluster;
        const float2 y = has >> i & 1 ? *x : make_float2(-INFINITY, 0.f);
        float M = y.x;
#pragma unroll
        for (int d = kMaxCluster / 2; d; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
        const float w = y.x == -INFINITY ? 0.f : ex2_approx(y.x - M);
        float sum = w * y.y;
#pragma unroll
        for (int d = kMaxCluster / 2; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (has >> i & 1) x->x = sum == 0.f ? NAN : w / sum;
      }
      bar_sync(5, S::SOFT);
      if (*fail == 0) {
        for (int e = threadIdx.x; e < rows << (log_s - 2); e += S::SOFT) {      // four dims of a row
          const int r = e >> (log_s - 2), ds = (e & ((slice >> 2) - 1)) * 4, row = row0 + r;
          float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int i = 0; i < a.cluster; ++i)
            if (has >> i & 1) {
              const float4 y = *reinterpret_cast<const float4*>(pieces + ((i * N + r) << log_s) + ds);
              const float w = stats[i * N + r].x;
              o.x += w * y.x;
              o.y += w * y.y;
              o.z += w * y.z;
              o.w += w * y.w;
            }
          if (len <= 0 && blind_rows<1>(a, len, b, row)) o = make_float4(0.f, 0.f, 0.f, 0.f);
          const int64_t at = S::SHARED ? (int64_t)b * a.R + row
                                       : ((int64_t)b * a.n + (row >> a.log_g)) * a.H + kvh * a.G + (row & (a.G - 1));
          *reinterpret_cast<uint2*>(a.out + at * S::DV + (rank << log_s) + ds) =
              make_uint2(pack2<S::BF16>(o.x, o.y), pack2<S::BF16>(o.z, o.w));
        }
      }
    }
  }
  // teardown: the products issued are complete; after a failure so are the copies (each wait bounded)
  if (threadIdx.x == 0) {
    tc_mbar_wait(&ctl->drained, 0, kRoleWaitNs);
    if (ctl->fail) {
      if (ctl->q_loads > 0) tc_mbar_wait(&ctl->qfull, (uint32_t)((ctl->q_loads - 1) & 1), kRoleWaitNs);
      for (int g = std::max(0, ctl->k_loads - S::AHEAD); g < ctl->k_loads; ++g)
        tc_mbar_wait(&ctl->kfull[g % S::AHEAD], (uint32_t)((g / S::AHEAD) & 1), kRoleWaitNs);
      for (int g = std::max(0, ctl->v_loads - S::AHEAD); g < ctl->v_loads; ++g)
        tc_mbar_wait(&ctl->vfull[g % S::AHEAD], (uint32_t)((g / S::AHEAD) & 1), kRoleWaitNs);
    }
  }
  __syncthreads();
  tc_fence_after();
  if (warp == kMma) tc_dealloc(tbase, S::TMEM);
}

// The units that several runs share: out = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s over their pieces; zeros for
// the units of an entry without any token.  A CTA takes 512 / DV rows, a thread four dims of one; the weights of a
// row's pieces are worked out side by side first, so that the pieces' loads do not wait for one another.  With many
// pieces a row PARTS groups of 128 threads take kAt pieces in turn, and their sums are added in the groups' order.
constexpr int kJoinWeights = 160;      // at most one piece per run
constexpr int kJoinThreads = 128;      // of a group
template <bool BF16, int KT, int DV, int PARTS>
__global__ void __launch_bounds__(kJoinThreads * PARTS) join_kernel(const RowsArgs a, int N) {
  constexpr int kPer = 512 / DV, kGrp = DV / 4;          // rows a CTA, threads a row
  __shared__ float sw[kPer][kJoinWeights], sred[4 * PARTS][2];
  __shared__ float4 ssum[PARTS > 1 ? PARTS - 1 : 1][kJoinThreads];
  pdl_wait_and_trigger();
  const int part = threadIdx.x / kJoinThreads, tid = threadIdx.x % kJoinThreads;
  const int g = tid / kGrp, x = tid % kGrp;
  const int64_t rows = (int64_t)a.B * a.Hkv * a.R, want = (int64_t)blockIdx.x * kPer + g;
  const int64_t row = want < rows ? want : rows - 1;     // (b Hkv + kvh) R + r
  const int64_t bh = row / a.R;
  const int r = (int)(row - bh * a.R), b = (int)(bh / a.Hkv), kvh = (int)(bh - (int64_t)b * a.Hkv);
  const int tiles = entry_tiles<KT>(a, b);
  const Joint jt = a.joint[bh * a.row_blocks + r / N];     // (not written for an entry without tiles)
  const int count = tiles > 0 ? jt.count : 1;
  // a piece's place in the workspace; piece i is of run jt.run + i
  // (a.side CTAs share a run: the row's block tells which of them)
  const int rn = r % N, step = a.side * 2 * N, at0 = jt.run * step + (a.side > 1 ? r / N : 0) * 2 * N + rn;
  auto place = [&](int i) { return at0 + i * step + (i == 0 ? jt.slot * N : 0); };
  // a group's threads of one row: a maximum and a sum over all of its pieces (all threads of the CTA take part)
  auto all = [&](float v, bool maximum, int slot) {
#pragma unroll
    for (int d = (kGrp < 32 ? kGrp : 32) / 2; d; d >>= 1) {
      const float y = __shfl_xor_sync(0xffffffffu, v, d);
      v = maximum ? fmaxf(v, y) : v + y;
    }
    if constexpr (kGrp > 32) {                           // a row of several warps
      const int w = threadIdx.x >> 5, w0 = w / (kGrp / 32) * (kGrp / 32);
      if ((threadIdx.x & 31) == 0) sred[w][slot] = v;
      __syncthreads();
      v = sred[w0][slot];
      for (int k = 1; k < kGrp / 32; ++k) v = maximum ? fmaxf(v, sred[w0 + k][slot]) : v + sred[w0 + k][slot];
    }
    return v;
  };
  float2 ml[(kJoinWeights + kGrp - 1) / kGrp];
  float M = -INFINITY, L = 0.f;
#pragma unroll
  for (int k = 0; k < (kJoinWeights + kGrp - 1) / kGrp; ++k) {
    const int i = k * kGrp + x;
    ml[k] = count > 1 && i < count ? a.part_ml[place(i)] : make_float2(-INFINITY, 0.f);
    M = fmaxf(M, ml[k].x);
  }
  M = all(M, true, 0);
#pragma unroll
  for (int k = 0; k < (kJoinWeights + kGrp - 1) / kGrp; ++k) {
    const int i = k * kGrp + x;
    const float w = ml[k].x == -INFINITY ? 0.f : ex2_approx(ml[k].x - M);
    if (part == 0 && i < kJoinWeights) sw[g][i] = w;
    L += w * ml[k].y;
  }
  L = all(L, false, 1);
  __syncthreads();
  const bool live = want < rows && (count > 1 || tiles <= 0);   // (else one run held the whole unit)
  const int d = x * 4;
  const int64_t at =
      (a.log_g < 0 ? row : ((int64_t)b * a.n + (r >> a.log_g)) * a.H + kvh * a.G + (r & (a.G - 1))) * DV + d;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  const float inv = L == 0.f ? NAN : 1.f / L;            // (a unit of several pieces has cached tokens: its rows see them)
  if (live && tiles > 0) {
    // kAt pieces' loads under way together, none behind a condition (past the last piece it is loaded again, unused)
    constexpr int kAt = DV >= 256 && PARTS == 1 ? 16 : 8;
    for (int i0 = part * kAt; i0 < count; i0 += kAt * PARTS) {
      float4 y[kAt];
#pragma unroll
      for (int k = 0; k < kAt; ++k)
        y[k] = *reinterpret_cast<const float4*>(a.part_o + (int64_t)place(std::min(i0 + k, count - 1)) * DV + d);
#pragma unroll
      for (int k = 0; k < kAt; ++k) {
        // (every piece that exists counts, also with a weight that rounds to zero: 0 x infinity has to show)
        const bool is = i0 + k < count;
        const float w = is ? sw[g][i0 + k] * inv : 0.f;
        o.x = is ? o.x + w * y[k].x : o.x;
        o.y = is ? o.y + w * y[k].y : o.y;
        o.z = is ? o.z + w * y[k].z : o.z;
        o.w = is ? o.w + w * y[k].w : o.w;
      }
    }
  }
  if constexpr (PARTS > 1) {
    if (part > 0) ssum[part - 1][tid] = o;
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int k = 0; k < PARTS - 1; ++k) {
      const float4 y = ssum[k][tid];
      o = make_float4(o.x + y.x, o.y + y.y, o.z + y.z, o.w + y.w);
    }
  }
  if (!live) return;
  uint2 h;
  h.x = pack2<BF16>(o.x, o.y);
  h.y = pack2<BF16>(o.z, o.w);
  *reinterpret_cast<uint2*>(a.out + at) = h;
}

// ---------------------------------------------------------------- host side
struct Plan {
  int N, KT, R, row_blocks, ctas;
  int cluster;                 // CTAs a unit; 0: runs
  int side;                    // CTAs that take a run together
  int64_t tiles;               // of all units when every entry is full
  size_t joint_off, ml_off, o_off, bytes;
};

Plan plan_rows(const RowsCall& c) {
  Plan p{};
  p.R = c.n * (c.H / c.Hkv);
  p.N = p.R <= 16 ? 16 : p.R <= 32 ? 32 : 64;
  p.KT = c.latent ? 64 : 128;
  p.row_blocks = (int)ceil_div(p.R, p.N);
  p.tiles = (ceil_div(c.T_cap, p.KT) + 1) * c.B * c.Hkv * p.row_blocks;
  p.ctas = (int)std::min<int64_t>(p.tiles, kNumSMs);
  // Clusters where as many as there are units run beside each other (one CTA an SM: 76 of 2, 36 of 4, 15 of 8) and no
  // CTA's share is much longer than an equal one: joining through the workspace costs about four tiles' time (two of
  // the 64-row tiles, which take longer), and a seventh of a long run's where HBM is the bound.  Measured, clusters
  // against runs: 16 drafted tokens over 8 x 8K (64 units) 49 against 53 us, 8 over 3000 tokens (8 units) 10.1 against
  // 13.5, one latent token over 8 x 1000 (8 units) 11.2 against 12.2, 8 x 4K 20.9 against 21.8; but 32 against 27 for one
  // latent token over 8 x 8K, and 36.6 against 31.9 for 5 over 8 x 4K (24 units, ragged).  The rule is a rough one: on
  // the side of the crossing that it takes for clusters', one latent token over 2000 tokens 12.9 against 11.2, over 32 x
  // 16K 105.9 against 104.3 (32 x 8K 59.3 against 61.0); on the other, 16 drafted over 3 x 8K 27.1 against 29.9, 5 over
  // 24 x 1000 (16 heads) 24.5 against 29.7 (24 x 4K 62 against 54).
  const int64_t units = (int64_t)c.B * c.Hkv * p.row_blocks, per_unit = ceil_div(c.T_cap, p.KT) + 1;
  const int64_t equal = ceil_div(per_unit * units, kNumSMs);
  const int64_t spare = (p.N <= 32 ? 4 : 2) + (p.row_blocks == 1 ? equal / 7 : 0);
  const int k = units <= 15 ? 8 : units <= 36 ? 4 : units <= 76 ? 2 : 0;
  p.cluster = k > 0 && ceil_div(per_unit, k) <= equal + spare ? k : 0;
  // A run for all row blocks at once where that leaves few SMs without one (12 tokens of 32 heads over 32K rows, 6
  // blocks: 25 x 6 CTAs; as 152 runs of single blocks the keys came from HBM 3.6 times).
  p.side = 1;
  if (p.cluster == 0 && p.row_blocks > 1 && p.ctas / p.row_blocks * p.row_blocks >= p.ctas * 7 / 8)
    p.side = p.row_blocks;
  const size_t parts = (size_t)p.ctas * 2 * p.N;       // (of the runs, so that the size does not fall with T_cap or n)
  p.joint_off = kCounterBytes;
  p.ml_off = p.joint_off + align256((size_t)c.B * c.Hkv * p.row_blocks * sizeof(Joint));
  p.o_off = p.ml_off + align256(parts * sizeof(float2));
  p.bytes = p.o_off + align256(parts * c.dv * sizeof(float));
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
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)std::max(1, p.cluster), 1, 1};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.cluster > 0 ? (unsigned)(B * Hkv * p.row_blocks * p.cluster)
                                    : (unsigned)(p.ctas / p.side * p.side));
  cfg.blockDim = dim3(S::THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = p.cluster > 0 ? 2 : 1;
  e = cudaLaunchKernelEx(&cfg, rows_kernel<S>, qm, km, vm, ktm, vtm, a);
  if (e == cudaSuccess) e = cudaPeekAtLastError();
  if (e != cudaSuccess || p.cluster > 0) return e;
  const unsigned grid = (unsigned)ceil_div(B * Hkv * p.R, 512 / S::DV);
  // Four groups where a unit has more pieces (about) than one takes at a time and the CTAs fit beside each other (one
  // latent token over 32000 rows 35.5 -> 25.6 us, over 8 x 8K 28.7 -> 26.8, 16 x 4K of 16 heads, 256 CTAs, 24.5 -> 23.5;
  // but of 32 heads, 512 CTAs, 26.8 -> 28.8, and with six pieces a unit, 16 drafted over 3 x 8K, 29.8 -> 31.1).
  if (p.ctas / (B * Hkv * p.row_blocks) >= 8 && grid <= 2 * kNumSMs)
    return launch_pdl(join_kernel<S::BF16, S::KT, S::DV, 4>, dim3(grid), dim3(4 * kJoinThreads), 0, st, a, (int)S::N);
  return launch_pdl(join_kernel<S::BF16, S::KT, S::DV, 1>, dim3(grid), dim3(kJoinThreads), 0, st, a, (int)S::N);
}

// rows a block, ring slots, last-key-atom slots, weight buffers: what an SM's shared memory holds
template <bool BF16>
cudaError_t launch_latent(const RowsCall& c, const Plan& p, const RowsArgs& a, cudaStream_t st) {
  if (c.dv == 512) {
    if (p.N == 16) return launch_shape<Shape<BF16, 9, 8, true, 64, 16, 10, 3, 2>>(c, p, a, st);
    if (p.N == 32) return launch_shape<Shape<BF16, 9, 8, true, 64, 32, 9, 3, 2>>(c, p, a, st);
    return launch_shape<Shape<BF16, 9, 8, true, 64, 64, 8, 2, 1>>(c, p, a, st);
  }
  if (p.N == 16) return launch_shape<Shape<BF16, 5, 4, true, 64, 16, 10, 4, 2>>(c, p, a, st);
  if (p.N == 32) return launch_shape<Shape<BF16, 5, 4, true, 64, 32, 9, 4, 2>>(c, p, a, st);
  return launch_shape<Shape<BF16, 5, 4, true, 64, 64, 8, 4, 2>>(c, p, a, st);
}

template <int KA, int SL>
cudaError_t launch_tree(const RowsCall& c, const Plan& p, const RowsArgs& a, cudaStream_t st) {
  if (p.N == 16) return launch_shape<Shape<false, KA, KA, false, 128, 16, SL, 0, 2>>(c, p, a, st);
  if (p.N == 32) return launch_shape<Shape<false, KA, KA, false, 128, 32, SL, 0, 2>>(c, p, a, st);
  return launch_shape<Shape<false, KA, KA, false, 128, 64, KA == 2 ? 5 : SL, 0, 2>>(c, p, a, st);
}

}  // namespace

size_t rows_ws_bytes(const RowsCall& c) { return plan_rows(c).bytes; }
bool rows_countable(const RowsCall& c) { return plan_rows(c).tiles <= INT32_MAX / 2; }

cudaError_t launch_rows_attention(const RowsCall& c, void* ws, cudaStream_t st) {
  const Plan p = plan_rows(c);
  RowsArgs a{};
  const cudaError_t e = status_word(&a.status);
  if (e != cudaSuccess) return e;
  a.B = c.B;
  a.n = c.n;
  a.H = c.H;
  a.Hkv = c.Hkv;
  a.G = c.H / c.Hkv;
  a.R = p.R;
  a.row_blocks = p.row_blocks;
  a.side = p.side;
  a.in_run = p.row_blocks / p.side;
  a.cluster = p.cluster;
  for (a.log_cluster = 0; (1 << a.log_cluster) < a.cluster;) ++a.log_cluster;
  a.log_g = -1;
  if (!c.latent)
    for (a.log_g = 0; (1 << a.log_g) < a.G;) ++a.log_g;
  a.tree = c.k_tree != nullptr;
  a.T_cap = c.T_cap;
  a.scale_log2 = c.scale * kLog2e;
  a.T_len = c.T_len;
  a.mask = c.mask;
  a.v_tree = static_cast<const uint16_t*>(c.latent ? c.k_tree : c.v_tree);
  a.v_tok = c.latent ? c.dk : (int64_t)c.Hkv * c.dv;
  a.v_head = c.latent ? 0 : c.dv;
  a.out = static_cast<uint16_t*>(c.out);
  a.joint = reinterpret_cast<Joint*>(static_cast<uint8_t*>(ws) + p.joint_off);
  a.part_ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(ws) + p.ml_off);
  a.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + p.o_off);
  if (c.latent) return c.dtype == MKV_BF16 ? launch_latent<true>(c, p, a, st) : launch_latent<false>(c, p, a, st);
  return c.dv == 128 ? launch_tree<2, 6>(c, p, a, st) : launch_tree<1, 10>(c, p, a, st);
}

}  // namespace mkv
