// Attention of an entry's newest tokens, up to eight query rows of a key head (tokens x heads of a group), over its 8-bit
// pages:
//   s_rt = scale log2(e) ks (q_r . k_t),  out_r = sum_t p_rt vs v_t / sum_t p_rt,  p_rt = 2^(s_rt - m_r)
// with codes k, v and their page's scales ks, vs, over the tokens t up to the row's own.
//
// Bound by memory: a token is 2 D bytes a key head.  All rows that share a key head meet every code, so a code is loaded
// once.  A warp takes 32 tokens at a time, as two groups of 16 whose chains of instructions overlap; codes go from shared
// memory to registers, are widened to fp16 there (exactly) and meet the rows as the narrow side of both products:
//   S [16 tokens x 8 rows] = K Q^T         the widened keys as they lie in the lanes that loaded them
//   O [D dims x 8 rows]   += V^T W         pairs of tokens interleaved before they are widened; W = the weights, transposed
//                                          between lanes
// The order of the dims (and of the tokens) within a product is free as long as both operands agree, so each lane takes
// whole 16-byte pieces of its rows.  Queries are fp16 in registers (bf16 ones scaled by a power of two a row).  Statistics
// and accumulators are fp32.
//
// Work is shared out in runs of chunks (mkv_paged_work.cuh); one warp finds out its CTA's and loads it by TMA, a page a copy.
// A unit's pieces go to the workspace, and the CTA whose piece arrives last adds them up.  (Four times as many runs, taken in
// turn, even out what SMs get of HBM's bandwidth, but starting a piece costs more: 16 x 17-32K 146 against 130 us.)
//
// 16 x 17-32K tokens: 129 us, 0.94 of the measured copy rate; 8 x 8K: 31 us, 0.65 (a run of 14 chunks: the launch, the work's
// division and the first pages' chain take 6 us, a piece's end and the join 4); 777 tokens of one entry: 8.6 us, all of it that.
#include <math.h>

#include <algorithm>

#include "mkv_paged_softmax.cuh"
#include "mkv_paged_work.cuh"

namespace mkv {

namespace {

constexpr int N = 8;                // rows
constexpr int W = 4;                // warps that compute
static_assert(kTokens == 32 * W, "32 tokens of a chunk a warp");
constexpr int kComputing = 32 * W, kThreads = kComputing + 32;
constexpr int kCtas = 2;            // of them an SM
constexpr int kGrid = kCtas * kNumSMs;
struct DecodeArgs {
  PagedAttnCall c;
  uint32_t* status;
  Heads heads;
  WorkArgs w;
  int* tickets;                     // [B][Hkv], zero between calls
  float* part_o;                    // [kGrid][2][N][D]
  float4* part_st;                  // [kGrid][2][N]: m, sum, m2
};

template <int FMT_, int D_>
struct DShape {
  static constexpr int FMT = FMT_, D = D_, STAGES = D == 128 ? 3 : 6;
  static constexpr int TILE = kTokens * D;
  static constexpr int KV_OFF = 0;                         // [STAGES][K, V]
  static constexpr int SC_OFF = STAGES * 2 * TILE;         // scales of kBatches batches
  static constexpr int ST_OFF = SC_OFF + scale_bytes(kBatches);  // [W + 1][N] float4: the warps', the piece's
  static constexpr int HD_OFF = ST_OFF + (W + 1) * N * 16;      // [STAGES] Head
  static constexpr int Q_OFF = HD_OFF + STAGES * 64;       // [N][D] queries
  static constexpr int CTL_OFF = Q_OFF + N * D * 2;
  static constexpr int ALLOC = CTL_OFF + 256 + 1024;       // slack to align the base to 1024 B
  static constexpr int OROW = D + 16;                      // floats between rows of the warps' sums
  static_assert(STAGES < kBatches, "scales are kept");
  static_assert(kCtas * (ALLOC + 1024) <= 228 * 1024, "shared memory");
  static_assert(W * N * OROW * 4 <= 2 * TILE, "room for the warps' sums in a stage");
};

struct DecodeCtl {
  uint64_t full[6], empty[6], qfull, qempty, meet;
  int fail, loads, q_loads, last;
};
static_assert(sizeof(DecodeCtl) <= 256, "control block");

// Byte offset of 16-byte piece c of row r of a tile as TMA writes it (rows of 128 or 64 bytes, that swizzle).
template <int D>
__device__ __forceinline__ uint32_t code_offset(int r, int c) {
  return mn_offset<D / 2>(r, c);
}

__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

template <class S>
__global__ void __launch_bounds__(kThreads, kCtas)
    decode_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const DecodeArgs a) {
  constexpr int D = S::D, MB = D / 16, KS = D / 16;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  DecodeCtl* ctl = reinterpret_cast<DecodeCtl*>(sm + S::CTL_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PagedAttnCall& c = a.c;
  const int Hkv = c.s.Hkv;
  uint32_t* status = a.status;
  volatile int* fail = &ctl->fail;

  if (warp == W && lane == 0) {
    for (int s = 0; s < S::STAGES; ++s) {
      tc_mbar_init(&ctl->full[s], 2);                      // (its copies; its head and scales)
      tc_mbar_init(&ctl->empty[s], W);
    }
    tc_mbar_init(&ctl->qfull, 1);
    tc_mbar_init(&ctl->qempty, W);
    tc_mbar_init(&ctl->meet, W);
    tc_fence_mbar_init();
    ctl->fail = ctl->loads = ctl->q_loads = 0;
    prefetch_map(&kmap);
    prefetch_map(&vmap);
  }
  __syncthreads();
  pdl_wait_and_trigger();

  if (warp == W) {
    // ---------------------------------------------------------------- loads
    int g = 0, pieces = 0;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      return __all_sync(0xffffffffu, wait_or_fail(bar, parity, fail, status)) != 0;
    };
    auto free_stage = [&]() {
      return g < S::STAGES || wait(&ctl->empty[g % S::STAGES], (uint32_t)((g / S::STAGES - 1) & 1));
    };
    const int log_page = a.w.log_page;
    bool ok = work_through(
        c, a.w, status, reinterpret_cast<float2*>(sm + S::SC_OFF), lane,
        [&](const Piece& p) {                              // a piece's queries: one copy a token's heads
          if (pieces > 0 && !wait(&ctl->qempty, (uint32_t)((pieces - 1) & 1))) return false;
          const int bytes = a.heads.G * D * 2;
          if (lane == 0) {
            tc_mbar_expect_tx(&ctl->qfull, (uint32_t)(p.tokens * bytes));
            ctl->q_loads = pieces + 1;
          }
          __syncwarp();
          if (lane < p.tokens)
            bulk_load(sm + S::Q_OFF + lane * bytes, c.q + (int64_t)(p.row0 + lane) * c.q_stride + (int64_t)p.kvh * a.heads.G * D,
                      bytes, &ctl->qfull);
          ++pieces;
          return true;
        },
        [&](const Chunk& ch, const Piece& p, bool mine, int id, int at) {
          if (!free_stage()) return false;
          const int s = g % S::STAGES;
          if (lane == 0) {
            tc_mbar_expect_tx(&ctl->full[s], (uint32_t)(__popc(ch.copies) * 2 * D) << log_page);
            ctl->loads = g + 1;
          }
          __syncwarp();
          if (mine) {
            uint8_t* dst = sm + S::KV_OFF + s * 2 * S::TILE + (at << log_page) * D;
            const int z = id * Hkv + p.kvh;
            tma_load_4d(dst, &kmap, 0, 0, z, 0, &ctl->full[s]);
            tma_load_4d(dst + S::TILE, &vmap, 0, 0, z, 0, &ctl->full[s]);
          }
          return true;
        },
        [&](const Chunk& ch, const Piece& p) {
          Head* hd = reinterpret_cast<Head*>(sm + S::HD_OFF + g % S::STAGES * 64);
          if (lane == 31) hd->c = ch;
          if (lane == 31 && (ch.flags & kFirst)) hd->p = p;
          __syncwarp();
          if (lane == 0) tc_mbar_arrive(&ctl->full[g % S::STAGES]);
          ++g;
        });
    if (ok && free_stage()) {
      const int s = g % S::STAGES;
      if (lane == 0) {
        reinterpret_cast<Head*>(sm + S::HD_OFF + s * 64)->c.flags = kEnd;
        tc_mbar_arrive(&ctl->full[s]);
        tc_mbar_arrive(&ctl->full[s]);
      }
    }
  } else {
    // ---------------------------------------------------------------- attention
    const int lg = lane >> 2, lr = lane & 3;
    float4* stat = reinterpret_cast<float4*>(sm + S::ST_OFF);
    const bool bf16 = c.s.dtype == MKV_BF16;
    const int G = a.heads.G;
    bool dead = false;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (!dead) dead = !__all_sync(0xffffffffu, wait_or_fail(bar, parity, fail, status));
    };
    // A barrier of the computing warps whose waits are bounded too: one that gave up does not leave the others waiting.
    uint32_t met = 0;
    auto meet = [&]() {
      __syncwarp();
      if (lane == 0) tc_mbar_arrive(&ctl->meet);
      wait(&ctl->meet, met);
      met ^= 1;
    };
    // An output is o / sum 2^(m2 - m - 6); zeros for a row before position 0, which sees nothing; NaN where no score leaves a
    // weight.
    auto out_row = [&](const Piece& h, int row) {
      return c.out + (int64_t)(h.row0 + a.heads.token(row)) * c.out_stride + (int64_t)(h.kvh * G + a.heads.head(row)) * D;
    };
    auto finish = [&](const Piece& h, int row, float4 x, float mm, float sum, float mm2) {
      const float f = half_power(mm, mm2), inv = sum == 0.f ? NAN : 1.f / sum;
      x = make_float4(x.x * inv * f * f, x.y * inv * f * f, x.z * inv * f * f, x.w * inv * f * f);
      if (h.len - h.tokens + a.heads.token(row) < 0) x = make_float4(0.f, 0.f, 0.f, 0.f);
      return bf16 ? make_uint2(pack2<true>(x.x, x.y), pack2<true>(x.z, x.w))
                  : make_uint2(pack2<false>(x.x, x.y), pack2<false>(x.z, x.w));
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
        constexpr int VL = D / 32;                         // dims a lane
        for (int row = warp; row < owed.tokens * G; row += W) {   // a row a warp
          float mx, sum, mx2;
          const float4 y = add_pieces<VL>(owed, a.part_o, a.part_st, N, row, lane, mx, sum, mx2);
          const uint2 h = finish(owed, row, y, mx, sum, mx2);
          uint16_t* dst = out_row(owed, row) + lane * VL;
          if constexpr (VL == 4)
            *reinterpret_cast<uint2*>(dst) = h;
          else
            *reinterpret_cast<uint32_t*>(dst) = h.x;
        }
      }
      meet();                                              // (before `last` is set again)
      owed.count = 0;
    };

    uint32_t qf[2 * KS];
    float back[2], o[MB][4], m[2], m2[2], l[2];
    int pos0 = 0, own[2] = {0, 0}, pieces = 0;              // own: rows' own positions, the last that they see
    Piece hd;
    hd.len = hd.tokens = 0;
    // where this lane's pieces of a key row and of two value rows lie; further rows are whole swizzle periods away
    uint32_t kofs[D / 64], vofs[2];
#pragma unroll
    for (int h = 0; h < D / 64; ++h) kofs[h] = code_offset<D>(lg, lr * (D / 64) + h);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      vofs[i] = D == 128 ? code_offset<D>(2 * lr + i, lg) : code_offset<D>(2 * lr + i, lg >> 1) + (lg & 1) * 8;
    for (int g = 0;; ++g) {
      const int s = g % S::STAGES;
      wait(&ctl->full[s], (uint32_t)((g / S::STAGES) & 1));
      if (dead) break;
      const Head* from = reinterpret_cast<const Head*>(sm + S::HD_OFF + s * 64);
      const Chunk now = from->c;
      if (now.flags & kEnd) break;
      if (now.flags & kFirst) {
        hd = from->p;
        // ---------------------------------------------------------- queries: row lg, dims D / 4 lr ..
        wait(&ctl->qfull, (uint32_t)(pieces & 1));
        if (dead) break;
        ++pieces;
        const uint4* src = reinterpret_cast<const uint4*>(sm + S::Q_OFF + lg * D * 2 + lr * (D / 2));
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const uint4 y = lg < hd.tokens * G ? src[i] : make_uint4(0u, 0u, 0u, 0u);
          qf[4 * i] = y.x;
          qf[4 * i + 1] = y.y;
          qf[4 * i + 2] = y.z;
          qf[4 * i + 3] = y.w;
        }
        __syncwarp();
        if (lane == 0) tc_mbar_arrive(&ctl->qempty);
        back[0] = back[1] = 1.f;                           // what scores of rows 2 lr and 2 lr + 1 were scaled by
        if (bf16) {
          float most = 0.f;
#pragma unroll
          for (int i = 0; i < 2 * KS; ++i) {
            const float x0 = fabsf(widen<true>((uint16_t)qf[i])), x1 = fabsf(widen<true>((uint16_t)(qf[i] >> 16)));
            most = fmax3(most, x0 < INFINITY ? x0 : 0.f, x1 < INFINITY ? x1 : 0.f);
          }
          most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
          most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
          const int e = row_exponent(most);
          const float f = power_of_two(e);
#pragma unroll
          for (int i = 0; i < 2 * KS; ++i)
            qf[i] = pack2<false>(widen<true>((uint16_t)qf[i]) * f, widen<true>((uint16_t)(qf[i] >> 16)) * f);
#pragma unroll
          for (int j = 0; j < 2; ++j) back[j] = power_of_two(-__shfl_sync(0xffffffffu, e, (2 * lr + j) * 4));
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) o[mb][0] = o[mb][1] = o[mb][2] = o[mb][3] = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          m[j] = m2[j] = kNoMax;
          l[j] = 0.f;
        }
        pos0 = hd.len - hd.tokens;                         // the first new token's position
#pragma unroll
        for (int j = 0; j < 2; ++j) own[j] = pos0 + a.heads.token(2 * lr + j);
      }
      {
        const int ch = now.chunk;
        const int t0 = ch * kTokens + warp * 32;
        const float2* scales = reinterpret_cast<const float2*>(sm + S::SC_OFF) + now.scales;
        const int cp[2] = {(warp * 2) >> (a.w.log_page - 4), (warp * 2 + 1) >> (a.w.log_page - 4)};   // the groups' copies
        const float2 sc[2] = {scales[cp[0]], scales[cp[1]]};
        const bool in[2] = {(now.copies >> cp[0] & 1) != 0 && t0 < hd.len, (now.copies >> cp[1] & 1) != 0 && t0 + 16 < hd.len};
        if (in[0] || in[1]) {
          const uint8_t* K = sm + S::KV_OFF + s * 2 * S::TILE + warp * 32 * D;
          const uint8_t* V = K + S::TILE;
          // -------------------------------------------------------- scores of tokens lg and lg + 8 of each group
          uint32_t kw[2][2][D / 16];
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int h = 0; h < D / 64; ++h) {
                const uint4 y = *reinterpret_cast<const uint4*>(K + kofs[h] + (16 * u + 8 * i) * D);
                kw[u][i][4 * h] = y.x;
                kw[u][i][4 * h + 1] = y.y;
                kw[u][i][4 * h + 2] = y.z;
                kw[u][i][4 * h + 3] = y.w;
              }
          float x[2][4] = {};
#pragma unroll
          for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              uint32_t a0, a1, a2, a3;
              widen_codes<S::FMT>(kw[u][0][i], a0, a2);
              widen_codes<S::FMT>(kw[u][1][i], a1, a3);
              mma16816(x[u], a0, a1, a2, a3, qf[2 * i], qf[2 * i + 1]);
            }
          // -------------------------------------------------------- values: dims D / 8 lg .. of tokens 2 lr, + 1, + 8, + 9
          uint32_t v[2][4][D / 32];
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint8_t* src = V + vofs[i & 1] + (16 * u + 8 * (i >> 1)) * D;
              if constexpr (D == 128) {
                const uint4 y = *reinterpret_cast<const uint4*>(src);
                v[u][i][0] = y.x;
                v[u][i][1] = y.y;
                v[u][i][2] = y.z;
                v[u][i][3] = y.w;
              } else {
                const uint2 y = *reinterpret_cast<const uint2*>(src);
                v[u][i][0] = y.x;
                v[u][i][1] = y.y;
              }
            }
          if (!in[0] || !in[1] || t0 + 32 > hd.len) {      // (what no row may meet must not meet a zero weight as NaN)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (!in[u] || t0 + 16 * u + 2 * lr + (i & 1) + 8 * (i >> 1) >= hd.len)
#pragma unroll
                  for (int k = 0; k < D / 32; ++k) v[u][i][k] = 0u;
          }
          // -------------------------------------------------------- weights
          bool over = false;
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const bool part = !in[u] || t0 + 16 * u + 15 > pos0;     // some row does not see all 16 tokens
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float f = sc[u].x * back[j];
              x[u][j] *= f;
              x[u][2 + j] *= f;
              if (part) {
                if (!in[u] || t0 + 16 * u + lg > own[j]) x[u][j] = -INFINITY;
                if (!in[u] || t0 + 16 * u + lg + 8 > own[j]) x[u][2 + j] = -INFINITY;
              }
              const float t = fmaxf(x[u][j], x[u][2 + j]);
              over |= t > m[j] + kRaise || t + sc[u].y > m2[j] + kRaise;
            }
          }
          if (__any_sync(0xffffffffu, over)) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float y0 = fmaxf(x[0][j], x[0][2 + j]), y1 = fmaxf(x[1][j], x[1][2 + j]);
              float t = fmaxf(y0, y1), t2 = fmaxf(y0 + sc[0].y, y1 + sc[1].y);
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) {
                t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
                t2 = fmaxf(t2, __shfl_xor_sync(0xffffffffu, t2, d));
              }
              const float nm = fmaxf(m[j], t), nm2 = fmaxf(m2[j], t2);
              l[j] *= ex2_approx(m[j] - nm);
              const float w = ex2_approx(m2[j] - nm2);
              m[j] = nm;
              m2[j] = nm2;
#pragma unroll
              for (int mb = 0; mb < MB; ++mb) {
                o[mb][j] *= w;
                o[mb][2 + j] *= w;
              }
            }
          }
          uint32_t b0[2], b1[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            float w[4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float c2 = weight_shift(m[j], m2[j], sc[u].y);
              w[j] = ex2_approx(x[u][j] - m[j] + c2);
              w[2 + j] = ex2_approx(x[u][2 + j] - m[j] + c2);
              l[j] += (w[j] + w[2 + j]) * ex2_approx(-c2);
            }
            b0[u] = transpose8(pack2<false>(w[0], w[1]));
            b1[u] = transpose8(pack2<false>(w[2], w[3]));
          }
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
              for (int h = 0; h < 2; ++h) {                // dims 4 i + 2 h and the next, token pairs interleaved
                uint32_t a0, a1, a2, a3;
                widen_codes<S::FMT>(__byte_perm(v[u][0][i], v[u][1][i], h ? 0x7362 : 0x5140), a0, a1);
                widen_codes<S::FMT>(__byte_perm(v[u][2][i], v[u][3][i], h ? 0x7362 : 0x5140), a2, a3);
                mma16816(o[2 * i + h], a0, a1, a2, a3, b0[u], b1[u]);
              }
        }
        __syncwarp();
        if (lane == 0 && !(now.flags & kLast)) tc_mbar_arrive(&ctl->empty[s]);
      }
      if (!(now.flags & kLast)) continue;
      settle();                                            // (the piece before this one's unit)
      // ------------------------------------------------------------ the warps' parts joined, in their order
      // (As few instructions as will do: code that runs once a piece comes from a cold instruction cache.)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float t = l[j];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
        if (lg == 0) stat[warp * N + 2 * lr + j] = make_float4(m[j], t, m2[j], 0.f);
      }
      meet();
      if (dead) break;
      // The last chunk's stage, which no warp reads any more, takes the warps' sums: [W][N] rows, the dims that a lane holds
      // of each two 16 floats apart (lanes of a row then store 64 neighbouring bytes).
      float* ob = reinterpret_cast<float*>(sm + S::KV_OFF + s * 2 * S::TILE);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float4* x = stat + 2 * lr + j;
        float mx = kNoMax, mx2 = kNoMax, sum = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
          mx = fmaxf(mx, x[w * N].x);
          mx2 = fmaxf(mx2, x[w * N].z);
        }
#pragma unroll
        for (int w = 0; w < W; ++w) sum += x[w * N].y * ex2_approx(x[w * N].x - mx);
        const float f = ex2_approx(m2[j] - mx2);
        if (warp == 0 && lg == 0) stat[W * N + 2 * lr + j] = make_float4(mx, sum, mx2, 0.f);
        float* y = ob + (warp * N + 2 * lr + j) * S::OROW + 2 * lg;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
          *reinterpret_cast<float2*>(y + 16 * mb) = make_float2(o[mb][j] * f, o[mb][2 + j] * f);
      }
      meet();
      if (dead) break;
      // ------------------------------------------------------------ outputs, or a piece for the unit's last CTA
      const int R = hd.tokens * G;
      const bool whole = now.flags & kWhole;
      const int64_t mine = (int64_t)hd.mine * N;
#pragma unroll 1
      for (int e = threadIdx.x; e < R * (D / 4); e += kComputing) {
        const int row = e / (D / 4), d = e % (D / 4) * 4;
        const float* y = ob + row * S::OROW + d / (D / 8) * 2 + d % (D / 8) * 8;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const float2 y0 = *reinterpret_cast<const float2*>(y + w * N * S::OROW);
          const float2 y1 = *reinterpret_cast<const float2*>(y + w * N * S::OROW + 16);
          x = make_float4(x.x + y0.x, x.y + y0.y, x.z + y1.x, x.w + y1.y);
        }
        const float4 st = stat[W * N + row];
        if (whole) {
          *reinterpret_cast<uint2*>(out_row(hd, row) + d) = finish(hd, row, x, st.x, st.y, st.z);
        } else {
          __stcg(reinterpret_cast<float4*>(a.part_o + (mine + row) * D + d), x);
          if (d == 0) __stcg(a.part_st + mine + row, st);
        }
      }
      fence_async_smem();                                  // (before the stage is loaded again)
      meet();
      if (dead) break;
      if (lane == 0) tc_mbar_arrive(&ctl->empty[s]);
      if (!whole) {
        if (threadIdx.x == 0)
          asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(ticket) : "l"(a.tickets + hd.unit) : "memory");
        owed = hd;
      }
    }
    settle();
  }
  // teardown: after a failure the copies under way end first (each wait bounded)
  __syncthreads();
  if (threadIdx.x == 0 && ctl->fail) {
    if (ctl->q_loads > 0) tc_mbar_wait(&ctl->qfull, (uint32_t)((ctl->q_loads - 1) & 1), kRoleWaitNs);
    for (int x = std::max(0, ctl->loads - S::STAGES); x < ctl->loads; ++x)
      tc_mbar_wait(&ctl->full[x % S::STAGES], (uint32_t)((x / S::STAGES) & 1), kRoleWaitNs);
  }
  __syncthreads();
}

// ---------------------------------------------------------------- host side
template <class S>
cudaError_t launch_shape(const PagedAttnCall& c, DecodeArgs a, cudaStream_t st) {
  const int64_t heads = c.s.num_pages * c.s.Hkv;
  CUtensorMap km, vm;
  cudaError_t e = encode_code_map(&km, c.k, S::D, c.s.page, heads, c.s.page);
  if (e == cudaSuccess) e = encode_code_map(&vm, c.v, S::D, c.s.page, heads, c.s.page);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(decode_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::ALLOC);
  if (e != cudaSuccess) return e;
  return launch_pdl(decode_kernel<S>, dim3(kGrid), dim3(kThreads), S::ALLOC, st, km, vm, a);
}

}  // namespace

size_t paged_decode_ws_bytes(const PagedAttnCall& c) {
  return kCounterBytes + align256((size_t)kGrid * 2 * N * sizeof(float4)) + align256((size_t)kGrid * 2 * N * c.s.D * sizeof(float));
}

cudaError_t launch_paged_decode(const PagedAttnCall& c, void* ws, cudaStream_t st) {
  DecodeArgs a{};
  const cudaError_t e = status_word(&a.status);
  if (e != cudaSuccess) return e;
  a.c = c;
  a.heads = Heads(c.s.Hq / c.s.Hkv);
  a.w = work_args(c, kGrid, kAnyLost);
  uint8_t* base = static_cast<uint8_t*>(ws);
  a.tickets = reinterpret_cast<int*>(base);
  a.part_st = reinterpret_cast<float4*>(base + kCounterBytes);
  a.part_o = reinterpret_cast<float*>(base + kCounterBytes + align256((size_t)kGrid * 2 * N * sizeof(float4)));
  if (c.s.format == MKV_E4M3)
    return c.s.D == 128 ? launch_shape<DShape<MKV_E4M3, 128>>(c, a, st) : launch_shape<DShape<MKV_E4M3, 64>>(c, a, st);
  return c.s.D == 128 ? launch_shape<DShape<MKV_I8, 128>>(c, a, st) : launch_shape<DShape<MKV_I8, 64>>(c, a, st);
}

}  // namespace mkv
