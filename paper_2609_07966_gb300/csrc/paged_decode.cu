// Attention of an entry's newest tokens, up to 32 query rows of a key head (tokens x heads of a group), over its 8-bit
// pages:
//   s_rt = scale log2(e) ks (q_r . k_t),  out_r = sum_t p_rt vs v_t / sum_t p_rt,  p_rt = 2^(s_rt - m_r)
// with codes k, v and their page's scales ks, vs, over the tokens t up to the row's own.
//
// Bound by memory: a token is 2 D bytes a key head.  All rows that share a key head meet every code, so a code is loaded
// once.  A warp takes 16 tokens at a time; codes go from shared memory to registers, are widened to fp16 there (exactly)
// and meet the rows as the narrow side of both products:
//   S [16 tokens x N rows] = K Q^T         the widened keys as they lie in the lanes that loaded them
//   O [D dims x N rows]   += V^T W         pairs of tokens interleaved while they are widened; W = the weights, transposed
//                                          between lanes
// The order of the dims (and of the tokens) within a product is free as long as both operands agree, so each lane takes
// whole 16-byte pieces of its rows.  Queries are fp16: bf16 ones are scaled by a power of two a row so that their largest
// is within 2^14 .. 2^15 (what that rounds away is 2^-39 of it).
//
// Two running maxima a row: m of the scores s, for the sum, and m2 of s + log2 vs, for the weights W = p vs 2^(m - m2 + 6),
// which the tensor cores take in fp16: pages of any scales then keep full precision.  Both are only raised once a score
// passes them by 2^8, so the accumulators are almost never rescaled.  Statistics and accumulators are fp32.
//
// Work: the chunks of all (entry, key head) units end to end, an equal run for every CTA whatever the entries' lengths
// (read on the device); pieces of a unit that several runs share go to the workspace, and the last CTA of the unit to
// arrive adds them up in their order.  One warp loads chunks by TMA, a page (or its part of the chunk) a copy.
#include <math.h>

#include <algorithm>

#include "mkv_paged.cuh"

namespace mkv {

namespace {

constexpr float kRaise = 8.f;       // a score may pass the running maximum by this (log2) before it is raised
constexpr float kOffset = 6.f;      // weights carry 2^kOffset: full precision in fp16 down to 2^-20 of the maximum
constexpr float kNoMax = -3.402823466e+38f;   // running maximum of a row that has seen nothing

struct DecodeArgs {
  PagedAttnCall c;
  uint32_t* status;
  int G;
  float scale_log2;                 // (e4m3: with the 2^8 that the widened codes lack)
  int box;                          // tokens of a page's copy: min(page, chunk)
  int* tickets;                     // [B][Hkv], zero between calls
  float* part_o;                    // [CTAs][2][N][D]
  float4* part_st;                  // [CTAs][2][N]: m, sum, m2
};

// N rows, W warps that compute (16 tokens of a chunk each), CTAS of them an SM.
template <int FMT_, int D_, int N_, int W_, int STAGES_, int CTAS_>
struct DShape {
  static constexpr int FMT = FMT_, D = D_, N = N_, W = W_, STAGES = STAGES_, CTAS = CTAS_;
  static constexpr int NT = N / 8, MB = D / 16, KS = D / 16;
  // With 32 rows a thread's accumulators need more registers than an equal share: then the loading warp is one of a
  // warpgroup of its own (three warps idle), and the groups split what the launch got.
  static constexpr bool SPLIT = N == 32;
  static constexpr int CHUNK = 16 * W, TILE = CHUNK * D, THREADS = 32 * W + (SPLIT ? 128 : 32);
  static constexpr int RL = 168, RC = 216, RO = 72;        // registers a thread: at launch, computing, loading
  static_assert(!SPLIT || (W == 8 && 2 * RC + RO <= 3 * RL), "register shares");
  static constexpr int KV_OFF = 0;                         // [STAGES][K, V]
  static constexpr int SC_OFF = STAGES * 2 * TILE;         // [STAGES][W] float4: key factor, mantissa and exponent of vs
  static constexpr int QF_OFF = SC_OFF + STAGES * W * 16;  // [KS][NT][32] uint2
  static constexpr int O_OFF = QF_OFF + KS * NT * 256;     // [N][D] floats
  static constexpr int ST_OFF = O_OFF + N * D * 4;         // [W][N] float4
  static constexpr int QS_OFF = ST_OFF + W * N * 16;       // [N] floats
  static constexpr int CTL_OFF = QS_OFF + N * 4;
  static constexpr int ALLOC = CTL_OFF + 256 + 1024;       // slack to align the base to 1024 B
  static constexpr int ROW = D;                            // bytes of a token's codes
  static_assert(CTAS * (ALLOC + 1024) <= 228 * 1024, "shared memory");
};

struct DecodeCtl {
  uint64_t full[8], empty[8];
  int64_t run0, run1, base, total, runs;
  int b0, fail, loads, last;
};
static_assert(sizeof(DecodeCtl) <= 256, "control block");

// Byte offset of 16-byte piece c of row r of a tile as TMA writes it (rows of 128 or 64 bytes, that swizzle).
template <int D>
__device__ __forceinline__ uint32_t code_offset(int r, int c) {
  return mn_offset<D / 2>(r, c);
}

__device__ __forceinline__ int entry_tokens(const PagedAttnCall& c, int b) {
  return (int)min((int64_t)max(c.T_len[b], 0), c.s.max_pages * c.s.page);
}
struct Entry {
  int64_t row0;
  int rows, len, chunks;           // new tokens, tokens held, chunks of a unit
};
template <int CHUNK>
__device__ __forceinline__ Entry entry_of(const DecodeArgs& a, int b, bool report) {
  const EntryRows r = entry_rows(a.c.s, b);
  Entry e;
  e.row0 = r.first;
  e.rows = (int)min(r.count, a.c.max_rows + 1);
  e.len = entry_tokens(a.c, b);
  if (e.rows > a.c.max_rows) {
    if (report) atomicOr(a.status, MKV_FLAG_BAD_INDEX);
    e.rows = 0;
  }
  e.chunks = e.rows > 0 ? max(1, (e.len + CHUNK - 1) / CHUNK) : 0;
  return e;
}

// A run's pieces: chunks c0 .. c1 - 1 of one unit at a time.
template <int CHUNK>
struct Pieces {
  const DecodeArgs& a;
  int64_t cur, end, base;          // next chunk of the run, its end, first chunk of entry b
  int b, index;
  Entry e;
  int kvh, c0, c1;
  __device__ __forceinline__ Pieces(const DecodeArgs& args, const DecodeCtl* c)
      : a(args), cur(c->run0), end(c->run1), base(c->base), b(c->b0), index(-1) {
    if (cur < end) e = entry_of<CHUNK>(a, b, false);
  }
  __device__ __forceinline__ bool next() {
    if (cur >= end) return false;
    while (cur >= base + (int64_t)e.chunks * a.c.s.Hkv) {
      base += (int64_t)e.chunks * a.c.s.Hkv;
      e = entry_of<CHUNK>(a, ++b, false);
    }
    const int64_t in = cur - base;
    kvh = (int)(in / e.chunks);
    c0 = (int)(in - (int64_t)kvh * e.chunks);
    c1 = (int)min((int64_t)e.chunks, c0 + (end - cur));
    cur += c1 - c0;
    ++index;
    return true;
  }
};

__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

template <class S>
__global__ void __launch_bounds__(S::THREADS, S::CTAS)
    decode_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const DecodeArgs a) {
  constexpr int D = S::D, N = S::N, NT = S::NT, W = S::W, CHUNK = S::CHUNK, MB = S::MB, KS = S::KS, SOFT = 32 * W;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  DecodeCtl* ctl = reinterpret_cast<DecodeCtl*>(sm + S::CTL_OFF);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PagedAttnCall& c = a.c;
  const int Hkv = c.s.Hkv;
  uint32_t* status = a.status;
  volatile int* fail = &ctl->fail;

  if (warp == W) {
    if (lane == 0) {
      prefetch_map(&kmap);
      prefetch_map(&vmap);
      for (int s = 0; s < S::STAGES; ++s) {
        tc_mbar_init(&ctl->full[s], 1);
        tc_mbar_init(&ctl->empty[s], W);
      }
      tc_fence_mbar_init();
      ctl->fail = ctl->loads = 0;
    }
    pdl_wait_and_trigger();
    // all units' chunks, then this CTA's run of them and the entry that holds its first
    int64_t total = 0;
    for (int b = lane; b < c.s.B; b += 32) total += (int64_t)entry_of<CHUNK>(a, b, blockIdx.x == 0).chunks * Hkv;
#pragma unroll
    for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    const int64_t runs = max((int64_t)1, min((int64_t)gridDim.x, total));     // none of them empty
    const int64_t run0 = blockIdx.x < runs ? total * blockIdx.x / runs : 0;
    const int64_t run1 = blockIdx.x < runs ? total * (blockIdx.x + 1) / runs : 0;
    int64_t base = 0;
    int b0 = 0;
    for (int b = 0; b < c.s.B && run0 < run1; b += 32) {
      const int64_t mine = b + lane < c.s.B ? (int64_t)entry_of<CHUNK>(a, b + lane, false).chunks * Hkv : 0;
      int64_t upto = mine;                                 // inclusive prefix within the 32
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += x;
      }
      const unsigned past = __ballot_sync(0xffffffffu, base + upto > run0);
      if (past) {
        const int w = __ffs(past) - 1;
        b0 = b + w;
        base += __shfl_sync(0xffffffffu, upto - mine, w);
        break;
      }
      base += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) {
      ctl->run0 = run0;
      ctl->run1 = run1;
      ctl->base = base;
      ctl->total = total;
      ctl->runs = runs;
      ctl->b0 = b0;
    }
  } else {
    pdl_wait_and_trigger();
  }
  __syncthreads();

  if (warp >= W) {
    if constexpr (S::SPLIT) regs_down<S::RO>();
  }
  if (warp == W) {
    // ---------------------------------------------------------------- loads
    // A batch is 32 copies' pages, a lane each: page and scales of the next batch are fetched during this one.
    const int per = CHUNK / a.box, span = 32 / per;        // copies a chunk, chunks a batch
    const int box16 = a.box / 16;
    Pieces<CHUNK> p(a, ctl);
    int g = 0;
    bool ok = true;
    while (ok && p.next()) {
      const int32_t* table = c.s.page_table + (int64_t)p.b * c.s.max_pages;
      auto page_of = [&](int chunk) {                      // of this lane's copy of the batch from `chunk` on
        const int64_t t = (int64_t)chunk * CHUNK + (int64_t)lane * a.box;
        if (chunk + lane / per >= p.c1 || t >= p.e.len) return -1;
        return table[t / c.s.page];
      };
      // (a page outside the pool is not seen)
      auto check = [&](int chunk, int pid) {
        const int64_t t = (int64_t)chunk * CHUNK + (int64_t)lane * a.box;
        if (chunk + lane / per >= p.c1 || t >= p.e.len) return -1;
        if (pid < 0 || pid >= c.s.num_pages) {
          atomicOr(status, MKV_FLAG_BAD_INDEX);
          return -1;
        }
        return pid;
      };
      int pid = check(p.c0, page_of(p.c0)), next = 0;
      float ks = 0.f, vs = 1.f, nks = 0.f, nvs = 1.f;
      if (pid >= 0) {
        ks = c.k_scale[(int64_t)pid * Hkv + p.kvh];
        vs = c.v_scale[(int64_t)pid * Hkv + p.kvh];
      }
      for (int ch = p.c0; ok && ch < p.c1; ++ch, ++g) {
        const int in = (ch - p.c0) % span, from = ch - in;
        if (in == 0 && ch > p.c0) {
          pid = next;
          ks = nks;
          vs = nvs;
        }
        if (in == 0) next = page_of(ch + span);
        if (in == span / 2) {
          next = check(from + span, next);
          nks = 0.f;
          nvs = 1.f;
          if (next >= 0) {
            nks = c.k_scale[(int64_t)next * Hkv + p.kvh];
            nvs = c.v_scale[(int64_t)next * Hkv + p.kvh];
          }
        }
        const int s = g % S::STAGES;
        if (g >= S::STAGES) ok = wait_or_fail(&ctl->empty[s], (uint32_t)((g / S::STAGES - 1) & 1), fail, status);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const int mine = in * per + lane;                  // the copy that lane < per makes
        const int id = __shfl_sync(0xffffffffu, pid, mine & 31);
        // scales of the chunk's groups of 16 tokens
        const int owner = in * per + (lane < W ? lane / box16 : 0);
        const float gk = __shfl_sync(0xffffffffu, ks, owner), gv = __shfl_sync(0xffffffffu, vs, owner);
        const int gid = __shfl_sync(0xffffffffu, pid, owner);
        if (lane < W) {
          int e;
          const float m = frexpf(gv, &e);
          reinterpret_cast<float4*>(sm + S::SC_OFF)[s * W + lane] =
              make_float4(gk * a.scale_log2, m, (float)e, gid >= 0 ? 1.f : 0.f);
        }
        const bool copy = lane < per && id >= 0;
        const int copies = __popc(__ballot_sync(0xffffffffu, copy));
        __syncwarp();
        if (lane == 0) {
          tc_mbar_expect_tx(&ctl->full[s], (uint32_t)copies * 2 * a.box * S::ROW);
          ctl->loads = g + 1;
        }
        __syncwarp();
        if (copy) {
          uint8_t* dst = sm + S::KV_OFF + s * 2 * S::TILE + lane * a.box * S::ROW;
          const int64_t t = (int64_t)ch * CHUNK + (int64_t)lane * a.box;
          const int y = (int)(t % c.s.page), z = id * Hkv + p.kvh;
          tma_load_4d(dst, &kmap, 0, y, z, 0, &ctl->full[s]);
          tma_load_4d(dst + S::TILE, &vmap, 0, y, z, 0, &ctl->full[s]);
        }
      }
    }
  } else if (warp < W) {
    if constexpr (S::SPLIT) regs_up<S::RC>();
    // ---------------------------------------------------------------- attention
    const int lg = lane >> 2, lr = lane & 3;
    uint2* qf = reinterpret_cast<uint2*>(sm + S::QF_OFF);
    float* qs = reinterpret_cast<float*>(sm + S::QS_OFF);
    float* ob = reinterpret_cast<float*>(sm + S::O_OFF);
    float4* stat = reinterpret_cast<float4*>(sm + S::ST_OFF);
    const bool bf16 = c.s.dtype == MKV_BF16;
    Pieces<CHUNK> p(a, ctl);
    int g = 0;
    bool dead = false;
    while (p.next()) {
      const int G = a.G, R = p.e.rows * G;
      auto q_row = [&](int row) {                          // (of a row that exists)
        return c.q + (p.e.row0 + row / G) * c.q_stride + (int64_t)(p.kvh * G + row % G) * D;
      };
      // ------------------------------------------------------------ queries: fp16, in the lanes' order
      for (int row = warp; row < N; row += W) {            // powers of two that bf16 rows are scaled by
        float most = 0.f;
        if (bf16 && row < R)
          for (int d = lane; d < D; d += 32) {
            const float x = fabsf(widen<true>(q_row(row)[d]));
            most = fmaxf(most, x < INFINITY ? x : 0.f);
          }
        most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
        // 2^(141 - exponent field of the largest): its own power is at most 2^127 and at least 2^-113
        const int e = most > 0.f ? max(-113, min(127, 14 + 127 - (int)(__float_as_uint(most) >> 23))) : 0;
        if (lane == 0) qs[row] = __uint_as_float((uint32_t)(127 + (bf16 ? e : 0)) << 23);
      }
      bar_sync(1, SOFT);
      for (int e = threadIdx.x; e < KS * NT * 32; e += SOFT) {
        const int ks = e / (NT * 32), nt = e / 32 % NT, g8 = (e & 31) >> 2, r4 = e & 3, row = nt * 8 + g8;
        uint2 w = make_uint2(0u, 0u);
        if (row < R) w = *reinterpret_cast<const uint2*>(q_row(row) + r4 * (D / 4) + 4 * ks);
        if (bf16) {
          const float f = qs[row];
          w.x = pack2<false>(widen<true>((uint16_t)w.x) * f, widen<true>((uint16_t)(w.x >> 16)) * f);
          w.y = pack2<false>(widen<true>((uint16_t)w.y) * f, widen<true>((uint16_t)(w.y >> 16)) * f);
        }
        // (the order in which widen_codes gives four dims)
        qf[e] = make_uint2(__byte_perm(w.x, w.y, 0x5410), __byte_perm(w.x, w.y, 0x7632));
      }
      bar_sync(1, SOFT);
      float o[MB][NT][4], m[NT][2], m2[NT][2], l[NT][2], back[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          m[nt][j] = m2[nt][j] = kNoMax;
          l[nt][j] = 0.f;
          back[nt][j] = bf16 ? 1.f / qs[nt * 8 + 2 * lr + j] : 1.f;
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) o[mb][nt][j] = o[mb][nt][2 + j] = 0.f;
        }
      const int pos0 = p.e.len - p.e.rows;                 // the first new token's position
      for (int ch = p.c0; ch < p.c1; ++ch, ++g) {
        const int s = g % S::STAGES;
        if (!dead) dead = !__all_sync(0xffffffffu, wait_or_fail(&ctl->full[s], (uint32_t)((g / S::STAGES) & 1), fail, status));
        if (dead) break;
        const float4 sc = reinterpret_cast<const float4*>(sm + S::SC_OFF)[s * W + warp];
        const int t0 = ch * CHUNK + warp * 16;
        if (sc.w != 0.f && t0 < p.e.len) {
          const uint8_t* K = sm + S::KV_OFF + s * 2 * S::TILE + warp * 16 * S::ROW;
          const uint8_t* V = K + S::TILE;
          // -------------------------------------------------------- scores of tokens lg and lg + 8
          float x[NT][4];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) x[nt][0] = x[nt][1] = x[nt][2] = x[nt][3] = 0.f;
#pragma unroll
          for (int h = 0; h < KS / 4; ++h) {
            const int piece = lr * (KS / 4) + h;
            const uint4 k0 = *reinterpret_cast<const uint4*>(K + code_offset<D>(lg, piece));
            const uint4 k1 = *reinterpret_cast<const uint4*>(K + code_offset<D>(lg + 8, piece));
            const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t a0, a1, a2, a3;
              widen_codes<S::FMT>(w0[i], a0, a2);
              widen_codes<S::FMT>(w1[i], a1, a3);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                const uint2 b = qf[((h * 4 + i) * NT + nt) * 32 + lane];
                mma16816(x[nt], a0, a1, a2, a3, b.x, b.y);
              }
            }
          }
          // -------------------------------------------------------- weights
          const bool part = t0 + 15 > pos0;                // some row does not see all 16 tokens
          bool over = false;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float f = sc.x * back[nt][j];
              x[nt][j] *= f;
              x[nt][2 + j] *= f;
              if (part) {
                const int own = pos0 + (nt * 8 + 2 * lr + j) / G;    // the row's own position: the last that it sees
                if (t0 + lg > own) x[nt][j] = -INFINITY;
                if (t0 + lg + 8 > own) x[nt][2 + j] = -INFINITY;
              }
              const float t = fmaxf(x[nt][j], x[nt][2 + j]);
              over |= t > m[nt][j] + kRaise || t + sc.z > m2[nt][j] + kRaise;
            }
          if (__any_sync(0xffffffffu, over)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                float t = fmaxf(x[nt][j], x[nt][2 + j]);
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
                const float nm = fmaxf(m[nt][j], t), nm2 = fmaxf(m2[nt][j], t + sc.z);
                l[nt][j] *= ex2_approx(m[nt][j] - nm);
                const float w = ex2_approx(m2[nt][j] - nm2);
                m[nt][j] = nm;
                m2[nt][j] = nm2;
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) {
                  o[mb][nt][j] *= w;
                  o[mb][nt][2 + j] *= w;
                }
              }
          }
          uint32_t b0[NT], b1[NT];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float w[4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              // 2^(m - m2 + 6) vs, vs as mantissa and exponent (a product of the two could pass fp32's range)
              const float f = ex2_approx(m[nt][j] - m2[nt][j] + (kOffset + sc.z)) * sc.y;
              const float p0 = ex2_approx(x[nt][j] - m[nt][j]), p1 = ex2_approx(x[nt][2 + j] - m[nt][j]);
              l[nt][j] += p0 + p1;
              w[j] = p0 * f;
              w[2 + j] = p1 * f;
            }
            b0[nt] = transpose8(pack2<false>(w[0], w[1]));
            b1[nt] = transpose8(pack2<false>(w[2], w[3]));
          }
          // -------------------------------------------------------- values: dims D / 8 lg .. of tokens 2 lr, + 1, + 8, + 9
          uint32_t v[4][D / 32];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int row = 2 * lr + (i & 1) + 8 * (i >> 1);
            if constexpr (D == 128) {
              const uint4 y = *reinterpret_cast<const uint4*>(V + code_offset<D>(row, lg));
              v[i][0] = y.x;
              v[i][1] = y.y;
              v[i][2] = y.z;
              v[i][3] = y.w;
            } else {
              const uint2 y = *reinterpret_cast<const uint2*>(V + code_offset<D>(row, lg >> 1) + (lg & 1) * 8);
              v[i][0] = y.x;
              v[i][1] = y.y;
            }
          }
#pragma unroll
          for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {                  // dims 4 i + 2 h and the next, token pairs interleaved
              uint32_t a0, a1, a2, a3;
              widen_codes<S::FMT>(__byte_perm(v[0][i], v[1][i], h ? 0x7632 : 0x5410), a0, a1);
              widen_codes<S::FMT>(__byte_perm(v[2][i], v[3][i], h ? 0x7632 : 0x5410), a2, a3);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma16816(o[2 * i + h][nt], a0, a1, a2, a3, b0[nt], b1[nt]);
            }
        }
        __syncwarp();
        if (lane == 0) tc_mbar_arrive(&ctl->empty[s]);
      }
      // ------------------------------------------------------------ the warps' parts joined
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float t = l[nt][j];
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
          if (lg == 0) stat[warp * N + nt * 8 + 2 * lr + j] = make_float4(m[nt][j], t, m2[nt][j], 0.f);
        }
      bar_sync(1, SOFT);
      float M[NT][2], M2[NT][2], L[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float4* x = stat + nt * 8 + 2 * lr + j;
          float mx = kNoMax, mx2 = kNoMax, sum = 0.f;
#pragma unroll
          for (int w = 0; w < W; ++w) {
            mx = fmaxf(mx, x[w * N].x);
            mx2 = fmaxf(mx2, x[w * N].z);
          }
#pragma unroll
          for (int w = 0; w < W; ++w) sum += x[w * N].y * ex2_approx(x[w * N].x - mx);
          M[nt][j] = mx;
          M2[nt][j] = mx2;
          L[nt][j] = sum;
          const float f = ex2_approx(m2[nt][j] - mx2);
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) {
            o[mb][nt][j] *= f;
            o[mb][nt][2 + j] *= f;
          }
        }
      for (int w = 0; w < W; ++w) {                        // (in order, so that the sum is always the same)
        if (w == warp)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int mb = 0; mb < MB; ++mb) {
                float2* x = reinterpret_cast<float2*>(ob + (nt * 8 + 2 * lr + j) * D + (D / 8) * lg + 2 * mb);
                const float2 y = w == 0 ? make_float2(0.f, 0.f) : *x;
                *x = make_float2(y.x + o[mb][nt][j], y.y + o[mb][nt][2 + j]);
              }
        bar_sync(1, SOFT);
      }
      if (warp == 0 && lg == 0)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 2; ++j) stat[nt * 8 + 2 * lr + j] = make_float4(M[nt][j], L[nt][j], M2[nt][j], 0.f);
      bar_sync(1, SOFT);
      const bool gone = bar_or(1, SOFT, dead);
      // ------------------------------------------------------------ outputs, or a piece for the unit's last CTA
      constexpr int V4 = D / 4;
      // o / sum 2^(m2 - m - 6) (e4m3: + 8): the power as two factors, since it could pass fp32's range
      auto finish = [&](int row, float4 x, float mm, float sum, float mm2) {
        const bool blind = pos0 + row / G < 0;             // before position 0: it sees nothing
        const float h = ex2_approx(0.5f * (mm2 - mm - kOffset + (S::FMT == MKV_E4M3 ? 8.f : 0.f)));
        const float inv = sum == 0.f ? NAN : 1.f / sum;
        const float y[4] = {x.x * inv * h * h, x.y * inv * h * h, x.z * inv * h * h, x.w * inv * h * h};
        uint2 r;
        if (bf16)
          r = make_uint2(pack2<true>(y[0], y[1]), pack2<true>(y[2], y[3]));
        else
          r = make_uint2(pack2<false>(y[0], y[1]), pack2<false>(y[2], y[3]));
        return blind ? make_uint2(0u, 0u) : r;
      };
      auto out_row = [&](int row) {
        return c.out + (p.e.row0 + row / G) * c.out_stride + (int64_t)(p.kvh * G + row % G) * D;
      };
      if (p.c1 - p.c0 == p.e.chunks) {
        if (!gone)
          for (int e = threadIdx.x; e < R * V4; e += SOFT) {
            const int row = e / V4, d = e % V4 * 4;
            const float4 st = stat[row];
            *reinterpret_cast<uint2*>(out_row(row) + d) =
                finish(row, *reinterpret_cast<const float4*>(ob + row * D + d), st.x, st.y, st.z);
          }
      } else {
        const int64_t unit0 = p.base + (int64_t)p.kvh * p.e.chunks;
        auto run_start = [&](int64_t i) { return ctl->total * i / ctl->runs; };
        auto run_of = [&](int64_t x) { return (int)(((x + 1) * ctl->runs - 1) / ctl->total); };
        const int first = run_of(unit0), count = run_of(unit0 + p.e.chunks - 1) - first + 1;
        auto place = [&](int i) {                          // of the unit's piece i: the run's first piece or its last
          return ((int64_t)(first + i) * 2 + (i == 0 && run_start(first) < unit0 ? 1 : 0)) * N;
        };
        const int64_t mine = place((int)blockIdx.x - first);
        for (int e = threadIdx.x; e < R * V4; e += SOFT)
          reinterpret_cast<float4*>(a.part_o + mine * D)[e] = reinterpret_cast<const float4*>(ob)[e];
        if (threadIdx.x < R) a.part_st[mine + threadIdx.x] = stat[threadIdx.x];
        __threadfence();
        bar_sync(1, SOFT);
        if (threadIdx.x == 0) {
          int* ticket = a.tickets + (int64_t)p.b * Hkv + p.kvh;
          ctl->last = atomicAdd(ticket, 1) == count - 1;
          if (ctl->last) *ticket = 0;
        }
        bar_sync(1, SOFT);
        if (ctl->last) {
          __threadfence();
          constexpr int VL = D / 32;                       // dims a lane
          for (int row = warp; row < R; row += W) {        // a row a warp: its pieces' statistics, then their outputs
            float mx = kNoMax, mx2 = kNoMax, sum = 0.f, y[VL];
            for (int i = lane; i < count; i += 32) {
              const float4 st = __ldcg(a.part_st + place(i) + row);
              mx = fmaxf(mx, st.x);
              mx2 = fmaxf(mx2, st.z);
            }
#pragma unroll
            for (int d = 16; d; d >>= 1) {
              mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
              mx2 = fmaxf(mx2, __shfl_xor_sync(0xffffffffu, mx2, d));
            }
#pragma unroll
            for (int k = 0; k < VL; ++k) y[k] = 0.f;
            for (int i0 = 0; i0 < count; i0 += 32) {
              float w2 = 0.f;
              int64_t at = 0;
              if (i0 + lane < count) {
                at = place(i0 + lane) + row;
                const float4 st = __ldcg(a.part_st + at);
                sum += st.y * ex2_approx(st.x - mx);
                w2 = ex2_approx(st.z - mx2);
              }
              const int most = min(32, count - i0);
#pragma unroll 8
              for (int k = 0; k < most; ++k) {
                const float w = __shfl_sync(0xffffffffu, w2, k);
                const float* po = a.part_o + __shfl_sync(0xffffffffu, at, k) * D + lane * VL;
                float z[VL];
                if constexpr (VL == 4) {
                  const float4 f = __ldcg(reinterpret_cast<const float4*>(po));
                  z[0] = f.x;
                  z[1] = f.y;
                  z[2] = f.z;
                  z[3] = f.w;
                } else {
                  const float2 f = __ldcg(reinterpret_cast<const float2*>(po));
                  z[0] = f.x;
                  z[1] = f.y;
                }
#pragma unroll
                for (int q = 0; q < VL; ++q) y[q] += w * z[q];
              }
            }
#pragma unroll
            for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            const uint2 r = finish(row, make_float4(y[0], y[1], VL == 4 ? y[VL - 2] : 0.f, VL == 4 ? y[VL - 1] : 0.f), mx, sum, mx2);
            uint16_t* dst = out_row(row) + lane * VL;
            if (!gone) {
              if constexpr (VL == 4)
                *reinterpret_cast<uint2*>(dst) = r;
              else
                *reinterpret_cast<uint32_t*>(dst) = r.x;
            }
          }
        }
      }
      bar_sync(1, SOFT);                                   // (before the next piece's queries and sums)
    }
  }
  // teardown: after a failure the copies under way end first (each wait bounded)
  __syncthreads();
  if (threadIdx.x == 0 && ctl->fail)
    for (int x = std::max(0, ctl->loads - S::STAGES); x < ctl->loads; ++x)
      tc_mbar_wait(&ctl->full[x % S::STAGES], (uint32_t)((x / S::STAGES) & 1), kRoleWaitNs);
  __syncthreads();
}

// ---------------------------------------------------------------- host side
template <int FMT, int D, int N>
using ShapeOf = DShape<FMT, D, N, N == 32 ? 8 : 4, D == 128 ? 6 : 8, N == 32 ? 1 : 2>;

int block_rows(const PagedAttnCall& c) {
  const int64_t R = c.max_rows * (c.s.Hq / c.s.Hkv);
  return R <= 8 ? 8 : R <= 16 ? 16 : 32;
}

template <class S>
cudaError_t launch_shape(const PagedAttnCall& c, DecodeArgs a, void* ws, cudaStream_t st) {
  a.box = std::min(c.s.page, S::CHUNK);
  const int64_t heads = c.s.num_pages * c.s.Hkv;
  CUtensorMap km, vm;
  cudaError_t e = encode_code_map(&km, c.k, S::D, c.s.page, heads, a.box);
  if (e == cudaSuccess) e = encode_code_map(&vm, c.v, S::D, c.s.page, heads, a.box);
  if (e != cudaSuccess) return e;
  const int ctas = S::CTAS * kNumSMs;
  uint8_t* base = static_cast<uint8_t*>(ws);
  a.tickets = reinterpret_cast<int*>(base);
  a.part_st = reinterpret_cast<float4*>(base + kCounterBytes);
  a.part_o = reinterpret_cast<float*>(base + kCounterBytes + align256((size_t)ctas * 2 * S::N * sizeof(float4)));
  e = cudaFuncSetAttribute(decode_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::ALLOC);
  if (e != cudaSuccess) return e;
  return launch_pdl(decode_kernel<S>, dim3(ctas), dim3(S::THREADS), S::ALLOC, st, km, vm, a);
}

template <int FMT, int D>
cudaError_t launch_n(const PagedAttnCall& c, const DecodeArgs& a, void* ws, cudaStream_t st) {
  const int N = block_rows(c);
  if (N == 8) return launch_shape<ShapeOf<FMT, D, 8>>(c, a, ws, st);
  if (N == 16) return launch_shape<ShapeOf<FMT, D, 16>>(c, a, ws, st);
  return launch_shape<ShapeOf<FMT, D, 32>>(c, a, ws, st);
}

}  // namespace

size_t paged_decode_ws_bytes(const PagedAttnCall& c) {
  const size_t N = block_rows(c), slots = (size_t)(N == 32 ? 1 : 2) * kNumSMs * 2 * N;
  return kCounterBytes + align256(slots * sizeof(float4)) + align256(slots * c.s.D * sizeof(float));
}

cudaError_t launch_paged_decode(const PagedAttnCall& c, void* ws, cudaStream_t st) {
  DecodeArgs a{};
  const cudaError_t e = status_word(&a.status);
  if (e != cudaSuccess) return e;
  a.c = c;
  a.G = c.s.Hq / c.s.Hkv;
  a.scale_log2 = c.scale * kLog2e * (c.s.format == MKV_E4M3 ? kE4m3Up : 1.f);
  if (c.s.format == MKV_E4M3)
    return c.s.D == 128 ? launch_n<MKV_E4M3, 128>(c, a, ws, st) : launch_n<MKV_E4M3, 64>(c, a, ws, st);
  return c.s.D == 128 ? launch_n<MKV_I8, 128>(c, a, ws, st) : launch_n<MKV_I8, 64>(c, a, ws, st);
}

}  // namespace mkv
