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
// Work: the chunks of all (entry, key head) units end to end, an equal run for every CTA whatever the entries' lengths
// (read on the device); pieces of a unit that several runs share go to the workspace, and the last CTA of the unit to
// arrive adds them up in their order.  One warp loads chunks by TMA, a page (or its part of the chunk) a copy.
#include <math.h>

#include <algorithm>

#include "mkv_paged.cuh"

namespace mkv {

namespace {

constexpr int N = 8;                // rows
constexpr int W = 4;                // warps that compute
constexpr int kChunk = 32 * W;      // tokens
constexpr int kComputing = 32 * W, kThreads = kComputing + 32;
constexpr int kCtas = 2;            // of them an SM
constexpr size_t kRuns = kCtas * kNumSMs;

struct DecodeArgs {
  PagedAttnCall c;
  uint32_t* status;
  int G;
  float scale_log2;
  int box;                          // tokens of a page's copy: min(page, chunk)
  int* tickets;                     // [B][Hkv], zero between calls
  float* part_o;                    // [kRuns][2][N][D]
  float4* part_st;                  // [kRuns][2][N]: m, sum, m2
};

template <int FMT_, int D_>
struct DShape {
  static constexpr int FMT = FMT_, D = D_, STAGES = D == 128 ? 3 : 6;
  static constexpr int TILE = kChunk * D, GROUPS = kChunk / 16;
  static constexpr int KV_OFF = 0;                         // [STAGES][K, V]
  static constexpr int SC_OFF = STAGES * 2 * TILE;         // [STAGES][GROUPS] float4: key factor, mantissa and exponent of vs, seen
  static constexpr int O_OFF = SC_OFF + STAGES * GROUPS * 16;   // [W - 1][N][D] floats
  static constexpr int ST_OFF = O_OFF + (W - 1) * N * D * 4;    // [W][N] float4
  static constexpr int CTL_OFF = ST_OFF + W * N * 16;
  static constexpr int ALLOC = CTL_OFF + 256 + 1024;       // slack to align the base to 1024 B
  static_assert(kCtas * (ALLOC + 1024) <= 228 * 1024, "shared memory");
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
  e.chunks = e.rows > 0 ? max(1, (e.len + kChunk - 1) / kChunk) : 0;
  return e;
}

// A run's pieces: chunks c0 .. c1 - 1 of one unit at a time.
struct Pieces {
  const DecodeArgs& a;
  int64_t cur, end, base;          // next chunk of the run, its end, first chunk of entry b
  int b, index;
  Entry e;
  int kvh, c0, c1;
  __device__ __forceinline__ Pieces(const DecodeArgs& args, const DecodeCtl* c)
      : a(args), cur(c->run0), end(c->run1), base(c->base), b(c->b0), index(-1) {
    if (cur < end) e = entry_of(a, b, false);
  }
  __device__ __forceinline__ bool next() {
    if (cur >= end) return false;
    while (cur >= base + (int64_t)e.chunks * a.c.s.Hkv) {
      base += (int64_t)e.chunks * a.c.s.Hkv;
      e = entry_of(a, ++b, false);
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
    for (int b = lane; b < c.s.B; b += 32) total += (int64_t)entry_of(a, b, blockIdx.x == 0).chunks * Hkv;
#pragma unroll
    for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    const int64_t runs = max((int64_t)1, min((int64_t)gridDim.x, total));     // none of them empty
    const int64_t run0 = blockIdx.x < runs ? total * blockIdx.x / runs : 0;
    const int64_t run1 = blockIdx.x < runs ? total * (blockIdx.x + 1) / runs : 0;
    int64_t base = 0;
    int b0 = 0;
    for (int b = 0; b < c.s.B && run0 < run1; b += 32) {
      const int64_t mine = b + lane < c.s.B ? (int64_t)entry_of(a, b + lane, false).chunks * Hkv : 0;
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

  if (warp == W) {
    // ---------------------------------------------------------------- loads
    // A batch is 32 copies' pages, a lane each: page and scales of the next batch are fetched during this one.
    const int per = kChunk / a.box, span = 32 / per;        // copies a chunk, chunks a batch
    const int box16 = a.box / 16;
    Pieces p(a, ctl);
    int g = 0;
    bool ok = true;
    while (ok && p.next()) {
      const int32_t* table = c.s.page_table + (int64_t)p.b * c.s.max_pages;
      auto page_of = [&](int chunk) {                      // of this lane's copy of the batch from `chunk` on
        const int64_t t = (int64_t)chunk * kChunk + (int64_t)lane * a.box;
        if (chunk + lane / per >= p.c1 || t >= p.e.len) return -1;
        return table[t / c.s.page];
      };
      // (a page outside the pool is not seen)
      auto check = [&](int chunk, int pid) {
        const int64_t t = (int64_t)chunk * kChunk + (int64_t)lane * a.box;
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
        const int owner = in * per + (lane < S::GROUPS ? lane / box16 : 0);
        const float gk = __shfl_sync(0xffffffffu, ks, owner), gv = __shfl_sync(0xffffffffu, vs, owner);
        const int gid = __shfl_sync(0xffffffffu, pid, owner);
        if (lane < S::GROUPS) {
          int e;
          const float m = frexpf(gv, &e);
          reinterpret_cast<float4*>(sm + S::SC_OFF)[s * S::GROUPS + lane] =
              make_float4(gk * a.scale_log2, m, (float)e, gid >= 0 ? 1.f : 0.f);
        }
        const bool copy = lane < per && id >= 0;
        const int copies = __popc(__ballot_sync(0xffffffffu, copy));
        __syncwarp();
        if (lane == 0) {
          tc_mbar_expect_tx(&ctl->full[s], (uint32_t)copies * 2 * a.box * D);
          ctl->loads = g + 1;
        }
        __syncwarp();
        if (copy) {
          uint8_t* dst = sm + S::KV_OFF + s * 2 * S::TILE + lane * a.box * D;
          const int64_t t = (int64_t)ch * kChunk + (int64_t)lane * a.box;
          const int y = (int)(t % c.s.page), z = id * Hkv + p.kvh;
          tma_load_4d(dst, &kmap, 0, y, z, 0, &ctl->full[s]);
          tma_load_4d(dst + S::TILE, &vmap, 0, y, z, 0, &ctl->full[s]);
        }
      }
    }
  } else {
    // ---------------------------------------------------------------- attention
    const int lg = lane >> 2, lr = lane & 3;
    float* ob = reinterpret_cast<float*>(sm + S::O_OFF);
    float4* stat = reinterpret_cast<float4*>(sm + S::ST_OFF);
    const bool bf16 = c.s.dtype == MKV_BF16;
    Pieces p(a, ctl);
    int g = 0;
    bool dead = false;
    while (p.next()) {
      const int G = a.G, R = p.e.rows * G;
      // ------------------------------------------------------------ queries: row lg, dims D / 4 lr ..
      uint32_t qf[2 * KS];
      float back[2] = {1.f, 1.f};                          // what scores of rows 2 lr and 2 lr + 1 were scaled by
      {
        const uint4* src = reinterpret_cast<const uint4*>(c.q + (p.e.row0 + lg / G) * c.q_stride +
                                                          (int64_t)(p.kvh * G + lg % G) * D + lr * (D / 4));
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const uint4 y = lg < R ? src[i] : make_uint4(0u, 0u, 0u, 0u);
          qf[4 * i] = y.x;
          qf[4 * i + 1] = y.y;
          qf[4 * i + 2] = y.z;
          qf[4 * i + 3] = y.w;
        }
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
      }
      float o[MB][4], m[2] = {kNoMax, kNoMax}, m2[2] = {kNoMax, kNoMax}, l[2] = {0.f, 0.f};
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) o[mb][0] = o[mb][1] = o[mb][2] = o[mb][3] = 0.f;
      const int pos0 = p.e.len - p.e.rows;                 // the first new token's position
      for (int ch = p.c0; ch < p.c1; ++ch, ++g) {
        const int s = g % S::STAGES;
        if (!dead) dead = !__all_sync(0xffffffffu, wait_or_fail(&ctl->full[s], (uint32_t)((g / S::STAGES) & 1), fail, status));
        if (dead) break;
        const int t0 = ch * kChunk + warp * 32;
        const float4* scales = reinterpret_cast<const float4*>(sm + S::SC_OFF) + s * S::GROUPS + warp * 2;
        const float4 sc[2] = {scales[0], scales[1]};
        const bool in[2] = {sc[0].w != 0.f && t0 < p.e.len, sc[1].w != 0.f && t0 + 16 < p.e.len};
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
                const uint4 y = *reinterpret_cast<const uint4*>(K + code_offset<D>(16 * u + 8 * i + lg, lr * (D / 64) + h));
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
              const int row = 16 * u + 2 * lr + (i & 1) + 8 * (i >> 1);
              if constexpr (D == 128) {
                const uint4 y = *reinterpret_cast<const uint4*>(V + code_offset<D>(row, lg));
                v[u][i][0] = y.x;
                v[u][i][1] = y.y;
                v[u][i][2] = y.z;
                v[u][i][3] = y.w;
              } else {
                const uint2 y = *reinterpret_cast<const uint2*>(V + code_offset<D>(row, lg >> 1) + (lg & 1) * 8);
                v[u][i][0] = y.x;
                v[u][i][1] = y.y;
              }
              // (a token that no row may meet must not meet a zero weight as NaN)
              if (!in[u] || t0 + row >= p.e.len)
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
                const int own = in[u] ? pos0 + (2 * lr + j) / G : -1;    // the row's own position: the last that it sees
                if (t0 + 16 * u + lg > own) x[u][j] = -INFINITY;
                if (t0 + 16 * u + lg + 8 > own) x[u][2 + j] = -INFINITY;
              }
              const float t = fmaxf(x[u][j], x[u][2 + j]);
              over |= t > m[j] + kRaise || t + sc[u].z > m2[j] + kRaise;
            }
          }
          if (__any_sync(0xffffffffu, over)) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float y0 = fmaxf(x[0][j], x[0][2 + j]), y1 = fmaxf(x[1][j], x[1][2 + j]);
              float t = fmaxf(y0, y1), t2 = fmaxf(y0 + sc[0].z, y1 + sc[1].z);
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
              const float f = ex2_approx(m[j] - m2[j] + (kOffset + sc[u].z)) * sc[u].y;
              const float p0 = ex2_approx(x[u][j] - m[j]), p1 = ex2_approx(x[u][2 + j] - m[j]);
              l[j] += p0 + p1;
              w[j] = p0 * f;
              w[2 + j] = p1 * f;
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
        if (lane == 0) tc_mbar_arrive(&ctl->empty[s]);
      }
      // ------------------------------------------------------------ the warps' parts joined, in their order
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float t = l[j];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
        if (lg == 0) stat[warp * N + 2 * lr + j] = make_float4(m[j], t, m2[j], 0.f);
      }
      bar_sync(1, kComputing);
      float M[2], M2[2], L[2];
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
        M[j] = mx;
        M2[j] = mx2;
        L[j] = sum;
        const float f = ex2_approx(m2[j] - mx2);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
          o[mb][j] *= f;
          o[mb][2 + j] *= f;
          if (warp > 0)
            *reinterpret_cast<float2*>(ob + ((warp - 1) * N + 2 * lr + j) * D + (D / 8) * lg + 2 * mb) =
                make_float2(o[mb][j], o[mb][2 + j]);
        }
      }
      bar_sync(1, kComputing);
      if (warp == 0) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) {
            float2* x = reinterpret_cast<float2*>(ob + (2 * lr + j) * D + (D / 8) * lg + 2 * mb);
            float2 y = make_float2(o[mb][j], o[mb][2 + j]);
#pragma unroll
            for (int w = 0; w < W - 1; ++w) {
              y.x += x[w * N * D / 2].x;
              y.y += x[w * N * D / 2].y;
            }
            *x = y;
          }
          if (lg == 0) stat[2 * lr + j] = make_float4(M[j], L[j], M2[j], 0.f);
        }
      }
      const bool gone = bar_or(1, kComputing, dead);
      // ------------------------------------------------------------ outputs, or a piece for the unit's last CTA
      constexpr int V4 = D / 4;
      auto finish = [&](int row, float4 x, float mm, float sum, float mm2) {
        const bool blind = pos0 + row / G < 0;             // before position 0: it sees nothing
        const float h = half_power(mm, mm2);
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
          for (int e = threadIdx.x; e < R * V4; e += kComputing) {
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
        for (int e = threadIdx.x; e < R * V4; e += kComputing)
          reinterpret_cast<float4*>(a.part_o + mine * D)[e] = reinterpret_cast<const float4*>(ob)[e];
        if (threadIdx.x < R) a.part_st[mine + threadIdx.x] = stat[threadIdx.x];
        __threadfence();
        bar_sync(1, kComputing);
        if (threadIdx.x == 0) {
          int* ticket = a.tickets + (int64_t)p.b * Hkv + p.kvh;
          ctl->last = atomicAdd(ticket, 1) == count - 1;
          if (ctl->last) *ticket = 0;
        }
        bar_sync(1, kComputing);
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
      bar_sync(1, kComputing);                                   // (before the next piece's queries and sums)
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
template <class S>
cudaError_t launch_shape(const PagedAttnCall& c, DecodeArgs a, cudaStream_t st) {
  a.box = std::min(c.s.page, kChunk);
  const int64_t heads = c.s.num_pages * c.s.Hkv;
  CUtensorMap km, vm;
  cudaError_t e = encode_code_map(&km, c.k, S::D, c.s.page, heads, a.box);
  if (e == cudaSuccess) e = encode_code_map(&vm, c.v, S::D, c.s.page, heads, a.box);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(decode_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::ALLOC);
  if (e != cudaSuccess) return e;
  return launch_pdl(decode_kernel<S>, dim3(kRuns), dim3(kThreads), S::ALLOC, st, km, vm, a);
}

}  // namespace

size_t paged_decode_ws_bytes(const PagedAttnCall& c) {
  return kCounterBytes + align256(kRuns * 2 * N * sizeof(float4)) + align256((size_t)kRuns * 2 * N * c.s.D * sizeof(float));
}

cudaError_t launch_paged_decode(const PagedAttnCall& c, void* ws, cudaStream_t st) {
  DecodeArgs a{};
  const cudaError_t e = status_word(&a.status);
  if (e != cudaSuccess) return e;
  a.c = c;
  a.G = c.s.Hq / c.s.Hkv;
  a.scale_log2 = c.scale * kLog2e;
  uint8_t* base = static_cast<uint8_t*>(ws);
  a.tickets = reinterpret_cast<int*>(base);
  a.part_st = reinterpret_cast<float4*>(base + kCounterBytes);
  a.part_o = reinterpret_cast<float*>(base + kCounterBytes + align256(kRuns * 2 * N * sizeof(float4)));
  if (c.s.format == MKV_E4M3)
    return c.s.D == 128 ? launch_shape<DShape<MKV_E4M3, 128>>(c, a, st) : launch_shape<DShape<MKV_E4M3, 64>>(c, a, st);
  return c.s.D == 128 ? launch_shape<DShape<MKV_I8, 128>>(c, a, st) : launch_shape<DShape<MKV_I8, 64>>(c, a, st);
}

}  // namespace mkv
