// New tokens join an 8-bit paged cache, and their queries and keys are rotated on the way, in one launch:
//   e = least integer with max |x| <= top 2^e over a page's tokens of one head,  code = round(x 2^-e)
// (x a rotated key or a value, top 448 or 127).  A page that holds tokens already keeps its scale if the new ones fit it;
// else the codes that it holds are rounded again to the larger scale.
//
// Bound by memory: every row is read once, queries are written in 16 bits and keys and values in 8.  A slot is one page of
// one entry that the call writes into, with the rows that fall into it; its keys and values are units of one head each.
// A unit's rows stay in registers, as they were read, between its maximum and its codes (rotated twice: held in fp32 they left
// room for two CTAs an SM, and three prompts of 2-4K tokens took 80 us):
//   warps   a unit a warp, eight units a CTA: decode steps, and pages of 16 tokens (128 work columns);
//   blocks  a unit a CTA of 256 threads: larger pages filled by prompts.
// (One to nine rows of 64 entries: warps 8.9 us, blocks 22; three prompts in pages of 64 tokens: 76 and 63.)  One token of 8
// entries takes 5 us, its launch and two dependent loads.  One to nine rows of 64 entries are one wave (408 CTAs, three an SM):
// latency, a scheduler issues in a third of the cycles and a warp once in 13 (without the queries 8.1 us, without rotations
// too 6.3, 8 entries 6.7); a warp's unit spills 88 to 92 bytes at the 80 registers that three CTAs leave.  The three prompts, 10238 rows of 32 + 16 heads, run at 0.55 of the
// measured copy rate: keys and values alone take 30 us, bound by instructions (the maximum, the rotation twice, the codes) and
// by the latency of a unit's steps, which CTAs of the other kind fill in part.
// Other CTAs of the slot rotate its rows' queries, a thread the same dims of several heads.
//
// Every CTA reads its entry's length, and the last one to have read it (a ticket an entry) stores the new one.
#include <algorithm>

#include "mkv_paged.cuh"

namespace mkv {

namespace {

constexpr int kThreads = 256;
constexpr int kKeep = 4;            // columns of 16 dims that a thread holds
constexpr int kExpMin = -100, kExpMax = 120;

struct AppendArgs {
  PagedAppendCall c;
  uint32_t* status;
  int cap;                          // start null: slots of an entry
  int kv_ctas, q_ctas, q_heads;     // CTAs of a slot; heads of a query CTA
};

// Slots lie entry after entry: entry b's from slot_base(b) on, enough of them for m rows that begin anywhere in a page.
__device__ __forceinline__ int64_t slot_base(const AppendArgs& a, int b) {
  const int64_t r0 = min(max((int64_t)a.c.s.start[b], (int64_t)0), a.c.s.n);
  return (r0 + (int64_t)b * (2 * a.c.s.page - 2)) / a.c.s.page;
}
template <int FMT>
__device__ __forceinline__ constexpr float top_code() { return FMT == MKV_E4M3 ? 448.f : 127.f; }

// 2^e with e the least integer such that `most` <= top 2^e (its bits; finite and not negative).
template <int FMT>
__device__ __forceinline__ float least_scale(uint32_t most) {
  // most = m 2^x, 1/2 <= m < 1; top = 0.875 2^9 or (127/128) 2^7
  const int x = (int)(most >> 23) - 126;
  const uint32_t mant = most & 0x7fffffu;
  const bool over = FMT == MKV_E4M3 ? mant > 0x600000u : mant > 0x7e0000u;
  const int e = x - (FMT == MKV_E4M3 ? 9 : 7) + (over ? 1 : 0);
  return __uint_as_float((uint32_t)(127 + min(max(e, kExpMin), kExpMax)) << 23);
}

// The reciprocal of a power of two, exact; 0 for other scales (and the ends of the range), which have to be divided by.
__device__ __forceinline__ float exact_inverse(float s) {
  const uint32_t u = __float_as_uint(s), e = u >> 23;
  return (u & 0x7fffffu) == 0 && e >= 1 && e <= 253 ? __uint_as_float((254u - e) << 23) : 0.f;
}
// Eight codes, rounded to nearest even; SAFE: the largest ones beyond the range.
template <int FMT, bool SAFE>
__device__ __forceinline__ uint2 encode8(const float* x) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (FMT == MKV_E4M3) {
      uint16_t lo, hi;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[4 * i + 1]), "f"(x[4 * i]));
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[4 * i + 3]), "f"(x[4 * i + 2]));
      w[i] = (uint32_t)lo | (uint32_t)hi << 16;
    } else if (SAFE) {
      w[i] = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[i] |= ((uint32_t)min(max(__float2int_rn(x[4 * i + k]), -127), 127) & 0xffu) << (8 * k);
    } else {
      // (|x| <= 127: at 1.5 2^23 a unit is the last place, so the sum's low byte is x rounded)
      uint32_t u[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) u[k] = __float_as_uint(__fadd_rn(x[4 * i + k], 12582912.f));
      w[i] = __byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040), 0x5410);
    }
  }
  return make_uint2(w[0], w[1]);
}
// Four codes as their values.
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t w, float* x) {
  uint32_t lo, hi;
  widen_codes<FMT>(w, lo, hi);
  const float2 l = __half22float2(*reinterpret_cast<const __half2*>(&lo));
  const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  x[0] = l.x;
  x[1] = l.y;
  x[2] = h.x;
  x[3] = h.y;
}

// The rows of a slot: rows row0 .. row0 + count - 1 of the call, tokens at .. of page `pid`, which holds `held` tokens.
struct Slot {
  int64_t row0, token0;
  int count, at, held;
  int64_t pid;
};

// A column of 16 dims of a unit's row: two runs of eight dims, at lo and hi; `turn`: they are rotated.
struct Column {
  int i, col, lo, hi;
  bool turn;
};
template <int D>
__device__ __forceinline__ Column column_of(const AppendArgs& a, bool key, int e) {
  constexpr int kCols = D / 16;
  Column c;
  c.i = e / kCols;
  c.col = e % kCols;
  c.turn = key && c.col < a.c.rope.rot / 16;
  c.lo = c.turn ? turn_lo(c.col, a.c.rope.pairs) : 16 * c.col;
  c.hi = c.turn ? turn_hi(c.col, a.c.rope.rot, a.c.rope.pairs) : 16 * c.col + 8;
  return c;
}
template <int D>
__device__ __forceinline__ void load_column(const AppendArgs& a, const Slot& s, bool key, int h, int e, uint4& lo, uint4& hi) {
  const Column c = column_of<D>(a, key, e);
  const int64_t row = s.row0 + c.i;
  const uint16_t* p = (key ? a.c.k_new + row * a.c.k_stride : a.c.v_new + row * a.c.v_stride) + h * D;
  lo = *reinterpret_cast<const uint4*>(p + c.lo);
  hi = *reinterpret_cast<const uint4*>(p + c.hi);
}
// Its values, rotated.
template <int D, bool BF16>
__device__ __forceinline__ void turn_column(const AppendArgs& a, const Slot& s, const Column& c, const uint4& lo, const uint4& hi,
                                            float (&x)[16]) {
  widen8<BF16>(lo, x);
  widen8<BF16>(hi, x + 8);
  if (c.turn) {
    Turn8 t;
    t.load(turn_row(a.c.rope, a.c.pos != nullptr ? a.c.pos[s.row0 + c.i] : s.token0 + c.i, a.status), 8 * c.col);
    rotate16(x, t, a.c.rope.pairs, 1.f);
  }
}

// GROUP threads (a warp or the CTA) quantize one head's keys or values of a slot.  `lo`, `hi`: what this thread holds; `was`:
// the page's scale if it holds tokens.
template <int FMT, int D, bool BF16, int GROUP>
__device__ __forceinline__ void quantize_unit(const AppendArgs& a, const Slot& s, bool key, int h, const uint4 (&lo)[kKeep],
                                              const uint4 (&hi)[kKeep], float was) {
  constexpr int kCols = D / 16;
  const int tid = threadIdx.x % GROUP, items = s.count * kCols;
  const int64_t head = s.pid * a.c.s.Hkv + h;
  uint8_t* page = (key ? a.c.k : a.c.v) + head * a.c.s.page * D;
  uint32_t most = 0;
  bool bad = false;                                        // an infinity or NaN
  auto measure = [&](int e, const uint4& p0, const uint4& p1) {
    const Column c = column_of<D>(a, key, e);
    if (c.turn) {
      float y[16], top = 0.f, zero = 0.f;
      turn_column<D, BF16>(a, s, c, p0, p1, y);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        top = fmaxf(top, fabsf(y[i]));
        zero = fmaf(y[i], 0.f, zero);                      // (NaN if any value is not finite)
      }
      if (zero == 0.f) {
        most = max(most, __float_as_uint(top));
      } else {
        bad = true;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t u = __float_as_uint(y[i]) & 0x7fffffffu;
          most = max(most, u < 0x7f800000u ? u : 0u);
        }
      }
    } else {                                               // two values a word, as they are: their order is that of their bits
      constexpr uint32_t inf = BF16 ? 0x7f80u : 0x7c00u;
      const uint32_t w[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
      uint32_t top = max(m & 0xffffu, m >> 16);
      if (top >= inf) {
        bad = true;
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t x0 = w[i] & 0x7fffu, x1 = w[i] >> 16 & 0x7fffu;
          top = max(top, max(x0 < inf ? x0 : 0u, x1 < inf ? x1 : 0u));
        }
      }
      most = max(most, __float_as_uint(widen<BF16>((uint16_t)top)));
    }
  };
#pragma unroll
  for (int k = 0; k < kKeep; ++k)
    if (tid + k * GROUP < items) measure(tid + k * GROUP, lo[k], hi[k]);
  // (warps: more than 16 tokens of an entry that the others do not have; they are read again below)
  if (GROUP == 32)
    for (int e = tid + kKeep * GROUP; e < items; e += GROUP) {
      uint4 p0, p1;
      load_column<D>(a, s, key, h, e, p0, p1);
      measure(e, p0, p1);
    }
  if (bad) atomicOr(a.status, MKV_FLAG_NOT_FINITE);
  most = __reduce_max_sync(0xffffffffu, most);
  bool safe = __any_sync(0xffffffffu, bad);
  if constexpr (GROUP > 32) {
    __shared__ uint32_t of_warp[GROUP / 32];
    if ((tid & 31) == 0) of_warp[tid >> 5] = most;
    safe = __syncthreads_or(bad);
#pragma unroll
    for (int w = 0; w < GROUP / 32; ++w) most = max(most, of_warp[w]);
  }
  const bool fits = s.held > 0 && __uint_as_float(most) <= top_code<FMT>() * was;
  const float now = fits ? was : fmaxf(was, least_scale<FMT>(most));   // (a caller's scale may be above the largest)
  if (!fits) {
    if (tid == 0) (key ? a.c.k_scale : a.c.v_scale)[head] = now;
    if (s.held > 0) {
      const float less = __fdiv_rn(was, now);
      for (int e = tid; e < s.held * kCols; e += GROUP) {
        uint4* p = reinterpret_cast<uint4*>(page) + e;
        const uint4 old = *p;
        float y[16];
        decode4<FMT>(old.x, y);
        decode4<FMT>(old.y, y + 4);
        decode4<FMT>(old.z, y + 8);
        decode4<FMT>(old.w, y + 12);
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] *= less;
        const uint2 n0 = encode8<FMT, true>(y), n1 = encode8<FMT, true>(y + 8);
        *p = make_uint4(n0.x, n0.y, n1.x, n1.y);
      }
    }
  }
  safe |= __uint_as_float(most) > top_code<FMT>() * now;   // (beyond the largest scale)
  const float inv = exact_inverse(now);
  auto store = [&](int e, const uint4& p0, const uint4& p1) {
    const Column c = column_of<D>(a, key, e);
    float y[16];
    turn_column<D, BF16>(a, s, c, p0, p1, y);
    uint8_t* row = page + (int64_t)(s.at + c.i) * D;
    if (inv != 0.f && !safe) {
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] *= inv;
      *reinterpret_cast<uint2*>(row + c.lo) = encode8<FMT, false>(y);
      *reinterpret_cast<uint2*>(row + c.hi) = encode8<FMT, false>(y + 8);
    } else {
#pragma unroll 1
      for (int i = 0; i < 2; ++i) {
        float z[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float x = i == 0 ? y[k] : y[8 + k];
          z[k] = x == x ? __fdiv_rn(x, now) : 0.f;
        }
        *reinterpret_cast<uint2*>(row + (i == 0 ? c.lo : c.hi)) = encode8<FMT, true>(z);
      }
    }
  };
#pragma unroll
  for (int k = 0; k < kKeep; ++k)
    if (tid + k * GROUP < items) store(tid + k * GROUP, lo[k], hi[k]);
  if (GROUP == 32)
    for (int e = tid + kKeep * GROUP; e < items; e += GROUP) {
      uint4 p0, p1;
      load_column<D>(a, s, key, h, e, p0, p1);
      store(e, p0, p1);
    }
}

// The queries of a slot's rows, heads h0 .. h1 - 1.
template <int D, bool BF16>
__device__ __forceinline__ void rotate_queries(const AppendArgs& a, const Slot& s, int h0, int h1) {
  constexpr int kCols = D / 16;
  const PagedAppendCall& c = a.c;
  const int items = s.count * kCols, side = max(1, min(h1 - h0, kThreads / items));   // heads side by side
  for (int e = threadIdx.x; e < items * side; e += kThreads) {
    const int sh = e / items, item = e - sh * items, i = item / kCols, col = item % kCols;
    const int64_t row = s.row0 + i;
    const bool turn = col < c.rope.rot / 16;
    const int lo = turn ? turn_lo(col, c.rope.pairs) : 16 * col, hi = turn ? turn_hi(col, c.rope.rot, c.rope.pairs) : 16 * col + 8;
    Turn8 t;
    if (turn) t.load(turn_row(c.rope, c.pos != nullptr ? c.pos[row] : s.token0 + i, a.status), 8 * col);
    const uint16_t* x = c.q + row * c.q_stride;
    uint16_t* out = c.q_out + row * c.q_out_stride;
    constexpr int U = 2;                                  // heads whose loads are under way together
    for (int h = h0 + sh; h < h1; h += U * side) {
      uint4 p0[U], p1[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (h + u * side < h1) {
          p0[u] = *reinterpret_cast<const uint4*>(x + (h + u * side) * D + lo);
          p1[u] = *reinterpret_cast<const uint4*>(x + (h + u * side) * D + hi);
        }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h + u * side >= h1) break;
        if (turn) {
          float v[16];
          widen8<BF16>(p0[u], v);
          widen8<BF16>(p1[u], v + 8);
          rotate16(v, t, c.rope.pairs, 1.f);
          p0[u] = narrow8<BF16>(v);
          p1[u] = narrow8<BF16>(v + 8);
        }
        *reinterpret_cast<uint4*>(out + (h + u * side) * D + lo) = p0[u];
        *reinterpret_cast<uint4*>(out + (h + u * side) * D + hi) = p1[u];
      }
    }
  }
}

template <int FMT, int D, bool BF16, int GROUP>
__global__ void __launch_bounds__(kThreads, 3) append_kernel(const AppendArgs a) {
  pdl_wait_and_trigger();
  const PagedAppendCall& c = a.c;
  const int page = c.s.page;
  // A slot's CTAs follow one another, so that those of the queries, which bandwidth bounds, run beside those of keys and
  // values, which latency does (all keys and values first: 65 us for three prompts of 2-4K tokens).
  const int per = a.kv_ctas + a.q_ctas, slot = blockIdx.x / per, sub = blockIdx.x - slot * per;
  int b, j;                                                // the slot's entry; its page, counted from the entry's first
  int64_t slots;                                           // of the entry
  if (c.s.start == nullptr) {
    b = slot / a.cap;
    j = slot - b * a.cap;
    slots = a.cap;
  } else {
    b = find_entry(c.s.B, threadIdx.x & 31, [&](int e) { return slot_base(a, e) <= slot; });
    const int64_t base = slot_base(a, b);
    j = (int)(slot - base);
    slots = slot_base(a, b + 1) - base;
    if (j < 0 || j >= slots) return;                       // (behind the last entry's)
  }
  const EntryRows rows = entry_rows(c.s, b);
  if (rows.count == 0) return;
  const int t = c.T_len[b];
  const int64_t t0 = max(t, 0);
  Slot s;
  const int off = (int)(t0 & (page - 1)), i0 = max(0, j * page - off), i1 = min(rows.count, (j + 1) * page - off);
  s.row0 = rows.first + i0;
  s.token0 = (int64_t)t + i0;
  s.count = i1 - i0;
  s.at = j == 0 ? off : 0;
  s.held = s.at;
  const int64_t first = t0 / page, last = (t0 + (int64_t)rows.count - 1) / page;
  const bool ok = t >= 0 && last < c.s.max_pages;
  const int32_t* table = c.s.page_table + b * c.s.max_pages;
  const bool here = s.count > 0, keys = sub < a.kv_ctas;
  const int unit = sub * (kThreads / GROUP) + threadIdx.x / GROUP, h = unit < c.s.Hkv ? unit : unit - c.s.Hkv;
  const bool mine = here && keys && unit < 2 * c.s.Hkv, key = unit < c.s.Hkv;
  // what a unit needs is asked for before the entry's other pages are looked at
  s.pid = here && ok ? table[first + j] : -1;
  uint4 lo[kKeep], hi[kKeep];
  float was = 0.f;
  if (mine) {
#pragma unroll
    for (int k = 0; k < kKeep; ++k) {
      const int e = threadIdx.x % GROUP + k * GROUP;
      if (e < s.count * (D / 16)) load_column<D>(a, s, key, h, e, lo[k], hi[k]);
    }
    if (s.held > 0 && s.pid >= 0 && s.pid < c.s.num_pages) was = (key ? c.k_scale : c.v_scale)[s.pid * c.s.Hkv + h];
  }
  bool pages = true;
  if (ok)
    for (int64_t p = first + threadIdx.x; p <= last; p += kThreads) {
      const int pid = table[p];
      pages = pages && pid >= 0 && pid < c.s.num_pages;
    }
  pages = __syncthreads_and(pages);
  int ticket = 0;                                          // (looked at below, so that nothing waits for it)
  if (threadIdx.x == 0) ticket = atomicAdd(c.tickets + b, 1);
  if (here && !keys) {
    const int h0 = (sub - a.kv_ctas) * a.q_heads;
    rotate_queries<D, BF16>(a, s, h0, min(h0 + a.q_heads, c.s.Hq));
  } else if (mine && ok && pages) {
    quantize_unit<FMT, D, BF16, GROUP>(a, s, key, h, lo, hi, was);
  }
  if (threadIdx.x == 0 && ticket == (int)slots * per - 1) {   // every CTA of the entry has read its length
    c.tickets[b] = 0;
    if (!ok || !pages)
      atomicOr(a.status, ok ? MKV_FLAG_BAD_INDEX : MKV_FLAG_CACHE_FULL);
    else
      c.T_len[b] = (int)(t0 + rows.count);
  }
}

template <int FMT, int D, bool BF16>
cudaError_t launch_d(const AppendArgs& args, int64_t slots, bool warps, cudaStream_t st) {
  AppendArgs a = args;
  a.kv_ctas = warps ? (int)ceil_div(2 * a.c.s.Hkv, kThreads / 32) : 2 * a.c.s.Hkv;
  const int64_t ctas = slots * (a.kv_ctas + a.q_ctas);
  if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)ctas);
  if (warps) return launch_pdl(append_kernel<FMT, D, BF16, 32>, grid, dim3(kThreads), 0, st, a);
  return launch_pdl(append_kernel<FMT, D, BF16, kThreads>, grid, dim3(kThreads), 0, st, a);
}
template <int FMT>
cudaError_t launch_f(const AppendArgs& a, int64_t slots, bool warps, cudaStream_t st) {
  const bool bf16 = a.c.s.dtype == MKV_BF16;
  if (a.c.s.D == 128)
    return bf16 ? launch_d<FMT, 128, true>(a, slots, warps, st) : launch_d<FMT, 128, false>(a, slots, warps, st);
  return bf16 ? launch_d<FMT, 64, true>(a, slots, warps, st) : launch_d<FMT, 64, false>(a, slots, warps, st);
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppendCall& c, cudaStream_t st) {
  AppendArgs a{};
  const cudaError_t e = status_word(&a.status);
  if (e != cudaSuccess) return e;
  a.c = c;
  const int64_t m = ceil_div(c.s.n, c.s.B), page = c.s.page;
  a.cap = (int)((m + page - 2) / page + 1);
  const int64_t slots = c.s.start == nullptr ? c.s.B * (int64_t)a.cap : (c.s.n + c.s.B * (2 * page - 2)) / page;
  if (slots > INT32_MAX) return cudaErrorInvalidConfiguration;
  // A warp holds 128 columns: a page of 16 tokens, or the few tokens an entry of a decode step.
  const bool warps = std::min(m, page) * (c.s.D / 16) <= 32 * kKeep;
  // (without a rotation, queries that stay where they are need nothing)
  const bool queries = c.q != nullptr && !(c.rope.rot == 0 && c.q_out == c.q);
  // (heads of a query CTA, 32 and 8: one to nine rows of 64 entries 8.9 and 11.2 us, three prompts 81 and 63)
  a.q_heads = warps ? std::min(c.s.Hq, 32) : std::min(c.s.Hq, 8);
  a.q_ctas = queries ? (int)ceil_div(c.s.Hq, a.q_heads) : 0;
  return c.s.format == MKV_E4M3 ? launch_f<MKV_E4M3>(a, slots, warps, st) : launch_f<MKV_I8>(a, slots, warps, st);
}

}  // namespace mkv
