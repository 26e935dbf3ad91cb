// Pieces shared by the warp-specialised tcgen05 attention and product kernels: bounded waits, operand
// descriptors for both majors, tensor-memory loads and stores of a thread's columns, tensor maps.
#pragma once

#include <cuda.h>   // CUtensorMap and its enums; the encoder is fetched from the driver at run time
#include <cuda_bf16.h>

#include "mkv_tc.cuh"

namespace mkv {

constexpr uint64_t kRoleWaitNs = 1000000000ull;   // a bounded wait gives up after 1 s

// How a CTA ends, failed or not: the role that issues products commits them all to a barrier of their own as it leaves,
// wherever it stopped, and nothing of the CTA's is given back before that phase ends; on a failure the copies under way
// are waited for too, which end a phase each because the role that loads gives up the rest of a tile that it began.
//
// Bounded wait of one role: false when it ran out (the flag is raised and MKV_FLAG_WAIT_TIMEOUT set in
// *status) or another role's did.
__device__ __forceinline__ bool wait_or_fail(uint64_t* bar, uint32_t parity, volatile int* fail, uint32_t* status,
                                             uint64_t ns = kRoleWaitNs) {
  if (tc_mbar_try(bar, parity)) return true;
  const uint64_t t0 = globaltimer_ns();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 16; ++i)
      if (tc_mbar_try(bar, parity)) return true;
    if (*fail) return false;
    if (globaltimer_ns() - t0 > ns) break;
  }
  *fail = 1;
  atomicOr(status, MKV_FLAG_WAIT_TIMEOUT);
  return false;
}

// Arrives for the `left` pieces of a tile that will not be asked for: its phase ends with the copies that were.
__device__ __forceinline__ void give_up(uint64_t* bar, int left) {
  for (; left > 0; --left) tc_mbar_arrive(bar);
}

// One thread of a converged warp.  (Code behind this choice is known to run in a single thread, which matters for
// the instructions that take their operands from uniform registers: TMA copies and tensor-core products.)
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(p));
  return p != 0;
}

// One non-blocking test of phase `parity` of `bar`.
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{ .reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
      : "=r"(ok)
      : "r"(smem_addr(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}

// Instruction descriptor of kind::f16 with an fp32 accumulator: D format f32 in [4,6), A and B formats
// (0 fp16, 1 bf16) in [7,10) and [10,13), A / B stored with M / N contiguous in bits 15 / 16, N >> 3 in
// [17,23), M >> 4 in [24,29).
__host__ __device__ constexpr uint32_t tc_idesc(bool bf16, int M, int N, bool a_mn, bool b_mn) {
  return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((a_mn ? 1u : 0u) << 15) |
         ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// Shared-memory descriptor of an operand whose M (or N) index is contiguous: `width` elements of it per
// row (64, 32 or 16: the 128-, 64- or 32-byte swizzle), one row per K index, 8 rows a group; groups follow
// one another every 8 rows, blocks of `width` every `block` bytes.  A K step of 16 advances by 16 rows.
template <int width>
__device__ __forceinline__ uint64_t tc_desc_mn(uint32_t start, uint32_t block) {
  static_assert(width == 64 || width == 32 || width == 16, "row width");
  constexpr uint64_t layout = width == 64 ? 2 : width == 32 ? 4 : 6;
  return (uint64_t)((start >> 4) & 0x3fffu) | ((uint64_t)((block >> 4) & 0x3fffu) << 16) |
         ((uint64_t)(8 * width * 2 >> 4) << 32) | ((uint64_t)1u << 46) | (layout << 61);
}

// Byte offset of 16-byte piece `c` of row `r` in such a tile (the swizzle XORs the piece with the row's
// 128-byte line).
template <int width>
__device__ __forceinline__ uint32_t mn_offset(int r, int c) {
  if (width == 64) return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4));
  if (width == 32) return (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
  return (uint32_t)(r * 32 + ((c ^ ((r >> 2) & 1)) << 4));
}

// An operand descriptor as its two words: a product's offsets only touch the low one.  opaque() hides the low
// word's value from the compiler, which would otherwise keep every k step's sum in a register across tiles.
struct Desc {
  uint32_t lo, hi;
  __device__ __forceinline__ Desc(uint64_t d) : lo((uint32_t)d), hi((uint32_t)(d >> 32)) {}
  __device__ __forceinline__ Desc(uint32_t l, uint32_t h) : lo(l), hi(h) {}
  __device__ __forceinline__ Desc at(uint32_t bytes) const { return Desc(lo + (bytes >> 4), hi); }
  __device__ __forceinline__ Desc opaque() const {
    uint32_t x = lo;
    asm volatile("" : "+r"(x));
    return Desc(x, hi);
  }
};
// D[tmem] (+)= A[smem] B[smem], one K step of 16
__device__ __forceinline__ void tc_mma_ss(uint32_t d_tmem, Desc a, Desc b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{ .reg .pred p; .reg .b64 da, db; setp.ne.b32 p, %6, 0; mov.b64 da, {%1, %2}; mov.b64 db, {%3, %4};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p; }" ::"r"(d_tmem),
      "r"(a.lo), "r"(a.hi), "r"(b.lo), "r"(b.hi), "r"(idesc), "r"(acc)
      : "memory");
}
// the same with A in tensor memory: its rows are lanes, two 16-bit values of K a column
__device__ __forceinline__ void tc_mma_ts(uint32_t d_tmem, uint32_t a_tmem, Desc b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{ .reg .pred p; .reg .b64 db; setp.ne.b32 p, %5, 0; mov.b64 db, {%2, %3};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p; }" ::"r"(d_tmem),
      "r"(a_tmem), "r"(b.lo), "r"(b.hi), "r"(idesc), "r"(acc)
      : "memory");
}

__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void prefetch_map(const void* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// This warpgroup's registers per thread; every warp of it takes part, and the block's shares have to add up to no
// more than it was launched with.
template <int R>
__device__ __forceinline__ void regs_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R));
}
template <int R>
__device__ __forceinline__ void regs_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R));
}

// Thread-block clusters: this CTA's rank, a barrier over all threads of all CTAs (it orders their shared-memory
// accesses; whole or as its two halves), the address of a shared variable in another CTA, and stores there.
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_addr(const void* p, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_cluster(uint32_t a, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory");
}
__device__ __forceinline__ void st_cluster2(uint32_t a, float2 v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(a), "f"(v.x), "f"(v.y) : "memory");
}

// Named barrier over `count` threads: with and without an OR of a predicate.
__device__ __forceinline__ void bar_sync(int id, int count) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(count) : "memory");
}
__device__ __forceinline__ bool bar_or(int id, int count, bool p) {
  uint32_t r;
  asm volatile(
      "{ .reg .pred p, q; setp.ne.u32 p, %1, 0; barrier.cta.red.or.pred q, %2, %3, p; selp.u32 %0, 1, 0, q; }"
      : "=r"(r)
      : "r"((uint32_t)p), "r"(id), "r"(count)
      : "memory");
  return r != 0;
}

// C consecutive fp32 columns of the thread's tensor-memory lane.  The registers are valid after tm_wait, which
// names them, so no use is ordered before it (a second wait, already satisfied, covers more registers).
template <int C>
__device__ __forceinline__ void tm_issue(uint32_t addr, float (&v)[C]);
template <int C>
__device__ __forceinline__ void tm_wait(float (&v)[C]);
template <>
__device__ __forceinline__ void tm_issue<8>(uint32_t addr, float (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
               : "r"(addr));
}
template <>
__device__ __forceinline__ void tm_wait<8>(float (&v)[8]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7])
               :
               : "memory");
}
#define MKV_OUT16(m, v, o)                                                                                      \
  m(v[o + 0]), m(v[o + 1]), m(v[o + 2]), m(v[o + 3]), m(v[o + 4]), m(v[o + 5]), m(v[o + 6]), m(v[o + 7]),       \
      m(v[o + 8]), m(v[o + 9]), m(v[o + 10]), m(v[o + 11]), m(v[o + 12]), m(v[o + 13]), m(v[o + 14]), m(v[o + 15])
#define MKV_EQF(x) "=f"(x)
#define MKV_PLF(x) "+f"(x)
#define MKV_INF(x) "f"(x)
template <>
__device__ __forceinline__ void tm_issue<16>(uint32_t addr, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
      : MKV_OUT16(MKV_EQF, v, 0)
      : "r"(addr));
}
template <>
__device__ __forceinline__ void tm_wait<16>(float (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : MKV_OUT16(MKV_PLF, v, 0) : : "memory");
}
template <>
__device__ __forceinline__ void tm_issue<32>(uint32_t addr, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
      : MKV_OUT16(MKV_EQF, v, 0), MKV_OUT16(MKV_EQF, v, 16)
      : "r"(addr));
}
template <>
__device__ __forceinline__ void tm_wait<32>(float (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : MKV_OUT16(MKV_PLF, v, 0), MKV_OUT16(MKV_PLF, v, 16) : : "memory");
}
template <int C>
__device__ __forceinline__ void tm_load(uint32_t addr, float (&v)[C]) {
  tm_issue<C>(addr, v);
  tm_wait<C>(v);
}
// 16 tensor-memory lanes (an accumulator of 64 rows has 16 in each warp's quarter): lanes 0..15 of the warp get
// columns 0 .. C - 1 of them, lanes 16..31 columns C .. 2 C - 1.
template <int C>
__device__ __forceinline__ void tm_load_halves(uint32_t addr, float (&v)[C]);
template <>
__device__ __forceinline__ void tm_load_halves<4>(uint32_t addr, float (&v)[4]) {
  asm volatile("tcgen05.ld.sync.aligned.16x32bx2.x4.b32 {%0,%1,%2,%3}, [%4], 4;\n"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3])
               : "r"(addr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]) : : "memory");
}
template <>
__device__ __forceinline__ void tm_load_halves<8>(uint32_t addr, float (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.16x32bx2.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8], 8;\n"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
               : "r"(addr));
  tm_wait<8>(v);
}
template <>
__device__ __forceinline__ void tm_load_halves<16>(uint32_t addr, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x32bx2.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16], 16;\n"
      : MKV_OUT16(MKV_EQF, v, 0)
      : "r"(addr));
  tm_wait<16>(v);
}
// The stores complete at tm_store_wait().
template <int C>
__device__ __forceinline__ void tm_store(uint32_t addr, const float (&v)[C]);
template <>
__device__ __forceinline__ void tm_store<8>(uint32_t addr, const float (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};\n" ::"f"(v[0]), "f"(v[1]),
               "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "r"(addr)
               : "memory");
}
template <>
__device__ __forceinline__ void tm_store<16>(uint32_t addr, const float (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};\n" ::
          MKV_OUT16(MKV_INF, v, 0),
      "r"(addr)
      : "memory");
}
template <>
__device__ __forceinline__ void tm_store<32>(uint32_t addr, const float (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};\n" ::MKV_OUT16(MKV_INF, v, 0),
      MKV_OUT16(MKV_INF, v, 16), "r"(addr)
      : "memory");
}
#undef MKV_OUT16
#undef MKV_EQF
#undef MKV_PLF
#undef MKV_INF
__device__ __forceinline__ void tm_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two fp32 values rounded to the type and packed (lo in the low half).
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if (BF16)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool BF16>
__device__ __forceinline__ float widen(uint16_t x) {
  return BF16 ? __uint_as_float((uint32_t)x << 16) : __half2float(__ushort_as_half(x));
}
// Whether a 16-bit value is an infinity or NaN: its exponent bits are all ones.
template <bool BF16>
__device__ __forceinline__ bool non_finite(uint16_t x) {
  constexpr uint16_t e = BF16 ? 0x7f80 : 0x7c00;
  return (x & e) == e;
}

// Whether any of eight packed values is an infinity or NaN: adding one to an all-ones exponent carries into the sign.
template <bool BF16>
__device__ __forceinline__ bool any_non_finite(const uint4& x) {
  constexpr uint32_t one = BF16 ? 0x00800080u : 0x04000400u;
  const uint32_t a = ((x.x & 0x7fff7fffu) + one) | ((x.y & 0x7fff7fffu) + one);
  const uint32_t b = ((x.z & 0x7fff7fffu) + one) | ((x.w & 0x7fff7fffu) + one);
  return ((a | b) & 0x80008000u) != 0;
}
// Zeroes the non-finite values among eight packed ones; whether there were any.
template <bool BF16>
__device__ __forceinline__ bool bad_pairs(uint4& x) {
  constexpr uint32_t e = BF16 ? 0x7f80u : 0x7c00u;
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (w[i] & e) == e, hi = (w[i] & (e << 16)) == (e << 16);
    any |= lo | hi;
    w[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
  }
  x = make_uint4(w[0], w[1], w[2], w[3]);
  return any;
}

// 32 columns of a warp whose lane i holds output value 8 (i % 4) + i / 4 of each: rounded and exchanged between lanes so
// that lane i holds the eight values 8 (i % 4) .. + 7 of column 8 k + i / 4 in out[k] (three rounds of pairwise swaps);
// four neighbouring lanes then store 64 neighbouring bytes.
template <bool BF16>
__device__ __forceinline__ void gather_rows(const float (&v)[32], int lane, uint4 (&out)[4]) {
  const bool b0 = lane & 4, b1 = lane & 8, b2 = lane & 16;
  uint32_t h[16];                 // two values of column 2 p + b0
#pragma unroll
  for (int p = 0; p < 16; ++p) {
    const float y = __shfl_xor_sync(0xffffffffu, b0 ? v[2 * p] : v[2 * p + 1], 4);
    h[p] = b0 ? pack2<BF16>(y, v[2 * p + 1]) : pack2<BF16>(v[2 * p], y);
  }
  uint2 w[8];                     // four values of column 4 p + 2 b1 + b0
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const uint32_t y = __shfl_xor_sync(0xffffffffu, b1 ? h[2 * p] : h[2 * p + 1], 8);
    w[p] = b1 ? make_uint2(y, h[2 * p + 1]) : make_uint2(h[2 * p], y);
  }
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint2 s = b2 ? w[2 * p] : w[2 * p + 1];
    const uint32_t y0 = __shfl_xor_sync(0xffffffffu, s.x, 16), y1 = __shfl_xor_sync(0xffffffffu, s.y, 16);
    out[p] = b2 ? make_uint4(y0, y1, w[2 * p + 1].x, w[2 * p + 1].y) : make_uint4(w[2 * p].x, w[2 * p].y, y0, y1);
  }
}

// A reduction of each of C columns over each L neighbouring lanes: on return v[0] of lane i holds column
// (i % L) / (L / C).
template <int L, int C, typename Op>
__device__ __forceinline__ void reduce_columns(float (&v)[C], int lane, Op op) {
  static_assert(C <= L, "a column for every lane at most");
  int lb = L / 2;
#pragma unroll
  for (int w = C / 2; w >= 1; w >>= 1) {
    const bool up = (lane & lb) != 0;
#pragma unroll
    for (int i = 0; i < w; ++i) {
      const float keep = up ? v[i + w] : v[i], send = up ? v[i] : v[i + w];
      v[i] = op(keep, __shfl_xor_sync(0xffffffffu, send, lb));
    }
    lb >>= 1;
  }
  for (; lb >= 1; lb >>= 1) v[0] = op(v[0], __shfl_xor_sync(0xffffffffu, v[0], lb));
}

// A 4-D tensor map of 16-bit elements: dims and strides in elements (innermost stride 1), a box of
// 64 x box1 x box2 x box3 with the 128-byte swizzle; what lies outside reads as zero.
cudaError_t encode_map(CUtensorMap* m, const void* base, const int64_t (&dims)[4], const int64_t (&strides)[3],
                       int box1, int box2, int box3 = 1);
// A map of bytes [heads][rows][width], width 64 or 128: boxes of width x box_rows of one head, the swizzle of that width.
cudaError_t encode_code_map(CUtensorMap* m, const void* base, int width, int64_t rows, int64_t heads, int box_rows);

}  // namespace mkv
