// Device pieces of the rotary and 8-bit paged cache operators: a rotation of 16 dims, which rows belong to an entry, and
// 8-bit codes widened to fp16.
#pragma once

#include "mkv_paged.h"
#include "mkv_roles.cuh"

namespace mkv {

// Eight packed 16-bit values as fp32, and back (each rounded once).
template <bool BF16>
__device__ __forceinline__ void widen8(const uint4& p, float* x) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = widen<BF16>((uint16_t)w[i]);
    x[2 * i + 1] = widen<BF16>((uint16_t)(w[i] >> 16));
  }
}
template <bool BF16>
__device__ __forceinline__ uint4 narrow8(const float* x) {
  return make_uint4(pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3]), pack2<BF16>(x[4], x[5]), pack2<BF16>(x[6], x[7]));
}

// (x, y) -> (x c - y s, y c + x s), every product and sum rounded (no fused multiply-add), so that what is quantized
// afterwards does not depend on how the compiler contracts it.
__device__ __forceinline__ void rotate_pair(float& x, float& y, float c, float s) {
  const float a = __fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s)), b = __fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s));
  x = a;
  y = b;
}

// Eight pairs' (cos, sin): four 16-byte loads.
struct Turn8 {
  float4 v[4];
  __device__ __forceinline__ void load(const float2* row, int pair0) {
    const float4* p = reinterpret_cast<const float4*>(row + pair0);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __ldg(p + i);
  }
  __device__ __forceinline__ float c(int i) const { return i & 1 ? v[i >> 1].z : v[i >> 1].x; }
  __device__ __forceinline__ float s(int i) const { return i & 1 ? v[i >> 1].w : v[i >> 1].y; }
};
// Sixteen dims: PAIRS: in order (pair i is x[2i], x[2i + 1]); else eight of the first half, then their partners.
__device__ __forceinline__ void rotate16(float (&x)[16], const Turn8& t, bool pairs, float sign) {
  if (pairs) {
#pragma unroll
    for (int i = 0; i < 8; ++i) rotate_pair(x[2 * i], x[2 * i + 1], t.c(i), sign * t.s(i));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) rotate_pair(x[i], x[8 + i], t.c(i), sign * t.s(i));
  }
}
// Where the two runs of eight dims of rotated column c (of rot / 16) begin.
__device__ __forceinline__ int turn_lo(int c, bool pairs) { return pairs ? 16 * c : 8 * c; }
__device__ __forceinline__ int turn_hi(int c, int rot, bool pairs) { return pairs ? 16 * c + 8 : rot / 2 + 8 * c; }

// A position's row of the table, the nearest one if it lies outside.
__device__ __forceinline__ const float2* turn_row(const RopeCall& r, int64_t p, uint32_t* status) {
  if (p < 0 || p >= r.T_max) {
    atomicOr(status, MKV_FLAG_BAD_INDEX);
    p = p < 0 ? 0 : r.T_max - 1;
  }
  return r.table + p * (r.rot >> 1);
}

// Entry b's rows of the n flattened ones: the first, and how many.
struct EntryRows {
  int first, count;
};
__device__ __forceinline__ EntryRows entry_rows(const PagedShape& s, int b) {
  if (s.start == nullptr) return {b * s.each, s.each};
  const int n = (int)s.n, r0 = min(max(s.start[b], 0), n);
  return {r0, min(max(s.start[b + 1], r0), n) - r0};
}

// Division by the heads of a group, G <= 32, of numbers up to 2^26: x ceil(2^32 / G) / 2^32.
struct Heads {
  int G;
  uint32_t inv;                    // (0: G is 1)
  __host__ __device__ Heads(int g = 1) : G(g), inv(g == 1 ? 0u : (uint32_t)(((1ull << 32) + g - 1) / g)) {}
  __device__ __forceinline__ int token(int row) const { return inv == 0u ? row : (int)__umulhi((uint32_t)row, inv); }
  __device__ __forceinline__ int head(int row) const { return row - token(row) * G; }
};

// The last entry of B that begins at or before what is looked for (`begins(b)`, true up to it; 32 entries at a time, by a
// whole warp).
template <typename F>
__device__ __forceinline__ int find_entry(int B, int lane, F begins) {
  int lo = 0, count = B;
  for (;;) {
    const int step = (count + 31) / 32, at = lane * step;
    const unsigned upto = __ballot_sync(0xffffffffu, at < count && begins(lo + at));
    const int last = max(0, __popc(upto) - 1);
    lo += last * step;
    if (step == 1) return lo;
    count = min(step, count - last * step);
  }
}

// Four 8-bit codes as two pairs of fp16, bytes 0 and 1 and bytes 2 and 3; exact.  E4M3: one conversion a pair (shifting
// sign, exponent and mantissa into place takes 10 issue cycles of a scheduler for four codes, this 6); the NaN codes become
// NaN.  I8: 1024 + 128 + x by placing the biased byte in the mantissa, less 1152.
template <int FMT>
__device__ __forceinline__ void widen_codes(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (FMT == MKV_E4M3) {
    asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.rn.f16x2.e4m3x2 %0, a; cvt.rn.f16x2.e4m3x2 %1, b; }"
        : "=r"(lo), "=r"(hi)
        : "r"(w));
  } else {
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t l = __byte_perm(u, 0x64646464u, 0x4140), h = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 k = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));   // 1152
    const __half2 hl = __hsub2(*reinterpret_cast<const __half2*>(&l), k);
    const __half2 hh = __hsub2(*reinterpret_cast<const __half2*>(&h), k);
    lo = *reinterpret_cast<const uint32_t*>(&hl);
    hi = *reinterpret_cast<const uint32_t*>(&hh);
  }
}

// Softmax over 8-bit pages.  Two running maxima a row: m of the scores s (log2), for the sum of the weights p = 2^(s - m),
// and m2 of s + log2 vs, for the weights p vs 2^(m - m2 + 6) that the tensor cores take in fp16: pages of any value scales
// then keep full precision.  Either is only raised once a score passes it by 2^8, so accumulators are almost never rescaled
// and a weight stays below 2^14.
constexpr float kRaise = 8.f;
constexpr float kOffset = 6.f;      // (full precision in fp16 down to 2^-20 of the maximum)
constexpr float kNoMax = -3.402823466e+38f;   // the maxima of a row that has seen nothing: no score is below it
// An output is o / sum 2^(m2 - m - 6): the power's square root, applied twice after 1 / sum (it could pass fp32's range).
__device__ __forceinline__ float half_power(float m, float m2) { return ex2_approx(0.5f * (m2 - m - kOffset)); }

// What an fp32 power of two of `exponent` (within -126 .. 127) is.
__device__ __forceinline__ float power_of_two(int exponent) { return __uint_as_float((uint32_t)(127 + exponent) << 23); }
// The exponent of the power of two that a bf16 row is scaled by, so that it fits fp16: its largest finite magnitude comes to
// lie within 2^14 .. 2^15 (what that rounds away is 2^-39 of it).
__device__ __forceinline__ int row_exponent(float most) {
  return most > 0.f ? max(-113, min(126, 14 + 127 - (int)(__float_as_uint(most) >> 23))) : 0;
}

}  // namespace mkv
