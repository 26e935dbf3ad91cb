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
  int64_t first, count;
};
__device__ __forceinline__ EntryRows entry_rows(const PagedShape& s, int b) {
  if (s.start == nullptr) {
    const int64_t m = s.n / s.B;
    return {b * m, m};
  }
  const int64_t r0 = min(max((int64_t)s.start[b], (int64_t)0), s.n);
  return {r0, min(max((int64_t)s.start[b + 1], r0), s.n) - r0};
}

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

// Four 8-bit codes as two pairs of fp16: even holds bytes 0 and 2, odd bytes 1 and 3.  E4M3: an e4m3 code's sign,
// exponent and mantissa moved into fp16's places read as the code's value times 2^-8 (the two formats' exponent biases
// differ by 8), zero and subnormal codes alike; the NaN codes read as +-480, so no bits of a page give a non-finite
// number, which a weight of zero would not mask.  I8: 1024 + 128 + x by placing the biased byte in the mantissa, less
// 1152.  All exact.
constexpr float kE4m3Up = 256.f;    // what an e4m3 code's fp16 form is short of
template <int FMT>
__device__ __forceinline__ void widen_codes(uint32_t w, uint32_t& even, uint32_t& odd) {
  if (FMT == MKV_E4M3) {
    const uint32_t u = w << 7;
    even = ((w << 8) & 0x80008000u) | (u & 0x3f803f80u);
    odd = (w & 0x80008000u) | ((w >> 1) & 0x3f803f80u);
  } else {
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t e = (u & 0x00ff00ffu) | 0x64006400u, o = __byte_perm(u, 0x64646464u, 0x4341);
    const __half2 k = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));   // 1152
    const __half2 he = __hsub2(*reinterpret_cast<const __half2*>(&e), k);
    const __half2 ho = __hsub2(*reinterpret_cast<const __half2*>(&o), k);
    even = *reinterpret_cast<const uint32_t*>(&he);
    odd = *reinterpret_cast<const uint32_t*>(&ho);
  }
}

}  // namespace mkv
