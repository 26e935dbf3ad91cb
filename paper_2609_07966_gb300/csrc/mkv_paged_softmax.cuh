// A row's part of the softmax over a tile of 8-bit pages, a thread a row or a part of it: the columns' maxima, and weights.
//
// GC neighbouring columns (tokens) share a page's scales {kf, lv}: their scores are v kf back, and lv = log2 vs.  A weight as
// the tensor cores take it is p vs 2^(m - m2 + 6) = 2^(v kf back - m + c) with c = m - m2 + 6 + lv, one exponential; the row's
// sum gets their sum times 2^-c.  c is kept above -60: a weight below 2^-24 is zero in fp16 either way, and the sum keeps its
// digits (a page of zeros has the least scale and weights of its own in the sum).
#pragma once

#include "mkv_paged.cuh"

namespace mkv {

// Up to this maximum (log2) an unrounded product of score and scale is within a half of the rounded one.
constexpr float kFused = 16777216.f;
constexpr float kLeastShift = -60.f;

__device__ __forceinline__ float weight_shift(float m, float m2, float lv) { return fmaxf(m - m2 + kOffset + lv, kLeastShift); }
// (a factor of zero would make NaN of a masked score)
template <bool BACK>
__device__ __forceinline__ float score_factor(float kf, float back) {
  return fmaxf(BACK ? kf * back : kf, 1.17549435e-38f);
}

template <int N>
__device__ __forceinline__ float max_of(const float* y) {
  float x0 = fmax3(y[0], y[1], y[2]), x1 = fmax3(y[3], y[4], y[5]);
#pragma unroll
  for (int i = 6; i + 3 < N; i += 4) {
    x0 = fmax3(x0, y[i], y[i + 1]);
    x1 = fmax3(x1, y[i + 2], y[i + 3]);
  }
  return fmax3(x0, x1, fmaxf(y[N - 2], y[N - 1]));         // (N is a multiple of 4: two are left)
}

// 32 fp32 columns of the thread's tensor-memory lane, load and wait as one statement (as two, the wait names the registers
// again and the compiler copies them).
__device__ __forceinline__ void tm_read32(uint32_t addr, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
      "tcgen05.wait::ld.sync.aligned;\n"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
        "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
        "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(addr)
      : "memory");
}

// Raises mt and mt2 to the largest of N columns' scores and scores + log2 vs; GC of them share scale(g).
template <int N, int GC, bool BACK, typename Scale>
__device__ __forceinline__ void columns_max(const float (&v)[N], float back, Scale scale, float& mt, float& mt2) {
#pragma unroll
  for (int g = 0; g < N / GC; ++g) {
    const float2 s = scale(g);
    const float x = max_of<GC>(v + GC * g) * score_factor<BACK>(s.x, back);
    mt = fmaxf(mt, x);
    mt2 = fmaxf(mt2, x + s.y);
  }
}

// The weights of N columns as packed pairs, and their part of the row's sum.  `ends`: rows end among the columns: then the sum
// takes the weights as they were rounded, so that a row of few tokens is off by less (of one token, not at all).
template <int N, int GC, bool BACK, typename Scale>
__device__ __forceinline__ void columns_weights(float (&v)[N], bool ends, float m, float m2, float back, Scale scale, float& l,
                                                float (&pk)[N / 2]) {
  // (a maximum so large that its rounding alone passes the exponent's range: the products are rounded as it was)
  const bool plain = __any_sync(0xffffffffu, fabsf(m) > kFused && m != kNoMax);
  if (plain) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __fsub_rn(__fmul_rn(v[i], score_factor<BACK>(scale(i / GC).x, back)), m);
  }
#pragma unroll
  for (int g = 0; g < N / GC; ++g) {
    const float2 s = scale(g);
    const float c = weight_shift(m, m2, s.y), f = plain ? 1.f : score_factor<BACK>(s.x, back), off = plain ? c : c - m;
    const uint64_t f2 = pk2(f, f), off2 = pk2(off, off);
    uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
    for (int e = 0; e < GC / 2; ++e) {
      const int at = GC * g + 2 * e;
      const float2 y = upk2(ffma2(pk2(v[at], v[at + 1]), f2, off2));
      const float w0 = ex2_approx(y.x), w1 = ex2_approx(y.y);
      sum[e & 1] = fadd2(sum[e & 1], pk2(w0, w1));
      pk[GC / 2 * g + e] = __uint_as_float(pack2<false>(w0, w1));
    }
    if (ends && c > -kOffset) {                            // (weights of 2^-kOffset or less lose digits in fp16)
      sum[0] = sum[1] = 0ull;
#pragma unroll
      for (int e = 0; e < GC / 2; ++e) {
        const uint32_t h = __float_as_uint(pk[GC / 2 * g + e]);
        const float2 w = __half22float2(*reinterpret_cast<const __half2*>(&h));
        sum[e & 1] = fadd2(sum[e & 1], pk2(w.x, w.y));
      }
    }
    const float2 s0 = upk2(sum[0]), s1 = upk2(sum[1]);
    l += ((s0.x + s0.y) + (s1.x + s1.y)) * ex2_approx(-c);
  }
}

}  // namespace mkv
