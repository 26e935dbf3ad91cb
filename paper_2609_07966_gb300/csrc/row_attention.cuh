// Softmax attention of one query row, one key at a time per warp:
//   out = sum_j 2^(s_j - M) v_j / sum_j 2^(s_j - M),  s_j = scale log2(e) q . k_j over the visible keys,
// with the running maximum and sum in fp32; zeros when nothing is visible.
#pragma once

#include <cuda_bf16.h>

#include "mkv_common.cuh"

namespace mkv {

template <typename T>
struct Pair;
template <>
struct Pair<__half> {
  static __device__ __forceinline__ float2 get(const __half* p) {
    return __half22float2(*reinterpret_cast<const __half2*>(p));
  }
  static __device__ __forceinline__ __half put(float x) { return __float2half_rn(x); }
  static __device__ __forceinline__ float one(__half x) { return __half2float(x); }
};
template <>
struct Pair<__nv_bfloat16> {
  static __device__ __forceinline__ float2 get(const __nv_bfloat16* p) {
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(p));
  }
  static __device__ __forceinline__ __nv_bfloat16 put(float x) { return __float2bfloat16_rn(x); }
  static __device__ __forceinline__ float one(__nv_bfloat16 x) { return __bfloat162float(x); }
};

constexpr int kRowWarps = 4;

// A CTA of kRowWarps warps; key(j, k0, k1, v) gives the key's first DK0 values, its other DK - DK0 and
// its value, or false for a key the row does not see.
template <typename T, int DK0, int DK, int DV, typename KeyFn>
__device__ __forceinline__ void row_attention(const T* q, int64_t nkeys, float scale_log2, KeyFn key, T* out) {
  constexpr int NK = DK / 64, NV = DV / 64;
  __shared__ float sm[kRowWarps], sl[kRowWarps], so[kRowWarps][DV];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float2 qr[NK], o[NV];
#pragma unroll
  for (int i = 0; i < NK; ++i) qr[i] = Pair<T>::get(q + i * 64 + lane * 2);
#pragma unroll
  for (int i = 0; i < NV; ++i) o[i] = make_float2(0.f, 0.f);
  float m = -INFINITY, l = 0.f;
  for (int64_t j = warp; j < nkeys; j += kRowWarps) {
    const T *k0, *k1, *v;
    if (!key(j, k0, k1, v)) continue;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const float2 x = Pair<T>::get((i * 64 < DK0 ? k0 + i * 64 : k1 + (i * 64 - DK0)) + lane * 2);
      s = fmaf(qr[i].x, x.x, fmaf(qr[i].y, x.y, s));
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    s *= scale_log2;
    const float mn = fmaxf(m, s), a = m == -INFINITY ? 0.f : exp2f(m - mn), p = exp2f(s - mn);
    m = mn;
    l = l * a + p;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const float2 x = Pair<T>::get(v + i * 64 + lane * 2);
      o[i].x = o[i].x * a + p * x.x;
      o[i].y = o[i].y * a + p * x.y;
    }
  }
  if (lane == 0) {
    sm[warp] = m;
    sl[warp] = l;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    so[warp][i * 64 + lane * 2] = o[i].x;
    so[warp][i * 64 + lane * 2 + 1] = o[i].y;
  }
  __syncthreads();
  float M = -INFINITY, L = 0.f;
  for (int w = 0; w < kRowWarps; ++w) M = fmaxf(M, sm[w]);
  float f[kRowWarps];
  for (int w = 0; w < kRowWarps; ++w) {
    f[w] = sm[w] == -INFINITY ? 0.f : exp2f(sm[w] - M);
    L += sl[w] * f[w];
  }
  for (int d = threadIdx.x; d < DV; d += kRowWarps * 32) {
    float x = 0.f;
    for (int w = 0; w < kRowWarps; ++w) x += f[w] == 0.f ? 0.f : so[w][d] * f[w];
    out[d] = Pair<T>::put(L == 0.f ? 0.f : x / L);
  }
}

}  // namespace mkv
