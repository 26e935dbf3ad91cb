// The per-head products around latent attention: W_uk^T q (absorb), W_uv o (project), w_kv c (expand).
#include <algorithm>

#include "mkv_rows.h"
#include "row_attention.cuh"

namespace mkv {

namespace {

// One thread per output value: out[row][h][c] = sum_k x[row][h][k] w[h][..]
template <typename T, Product KIND>
__global__ void product_kernel(const ProductCall a) {
  const int d = a.nope + a.v_dim, r = a.rank;
  const int width = KIND == Product::kAbsorb ? r + a.rope : (KIND == Product::kProject ? a.v_dim : d);
  const int64_t e = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
  if (e >= (int64_t)a.B * a.rows * a.H * width) return;
  const int c = (int)(e % width);
  const T* x = static_cast<const T*>(a.x);
  const T* w = static_cast<const T*>(a.w);
  float s = 0.f;
  if (KIND == Product::kExpand) {                     // out [B][H][rows][d]
    const int64_t t = e / width % a.rows, bh = e / width / a.rows, h = bh % a.H, b = bh / a.H;
    if (t >= a.T_len[b]) return;
    x += (b * a.T_cap + t) * (r + a.rope);
    w += (h * d + c) * r;
    for (int k = 0; k < r; ++k) s = fmaf(Pair<T>::one(x[k]), Pair<T>::one(w[k]), s);
  } else {                                            // out [B rows][H][width]
    const int64_t h = e / width % a.H, row = e / width / a.H;
    if (KIND == Product::kAbsorb) {
      x += (row * a.H + h) * (a.nope + a.rope);
      w += h * d * r + c;
      if (c >= r) {
        static_cast<T*>(a.out)[e] = x[a.nope + c - r];
        return;
      }
      for (int k = 0; k < a.nope; ++k) s = fmaf(Pair<T>::one(x[k]), Pair<T>::one(w[(int64_t)k * r]), s);
    } else {
      x += (row * a.H + h) * r;
      w += (h * d + a.nope + c) * r;
      for (int k = 0; k < r; ++k) s = fmaf(Pair<T>::one(x[k]), Pair<T>::one(w[k]), s);
    }
  }
  static_cast<T*>(a.out)[e] = Pair<T>::put(s);
}

template <typename T>
cudaError_t launch_t(const ProductCall& c, cudaStream_t st) {
  const int width = c.kind == Product::kAbsorb ? c.rank + c.rope
                    : c.kind == Product::kProject ? c.v_dim : c.nope + c.v_dim;
  const unsigned grid = (unsigned)ceil_div((int64_t)c.B * c.rows * c.H * width, 256);
  if (c.kind == Product::kAbsorb)
    product_kernel<T, Product::kAbsorb><<<grid, 256, 0, st>>>(c);
  else if (c.kind == Product::kProject)
    product_kernel<T, Product::kProject><<<grid, 256, 0, st>>>(c);
  else
    product_kernel<T, Product::kExpand><<<grid, 256, 0, st>>>(c);
  return cudaPeekAtLastError();
}

}  // namespace

cudaError_t launch_latent_product(const ProductCall& c, cudaStream_t st) {
  return c.dtype == MKV_BF16 ? launch_t<__nv_bfloat16>(c, st) : launch_t<__half>(c, st);
}

}  // namespace mkv
