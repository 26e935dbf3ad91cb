// Attention of a few tokens' query rows over a cache and the drafted tokens behind it: the tree form of an
// FP16 cache's decode step and the absorbed form of latent attention.
#include <algorithm>

#include "mkv_rows.h"
#include "row_attention.cuh"

namespace mkv {

__device__ uint32_t g_status_rows;   // MKV_FLAG_* bits raised here

cudaError_t take_status_rows(uint32_t* flags, cudaStream_t st) {
  uint32_t v = 0, zero = 0;
  cudaError_t e = cudaMemcpyFromSymbolAsync(&v, g_status_rows, sizeof(v), 0, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaMemcpyToSymbolAsync(g_status_rows, &zero, sizeof(zero), 0, cudaMemcpyHostToDevice, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  *flags |= v;
  return e;
}

namespace {

template <typename T, int DK, int DV>
__global__ void __launch_bounds__(kRowWarps * 32) rows_kernel(const RowsCall a) {
  const int64_t row = blockIdx.x;                     // (b n + i) H + h
  const int h = (int)(row % a.H), g = h / (a.H / a.Hkv);
  const int64_t bi = row / a.H, b = bi / a.n;
  const int64_t len = std::min<int64_t>(std::max(a.T_len[b], 0), a.T_cap);
  const T* k = static_cast<const T*>(a.k) + (b * a.Hkv + g) * a.T_cap * DK;
  const T* v = a.latent ? k : static_cast<const T*>(a.v) + (b * a.Hkv + g) * a.T_cap * DV;
  const T* kt = static_cast<const T*>(a.k_tree);
  const T* vt = a.latent ? kt : static_cast<const T*>(a.v_tree);
  const uint64_t mask = kt != nullptr ? a.mask[bi] : 0;
  row_attention<T, DK, DK, DV>(
      static_cast<const T*>(a.q) + row * DK, len + (kt != nullptr ? a.n : 0), a.scale * kLog2e,
      [&](int64_t j, const T*& k0, const T*& k1, const T*& vj) {
        k1 = nullptr;
        if (j < len) {
          k0 = k + j * DK;
          vj = v + j * (a.latent ? DK : DV);
          return true;
        }
        j -= len;
        k0 = kt + ((b * a.n + j) * a.Hkv + g) * DK;
        vj = vt + ((b * a.n + j) * a.Hkv + g) * (a.latent ? DK : DV);
        return (mask >> j & 1) != 0;
      },
      static_cast<T*>(a.out) + row * DV);
}

template <typename T>
cudaError_t launch_t(const RowsCall& c, cudaStream_t st) {
  const unsigned grid = (unsigned)((int64_t)c.B * c.n * c.H);
  if (c.latent && c.dv == 512)
    rows_kernel<T, 576, 512><<<grid, kRowWarps * 32, 0, st>>>(c);
  else if (c.latent)
    rows_kernel<T, 320, 256><<<grid, kRowWarps * 32, 0, st>>>(c);
  else if (c.dv == 128)
    rows_kernel<T, 128, 128><<<grid, kRowWarps * 32, 0, st>>>(c);
  else
    rows_kernel<T, 64, 64><<<grid, kRowWarps * 32, 0, st>>>(c);
  return cudaPeekAtLastError();
}

}  // namespace

size_t rows_ws_bytes(const RowsCall&) { return kCounterBytes; }

cudaError_t launch_rows_attention(const RowsCall& c, void*, cudaStream_t st) {
  return c.dtype == MKV_BF16 ? launch_t<__nv_bfloat16>(c, st) : launch_t<__half>(c, st);
}

}  // namespace mkv
