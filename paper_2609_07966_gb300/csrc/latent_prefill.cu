// Causal attention of a prompt's queries over expanded latent keys and values.
#include <algorithm>

#include "mkv_rows.h"
#include "row_attention.cuh"

namespace mkv {

namespace {

template <typename T, int DN, int DV>
__global__ void __launch_bounds__(kRowWarps * 32) prefill_kernel(const PrefillCall a) {
  constexpr int DK = DN + 64;
  const int64_t row = blockIdx.x;                     // (b n + i) H + h
  const int h = (int)(row % a.H);
  const int64_t b = row / a.H / a.n, i = row / a.H % a.n;
  const int64_t len = std::min<int64_t>(std::max(a.T_len[b], 0), a.T_max);
  const int64_t ql = a.q_len != nullptr ? std::min(std::max(a.q_len[b], 0), a.n) : a.n;
  const int64_t seen = i < ql ? std::min<int64_t>(len, (int64_t)a.T_len[b] - ql + i + 1) : 0;
  const T* kv = static_cast<const T*>(a.kv) + (b * a.H + h) * a.T_max * (DN + DV);
  const T* rows = static_cast<const T*>(a.rows) + b * a.T_cap * (a.rank + 64) + a.rank;
  row_attention<T, DN, DK, DV>(
      static_cast<const T*>(a.q) + row * DK, seen, a.scale * kLog2e,
      [&](int64_t j, const T*& k0, const T*& k1, const T*& v) {
        k0 = kv + j * (DN + DV);
        v = k0 + DN;
        k1 = rows + j * (a.rank + 64);
        return true;
      },
      static_cast<T*>(a.out) + row * DV);
}

template <typename T>
cudaError_t launch_t(const PrefillCall& c, cudaStream_t st) {
  const unsigned grid = (unsigned)((int64_t)c.B * c.n * c.H);
  if (c.nope == 128 && c.v_dim == 128)
    prefill_kernel<T, 128, 128><<<grid, kRowWarps * 32, 0, st>>>(c);
  else if (c.nope == 128)
    prefill_kernel<T, 128, 64><<<grid, kRowWarps * 32, 0, st>>>(c);
  else if (c.v_dim == 128)
    prefill_kernel<T, 64, 128><<<grid, kRowWarps * 32, 0, st>>>(c);
  else
    prefill_kernel<T, 64, 64><<<grid, kRowWarps * 32, 0, st>>>(c);
  return cudaPeekAtLastError();
}

}  // namespace

cudaError_t launch_latent_prefill(const PrefillCall& c, cudaStream_t st) {
  return c.dtype == MKV_BF16 ? launch_t<__nv_bfloat16>(c, st) : launch_t<__half>(c, st);
}

}  // namespace mkv
