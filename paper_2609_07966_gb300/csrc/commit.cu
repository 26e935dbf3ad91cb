// The accepted path of a tree of drafted tokens joins a cache: for i < n_path[b] the rows of token
// path[b][i] are copied to slot T_len[b] + i, then T_len[b] += n_path[b].  Bound by memory latency (a few
// tens of KB an entry) and, for a whole prompt's rows, by bandwidth.
//
// A cluster of CTAs per entry shares the copies; every CTA reads the length and checks the whole path, a
// cluster barrier separates those reads from the first CTA's store of the new length.
#include <algorithm>

#include "mkv_common.cuh"
#include "mkv_rows.h"

namespace mkv {

namespace {

__device__ uint32_t g_status_commit;

constexpr int kCommitThreads = 512;

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;\n" ::: "memory");
}

__global__ void __launch_bounds__(kCommitThreads) commit_kernel(const CommitCall a) {
  const int b = blockIdx.y, parts = gridDim.x;
  const int t0 = a.T_len[b];
  const int np = a.n_path != nullptr ? a.n_path[b] : a.n;
  bool ok = t0 >= 0 && np >= 0 && np <= a.n && (int64_t)t0 + np <= a.T_cap;
  if (ok && a.path != nullptr)
    for (int i = threadIdx.x; i < np; i += kCommitThreads) {
      const int p = a.path[(int64_t)b * a.n + i];
      ok = ok && p >= 0 && p < a.n;
    }
  ok = __syncthreads_and(ok);
  cluster_sync();                                       // every CTA of the entry has read its length
  if (cluster_rank() == 0 && threadIdx.x == 0) {
    if (ok)
      a.T_len[b] = t0 + np;
    else
      atomicOr(&g_status_commit, MKV_FLAG_CACHE_FULL);
  }
  if (!ok) return;
  // (cache, token, head, 16-byte piece), pieces fastest
  const int per = a.row_bytes / 16;
  const int64_t one = (int64_t)np * a.heads * per, total = a.src1 != nullptr ? 2 * one : one;
  for (int64_t e = (int64_t)blockIdx.x * kCommitThreads + threadIdx.x; e < total;
       e += (int64_t)parts * kCommitThreads) {
    const bool second = e >= one;
    const int64_t x = second ? e - one : e;
    const int c = (int)(x % per), h = (int)(x / per % a.heads);
    const int64_t i = x / per / a.heads;
    const int64_t tok = a.path != nullptr ? a.path[(int64_t)b * a.n + i] : i;
    const uint4* src = static_cast<const uint4*>(second ? a.src1 : a.src0);
    uint4* dst = static_cast<uint4*>(second ? a.dst1 : a.dst0);
    dst[(((int64_t)b * a.heads + h) * a.T_cap + t0 + i) * per + c] =
        src[(((int64_t)b * a.n + tok) * a.heads + h) * per + c];
  }
}

}  // namespace

cudaError_t take_status_commit(uint32_t* flags, cudaStream_t st) {
  uint32_t v = 0, zero = 0;
  cudaError_t e = cudaMemcpyFromSymbolAsync(&v, g_status_commit, sizeof(v), 0, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaMemcpyToSymbolAsync(g_status_commit, &zero, sizeof(zero), 0, cudaMemcpyHostToDevice, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  *flags |= v;
  return e;
}

cudaError_t launch_commit(const CommitCall& c, cudaStream_t st) {
  constexpr int kParts = 8;                             // the largest portable cluster
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {kParts, 1, 1};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kParts, c.B);
  cfg.blockDim = dim3(kCommitThreads);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, commit_kernel, c);
  return e != cudaSuccess ? e : cudaPeekAtLastError();
}

}  // namespace mkv
