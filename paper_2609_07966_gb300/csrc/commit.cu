// The accepted path of a tree of drafted tokens joins a cache: for i < n_path[b] the rows of token
// path[b][i] are copied to slot T_len[b] + i, then T_len[b] += n_path[b].  A step's few tens of KB an entry are bound
// by latency, a whole prompt's rows by bandwidth; a warp moves one token's row of one cache at a time (its heads lie
// together in the source), four 16-byte pieces a lane in flight.
//
// Every CTA that reads an entry's length has to do so before it changes.  A step's rows are shared by a cluster of
// CTAs per entry, whose barrier separates the reads from the first CTA's store of the new length: one launch.  A
// prompt's rows are shared by as many CTAs as the GPU holds, and a second launch stores the lengths.
#include <algorithm>

#include "mkv_roles.cuh"
#include "mkv_rows.h"

namespace mkv {

namespace {

constexpr int kCommitThreads = 512;

// Whether entry b's path fits (all threads of the CTA take part); its length and path length.
__device__ __forceinline__ bool path_fits(const CommitCall& a, int b, int& t0, int& np) {
  t0 = a.T_len[b];
  np = a.n_path != nullptr ? a.n_path[b] : a.n;
  bool ok = t0 >= 0 && np >= 0 && np <= a.n && (int64_t)t0 + np <= a.T_cap;
  if (ok && a.path != nullptr)
    for (int i = threadIdx.x; i < np; i += kCommitThreads) {
      const int p = a.path[(int64_t)b * a.n + i];
      ok = ok && p >= 0 && p < a.n;
    }
  return __syncthreads_and(ok);
}

__device__ __forceinline__ void store_length(const CommitCall& a, int b, bool ok, int t) {
  if (threadIdx.x != 0) return;
  if (ok)
    a.T_len[b] = t;
  else
    atomicOr(a.status, MKV_FLAG_CACHE_FULL);
}

template <bool kCluster>
__global__ void __launch_bounds__(kCommitThreads) commit_kernel(const CommitCall a) {
  pdl_wait_and_trigger();
  const int b = blockIdx.y;
  int t0, np;
  const bool ok = path_fits(a, b, t0, np);
  if (kCluster) {
    cluster_sync();                                     // every CTA of the entry has read its length
    if (cluster_rank() == 0) store_length(a, b, ok, t0 + np);
  }
  if (!ok) return;
  const int lane = threadIdx.x & 31, per = a.row_bytes / 16, row = a.heads * per;   // pieces of a token's row
  const int64_t jobs = a.src1 != nullptr ? 2 * (int64_t)np : np;
  for (int64_t j = (int64_t)blockIdx.x * (kCommitThreads / 32) + (threadIdx.x >> 5); j < jobs;
       j += (int64_t)gridDim.x * (kCommitThreads / 32)) {
    const bool second = j >= np;
    const int i = (int)(second ? j - np : j);
    const int tok = a.path != nullptr ? a.path[(int64_t)b * a.n + i] : i;
    const uint4* src = static_cast<const uint4*>(second ? a.src1 : a.src0) + ((int64_t)b * a.n + tok) * row;
    uint4* dst = static_cast<uint4*>(second ? a.dst1 : a.dst0) + ((int64_t)b * a.heads * a.T_cap + t0 + i) * per;
    for (int e0 = lane; e0 < row; e0 += 128) {
      uint4 x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (e0 + 32 * k < row) x[k] = src[e0 + 32 * k];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int e = e0 + 32 * k, h = e / per;
        if (e < row) dst[(int64_t)h * a.T_cap * per + (e - h * per)] = x[k];
      }
    }
  }
}

__global__ void __launch_bounds__(kCommitThreads) length_kernel(const CommitCall a) {
  pdl_wait_and_trigger();
  int t0, np;
  const bool ok = path_fits(a, blockIdx.x, t0, np);
  store_length(a, blockIdx.x, ok, t0 + np);
}

}  // namespace

cudaError_t launch_commit(const CommitCall& call, cudaStream_t st) {
  CommitCall c = call;
  cudaError_t e = status_word(&c.status);
  if (e != cudaSuccess) return e;
  constexpr int kParts = 8;                             // the largest portable cluster
  // One launch up to 1 MiB an entry (measured: 16 rows of 4 KB x 8 entries 4.2 us; but 9.4 MB of one entry 86 us through
  // one cluster and 7.9 us in two launches, each with a copy of the length before it).
  const int64_t bytes = (int64_t)c.n * c.heads * c.row_bytes * (c.src1 != nullptr ? 2 : 1);
  if (bytes > (1 << 20)) {
    const int64_t want = ceil_div((int64_t)4 * kNumSMs, (int64_t)c.B), most = ceil_div(c.n, kCommitThreads / 32);
    e = launch_pdl(commit_kernel<false>, dim3((unsigned)std::min(want, most), c.B), dim3(kCommitThreads), 0, st, c);
    return e != cudaSuccess ? e : launch_pdl(length_kernel, dim3(c.B), dim3(kCommitThreads), 0, st, c);
  }
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {kParts, 1, 1};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kParts, c.B);
  cfg.blockDim = dim3(kCommitThreads);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, commit_kernel<true>, c);
  return e != cudaSuccess ? e : cudaPeekAtLastError();
}

}  // namespace mkv
