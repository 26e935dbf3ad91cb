// Host side of mkv_roles.cuh: tensor-map encoding; and the self-test of its waits and of a CTA's end after a failure.
#include "mkv_roles.cuh"
#include "mkv_rows.h"

namespace mkv {

namespace {

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder() {
  static const EncodeTiled fn = []() -> EncodeTiled {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q{};
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      return nullptr;
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return fn;
}

}  // namespace

// fp16 and bf16 tensors alike: a map only moves 16-bit elements, and zero fill is the same bits.
cudaError_t encode_map(CUtensorMap* m, const void* base, const int64_t (&dims)[4], const int64_t (&strides)[3],
                       int box1, int box2, int box3) {
  const EncodeTiled enc = encoder();
  if (enc == nullptr) return cudaErrorNotSupported;
  cuuint64_t d[4], s[3];
  for (int i = 0; i < 4; ++i) d[i] = (cuuint64_t)dims[i];
  for (int i = 0; i < 3; ++i) s[i] = (cuuint64_t)strides[i] * 2;
  const cuuint32_t box[4] = {64, (cuuint32_t)box1, (cuuint32_t)box2, (cuuint32_t)box3};
  const cuuint32_t es[4] = {1, 1, 1, 1};
  const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(base), d, s, box, es,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

namespace {

// The roles of a CTA that fails: one has asked for half of a tile, one has products under way, and both wait for what
// never comes.  The first gives up after ns, the other with it or by itself; the CTA then ends as the kernels do.
// (A products' tile of zeros: 128 x 64 and 16 x 64.)
struct SelftestCtl {
  uint64_t never, full, drained;
  uint32_t tslot;
  int fail;
};
constexpr int kHalf = 1024;
__device__ __align__(16) uint8_t g_half_tile[kHalf];

__global__ void __launch_bounds__(96) role_wait_selftest_kernel(uint64_t ns, uint32_t* status) {
  __shared__ __align__(1024) uint8_t sm[(128 + 16) * 128 + kHalf];
  __shared__ SelftestCtl ctl;
  uint8_t* copy = sm + (128 + 16) * 128;
  const int warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < (128 + 16) * 128 / 16; i += 96) reinterpret_cast<uint4*>(sm)[i] = make_uint4(0, 0, 0, 0);
  if (warp == 0) tc_alloc(&ctl.tslot, 32);
  if (threadIdx.x == 0) {
    tc_mbar_init(&ctl.never, 1);
    tc_mbar_init(&ctl.full, 2);
    tc_mbar_init(&ctl.drained, 1);
    tc_fence_mbar_init();
    ctl.fail = 0;
  }
  fence_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = ctl.tslot;
  if (warp == 1 && elect_one()) {
    tc_mbar_expect_tx(&ctl.full, kHalf);
    bulk_load(copy, g_half_tile, kHalf, &ctl.full);
    if (!wait_or_fail(&ctl.never, 0, &ctl.fail, status, ns)) give_up(&ctl.full, 1);
  } else if (warp == 2 && elect_one()) {
    const Desc a = tc_desc_sw128(smem_addr(sm)), b = tc_desc_sw128(smem_addr(sm + 128 * 128));
    for (int k = 0; k < 4; ++k) tc_mma_ss(tbase, a.at(k * 32), b.at(k * 32), tc_idesc(false, 128, 16, false, false), k > 0);
    wait_or_fail(&ctl.never, 0, &ctl.fail, status, ns);
    tc_commit(&ctl.drained);
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0) {
    tc_mbar_wait(&ctl.drained, 0, kRoleWaitNs);
    tc_mbar_wait(&ctl.full, 0, kRoleWaitNs);
  }
  __syncthreads();
  tc_fence_after();
  if (warp == 0) tc_dealloc(tbase, 32);
}

}  // namespace

cudaError_t launch_role_wait_selftest(int ms, cudaStream_t st) {
  uint32_t* status;
  const cudaError_t e = status_word(&status);
  if (e != cudaSuccess) return e;
  role_wait_selftest_kernel<<<1, 96, 0, st>>>((uint64_t)ms * 1000000ull, status);
  return cudaPeekAtLastError();
}

}  // namespace mkv
