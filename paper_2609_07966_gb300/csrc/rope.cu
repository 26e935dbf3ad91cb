// Rotary positions: the table of (cos, sin) for every position and pair, and its application to heads.
//   (x, y) -> (x c - y s, y c + x s),  (c, s) = magnitude (cos, sin)(p f_i)
//
// The table is computed in fp64 (angles of far positions lose all of fp32's digits) and rounded once; programs keep it
// for all of their layers.  Applying it is bound by memory: every value is read and written once.  A thread holds the
// (cos, sin) of eight pairs and takes those pairs in several heads of its token, so that the table (8 bytes a pair, as
// much as a head's values) is read once a token rather than once a head; small calls take one head a thread, since they
// only pay latency.  8192 tokens x 40 heads of 128 dims: 31 us, 0.81 of the measured copy rate; 8 tokens: 2.1 us, the launch.
#include <algorithm>

#include "mkv_paged.cuh"

namespace mkv {

namespace {

constexpr int kThreads = 256;

__global__ void __launch_bounds__(kThreads) table_kernel(const RopeTableCall c) {
  __shared__ double f[128];
  if (threadIdx.x < c.half) {
    const int i = threadIdx.x;
    double w = pow(c.theta, -2.0 * (double)i / (2.0 * c.half));
    if (c.scaling == MKV_ROPE_LINEAR) {
      w /= c.factor;
    } else if (c.scaling == MKV_ROPE_BANDS) {
      const double turns = c.context * w / 6.283185307179586, mix = fmin(fmax((turns - c.low) / (c.high - c.low), 0.0), 1.0);
      w = (1.0 - mix) * w / c.factor + mix * w;
    } else if (c.scaling == MKV_ROPE_RAMP) {
      const double mix = 1.0 - fmin(fmax((i - c.low) / fmax(c.high - c.low, 0.001), 0.0), 1.0);
      w = (1.0 - mix) * w / c.factor + mix * w;
    }
    f[i] = w;
  }
  __syncthreads();
  const int64_t total = c.T_max * c.half;
  for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < total; e += (int64_t)gridDim.x * kThreads) {
    const int64_t p = e / c.half;
    double s, co;
    sincos((double)p * f[(int)(e - p * c.half)], &s, &co);
    c.table[e] = make_float2((float)(co * c.magnitude), (float)(s * c.magnitude));
  }
}

struct ApplyArgs {
  RopeApplyCall c;
  uint32_t* status;
  int cols, turns;      // 16-byte work columns of a head: `turns` of rotated 16 dims, the others of 8 copied dims
  int slots;            // heads that a token's threads take side by side
  int tokens;           // tokens of a block
  int loops;            // heads a thread takes, `slots` apart
};

// Rows, strides and rotated dims that allow 16-byte accesses.
template <bool BF16>
__global__ void __launch_bounds__(kThreads) apply_kernel(const ApplyArgs a) {
  pdl_wait_and_trigger();
  const RopeApplyCall& c = a.c;
  const int per = a.slots * a.cols, tok = threadIdx.x / per, in = threadIdx.x - tok * per;
  const int64_t i = (int64_t)blockIdx.x * a.tokens + tok;
  if (tok >= a.tokens || i >= c.n) return;
  const int slot = in / a.cols, col = in - slot * a.cols;
  const int h0 = blockIdx.y * a.slots * a.loops + slot, h1 = min(c.heads, (int)(blockIdx.y + 1) * a.slots * a.loops);
  const uint16_t* x = c.x + i * c.x_stride;
  uint16_t* out = c.out + i * c.out_stride;
  if (col >= a.turns) {                                   // dims that are not rotated
    const int d = c.rope.rot + 8 * (col - a.turns);
#pragma unroll 4
    for (int h = h0; h < h1; h += a.slots)
      *reinterpret_cast<uint4*>(out + (int64_t)h * c.D + d) = *reinterpret_cast<const uint4*>(x + (int64_t)h * c.D + d);
    return;
  }
  Turn8 t;
  t.load(turn_row(c.rope, c.pos[i], a.status), 8 * col);
  const int lo = turn_lo(col, c.rope.pairs), hi = turn_hi(col, c.rope.rot, c.rope.pairs);
  const float sign = c.transposed ? -1.f : 1.f;
  // (the loads of four heads are under way together)
  constexpr int U = 4;
  for (int h = h0; h < h1; h += U * a.slots) {
    uint4 p0[U], p1[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint16_t* y = x + (int64_t)min(h + u * a.slots, h1 - 1) * c.D;
      if (h + u * a.slots < h1) {
        p0[u] = *reinterpret_cast<const uint4*>(y + lo);
        p1[u] = *reinterpret_cast<const uint4*>(y + hi);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (h + u * a.slots >= h1) break;
      float v[16];
      widen8<BF16>(p0[u], v);
      widen8<BF16>(p1[u], v + 8);
      rotate16(v, t, c.rope.pairs, sign);
      uint16_t* y = out + (int64_t)(h + u * a.slots) * c.D;
      *reinterpret_cast<uint4*>(y + lo) = narrow8<BF16>(v);
      *reinterpret_cast<uint4*>(y + hi) = narrow8<BF16>(v + 8);
    }
  }
}

// Any alignment, stride and even number of rotated dims: a pair or a copied dim a thread.
template <bool BF16>
__global__ void __launch_bounds__(kThreads) apply_any_kernel(const ApplyArgs a) {
  pdl_wait_and_trigger();
  const RopeApplyCall& c = a.c;
  const int half = c.rope.rot / 2, per = half + (c.D - c.rope.rot), total = c.heads * per;
  for (int64_t i = blockIdx.x; i < c.n; i += gridDim.x) {
    const float2* row = turn_row(c.rope, c.pos[i], a.status);
    for (int e = threadIdx.x; e < total; e += kThreads) {
      const int h = e / per, k = e - h * per;
      const uint16_t* x = c.x + i * c.x_stride + (int64_t)h * c.D;
      uint16_t* out = c.out + i * c.out_stride + (int64_t)h * c.D;
      if (k >= half) {
        out[k + half] = x[k + half];
        continue;
      }
      const int d0 = c.rope.pairs ? 2 * k : k, d1 = c.rope.pairs ? 2 * k + 1 : half + k;
      float v0 = widen<BF16>(x[d0]), v1 = widen<BF16>(x[d1]);
      const float2 t = row[k];
      rotate_pair(v0, v1, t.x, c.transposed ? -t.y : t.y);
      const uint32_t p = pack2<BF16>(v0, v1);
      out[d0] = (uint16_t)p;
      out[d1] = (uint16_t)(p >> 16);
    }
  }
}

}  // namespace

cudaError_t launch_rope_scaled_table(const RopeTableCall& c, cudaStream_t st) {
  const int blocks = (int)std::min<int64_t>(ceil_div(c.T_max * c.half, kThreads), (int64_t)kNumSMs * 32);
  table_kernel<<<blocks, kThreads, 0, st>>>(c);
  return cudaPeekAtLastError();
}

cudaError_t launch_rope_apply(const RopeApplyCall& c, cudaStream_t st) {
  ApplyArgs a{};
  const cudaError_t e = status_word(&a.status);
  if (e != cudaSuccess) return e;
  a.c = c;
  const bool bf16 = c.dtype == MKV_BF16;
  auto multiple = [](const void* p, size_t b) { return (reinterpret_cast<uintptr_t>(p) & (b - 1)) == 0; };
  const bool wide = c.rope.rot % 16 == 0 && c.D % 8 == 0 && c.x_stride % 8 == 0 && c.out_stride % 8 == 0 &&
                    multiple(c.x, 16) && multiple(c.out, 16) && multiple(c.rope.table, 16);
  if (!wide) {
    const unsigned grid = (unsigned)std::min<int64_t>(c.n, INT32_MAX);
    return bf16 ? launch_pdl(apply_any_kernel<true>, dim3(grid), dim3(kThreads), 0, st, a)
                : launch_pdl(apply_any_kernel<false>, dim3(grid), dim3(kThreads), 0, st, a);
  }
  a.turns = c.rope.rot / 16;
  a.cols = a.turns + (c.out == c.x ? 0 : (c.D - c.rope.rot) / 8);
  // One head a thread until the GPU's threads (2048 an SM) are taken, then up to eight.  (8192 tokens x 40 heads: eight 31 us,
  // one 99; 8 tokens: 3.4 against 2.1; 1001 tokens of 12 heads of 64: 4.3 against 3.8.)
  const int64_t work = c.n * c.heads * a.cols;
  a.loops = (int)std::min<int64_t>(8, std::max<int64_t>(1, work / (2048 * kNumSMs)));
  a.slots = (int)std::min<int64_t>(ceil_div(c.heads, a.loops), kThreads / a.cols);
  a.tokens = kThreads / (a.slots * a.cols);
  const int64_t gx = ceil_div(c.n, a.tokens);
  if (gx > INT32_MAX) return cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)gx, (unsigned)ceil_div(c.heads, a.slots * a.loops));
  return bf16 ? launch_pdl(apply_kernel<true>, grid, dim3(kThreads), 0, st, a)
              : launch_pdl(apply_kernel<false>, grid, dim3(kThreads), 0, st, a);
}

}  // namespace mkv
