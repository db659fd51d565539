// Attention over the paged cache, the plain way: one CTA per (token, query head), which walks the visible
// keys 128 at a time with the running maximum and sum of the softmax.
#include <cuda_fp16.h>

#include "common.cuh"
#include "kv.h"

namespace icc {

namespace {

constexpr int THREADS = 128;

template <bool F16>
__device__ __forceinline__ float to_f32(uint16_t x) {
  if (F16) return __half2float(__ushort_as_half(x));
  return __uint_as_float((uint32_t)x << 16);
}
template <bool F16>
__device__ __forceinline__ uint16_t from_f32(float x) {
  if (F16) return __half_as_ushort(__float2half_rn(x));
  return __bfloat16_as_ushort(__float2bfloat16_rn(x));
}

__device__ float block_reduce(float x, bool maximum, float* sums) {
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const float y = __shfl_xor_sync(FULL_MASK, x, d);
    x = maximum ? fmaxf(x, y) : x + y;
  }
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = x;
  __syncthreads();
  x = sums[0];
  for (int w = 1; w < THREADS / 32; ++w) x = maximum ? fmaxf(x, sums[w]) : x + sums[w];
  __syncthreads();
  return x;
}

template <bool F16>
__global__ void __launch_bounds__(THREADS) kv_attend_simple_kernel(const KvAttendParams p) {
  __shared__ float q[256], w[THREADS], sums[4];
  __shared__ const unsigned char* rows[THREADS];
  const KvView& v = p.v;
  const int64_t t = blockIdx.x;
  const int head = blockIdx.y, kvh = head / p.group, D = v.head_dim, tid = threadIdx.x;
  int i = (int)t, end = (int)t + 1;
  if (p.starts) {
    for (i = 0; i + 1 < p.n && p.starts[i + 1] <= t; ++i) {}
    end = p.starts[i + 1];
  }
  const int s = p.seqs[i];
  int64_t pos = -1;
  if (s >= 0 && s < v.max_seqs && t < end) pos = (int64_t)v.lengths[s] - end + t;
  else if (tid == 0) kv_report(v, KV_INVALID);
  if (pos >= ((int64_t)v.max_pages << v.page_shift)) pos = -1;
  const uint16_t* qg = reinterpret_cast<const uint16_t*>(p.q) + t * p.q_token_stride + head * p.q_head_stride;
  for (int d = tid; d < D; d += THREADS) q[d] = to_f32<F16>(qg[d]);
  float m = -INFINITY, l = 0.0f, acc[2] = {0.0f, 0.0f};
  const int64_t first = p.window ? max((int64_t)0, pos - p.window + 1) : 0;
  const int64_t sinks = min((int64_t)(p.window ? p.sinks : 0), first);
  const size_t block = ((size_t)D * 2) << v.page_shift;
  for (int64_t j0 = sinks > 0 ? 0 : first / THREADS * THREADS; j0 <= pos;) {
    const int64_t j = j0 + tid;
    const bool seen = j <= pos && (j >= first || j < sinks);
    float x = -INFINITY;
    __syncthreads();
    rows[tid] = nullptr;
    if (seen) {
      const int page = v.tables[(size_t)s * v.max_pages + (j >> v.page_shift)];
      if (page >= 0 && page < v.n_pages) {
        const unsigned char* kr = v.pool + (size_t)page * v.page_bytes + ((size_t)p.layer * 2 * v.n_kv_heads + kvh) * block +
                                  (size_t)(j & ((1 << v.page_shift) - 1)) * D * 2;
        float dot = 0.0f;
        for (int d = 0; d < D; ++d) dot += q[d] * to_f32<F16>(reinterpret_cast<const uint16_t*>(kr)[d]);
        x = dot * p.scale_log2;
        rows[tid] = kr + (size_t)v.n_kv_heads * block;
      }
    }
    const float top = fmaxf(m, block_reduce(x, true, sums));
    const float e = rows[tid] ? exp2f(x - (top == -INFINITY ? 0.0f : top)) : 0.0f;
    w[tid] = e;
    const float shrink = m == -INFINITY ? 0.0f : exp2f(m - top);
    l = l * shrink + block_reduce(e, false, sums);
    m = top;
    for (int c = 0; c < 2; ++c) {
      const int d = tid + c * THREADS;
      if (d >= D) continue;
      float a = acc[c] * shrink;
      for (int y = 0; y < THREADS; ++y)
        if (rows[y]) a += w[y] * to_f32<F16>(reinterpret_cast<const uint16_t*>(rows[y])[d]);
      acc[c] = a;
    }
    j0 += THREADS;
    if (j0 >= sinks && j0 < first / THREADS * THREADS) j0 = first / THREADS * THREADS;
  }
  uint16_t* og = reinterpret_cast<uint16_t*>(p.out) + t * p.out_token_stride + head * p.out_head_stride;
  for (int c = 0; c < 2; ++c) {
    const int d = tid + c * THREADS;
    if (d < D) og[d] = from_f32<F16>(l == 0.0f ? 0.0f : acc[c] / l);
  }
}

}  // namespace

cudaError_t kv_attend_simple_launch(const KvAttendParams& p, bool f16, cudaStream_t st) {
  const dim3 grid((unsigned)p.n_tokens, (unsigned)p.n_heads);
  if (f16) kv_attend_simple_kernel<true><<<grid, THREADS, 0, st>>>(p);
  else kv_attend_simple_kernel<false><<<grid, THREADS, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace icc
