// Linear attention with a decay per head, token by token; forks and resets of states.
//
//   S <- e^(-rate) S + k v^T,   out = scale q S
//
// A CTA holds a slice of SLICE value columns of one sequence and head in registers: four columns of every RP-th row a thread.  The bound is the
// state, read and written once, 8 bytes an element against two fused products; all of a thread's loads are under way
// together, and while they are the call is looked over.  64 sequences, 32 heads of 128 x 128: 50 us, 5.3 TB/s.
// e^(-rate) is kept as two floats: over several tokens its rounding would add up.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kernels.h"
#include "kv_mma.cuh"
#include "kv_pages.cuh"
#include "pipeline.cuh"
#include "state_check.cuh"

namespace icc {

namespace {

constexpr int THREADS = 256;

template <bool F16>
__device__ __forceinline__ float to_float(uint16_t x) {
  return F16 ? __half2float(__ushort_as_half(x)) : __uint_as_float((uint32_t)x << 16);
}
template <bool F16>
__device__ __forceinline__ float4 load4(const uint16_t* p) {
  const uint2 x = *reinterpret_cast<const uint2*>(p);
  return make_float4(to_float<F16>((uint16_t)x.x), to_float<F16>((uint16_t)(x.x >> 16)), to_float<F16>((uint16_t)x.y), to_float<F16>((uint16_t)(x.y >> 16)));
}

template <bool F16, int SLICE, int ROUNDS>
__global__ void __launch_bounds__(THREADS) state_step_kernel(const StateAttendParams p) {
  constexpr int PER_ROW = SLICE / 4, RP = THREADS / PER_ROW;     // threads of a row; rows at a time
  __shared__ uint32_t seen[STATE_MAX_SEQS / 32];
  __shared__ float qs[2][RP * ROUNDS], ks[2][RP * ROUNDS];
  __shared__ float parts[THREADS / 32][SLICE];
  grid_dep_launch_dependents();
  grid_dep_wait();
  const StateView& v = p.v;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int slices = (v.value_dim + SLICE - 1) / SLICE;
  int x = blockIdx.x;
  const int slice = x % slices;
  x /= slices;
  const int head = x % v.n_heads, i = x / v.n_heads;
  const int first = p.starts ? p.starts[i] : i, count = p.starts ? p.starts[i + 1] - first : 1, seq = p.seqs[i];
  const int r0 = tid / PER_ROW, col = slice * SLICE + tid % PER_ROW * 4;
  const bool here = col < v.value_dim;
  // the state is on its way while the call is looked over
  const bool some = count > 0 && count <= p.most && seq >= 0 && seq < v.max_seqs;
  float* state = v.pool + (((size_t)seq * v.n_layers + p.layer) * v.n_heads + head) * v.head_floats() + col;
  float4 s[ROUNDS];
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    const int r = j * RP + r0;
    s[j] = some && here && r < v.key_dim ? *reinterpret_cast<const float4*>(state + (size_t)r * v.value_dim) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  }
  const uint16_t* q = reinterpret_cast<const uint16_t*>(p.q.at) + first * p.q.token_stride + head * p.q.head_stride;
  const uint16_t* k = reinterpret_cast<const uint16_t*>(p.k.at) + first * p.k.token_stride + head * p.k.head_stride;
  const uint16_t* val = reinterpret_cast<const uint16_t*>(p.val.at) + first * p.val.token_stride + head * p.val.head_stride + col;
  uint16_t* out = reinterpret_cast<uint16_t*>(const_cast<unsigned char*>(p.out.at)) + first * p.out.token_stride + head * p.out.head_stride;
  __shared__ float2 decay_of;
  if (tid == 0) {                  // (one thread: 64-bit exponentials are slow)
    const double decay = exp(-(double)p.rates[head]);
    decay_of = make_float2((float)decay, (float)(decay - (double)(float)decay));
  }
  if (!state_call_holds(p, seen) || count == 0 || count > p.most) return;
  auto fetch = [&](int t) {
    for (int d = tid; d < 2 * RP * ROUNDS; d += THREADS) {
      const bool of_k = d >= RP * ROUNDS;
      const int e = of_k ? d - RP * ROUNDS : d;
      float y = 0.0f;
      if (e < v.key_dim) y = to_float<F16>(of_k ? k[t * p.k.token_stride + e] : q[t * p.q.token_stride + e]);
      (of_k ? ks : qs)[t & 1][e] = y;
    }
  };
  fetch(0);
  for (int t = 0; t < count; ++t) {
    const float4 w = here ? load4<F16>(val + t * p.val.token_stride) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    __syncthreads();                 // this token's q and k are there, and the last one's parts have been read
    if (t + 1 < count) fetch(t + 1);
    const float high = decay_of.x, low = decay_of.y;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < ROUNDS; ++j) {
      const float kk = ks[t & 1][j * RP + r0], qq = qs[t & 1][j * RP + r0];
      s[j].x = fmaf(s[j].x, high, fmaf(s[j].x, low, kk * w.x));
      s[j].y = fmaf(s[j].y, high, fmaf(s[j].y, low, kk * w.y));
      s[j].z = fmaf(s[j].z, high, fmaf(s[j].z, low, kk * w.z));
      s[j].w = fmaf(s[j].w, high, fmaf(s[j].w, low, kk * w.w));
      o.x = fmaf(qq, s[j].x, o.x);
      o.y = fmaf(qq, s[j].y, o.y);
      o.z = fmaf(qq, s[j].z, o.z);
      o.w = fmaf(qq, s[j].w, o.w);
    }
#pragma unroll
    for (int d = 16; d >= PER_ROW; d >>= 1) {
      o.x += __shfl_xor_sync(FULL_MASK, o.x, d);
      o.y += __shfl_xor_sync(FULL_MASK, o.y, d);
      o.z += __shfl_xor_sync(FULL_MASK, o.z, d);
      o.w += __shfl_xor_sync(FULL_MASK, o.w, d);
    }
    if (lane < PER_ROW) *reinterpret_cast<float4*>(&parts[warp][lane * 4]) = o;
    __syncthreads();
    if (tid < SLICE && slice * SLICE + tid < v.value_dim) {
      float sum = 0.0f;
#pragma unroll
      for (int y = 0; y < THREADS / 32; ++y) sum += parts[y][tid];
      out[t * p.out.token_stride + slice * SLICE + tid] = round16<F16>(sum * p.scale);
    }
  }
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    const int r = j * RP + r0;
    if (here && r < v.key_dim) *reinterpret_cast<float4*>(state + (size_t)r * v.value_dim) = s[j];
  }
}

// ---------------------------------------------------------------- checks ahead of a launch
constexpr int PLAN_THREADS = 1024;

__global__ void __launch_bounds__(PLAN_THREADS) state_check_kernel(const StateAttendParams p) {
  __shared__ uint32_t seen[STATE_MAX_SEQS / 32];
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (*p.v.err != KV_OK) return;
  if (!state_check_attend(p, seen)) {
    if (threadIdx.x == 0) state_report(p.v, KV_INVALID);
    return;
  }
  // the sequences that are left to the chunks
  if (p.n_long == 0) return;
  __shared__ unsigned sums[33];
  int* const list[3] = {p.long_ones, p.long_ones + p.v.max_seqs, p.long_ones + 2 * p.v.max_seqs};
  unsigned found = 0, total;
  for (int i0 = 0; i0 < p.n; i0 += PLAN_THREADS) {
    const int i = i0 + threadIdx.x;
    const bool some = i < p.n && p.starts[i + 1] - p.starts[i] > p.most;
    const unsigned at = found + block_scan(some, sums, &total);
    if (some) {                           // (at most n_long, as each has more than `most` of the call's tokens)
      list[0][at] = p.seqs[i];
      list[1][at] = p.starts[i];
      list[2][at] = p.starts[i + 1];
    }
    found += total;
  }
  for (int at = (int)found + threadIdx.x; at < p.n_long; at += PLAN_THREADS) list[0][at] = list[1][at] = list[2][at] = 0;
}

// ---------------------------------------------------------------- fork
__global__ void __launch_bounds__(PLAN_THREADS) state_fork_plan_kernel(const StateView v, const int* __restrict__ parents, const int* __restrict__ children,
                                                                       int n) {
  __shared__ uint32_t seen[STATE_MAX_SEQS / 32];
  grid_dep_launch_dependents();
  grid_dep_wait();
  bool fine = *v.err == KV_OK;
  for (int i = threadIdx.x; i < n; i += PLAN_THREADS) fine &= parents[i] >= 0 && parents[i] < v.max_seqs;
  fine = state_check_seqs(v, children, n, seen) & __syncthreads_and(fine);
  if (threadIdx.x == 0) {
    v.meta[0] = fine;
    if (!fine && *v.err == KV_OK) state_report(v, KV_INVALID);
  }
}

// A CTA takes the same `tile` vectors of 16 bytes of all n parents into shared memory and then writes them to the children, so that any exchange
// among them comes out right.
__global__ void __launch_bounds__(THREADS) state_fork_kernel(const StateView v, const int* __restrict__ parents, const int* __restrict__ children, int n,
                                                             int tile) {
  extern __shared__ uint4 held[];          // [n, tile]
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (v.meta[0] == 0) return;
  const size_t vectors = v.seq_floats() / 4;
  uint4* pool = reinterpret_cast<uint4*>(v.pool);
  for (size_t c = (size_t)blockIdx.x * tile; c < vectors; c += (size_t)gridDim.x * tile) {
    for (int u = threadIdx.x; u < n * tile; u += THREADS) {
      const int i = u / tile, j = u - i * tile, a = parents[i];
      if (a != children[i] && c + j < vectors) held[u] = pool[a * vectors + c + j];
    }
    __syncthreads();
    for (int u = threadIdx.x; u < n * tile; u += THREADS) {
      const int i = u / tile, j = u - i * tile, b = children[i];
      if (b != parents[i] && c + j < vectors) pool[b * vectors + c + j] = held[u];
    }
    __syncthreads();
  }
}

// A bad number is passed over and the others cleared, so it is reported by the CTA that finishes last: an error that stood while others begin would
// stop them.
__global__ void __launch_bounds__(THREADS) state_clear_kernel(const StateView v, const int* __restrict__ seqs, int n) {
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (*v.err != KV_OK) return;
  const size_t vectors = v.seq_floats() / 4;
  uint4* pool = reinterpret_cast<uint4*>(v.pool);
  bool bad = false;
  for (int i = blockIdx.y; i < n; i += gridDim.y) {
    const int s = seqs[i];
    if (s < 0 || s >= v.max_seqs) {
      bad = true;
      continue;
    }
    for (size_t c = (size_t)blockIdx.x * THREADS + threadIdx.x; c < vectors; c += (size_t)gridDim.x * THREADS)
      pool[s * vectors + c] = make_uint4(0, 0, 0, 0);
  }
  __syncthreads();                         // all threads have looked at the error
  if (threadIdx.x == 0) {
    if (bad) atomicExch(&v.meta[1], 1);
    __threadfence();
    if (atomicAdd(&v.meta[2], 1) == (int)(gridDim.x * gridDim.y) - 1) {
      v.meta[2] = 0;
      if (atomicExch(&v.meta[1], 0) != 0) state_report(v, KV_INVALID);
    }
  }
}

constexpr int FORK_SMEM = STATE_MAX_SEQS * 16;

template <bool F16, int SLICE>
cudaError_t step_launch(const StateAttendParams& p, cudaStream_t st) {
  const int slices = (p.v.value_dim + SLICE - 1) / SLICE, rows = THREADS / (SLICE / 4), rounds = (p.v.key_dim + rows - 1) / rows;
  constexpr int MOST = 128 / (THREADS / (SLICE / 4));         // rounds for the largest key_dim
  auto* kernel = rounds <= MOST / 4 ? state_step_kernel<F16, SLICE, MOST / 4> : rounds <= MOST / 2 ? state_step_kernel<F16, SLICE, MOST / 2> : state_step_kernel<F16, SLICE, MOST>;
  return launch_overlapped(kernel, dim3((unsigned)p.n * p.v.n_heads * slices), dim3(THREADS), 0, st, 1, p);
}

}  // namespace

cudaError_t state_configure(int smem_optin) {
  (void)smem_optin;
  return cudaFuncSetAttribute(state_fork_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FORK_SMEM);
}

cudaError_t state_check_launch(const StateAttendParams& p, cudaStream_t st) {
  return launch_overlapped(state_check_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, 1, p);
}

cudaError_t state_step_launch(const StateAttendParams& p, bool f16, int sm_count, cudaStream_t st) {
  // Slices of 64 columns, 32 KB of a state of 128 x 128, have the memory busy all the time (64 sequences, 32 heads of 128 x 128: 50 us; with 128 columns
  // 55, with 32 columns 64).  Below two CTAs an SM the narrower ones wait less (4 sequences 6.6 us; 6, as 64 columns, 8.4, as 32 9.4).
  const bool narrow = (int64_t)p.n * p.v.n_heads * ((p.v.value_dim + 63) / 64) < 2 * sm_count;
  if (narrow) return f16 ? step_launch<true, 32>(p, st) : step_launch<false, 32>(p, st);
  return f16 ? step_launch<true, 64>(p, st) : step_launch<false, 64>(p, st);
}

cudaError_t state_fork_launch(const StateView& v, const int* parents, const int* children, int n, int sm_count, int* launches, cudaStream_t st) {
  *launches = 2;
  cudaError_t e = launch_overlapped(state_fork_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, 1, v, parents, children, n);
  if (e != cudaSuccess) return e;
  int tile = FORK_SMEM / 2 / 16 / n;       // two CTAs an SM, or what one sequence after the other needs
  tile = tile > 256 ? 256 : tile < 1 ? 1 : tile;
  return launch_overlapped(state_fork_kernel, dim3((unsigned)(2 * sm_count)), dim3(THREADS), (size_t)n * tile * 16, st, 1, v, parents, children, n, tile);
}

cudaError_t state_clear_launch(const StateView& v, const int* seqs, int n, int sm_count, cudaStream_t st) {
  const size_t parts = (v.seq_floats() / 4 + 8 * THREADS - 1) / (8 * THREADS);
  const unsigned y = n < 1024 ? n : 1024, most = (unsigned)(8 * sm_count + y - 1) / y;
  return launch_overlapped(state_clear_kernel, dim3((unsigned)(parts < most ? parts : most), y), dim3(THREADS), 0, st, 1, v, seqs, n);
}

}  // namespace icc
