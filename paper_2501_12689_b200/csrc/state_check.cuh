// The arguments of a call over the states, looked over by a whole CTA.
#pragma once
#include "common.cuh"
#include "kv.h"
#include "state.h"

namespace icc {

__device__ __forceinline__ void state_report(const StateView& v, int code) {
  if (atomicCAS(v.err, KV_OK, code) == KV_OK) {
    *reinterpret_cast<volatile int*>(v.host_status) = code;
    __threadfence_system();
  }
}

// seen: STATE_MAX_SEQS bits of shared memory.  Every thread of the CTA calls it; all get the same answer.
__device__ __forceinline__ bool state_check_seqs(const StateView& v, const int* seqs, int n, uint32_t* seen) {
  for (int i = threadIdx.x; i < STATE_MAX_SEQS / 32; i += blockDim.x) seen[i] = 0;
  __syncthreads();
  bool fine = true;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int s = seqs[i];
    if (s < 0 || s >= v.max_seqs) fine = false;
    else if (atomicOr(&seen[s >> 5], 1u << (s & 31)) >> (s & 31) & 1) fine = false;      // twice
  }
  return __syncthreads_and(fine);
}
__device__ __forceinline__ bool state_check_attend(const StateAttendParams& p, uint32_t* seen) {
  bool fine = true;
  for (int h = threadIdx.x; h < p.v.n_heads; h += blockDim.x) fine &= p.rates[h] >= 0.0f;
  if (p.starts)
    for (int i = threadIdx.x; i < p.n; i += blockDim.x) {
      const int a = p.starts[i], b = p.starts[i + 1];
      fine &= a <= b && (i > 0 || a == 0) && (i + 1 < p.n || b == p.n_tokens);
    }
  return state_check_seqs(p.v, p.seqs, p.n, seen) & __syncthreads_and(fine);
}

// Whether the call goes on: nothing was wrong before it, and its arguments hold.  Whole CTA; ends with a barrier.
// (Another CTA of the launch may set the error while this one's threads look at it: they decide together, no thread leaves by itself.)
__device__ __forceinline__ bool state_call_holds(const StateAttendParams& p, uint32_t* seen) {
  if (__syncthreads_or(*p.v.err != KV_OK)) return false;
  if (p.checked || state_check_attend(p, seen)) return true;
  if (threadIdx.x == 0) state_report(p.v, KV_INVALID);
  return false;
}

}  // namespace icc
