// What the page operations share: prefix sums over a CTA, the checks of borrowed books, and where a token lies.
#pragma once
#include "common.cuh"
#include "kv.h"

namespace icc {

// Exclusive prefix sum over the CTA; *total gets the sum.  Unsigned, so that two packed counters may be
// summed at once.  `sums`: 33 words of shared memory; ends with a barrier.
__device__ __forceinline__ unsigned block_scan(unsigned x, unsigned* sums, unsigned* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned inc = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned y = __shfl_up_sync(FULL_MASK, inc, d);
    if (lane >= d) inc += y;
  }
  if (lane == 31) sums[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    const unsigned w = lane < (int)(blockDim.x >> 5) ? sums[lane] : 0u;
    unsigned winc = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned y = __shfl_up_sync(FULL_MASK, winc, d);
      if (lane >= d) winc += y;
    }
    sums[lane] = winc - w;
    if (lane == 31) sums[32] = winc;
  }
  __syncthreads();
  const unsigned before = sums[warp] + inc - x;
  *total = sums[32];
  __syncthreads();
  return before;
}

// Which of begin[0..n) holds rank r (begin ascends; entries without pages repeat their successor's value).
__device__ __forceinline__ int owner_of(const int* begin, int n, int r) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (begin[mid] <= r) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// A length is one that the sequence's row holds.  Lent lengths that are not an earlier cache's may be anything, and
// the rows' entries are counted by them.
__device__ __forceinline__ bool length_fits(const KvView& v, int tokens) {
  return tokens >= 0 && tokens <= (v.max_pages << v.page_shift);
}

// An owned table entry names a page of the pool.  One that does not (lent tables that are not an earlier cache's) is
// reported.
__device__ __forceinline__ bool page_exists(const KvView& v, int page) {
  if ((unsigned)page < (unsigned)v.n_pages) return true;
  kv_report(v, KV_INVALID);
  return false;
}

// What a write needs to be right of sequence i of the call: the sequence, where its tokens begin and end, and its length.
struct WriteSeq {
  int s, length;
  int64_t begin, end;
  bool fine;
  __device__ __forceinline__ WriteSeq(const KvView& v, const int* seqs, const int* starts, int i, int n, int64_t n_tokens) {
    s = seqs[i];
    begin = starts ? starts[i] : i;
    end = starts ? starts[i + 1] : i + 1;
    length = 0;
    fine = s >= 0 && s < v.max_seqs && begin <= end && (i > 0 || begin == 0) && (i + 1 < n || end == n_tokens);
    if (fine) {
      length = v.lengths[s];
      fine = length_fits(v, length) && end - begin <= length;
    }
  }
};

// First byte of a token's key row of head 0, or null.
__device__ __forceinline__ unsigned char* token_place(const KvView& v, int layer, int s, int pos) {
  const int page = v.tables[(size_t)s * v.max_pages + (pos >> v.page_shift)];
  if (!page_exists(v, page)) return nullptr;
  const size_t row = (size_t)layer * 2 * v.n_kv_heads << v.page_shift;
  return v.pool + (size_t)page * v.page_bytes + (row + (size_t)(pos & ((1 << v.page_shift) - 1))) * v.head_dim * 2;
}

}  // namespace icc
