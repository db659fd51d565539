// Paged key-value cache: what its kernels are given, and the launch functions that kv_cache.cu calls.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace icc {

// What a kernel finds wrong with a call.  The first code is kept in device memory (the kernels that
// change the cache look there and do nothing) and in the handle's mapped host word.
enum : int { KV_OK = 0, KV_TIMEOUT = 2, KV_FULL = 4, KV_INVALID = 5 };

// The cache as the kernels see it.  A page is page_bytes long and holds all layers; the block of one
// (layer, keys or values, head) in it is page_size rows of head_dim 2-byte elements.
struct KvView {
  unsigned char* pool;
  int* tables;
  int* lengths;
  int* refs;
  int n_pages, n_layers, n_kv_heads, head_dim, max_seqs, max_pages;
  int page_shift;           // page_size = 1 << page_shift
  size_t page_bytes;
  // scratch of the page operations
  int* err;                 // first error since the last ic_kv_sync
  int* host_status;         // mapped host word, the same
  int* meta;                // [0] 1 = the plan of this call holds, [1] pages to copy, [2] live pages
  int* had;                 // [max_seqs] fork: a child's tokens before the call
  int* upto;                // [max_seqs] fork: its tokens after the call; -1 = nothing to do
  int* shared;              // [max_seqs] fork: leading pages shared with the parent
  int* begin;               // [max_seqs] fork: its first entry in `fresh`
  int* mark;                // [max_seqs] zero between calls; a sequence that came up in this call
  int* fresh;               // [n_pages] pages handed out; compact: rank of a page that moves
  int2* jobs;               // [n_pages] pages to copy: from, to
  int* staged;              // [max_seqs, max_pages] fork: the children's new rows
};

__device__ __forceinline__ int kv_pages_of(int tokens, int page_shift) {
  return (int)(((unsigned)tokens + (1u << page_shift) - 1u) >> page_shift);
}

// Keep the first error: device word for later kernels, host word for the caller.
__device__ __forceinline__ void kv_report(const KvView& v, int code) {
  if (atomicCAS(v.err, KV_OK, code) == KV_OK) {
    *reinterpret_cast<volatile int*>(v.host_status) = code;
    __threadfence_system();
  }
}

// One attention call, as the kernels see it.
struct KvAttendParams {
  KvView v;
  const unsigned char* q;
  unsigned char* out;
  int64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;   // elements
  const int* seqs;
  const int* starts;        // null: one token per sequence
  int n, n_heads, group, layer;
  int64_t n_tokens;         // of the whole call: `starts` and first_seq index its q
  int first_seq, n_seqs;    // where in the call this launch's sequences begin (starts null: its first token), and how many that has
  int window, sinks;
  unsigned group_magic;     // x / group = x * group_magic >> group_shift for 0 <= x < 2^31
  int group_shift;
  float scale_log2;         // scale * log2(e): the softmax works in powers of two
  // pieces of items that span CTAs: two slots per CTA, and per CTA (and row tile, where an item has two)
  // how many pieces of the item that begins in it and goes on have arrived (zero between launches)
  float* partials;
  int* arrivals;
  size_t partial_floats;    // of one slot
};

__device__ __forceinline__ int kv_token_of(const KvAttendParams& p, int row) {
  return (int)(((unsigned long long)(unsigned)row * p.group_magic) >> p.group_shift);
}

cudaError_t kv_reserve_launch(const KvView& v, const int* seqs, const int* counts, int n, cudaStream_t st);
cudaError_t kv_write_launch(const KvView& v, int layer, const void* k, const void* val, int64_t token_stride, int64_t head_stride,
                            const int* seqs, const int* starts, int n, int64_t n_tokens, int sm_count, int* launches, cudaStream_t st);
cudaError_t kv_fork_launch(const KvView& v, const int* parents, const int* children, const int* upto, int n, int copy,
                           int sm_count, int* launches, cudaStream_t st);
cudaError_t kv_free_launch(const KvView& v, const int* seqs, int n, int sm_count, cudaStream_t st);
cudaError_t kv_compact_launch(const KvView& v, int sm_count, int* launches, cudaStream_t st);
cudaError_t kv_pages_configure(int smem_optin);

cudaError_t kv_decode_configure(int smem_optin);
// tmap: the pool as rows of head_dim elements, box of 64 elements x min(page_size, 64) rows, 128-byte swizzle.
// two: 16 rows per item instead of 8.
cudaError_t kv_decode_launch(const KvAttendParams& p, const CUtensorMap& tmap, bool f16, bool two, int sm_count, int smem_optin, cudaStream_t st);
cudaError_t kv_extend_configure(int smem_optin);
size_t kv_extend_partial_floats(int head_dim);
cudaError_t kv_extend_launch(const KvAttendParams& p, const CUtensorMap& tmap, bool f16, int sm_count, int smem_optin, cudaStream_t st);
constexpr int KV_BATCH = 256;      // sequences per attention launch
constexpr int KV_MAX_CTAS = 160;   // attention kernels run one CTA per SM, of which there are at most this many

}  // namespace icc
