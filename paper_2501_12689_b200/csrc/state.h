// State cache: what its kernels are given, and the launch functions that state_cache.cu calls.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace icc {

constexpr int STATE_MAX_SEQS = 8192, STATE_MAX_HEADS = 1024;

// The cache as the kernels see it.
struct StateView {
  float* pool;
  int n_layers, n_heads, key_dim, value_dim, max_seqs;
  int* err;                 // first error since the last ic_state_sync (codes as in kv.h)
  int* host_status;         // mapped host word, the same
  int* meta;                // [0] 1 = the arguments of this call hold; zero between calls: [1] clear: a number was bad, [2] its CTAs that have finished
  __host__ __device__ size_t head_floats() const { return (size_t)key_dim * value_dim; }
  __host__ __device__ size_t seq_floats() const { return head_floats() * n_layers * n_heads; }
};

// Rows of tokens and heads; strides in elements.
struct StateRows {
  const unsigned char* at;
  int64_t token_stride, head_stride;
};

struct StateAttendParams {
  StateView v;
  StateRows q, k, val, out;
  const float* rates;
  const int* seqs;
  const int* starts;        // null: one token per sequence
  int n, layer, checked;    // checked: a kernel before has looked over the arguments
  const int* ends;          // in chunks: where each sequence's tokens end
  int most, least;          // token by token: sequences of up to `most` tokens; in chunks: of more than `least`
  int n_long;               // sequences for the chunks, at most; 0 = none
  int* long_ones;           // [3, max_seqs] their numbers, starts and ends, in their order, and empty ones up to n_long: made by the check ahead of a call
  int64_t n_tokens;
  float scale;
  // calls of many tokens: value slices of a head; states that CTAs publish for one another, and how much of each is there
  int slices, first_item, n_items;        // (heads times slices) items of a launch
  float* slots;
  size_t slot_floats;       // of one CTA's
  unsigned* flags;          // [CTAs + 1], zero between launches
};

cudaError_t state_configure(int smem_optin);
cudaError_t state_check_launch(const StateAttendParams& p, cudaStream_t st);
// Few tokens a sequence: one after the other.
cudaError_t state_step_launch(const StateAttendParams& p, bool f16, int sm_count, cudaStream_t st);
cudaError_t state_fork_launch(const StateView& v, const int* parents, const int* children, int n, int sm_count, int* launches, cudaStream_t st);
cudaError_t state_clear_launch(const StateView& v, const int* seqs, int n, int sm_count, cudaStream_t st);

// Many tokens a sequence: chunks of them, on the tensor cores.  At most STATE_BATCH sequences a launch.
cudaError_t state_chunk_configure(int smem_optin);
size_t state_slot_floats(int key_dim, int value_dim);
// Rows of q, k and v as tensor maps [heads, tokens, dim] of boxes of 64 tokens and 64 elements; there: all three could be made.
struct StateMaps {
  CUtensorMap q, k, val;
  int there;
};
cudaError_t state_chunk_launch(StateAttendParams p, const StateMaps& maps, bool f16, int sm_count, int smem_optin, cudaStream_t st);

constexpr int STATE_CHECK_THREADS = 256;  // sequences that every CTA looks over by itself

}  // namespace icc
