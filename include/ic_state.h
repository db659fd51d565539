/*
 * ic_state.h - C ABI of the state cache: linear attention with a decay per head.
 *
 * The recurrent layers that stand between a model's attention layers keep no pages: what a sequence has seen is one matrix per layer
 * and head.  As with the pages of ic_kv.h, a retrieved example is run through the model once, requests that
 * begin with it fork from its state, and go on with their own tokens.
 *
 *     S_t = e^(-rate) S_(t-1) + k_t v_t^T          S [key_dim, value_dim], in fp32
 *     out_t = scale * q_t S_t
 *
 * token by token, for every sequence, head and layer on its own.
 *
 * Storage, on the device: pool [max_seqs, n_layers, n_heads, key_dim, value_dim], fp32.  The state of a sequence that has seen nothing is
 * zeros.
 *
 * Conventions as in ic_kv.h: index arrays are device arrays, calls enqueue on the handle's stream without synchronising and can be
 * captured; what only the device can see (a sequence out of range or twice, starts that do not ascend, a rate that is
 * negative or NaN) is found by the kernels: such a call changes nothing and writes no result, the error is kept, later calls
 * do nothing until ic_state_sync has reported and cleared it.  (ic_state_clear skips a bad number and clears the others.)  One
 * handle per stream, not thread-safe.  Graphs captured from one handle share its workspace and its states: they must not run at the
 * same time.  There is no CPU fallback.
 */
#ifndef IC_STATE_H_
#define IC_STATE_H_

#include "ic_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ic_state ic_state_t; /* opaque, owned by the library */

enum ic_state_dtype { IC_STATE_BF16 = 0, IC_STATE_F16 = 1 };

#define IC_STATE_MAX_KEY_DIM 128   /* key_dim: a multiple of 8 up to this                      */
#define IC_STATE_MAX_VALUE_DIM 256 /* value_dim: a multiple of 8 up to this                    */
#define IC_STATE_MAX_SEQS 8192     /* largest max_seqs                                         */

/* Zero-initialise, set struct_size = sizeof, then fill. */
typedef struct ic_state_opts {
  uint32_t struct_size; /* sizeof(ic_state_opts_t) of the caller's build                      */
  int32_t device;       /* CUDA device ordinal; -1 = the current device                       */
  int32_t dtype;        /* ic_state_dtype of q, k, v and out                                  */
  int32_t n_layers;     /* 1 .. 1024                                                          */
  int32_t n_heads;      /* 1 .. 1024                                                          */
  int32_t key_dim;
  int32_t value_dim;
  int32_t max_seqs;     /* states of the pool                                                 */
  float* pool;          /* optional caller-owned device buffer, 256-byte aligned, taken as it is; NULL = the */
                        /*   library allocates one of zeros                                   */
  void* stream;         /* cudaStream_t; NULL = the legacy default stream                     */
  void* workspace;      /* optional caller-owned scratch, 256-byte aligned; NULL = library    */
  size_t workspace_bytes; /* its size, at least ic_state_workspace_bytes                      */
} ic_state_opts_t;

/* NULL on failure; ic_cache_last_error() then describes why.  No later call allocates. */
ic_state_t* ic_state_create(const ic_state_opts_t* opts);

/* Bytes of workspace for these options; 0 for invalid options. */
size_t ic_state_workspace_bytes(const ic_state_opts_t* opts);

/*
 * The newest tokens of sequences seqs[i], i < n (no sequence twice), through one layer: their states are brought up to date, and
 * every token's result is written.  Sums are held in fp32.  In calls of several tokens a sequence, products of two computed numbers
 * (scores with values, queries with states) round one of them to the 16-bit type first; the state itself is not rounded.
 * An infinite or NaN value may also reach its sequence and head's other tokens in the call, and where the formula gives an infinity the result
 * may be a NaN.
 */
typedef struct ic_state_attend {
  uint32_t struct_size; /* sizeof(ic_state_attend_t) of the caller's build                    */
  int32_t layer;
  int32_t n;            /* sequences                                                          */
  float scale;          /* of the results, finite; 1 / sqrt(key_dim) as a rule                */
  int64_t n_tokens;     /* tokens in all                                                      */
  const void* q;        /* [n_tokens, n_heads, key_dim]: token t, head h at element           */
  int64_t q_token_stride; /*   t * q_token_stride + h * q_head_stride; 16-byte aligned,       */
  int64_t q_head_stride;  /*   strides non-negative multiples of 8 elements (0: shared)       */
  const void* k;        /* the same                                                           */
  int64_t k_token_stride;
  int64_t k_head_stride;
  const void* v;        /* [n_tokens, n_heads, value_dim]                                     */
  int64_t v_token_stride;
  int64_t v_head_stride;
  void* out;            /* [n_tokens, n_heads, value_dim]; no two rows may overlap, nor a row with q, k or v */
  int64_t out_token_stride;
  int64_t out_head_stride;
  const float* rates;   /* [n_heads] >= 0, what a token's weight falls by in nats per token (infinity: at once) */
  const int32_t* seqs;  /* [n]                                                                */
  const int32_t* starts;/* [n+1] ascending from 0 to n_tokens; NULL = one token per sequence  */
} ic_state_attend_t;

int ic_state_attend(ic_state_t* s, const ic_state_attend_t* a);

/* Sequence children[i] gets the state of parents[i], in all layers, i < n, all at once: parents are taken as they are before
 * the call, also where they are children themselves.  No child twice. */
int ic_state_fork(ic_state_t* s, const int32_t* parents, const int32_t* children, int32_t n);

/* Sequences seqs[0..n) have seen nothing.  A number that comes twice counts once. */
int ic_state_clear(ic_state_t* s, const int32_t* seqs, int32_t n);

/* Synchronise the stream and report and clear the error that a kernel found: IC_ERR_INVALID, IC_ERR_TIMEOUT (a bounded wait ran
 * out; the states of that call are then undefined), IC_ERR_CUDA, else IC_OK. */
int ic_state_sync(ic_state_t* s);

/* Bind the handle to another stream; ordering between the two is the caller's. */
int ic_state_set_stream(ic_state_t* s, void* cuda_stream);

/* Kernels launched by this handle so far. */
int64_t ic_state_launch_count(const ic_state_t* s);

/* Synchronise the stream and free what the library allocated.  NULL is a no-op. */
void ic_state_destroy(ic_state_t* s);

#ifdef __cplusplus
}
#endif
#endif /* IC_STATE_H_ */
