/*
 * ic_score.h - C ABI of token scores: what tokens are worth under a model's logits.
 *
 * The cache of ic_cache.h keeps a utility per example (paper Sec. 4.3, "Example Manager"), and requests are routed by how sure a model is
 * (Sec. 4.2).  Both come from the served model's logits: the log-probabilities of an answer's tokens with and without an example in
 * front of them, the entropy of the next token, and the alternatives to it.  One pass over the logits gives all of these.
 *
 * For a row x[0..vocab) of logits, y = scale * x:
 *     log_prob(t) = y_t - log sum_j e^(y_j)         entropy = - sum_j p_j log p_j,  p_j = e^(log_prob(j))
 *     top alternatives: the n_top largest logits, in order, the lowest index first among equal ones (-0 equals 0)
 * Differences to a row's largest logit, products, sums and maxima are held in fp32.  A logit of minus infinity is a banned token:
 * probability 0, and nothing to the entropy.  A row that bans every token has log-probabilities of minus infinity and an entropy of 0.
 * A row with a NaN, or whose largest y is plus infinity, has none: log-probabilities and entropy are NaN, its top ids -1.
 *
 * Conventions as in ic_kv.h: device arrays, work enqueued on the handle's stream without synchronising, one handle per stream, not
 * thread-safe.  A call needs no more memory than the handle has, whatever its size.  Graphs captured from one handle share its
 * workspace: they must not run at the same time.  There is no CPU fallback.
 */
#ifndef IC_SCORE_H_
#define IC_SCORE_H_

#include "ic_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ic_score ic_score_t; /* opaque, owned by the library */

enum ic_score_dtype { IC_SCORE_BF16 = 0, IC_SCORE_F16 = 1, IC_SCORE_F32 = 2 };

#define IC_SCORE_MAX_TOP 32          /* largest n_top                                         */
#define IC_SCORE_MAX_VOCAB 16777216  /* largest vocab                                         */

/* Zero-initialise, set struct_size = sizeof, then fill. */
typedef struct ic_score_opts {
  uint32_t struct_size; /* sizeof(ic_score_opts_t) of the caller's build                      */
  int32_t device;       /* CUDA device ordinal; -1 = the current device                       */
  int32_t dtype;        /* ic_score_dtype of the logits                                       */
  int32_t vocab;        /* logits of a row, 1 .. IC_SCORE_MAX_VOCAB                           */
  void* stream;         /* cudaStream_t; NULL = the legacy default stream                     */
  void* workspace;      /* optional caller-owned scratch, 256-byte aligned; NULL = library    */
  size_t workspace_bytes; /* its size, at least ic_score_workspace_bytes                      */
} ic_score_opts_t;

/* NULL on failure; ic_cache_last_error() then describes why. */
ic_score_t* ic_score_create(const ic_score_opts_t* opts);

/* Bytes of workspace: partial results of rows that are split over several CTAs, 0.3 MB.  0 for invalid options. */
size_t ic_score_workspace_bytes(const ic_score_opts_t* opts);

typedef struct ic_score_args {
  uint32_t struct_size; /* sizeof(ic_score_args_t) of the caller's build                      */
  int32_t n_top;        /* 0 .. IC_SCORE_MAX_TOP, at most vocab                               */
  int64_t n_rows;       /* 0 .. 2^26                                                          */
  float scale;          /* of the logits, above 0 (one over the temperature); finite, also times log2(e) */
  int32_t reserved;     /* 0                                                                  */
  const void* logits;   /* row r at element r * row_stride, `vocab` contiguous values; any    */
  int64_t row_stride;   /*   stride >= 0, aligned to an element                               */
  const int32_t* targets; /* [n_rows] or NULL: the tokens asked for; -1 = none (its result is 0).  Another */
                        /*   index outside the vocabulary is IC_ERR_INVALID (on the device), its result NaN */
  float* log_probs;     /* [n_rows], with targets                                             */
  float* entropy;       /* [n_rows] or NULL                                                   */
  int32_t* top_ids;     /* [n_rows, n_top], NULL if n_top is 0                                */
  float* top_log_probs; /* the same                                                           */
} ic_score_args_t;

int ic_score_tokens(ic_score_t* s, const ic_score_args_t* a);

/* Synchronise the stream and report and clear the error that a kernel found (IC_ERR_INVALID; later calls report it too). */
int ic_score_sync(ic_score_t* s);

/* Bind the handle to another stream; ordering between the two is the caller's. */
int ic_score_set_stream(ic_score_t* s, void* cuda_stream);

/* Kernels launched by this handle so far. */
int64_t ic_score_launch_count(const ic_score_t* s);

/* Synchronise the stream and free what the library allocated.  NULL is a no-op. */
void ic_score_destroy(ic_score_t* s);

#ifdef __cplusplus
}
#endif
#endif /* IC_SCORE_H_ */
