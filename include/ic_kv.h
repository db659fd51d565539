/*
 * ic_kv.h - C ABI of the paged key-value cache that serves the retrieved examples.
 *
 * Example selection (ic_cache.h) returns the cached examples that go in front of a request's
 * prompt (paper Sec. 4.1; Algorithm 1, GenerateResponse on "examples + request").  The keys and
 * values that a causal model computes for the front of a prompt are the same whatever follows.  This
 * cache keeps them in pages of a fixed number of tokens: an example is run through the model
 * once, requests that begin with it fork from it and share its full pages, append their own tokens, attend
 * to all of it, and give the pages back.  (What stands behind the first example depends on it: a second
 * example's keys and values are part of the request's own tokens, unless the pair is kept as a sequence
 * too.  A sequence has one parent; there is no call that joins two.)
 *
 * Storage, all on the device (bf16 or fp16, int32):
 *   pool    [n_pages, n_layers, 2, n_kv_heads, page_size, head_dim]   index 2: 0 = keys, 1 = values
 *   tables  [max_seqs, max_pages]   row s: the pages of sequence s, in order
 *   lengths [max_seqs]              tokens of sequence s; it owns ceil(length / page_size) entries of
 *                                   its row, the entries behind those mean nothing
 *   refs    [n_pages]               how many owned table entries name the page; 0 = free
 * Only full pages are ever shared: a sequence's partly filled last page has one owner, so
 * appending never has to copy.  Pages are taken lowest number first, in the order of the call's
 * arguments, so that the tables are a function of the calls alone.
 *
 * Conventions
 *   - Arrays that a call takes (sequence numbers, counts, starts) are DEVICE arrays: what a step
 *     does next may come from the device (the parents chosen by a beam search) without a copy to
 *     the host, and a whole step can be captured in a CUDA graph.
 *   - Calls validate what the host can see, enqueue kernels on the handle's stream and return
 *     without synchronising; a non-OK return enqueued nothing.
 *   - What only the device can see (a sequence number out of range, the same child twice, a pool
 *     with too few free pages) is found by the kernels.  A call that meets it changes nothing at
 *     all, the error is kept, and every later call that would change the cache does nothing either
 *     until ic_kv_sync has reported the error and cleared it: IC_ERR_FULL or IC_ERR_INVALID, also
 *     returned by later calls as soon as the host sees it.  (ic_kv_free skips a bad number and frees
 *     the others.)
 *   - Borrowed tables, lengths and refs are trusted to be a cache's, but where they are not, no kernel
 *     leaves the pool and the books because of them: a length that the row cannot hold, or an owned entry
 *     that names no page, is reported as a bad argument of the call that meets it.  (Where it is an
 *     entry, ic_kv_free and ic_kv_compact pass over it and do the rest; ic_kv_write may have stored other
 *     tokens.)
 *   - One handle is bound to one stream and is not thread-safe; handles are independent.  Buffers
 *     are borrowed or owned as in ic_cache.h.  There is no CPU fallback.
 */
#ifndef IC_KV_H_
#define IC_KV_H_

#include "ic_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ic_kv ic_kv_t; /* opaque, owned by the library */

enum ic_kv_dtype { IC_KV_BF16 = 0, IC_KV_F16 = 1 };

#define IC_KV_MAX_HEAD_DIM 256 /* head_dim: a multiple of 8 up to this                       */
#define IC_KV_MAX_PAGE 256     /* page_size: a power of two, 8 .. 256                        */
#define IC_KV_MAX_SEQS 16384   /* largest max_seqs                                           */

/* Zero-initialise, set struct_size = sizeof, then fill. */
typedef struct ic_kv_opts {
  uint32_t struct_size; /* sizeof(ic_kv_opts_t) of the caller's build                        */
  int32_t device;       /* CUDA device ordinal; -1 = the current device                      */
  int32_t dtype;        /* ic_kv_dtype of the pool and of q, k, v and out                    */
  int32_t n_pages;      /* pages of the pool                                                 */
  int32_t n_layers;
  int32_t n_kv_heads;
  int32_t page_size;    /* tokens per page                                                   */
  int32_t head_dim;
  int32_t max_seqs;     /* rows of the page tables                                           */
  int32_t max_pages;    /* entries per row                                                   */
  void* pool;           /* optional caller-owned device buffers, 16-byte aligned (pool: 256); */
  int32_t* tables;      /*   NULL = the library allocates.  Borrowed tables, lengths and refs */
  int32_t* lengths;     /*   are taken as they are: zeros for an empty cache, or the state of */
  int32_t* refs;        /*   an earlier one (together with its pool)                          */
  void* stream;         /* cudaStream_t; NULL = the legacy default stream                    */
  void* workspace;      /* optional caller-owned scratch, 256-byte aligned; NULL = library    */
  size_t workspace_bytes; /* its size, at least ic_kv_workspace_bytes                         */
} ic_kv_opts_t;

/* Create the cache.  NULL on failure; ic_cache_last_error() then describes why.  Everything the
 * handle will ever need is allocated here: no later call allocates. */
ic_kv_t* ic_kv_create(const ic_kv_opts_t* opts);

/* Bytes of workspace for these options: 4 for every entry of the page tables, 12 a page, and the partial
 * results of attention that is split over a cache's length, whatever the model's size: 22 MB for a
 * head_dim of up to 64, 43 MB up to 128, 32 MB up to 192, 42 MB above.  0 for invalid options. */
size_t ic_kv_workspace_bytes(const ic_kv_opts_t* opts);

/*
 * Append: make room for counts[i] >= 0 new tokens at the end of sequence seqs[i], i < n (no
 * sequence twice), then write each layer's keys and values as the model computes them.
 *
 * ic_kv_reserve takes the pages that the longer sequences need and adds counts to lengths.
 * IC_ERR_FULL (on the device, see above) if the pool has too few free pages or a row too few
 * entries; nothing is reserved then.
 *
 * ic_kv_write stores the last starts[i+1] - starts[i] tokens of sequence seqs[i] in one layer.
 * k, v: token t, head h at element t * token_stride + h * head_stride, n_kv_heads x head_dim
 * values per token, 16-byte aligned, strides multiples of 8 elements.  starts: [n+1] ascending from 0
 * to n_tokens, or NULL for one token per sequence (n_tokens = n).
 */
int ic_kv_reserve(ic_kv_t* kv, const int32_t* seqs, const int32_t* counts, int32_t n);
int ic_kv_write(ic_kv_t* kv, int32_t layer, const void* k, const void* v, int64_t token_stride,
                int64_t head_stride, const int32_t* seqs, const int32_t* starts, int32_t n,
                int64_t n_tokens);

/*
 * Attention of the newest tokens of each sequence over its pages (n <= IC_KV_MAX_SEQS; a sequence may come
 * more than once).  Token t of sequence i is at
 * position p = length - (starts[i+1] - starts[i]) + t - starts[i] and sees the keys
 *     j <= p   and   (window == 0  or  j > p - window  or  j < sinks)
 * (all earlier tokens; or a sliding window and the first `sinks` tokens, which stay visible).
 *     out = sum_j softmax_j(scale * q.k_j) v_j        query head h reads kv head h / (n_heads / n_kv_heads)
 * A token that sees nothing (an empty sequence) gets zeros.  Scores, the softmax's maximum and sum, and
 * the weighted sum are held in fp32.  The weights are rounded to the cache's type for the product with the
 * values.  A call of at most 16 query rows (tokens x query heads per kv head) per sequence on average keeps
 * what the rounding leaves over as a second number; a call of more rows does not, so that a token's last
 * bits depend on the call that it is in.  In fp16 a key has no weight if its score is 27 nats (22 in a
 * call of more rows) below the largest one.
 * Rows of `out` that `starts` leaves out are not written; that is reported.  Bad sequences get zeros.
 * A value that no query of the call sees (a page's unused slots, keys outside the window) has no
 * influence, whatever it holds, infinities and NaN included.  An infinite or NaN value that a query sees
 * may also reach the sequence's other queries in the call, as a weight of zero does not undo it.
 */
typedef struct ic_kv_attend {
  uint32_t struct_size; /* sizeof(ic_kv_attend_t) of the caller's build                      */
  int32_t layer;
  int32_t n;            /* sequences                                                         */
  int32_t n_heads;      /* query heads, a multiple of n_kv_heads                             */
  int64_t n_tokens;     /* tokens in all                                                     */
  int32_t window;       /* >= 0; 0 = no window                                               */
  int32_t sinks;        /* >= 0; without a window it changes nothing                         */
  float scale;          /* of the scores; 1 / sqrt(head_dim) as a rule, below 2e38 in size    */
  int32_t reserved;     /* 0                                                                 */
  const void* q;        /* [n_tokens, n_heads, head_dim]: token t, head h at element         */
  int64_t q_token_stride; /*   t * q_token_stride + h * q_head_stride; 16-byte aligned,      */
  int64_t q_head_stride;  /*   strides multiples of 8 elements                               */
  void* out;            /* the same for the result; no two rows may overlap.  q itself, with */
  int64_t out_token_stride; /* its strides, is fine; any other overlap with q is not         */
  int64_t out_head_stride;
  const int32_t* seqs;  /* [n]                                                               */
  const int32_t* starts;/* [n+1] ascending from 0 to n_tokens; NULL = one token per sequence */
} ic_kv_attend_t;

int ic_kv_attend(ic_kv_t* kv, const ic_kv_attend_t* a);

/*
 * Rotary positions.  ic_kv_set_rotary says how the model behind the cache turns its queries and keys: pair i of a
 * head at position p by the angle p * f_i,
 *     (a, b) -> magnitude * (a cos - b sin, a sin + b cos),
 * where (a, b) are the elements i and i + rotary_dim / 2 (halves) or 2 i and 2 i + 1 (neighbours); elements from rotary_dim on are left as
 * they are.  f_i = base^(-2 i / rotary_dim) radians per token, scaled for contexts longer than the model was trained on:
 *     LINEAR  f_i / factor
 *     BASE    with the base  base * factor^(rotary_dim / (rotary_dim - 2))  (rotary_dim 2: no change)
 *     BANDS   by how many turns r = original * f_i / 2 pi the pair makes over `original` tokens:  w f_i + (1 - w) f_i / factor
 *             with w = (r - low) / (high - low), between 0 and 1
 * or `frequencies` gives the f_i themselves (for instance where w is to go by the pair's number between rounded borders, as some checkpoints have it).
 * Angles are off by less than 2^-24 of a half turn at every position (frequencies below 100).  Rows are computed in fp32 and rounded once to the cache's
 * type; elements from rotary_dim on keep their bits.  The call changes the handle only: later calls use it, a captured graph keeps what it was captured with.
 * ic_kv_rotary_frequencies writes the f_i of these options to host memory (rotary_dim / 2 numbers).
 */
enum ic_kv_rotary_layout { IC_KV_ROTARY_HALVES = 0, IC_KV_ROTARY_NEIGHBOURS = 1 };
enum ic_kv_rotary_scaling { IC_KV_ROTARY_NONE = 0, IC_KV_ROTARY_LINEAR = 1, IC_KV_ROTARY_BASE = 2, IC_KV_ROTARY_BANDS = 3 };

typedef struct ic_kv_rotary {
  uint32_t struct_size; /* sizeof(ic_kv_rotary_t) of the caller's build                      */
  int32_t rotary_dim;   /* even, 2 .. head_dim                                               */
  int32_t layout;       /* ic_kv_rotary_layout                                               */
  int32_t scaling;      /* ic_kv_rotary_scaling                                              */
  double base;          /* > 0; 0 = 10000                                                    */
  double factor;        /* > 0; 0 = 1                                                        */
  double low;           /* BANDS: 0 <= low < high                                            */
  double high;
  double original;      /* BANDS: > 0                                                        */
  double magnitude;     /* of ic_kv_rotate's results; 0 = 1                                  */
  const double* frequencies; /* optional HOST array [rotary_dim / 2], instead of base and scaling */
} ic_kv_rotary_t;

int ic_kv_set_rotary(ic_kv_t* kv, const ic_kv_rotary_t* r);
int ic_kv_rotary_frequencies(const ic_kv_rotary_t* r, double* frequencies);

/*
 * Turn new tokens' queries and keys, and store the keys with their values: ic_kv_write with rotary positions, and the queries
 * of the same tokens on the way.  Without k and v only queries (or any rows) are turned; without q only keys are stored.
 * A token stands where it stands in its sequence (as for ic_kv_attend), or at positions[t] (any int32, also below 0);
 * where it is stored does not depend on positions.  Without k and v, and with positions, seqs may be NULL (n = 0).
 * inverse != 0 turns back: by minus the angle, still times the magnitude.
 * A bad sequence or start anywhere in the call means that nothing is turned or stored; where a table entry is bad, other tokens may have
 * been turned and stored.
 */
typedef struct ic_kv_rotate {
  uint32_t struct_size; /* sizeof(ic_kv_rotate_t) of the caller's build                      */
  int32_t layer;        /* that k and v are stored in                                        */
  int32_t n;            /* sequences                                                         */
  int32_t n_heads;      /* of q; 0 without                                                   */
  int64_t n_tokens;     /* tokens in all                                                     */
  int32_t inverse;
  int32_t reserved;     /* 0                                                                 */
  const void* q;        /* [n_tokens, n_heads, head_dim], strides and alignment as for ic_kv_attend */
  int64_t q_token_stride;
  int64_t q_head_stride;
  void* out;            /* the same for the result; q itself, with its strides, is fine      */
  int64_t out_token_stride;
  int64_t out_head_stride;
  const void* k;        /* [n_tokens, n_kv_heads, head_dim], as for ic_kv_write              */
  const void* v;
  int64_t kv_token_stride;
  int64_t kv_head_stride;
  const int32_t* positions; /* [n_tokens], or NULL                                           */
  const int32_t* seqs;  /* [n]                                                               */
  const int32_t* starts;/* [n+1] ascending from 0 to n_tokens; NULL = one token per sequence */
} ic_kv_rotate_t;

int ic_kv_rotate(ic_kv_t* kv, const ic_kv_rotate_t* a);

/*
 * Move what is cached of sequence seqs[i], i < n (no sequence twice), by by[i] positions: its keys, in all layers, are turned by
 * by[i] * f_j (without the magnitude, which they have).  For a copy of an example (ic_kv_fork with copy) that stands
 * elsewhere in the request than where it was computed.  The keys are rounded to the cache's type once more.
 * Every page of the sequences must be theirs alone: one that is shared is IC_ERR_INVALID (on the device), and nothing is changed.
 */
int ic_kv_shift(ic_kv_t* kv, const int32_t* seqs, const int32_t* by, int32_t n);

/*
 * Make sequence children[i] the first upto[i] tokens of sequence parents[i], i < n, all at once: parents
 * are taken as they are before the call, also where they are children themselves (the reordering of
 * a beam search).  No child twice; upto: 0 <= upto[i] <= the parent's length, NULL = the whole parent.
 * Full pages are shared; the partly filled last page is copied to a fresh one (all layers).
 * copy != 0: every page is copied (a request that will rewrite what it takes over, such as keys that
 * move to other positions).  The pages that a child held before are given back after the copies; they
 * are not handed out within the call.  copy == 0, a child that is its own parent at full length:
 * nothing to do.  IC_ERR_FULL (on the device) if there are too few free pages.
 */
int ic_kv_fork(ic_kv_t* kv, const int32_t* parents, const int32_t* children, const int32_t* upto,
               int32_t n, int32_t copy);

/* Give back the pages of sequences seqs[0..n); their lengths become 0.  A number that comes twice
 * counts once.  (Paper Sec. 4.3: an evicted example's memory.) */
int ic_kv_free(ic_kv_t* kv, const int32_t* seqs, int32_t n);

/* Move the live pages to the front of the pool: those at or above the number of live pages go, in
 * order, into the free pages below it; tables and refs follow.  The back of the pool is then one
 * free range (to shrink the pool, or to write a checkpoint of its front). */
int ic_kv_compact(ic_kv_t* kv);

/* Synchronise the stream and report and clear the error that a kernel found: IC_ERR_FULL,
 * IC_ERR_INVALID, IC_ERR_TIMEOUT (a bounded wait ran out), IC_ERR_CUDA, else IC_OK. */
int ic_kv_sync(ic_kv_t* kv);

/* Bind the handle to another stream; ordering between the two is the caller's. */
int ic_kv_set_stream(ic_kv_t* kv, void* cuda_stream);

/* Kernels launched by this handle so far. */
int64_t ic_kv_launch_count(const ic_kv_t* kv);

/* Synchronise the stream and free what the library allocated.  NULL is a no-op. */
void ic_kv_destroy(ic_kv_t* kv);

#ifdef __cplusplus
}
#endif
#endif /* IC_KV_H_ */
