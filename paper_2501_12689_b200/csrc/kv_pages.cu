// Page operations of the paged key-value cache: reserve, write, fork, free, compact.
//
// The state is three integer arrays on the device (page tables, lengths, reference counts) and there is
// no free list beside them: a page is free if its count is 0, and pages are handed out lowest number
// first.  That makes the tables a function of the calls alone, needs nothing rebuilt after a restore, and
// costs one pass over the counts per allocation, 4 bytes a page.
//
// Nothing is computed: the bound is the bytes moved, or for few of them the launches, which overlap their predecessors'
// tails.  Measured (us; the floor at a copy's rate in brackets): 32 K tokens appended 55 (40), forks of 48 examples with
// copies of all pages 177 (163), a large compaction 94 (72); small calls of each kind 13 to 19, of which the host's own
// part of its two to four calls is most.
#include "common.cuh"
#include "kernels.h"
#include "kv.h"
#include "pipeline.cuh"

namespace icc {

namespace {

constexpr int PLAN_THREADS = 1024;        // planning kernels: one CTA, so that its barriers order the steps
constexpr int PAGES_PER_THREAD = 32;      // counts that a thread of a planning kernel looks at per round
constexpr int COPY_THREADS = 256;
constexpr int COPY_UNIT = COPY_THREADS * 16 * 4;   // bytes of a page that a CTA copies at a time
constexpr int ROW_UNIT = 1024;            // table entries that a CTA updates at a time

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

// Bit b of the result: page p0 + b exists and its reference count is 0.
__device__ __forceinline__ unsigned free_mask(const int* refs, int n_pages, int p0) {
  unsigned m = 0;
  if (p0 + PAGES_PER_THREAD <= n_pages) {
    int4 r[PAGES_PER_THREAD / 4];
#pragma unroll
    for (int j = 0; j < PAGES_PER_THREAD / 4; ++j) r[j] = reinterpret_cast<const int4*>(refs + p0)[j];
#pragma unroll
    for (int j = 0; j < PAGES_PER_THREAD / 4; ++j)
      m |= ((r[j].x == 0 ? 1u : 0u) | (r[j].y == 0 ? 2u : 0u) | (r[j].z == 0 ? 4u : 0u) | (r[j].w == 0 ? 8u : 0u)) << (4 * j);
  } else {
    for (int b = 0; p0 + b < n_pages; ++b) m |= (refs[p0 + b] == 0 ? 1u : 0u) << b;
  }
  return m;
}

// The lowest `need` free pages, in order, into `list`; returns how many were found (at least `need` if
// there are that many).  Whole CTA; ends with a barrier.
__device__ int take_free_pages(const KvView& v, int need, int* list, unsigned* sums) {
  int found = 0;
  for (int base = 0; base < v.n_pages && found < need; base += PLAN_THREADS * PAGES_PER_THREAD) {
    const int p0 = base + threadIdx.x * PAGES_PER_THREAD;
    unsigned m = p0 < v.n_pages ? free_mask(v.refs, v.n_pages, p0) : 0u;
    unsigned total;
    int r = found + (int)block_scan(__popc(m), sums, &total);
    while (m && r < need) {
      list[r++] = p0 + __ffs(m) - 1;
      m &= m - 1;
    }
    found += (int)total;
  }
  __syncthreads();
  return found;
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

// ---------------------------------------------------------------- reserve
// One CTA: check the arguments and sum up the pages they need, find that many free pages, and only then
// write tables, counts and lengths.
__global__ void __launch_bounds__(PLAN_THREADS) kv_reserve_kernel(const KvView v, const int* __restrict__ seqs,
                                                                  const int* __restrict__ counts, int n) {
  extern __shared__ int begin[];          // [n] rank of a sequence's first fresh page
  __shared__ unsigned sums[33];
  __shared__ int bad;
  grid_dep_launch_dependents();
  grid_dep_wait();   // arguments and state come from earlier kernels in the stream
  if (*v.err != KV_OK) return;
  if (threadIdx.x == 0) bad = KV_OK;
  __syncthreads();
  long long need = 0;
  for (int i0 = 0; i0 < n; i0 += PLAN_THREADS) {
    const int i = i0 + threadIdx.x;
    unsigned mine = 0;
    if (i < n) {
      const int s = seqs[i], c = counts[i];
      if (s < 0 || s >= v.max_seqs || c < 0) {
        bad = KV_INVALID;
      } else if (atomicExch(&v.mark[s], 1) != 0) {
        bad = KV_INVALID;
      } else {
        const int had = v.lengths[s];
        const long long will = (long long)had + c;
        if (!length_fits(v, had)) bad = KV_INVALID;
        else if (will > ((long long)v.max_pages << v.page_shift)) atomicCAS(&bad, KV_OK, KV_FULL);
        else mine = kv_pages_of((int)will, v.page_shift) - kv_pages_of(had, v.page_shift);
      }
    }
    unsigned total;
    const unsigned before = block_scan(mine, sums, &total);
    if (i < n) begin[i] = (int)min(need + before, 0x7fffffffll);
    need += total;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += PLAN_THREADS) {
    const int s = seqs[i];
    if (s >= 0 && s < v.max_seqs) v.mark[s] = 0;
  }
  int why = bad;
  if (why == KV_OK && need > v.n_pages) why = KV_FULL;
  if (why == KV_OK && need > 0 && take_free_pages(v, (int)need, v.fresh, sums) < need) why = KV_FULL;
  if (why != KV_OK) {
    if (threadIdx.x == 0) kv_report(v, why);
    return;
  }
  for (int r = threadIdx.x; r < (int)need; r += PLAN_THREADS) {
    const int i = owner_of(begin, n, r), s = seqs[i], page = v.fresh[r];
    v.tables[(size_t)s * v.max_pages + kv_pages_of(v.lengths[s], v.page_shift) + (r - begin[i])] = page;
    v.refs[page] = 1;
  }
  __syncthreads();                        // every old length has been read
  for (int i = threadIdx.x; i < n; i += PLAN_THREADS) v.lengths[seqs[i]] += counts[i];
}

// ---------------------------------------------------------------- write
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

__global__ void __launch_bounds__(COPY_THREADS) kv_write_check_kernel(const KvView v, const int* __restrict__ seqs, const int* __restrict__ starts,
                                                                      int n, int64_t n_tokens) {
  grid_dep_launch_dependents();
  grid_dep_wait();
  const int i = blockIdx.x * COPY_THREADS + threadIdx.x;
  if (*v.err != KV_OK || i >= n) return;
  if (!WriteSeq(v, seqs, starts, i, n, n_tokens).fine) kv_report(v, KV_INVALID);
}

// First byte of a token's key row of head 0, or null.
__device__ __forceinline__ unsigned char* token_place(const KvView& v, int layer, int s, int pos) {
  const int page = v.tables[(size_t)s * v.max_pages + (pos >> v.page_shift)];
  if (!page_exists(v, page)) return nullptr;
  const size_t row = (size_t)layer * 2 * v.n_kv_heads << v.page_shift;
  return v.pool + (size_t)page * v.page_bytes + (row + (size_t)(pos & ((1 << v.page_shift) - 1))) * v.head_dim * 2;
}

// TOKENS tokens per CTA.  A bad sequence anywhere in the call means that nothing is stored, so every CTA looks over all of them,
// one per thread, and on its way finds the places of its own tokens; more than COPY_THREADS sequences are CHECKED by a
// kernel of their own before this one.  (Looked over here | before, us a write: 1,024 single tokens 5.4 | 5.2, 4,096 11.7 | 6.6,
// 16,384 99 | 25; 256 and fewer take 2.2 to 2.9 here, and a launch more would add 1.2.)  Then all threads move 16-byte pieces.
// A head's rows of one page are contiguous, so the pieces of neighbouring tokens fill whole lines.
template <int TOKENS, bool CHECKED>
__global__ void __launch_bounds__(COPY_THREADS) kv_write_kernel(const KvView v, int layer, const uint4* __restrict__ k,
                                                                const uint4* __restrict__ val, int64_t token_stride, int64_t head_stride,
                                                                const int* __restrict__ seqs, const int* __restrict__ starts, int n,
                                                                int64_t n_tokens) {
  __shared__ unsigned char* place[TOKENS];
  __shared__ int row_of[TOKENS], pos_of[TOKENS];
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (*v.err != KV_OK) return;
  const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
  if (CHECKED) {
    const int64_t t = t0 + threadIdx.x;
    if (threadIdx.x < TOKENS) {
      unsigned char* at = nullptr;
      if (t < n_tokens) {
        const WriteSeq seq(v, seqs, starts, starts ? owner_of(starts, n, (int)t) : (int)t, n, n_tokens);
        at = token_place(v, layer, seq.s, (int)(seq.length - seq.end + t));
      }
      place[threadIdx.x] = at;
    }
  } else {
    bool fine = true;
    const int i = threadIdx.x;
    if (i < n) {
      const WriteSeq seq(v, seqs, starts, i, n, n_tokens);
      fine = seq.fine;
      if (fine)
        for (int64_t t = max(seq.begin, t0); t < min(seq.end, t0 + TOKENS); ++t) {
          const int pos = (int)(seq.length - seq.end + t);
          if (TOKENS == 1) {
            place[0] = token_place(v, layer, seq.s, pos);
          } else {
            row_of[t - t0] = seq.s;
            pos_of[t - t0] = pos;
          }
        }
    }
    if (!__syncthreads_and(fine)) {
      if (threadIdx.x == 0) kv_report(v, KV_INVALID);
      return;
    }
    if (TOKENS > 1 && i < TOKENS) place[i] = t0 + i < n_tokens ? token_place(v, layer, row_of[i], pos_of[i]) : nullptr;
  }
  if (CHECKED || TOKENS > 1) __syncthreads();
  // a thread takes one place in the tokens (keys or values, head, piece) at a time and all TOKENS tokens there: their
  // loads are under way together
  const int pieces = v.head_dim >> 3, per_token = v.n_kv_heads * pieces;
  const size_t block = ((size_t)v.head_dim * 2) << v.page_shift;      // bytes of one head's keys in a page
  for (int u = threadIdx.x; u < 2 * per_token; u += COPY_THREADS) {
    const int is_v = u >= per_token, hp = is_v ? u - per_token : u;
    const int h = hp / pieces, piece = hp - h * pieces;
    const uint4* from = (is_v ? val : k) + (t0 * token_stride + h * head_stride) / 8 + piece;
    const size_t off = (size_t)(is_v * v.n_kv_heads + h) * block + (size_t)piece * 16;
    uint4 w[TOKENS];
#pragma unroll
    for (int x = 0; x < TOKENS; ++x)
      if (place[x]) w[x] = ld_stream_16B(from + x * (token_stride / 8));
#pragma unroll
    for (int x = 0; x < TOKENS; ++x)
      if (place[x]) *reinterpret_cast<uint4*>(place[x] + off) = w[x];
  }
}

// ---------------------------------------------------------------- copying whole pages
// All CTAs of the grid share the pages jobs[0..n_jobs), a COPY_UNIT at a time.
__device__ __forceinline__ void copy_pages(const KvView& v, int n_jobs) {
  const long long units_per_page = (long long)((v.page_bytes + COPY_UNIT - 1) / COPY_UNIT);
  for (long long u = blockIdx.x; u < n_jobs * units_per_page; u += gridDim.x) {
    const int j = (int)(u / units_per_page);
    const size_t off = (size_t)(u - j * units_per_page) * COPY_UNIT + threadIdx.x * 16;
    const int2 job = v.jobs[j];
    const unsigned char* from = v.pool + (size_t)job.x * v.page_bytes;
    unsigned char* to = v.pool + (size_t)job.y * v.page_bytes;
    uint4 w[4];
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (off + x * COPY_THREADS * 16 < v.page_bytes) w[x] = ld_stream_16B(from + off + x * COPY_THREADS * 16);
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (off + x * COPY_THREADS * 16 < v.page_bytes) __stcs(reinterpret_cast<uint4*>(to + off + x * COPY_THREADS * 16), w[x]);
  }
}

// ---------------------------------------------------------------- fork
// Three steps: the plan (arguments, pages needed, free pages), by one CTA; the children's new rows, made
// beside the old ones while all parents still stand; and the exchange of rows with its counts, and the copies of pages.
// Only the last step changes the cache, and it is left out if one of the first two has found something wrong.  The plan's
// CTA does the rows too where there are few table entries (SMALL_FORK), which saves a launch; otherwise the rows are
// spread over CTAs, and each step is a launch.
constexpr int SMALL_FORK = 8192;          // table entries: eight per thread of the plan's CTA, about what a launch takes

// Entries c0 .. c_end of child i's new row; n_threads threads.  False if an entry that is taken over or given back names no page.
__device__ __forceinline__ bool stage_row(const KvView& v, const int* parents, const int* children, int i, int c0, int c_end, int thread,
                                          int n_threads) {
  const int want = v.upto[i];
  if (want < 0) return true;
  const int left = kv_pages_of(v.had[i], v.page_shift), pages = kv_pages_of(want, v.page_shift);
  const int end = min(max(left, pages), c_end), shared = v.shared[i], begin = v.begin[i];
  const int* row = v.tables + (size_t)parents[i] * v.max_pages;
  const int* old = v.tables + (size_t)children[i] * v.max_pages;
  int* to = v.staged + (size_t)i * v.max_pages;
  bool fine = true;
  for (int c = c0 + thread; c < end; c += n_threads) {
    if (c < left) fine &= page_exists(v, old[c]);
    if (c < pages) {
      const int page = row[c];
      fine &= page_exists(v, page);
      if (c < shared) {
        to[c] = page;
      } else {
        const int r = begin + c - shared, mine = v.fresh[r];
        v.jobs[r] = make_int2(page, mine);
        to[c] = mine;
      }
    }
  }
  return fine;
}

__device__ __forceinline__ void exchange_row(const KvView& v, const int* children, int i, int c0, int c_end, int thread, int n_threads) {
  const int want = v.upto[i];
  if (want < 0) return;
  const int b = children[i], left = kv_pages_of(v.had[i], v.page_shift), pages = kv_pages_of(want, v.page_shift), shared = v.shared[i];
  const int end = min(max(left, pages), c_end);
  int* row = v.tables + (size_t)b * v.max_pages;
  const int* from = v.staged + (size_t)i * v.max_pages;
  for (int c = c0 + thread; c < end; c += n_threads) {
    if (c < left) atomicSub(&v.refs[row[c]], 1);
    if (c < pages) {
      const int page = from[c];
      if (c < shared) atomicAdd(&v.refs[page], 1);
      else v.refs[page] = 1;
      row[c] = page;
    }
  }
  if (c0 == 0 && thread == 0) v.lengths[b] = want;
}

__global__ void __launch_bounds__(PLAN_THREADS) kv_fork_plan_kernel(const KvView v, const int* __restrict__ parents,
                                                                    const int* __restrict__ children, const int* __restrict__ upto,
                                                                    int n, int copy, int rows_too) {
  __shared__ unsigned sums[33];
  __shared__ int bad;
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (threadIdx.x == 0) {
    bad = KV_OK;
    v.meta[0] = 0;
  }
  __syncthreads();
  if (*v.err != KV_OK) return;
  long long need = 0;
  for (int i0 = 0; i0 < n; i0 += PLAN_THREADS) {
    const int i = i0 + threadIdx.x;
    unsigned mine = 0;
    if (i < n) {
      const int a = parents[i], b = children[i];
      if (a < 0 || a >= v.max_seqs || b < 0 || b >= v.max_seqs || atomicExch(&v.mark[b], 1) != 0) {
        bad = KV_INVALID;
      } else {
        const int len = v.lengths[a], had = v.lengths[b], want = upto ? upto[i] : len;
        if (want < 0 || want > len || !length_fits(v, len) || !length_fits(v, had)) {
          bad = KV_INVALID;
        } else {
          const bool nothing = !copy && a == b && want == len;
          const int pages = kv_pages_of(want, v.page_shift);
          const int shared = copy ? 0 : (nothing ? pages : want >> v.page_shift);
          v.had[i] = had;
          v.upto[i] = nothing ? -1 : want;
          v.shared[i] = shared;
          mine = pages - shared;
        }
      }
    }
    unsigned total;
    const unsigned before = block_scan(mine, sums, &total);
    if (i < n) v.begin[i] = (int)min(need + before, 0x7fffffffll);
    need += total;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += PLAN_THREADS) {
    const int b = children[i];
    if (b >= 0 && b < v.max_seqs) v.mark[b] = 0;
  }
  int why = bad;
  if (why == KV_OK && need > v.n_pages) why = KV_FULL;
  if (why == KV_OK && need > 0 && take_free_pages(v, (int)need, v.fresh, sums) < need) why = KV_FULL;
  if (why != KV_OK) {
    if (threadIdx.x == 0) kv_report(v, why);
    return;
  }
  if (rows_too) {                         // a warp per row
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();
    bool fine = true;
    for (int i = warp; i < n; i += PLAN_THREADS / 32) fine &= stage_row(v, parents, children, i, 0, v.max_pages, lane, 32);
    if (!__syncthreads_and(fine)) return;
    for (int i = warp; i < n; i += PLAN_THREADS / 32) exchange_row(v, children, i, 0, v.max_pages, lane, 32);
  }
  if (threadIdx.x == 0) {
    v.meta[0] = 1;
    v.meta[1] = (int)need;
  }
}

__global__ void __launch_bounds__(COPY_THREADS) kv_fork_stage_kernel(const KvView v, const int* __restrict__ parents,
                                                                     const int* __restrict__ children, int n) {
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (v.meta[0] == 0) return;
  const int chunks = (v.max_pages + ROW_UNIT - 1) / ROW_UNIT;
  for (long long u = blockIdx.x; u < (long long)n * chunks; u += gridDim.x) {
    const int i = (int)(u / chunks), c0 = (int)(u - (long long)i * chunks) * ROW_UNIT;
    if (!stage_row(v, parents, children, i, c0, min(c0 + ROW_UNIT, v.max_pages), threadIdx.x, COPY_THREADS)) v.meta[0] = 0;
  }
}

__global__ void __launch_bounds__(COPY_THREADS) kv_fork_apply_kernel(const KvView v, const int* __restrict__ children, int n, int rows_done) {
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (v.meta[0] == 0) return;
  if (!rows_done) {
    const int chunks = (v.max_pages + ROW_UNIT - 1) / ROW_UNIT;
    for (long long u = blockIdx.x; u < (long long)n * chunks; u += gridDim.x) {
      const int i = (int)(u / chunks), c0 = (int)(u - (long long)i * chunks) * ROW_UNIT;
      exchange_row(v, children, i, c0, min(c0 + ROW_UNIT, v.max_pages), threadIdx.x, COPY_THREADS);
    }
  }
  copy_pages(v, v.meta[1]);
}

// ---------------------------------------------------------------- free
// A CTA per sequence.  Whoever takes the length away owns the release, so a number that comes twice counts once.
__global__ void __launch_bounds__(COPY_THREADS) kv_free_kernel(const KvView v, const int* __restrict__ seqs, int n) {
  __shared__ int had;
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (*v.err != KV_OK) return;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int s = seqs[i];
    if (threadIdx.x == 0) {
      had = 0;
      if (s < 0 || s >= v.max_seqs || !length_fits(v, v.lengths[s])) kv_report(v, KV_INVALID);
      else had = atomicExch(&v.lengths[s], 0);
    }
    __syncthreads();
    const int pages = kv_pages_of(had, v.page_shift);
    const int* row = v.tables + (size_t)s * v.max_pages;
    for (int c = threadIdx.x; c < pages; c += COPY_THREADS)
      if (page_exists(v, row[c])) atomicSub(&v.refs[row[c]], 1);
    __syncthreads();
  }
}

// ---------------------------------------------------------------- compact
// The plan: count the live pages, then give the holes below that number and the live pages above it
// their ranks; rank r's page moves to rank r's hole.
__global__ void __launch_bounds__(PLAN_THREADS) kv_compact_plan_kernel(const KvView v) {
  __shared__ unsigned sums[33];
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (threadIdx.x == 0) v.meta[0] = 0;
  if (*v.err != KV_OK) return;
  int bad = 0;
  for (int s = threadIdx.x; s < v.max_seqs; s += PLAN_THREADS) bad |= !length_fits(v, v.lengths[s]);
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) kv_report(v, KV_INVALID);
    return;
  }
  constexpr int ROUND = PLAN_THREADS * PAGES_PER_THREAD;
  int n_free = 0;
  for (int base = 0; base < v.n_pages; base += ROUND) {
    const int p0 = base + threadIdx.x * PAGES_PER_THREAD;
    unsigned total;
    block_scan(p0 < v.n_pages ? __popc(free_mask(v.refs, v.n_pages, p0)) : 0, sums, &total);
    n_free += (int)total;
  }
  const int n_live = v.n_pages - n_free;
  int holes = 0, movers = 0;
  for (int base = 0; base < v.n_pages; base += ROUND) {
    const int p0 = base + threadIdx.x * PAGES_PER_THREAD;
    unsigned hole = 0, move = 0;
    if (p0 < v.n_pages) {
      const unsigned f = free_mask(v.refs, v.n_pages, p0);
      const int here = min(PAGES_PER_THREAD, v.n_pages - p0), below = max(0, min(PAGES_PER_THREAD, n_live - p0));
      const unsigned exist = here == 32 ? ~0u : (1u << here) - 1u, low = below == 32 ? ~0u : (1u << below) - 1u;
      hole = f & low;
      move = ~f & exist & ~low;
    }
    unsigned total;      // two counts in one scan: at most 32,768 pages a round, so neither overflows its half
    const unsigned before = block_scan((unsigned)__popc(hole) | ((unsigned)__popc(move) << 16), sums, &total);
    int r = holes + (int)(before & 0xffffu);
    for (unsigned m = hole; m; m &= m - 1) v.jobs[r++].y = p0 + __ffs(m) - 1;
    r = movers + (int)(before >> 16);
    for (unsigned m = move; m; m &= m - 1) {
      const int p = p0 + __ffs(m) - 1;
      v.jobs[r].x = p;
      v.fresh[p] = r++;
    }
    holes += (int)(total & 0xffffu);
    movers += (int)(total >> 16);
  }
  if (threadIdx.x == 0) {
    v.meta[0] = 1;
    v.meta[1] = movers;
    v.meta[2] = n_live;
  }
}

__global__ void __launch_bounds__(COPY_THREADS) kv_compact_apply_kernel(const KvView v) {
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (v.meta[0] == 0) return;
  const int n_jobs = v.meta[1], n_live = v.meta[2];
  if (n_jobs == 0) return;
  const int chunks = (v.max_pages + ROW_UNIT - 1) / ROW_UNIT;
  for (long long u = blockIdx.x; u < (long long)v.max_seqs * chunks; u += gridDim.x) {
    const int s = (int)(u / chunks), c0 = (int)(u - (long long)s * chunks) * ROW_UNIT;
    const int end = min(kv_pages_of(v.lengths[s], v.page_shift), c0 + ROW_UNIT);
    int* row = v.tables + (size_t)s * v.max_pages;
    for (int c = c0 + threadIdx.x; c < end; c += COPY_THREADS) {
      const int page = row[c];
      if (!page_exists(v, page) || page < n_live) continue;
      // (an entry of lent tables may name a page that nobody holds: it has no rank, and its word of `fresh` may be anything)
      const int r = v.fresh[page];
      const int2 job = (unsigned)r < (unsigned)n_jobs ? v.jobs[r] : make_int2(-1, -1);
      if (job.x == page) row[c] = job.y;
      else kv_report(v, KV_INVALID);
    }
  }
  for (int r = blockIdx.x * COPY_THREADS + threadIdx.x; r < n_jobs; r += gridDim.x * COPY_THREADS) {
    const int2 job = v.jobs[r];
    v.refs[job.y] = v.refs[job.x];
    v.refs[job.x] = 0;
  }
  copy_pages(v, n_jobs);
}

}  // namespace

cudaError_t kv_pages_configure(int smem_optin) {
  (void)smem_optin;
  return cudaFuncSetAttribute(kv_reserve_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 16384 * 4);
}

cudaError_t kv_reserve_launch(const KvView& v, const int* seqs, const int* counts, int n, cudaStream_t st) {
  return launch_overlapped(kv_reserve_kernel, dim3(1), dim3(PLAN_THREADS), (size_t)n * 4, st, 1, v, seqs, counts, n);
}

cudaError_t kv_write_launch(const KvView& v, int layer, const void* k, const void* val, int64_t token_stride, int64_t head_stride,
                            const int* seqs, const int* starts, int n, int64_t n_tokens, int sm_count, int* launches, cudaStream_t st) {
  const uint4* k4 = static_cast<const uint4*>(k);
  const uint4* v4 = static_cast<const uint4*>(val);
  const bool checked = n > COPY_THREADS, single = n_tokens <= 4 * sm_count;
  *launches = checked ? 2 : 1;
  if (checked) {
    const cudaError_t e = launch_overlapped(kv_write_check_kernel, dim3((unsigned)((n + COPY_THREADS - 1) / COPY_THREADS)), dim3(COPY_THREADS), 0, st, 1, v,
                                            seqs, starts, n, n_tokens);
    if (e != cudaSuccess) return e;
  }
  auto* kernel = single ? (checked ? kv_write_kernel<1, true> : kv_write_kernel<1, false>) : (checked ? kv_write_kernel<8, true> : kv_write_kernel<8, false>);
  return launch_overlapped(kernel, dim3((unsigned)(single ? n_tokens : (n_tokens + 7) / 8)), dim3(COPY_THREADS), 0, st, 1, v, layer, k4, v4, token_stride,
                           head_stride, seqs, starts, n, n_tokens);
}

cudaError_t kv_fork_launch(const KvView& v, const int* parents, const int* children, const int* upto, int n, int copy,
                           int sm_count, int* launches, cudaStream_t st) {
  const bool small = (long long)n * v.max_pages <= SMALL_FORK;
  const long long rows = (long long)n * ((v.max_pages + ROW_UNIT - 1) / ROW_UNIT);
  const int most = 8 * sm_count;
  *launches = small ? 2 : 3;
  cudaError_t e = launch_overlapped(kv_fork_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, 1, v, parents, children, upto, n, copy, (int)small);
  if (e == cudaSuccess && !small)
    e = launch_overlapped(kv_fork_stage_kernel, dim3((unsigned)(rows < most ? rows : most)), dim3(COPY_THREADS), 0, st, 1, v, parents, children, n);
  if (e == cudaSuccess)
    e = launch_overlapped(kv_fork_apply_kernel, dim3((unsigned)most), dim3(COPY_THREADS), 0, st, 1, v, children, n, (int)small);
  return e;
}

cudaError_t kv_free_launch(const KvView& v, const int* seqs, int n, int sm_count, cudaStream_t st) {
  return launch_overlapped(kv_free_kernel, dim3((unsigned)(n < 8 * sm_count ? n : 8 * sm_count)), dim3(COPY_THREADS), 0, st, 1, v, seqs, n);
}

cudaError_t kv_compact_launch(const KvView& v, int sm_count, int* launches, cudaStream_t st) {
  *launches = 2;
  const cudaError_t e = launch_overlapped(kv_compact_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, 1, v);
  return e == cudaSuccess ? launch_overlapped(kv_compact_apply_kernel, dim3((unsigned)(8 * sm_count)), dim3(COPY_THREADS), 0, st, 1, v) : e;
}

}  // namespace icc
