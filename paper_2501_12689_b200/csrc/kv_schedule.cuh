// How the attention kernels divide their work.
//
// The query rows of one sequence and kv head are its tokens times the query heads of that kv head
// (row = token * group + head in group), cut into tiles of ROWS rows.  A tile's work is the tiles of KEYS
// keys that any of its rows sees.  All of a launch's key tiles, in the order sequence, kv head, row
// tile, key tile, form one line, and each CTA takes an equal stretch of it, whatever the lengths: a CTA
// holds whole (row tile, head) items and at most two pieces of items, and the pieces of an item that
// spans CTAs are joined by the CTA that finishes last.  A piece costs its way through memory and the join, as much as
// some key tiles: an item of up to WHOLE tiles, and no longer than a stretch, is not cut (the cut moves to its nearer end).
// Lengths live on the device, so the CTAs work the
// line out for themselves; sequences are few and their data sits in shared memory.
#pragma once
#include "common.cuh"
#include "kv.h"

namespace icc {

struct KvSeq {
  int slot, length, first, count;        // table row, tokens, first row of q, number of q's rows
};

// What the CTAs of one launch share about the batch, in shared memory.
struct KvBatch {
  KvSeq seq[KV_BATCH];
  long long before[KV_BATCH + 1];  // key tiles of the sequences before this one, all heads
};

// The key tiles of one row tile: the sinks' tiles [0, sink_tiles) and then [first, end).
struct KvRange {
  int sink_tiles, first, n;              // n = tiles in all, at least 1
  __device__ __forceinline__ int tile(int k) const { return k < sink_tiles ? k : first + (k - sink_tiles); }
};

template <int ROWS, int KEYS>
struct KvSchedule {
  const KvAttendParams* p;
  const KvBatch* b;
  __device__ KvSchedule(const KvAttendParams& p_, const KvBatch& b_) : p(&p_), b(&b_) {}

  __device__ __forceinline__ int row_tiles(const KvSeq& s) const { return (int)(((unsigned)s.count * (unsigned)p->group + ROWS - 1u) / ROWS); }

  // Positions of the first and the last row of row tile rt.
  __device__ __forceinline__ void positions(const KvSeq& s, int rt, int* lowest, int* highest) const {
    const unsigned r0 = (unsigned)rt * ROWS, r1 = min(r0 + ROWS, (unsigned)s.count * (unsigned)p->group) - 1u;
    *lowest = s.length - s.count + kv_token_of(*p, (int)r0);
    *highest = s.length - s.count + kv_token_of(*p, (int)r1);
  }

  __device__ __forceinline__ KvRange range(const KvSeq& s, int rt) const {
    int lowest, highest;
    positions(s, rt, &lowest, &highest);
    KvRange r;
    const int end = highest < 0 ? 0 : highest / KEYS + 1;
    r.first = (p->window && lowest >= p->window) ? (lowest - p->window + 1) / KEYS : 0;
    // the sinks' tiles, as far as they lie before the window's
    const int sink_tiles = (int)(((unsigned)p->sinks + KEYS - 1u) / KEYS);
    r.sink_tiles = min(sink_tiles, r.first);
    r.n = max(1, r.sink_tiles + end - r.first);      // a row tile that sees nothing writes zeros
    return r;
  }
};

// Fill the batch table; all threads of the CTA, which synchronise afterwards.
template <int ROWS, int KEYS>
__device__ __forceinline__ void kv_load_batch(const KvAttendParams& p, KvBatch* b) {
  const KvSchedule<ROWS, KEYS> sched(p, *b);
  for (int i = threadIdx.x; i < p.n; i += blockDim.x) {
    KvSeq s;
    s.slot = p.seqs[i];
    bool fine = s.slot >= 0 && s.slot < p.v.max_seqs;
    s.length = fine ? p.v.lengths[s.slot] : 0;
    long long first = p.first_seq + i, end = first + 1;
    bool covered = true;               // no token is left out before the first or after the last sequence
    if (p.starts) {
      covered = first > 0 || p.starts[i] == 0;
      covered &= end < p.n_seqs || p.starts[i + 1] == p.n_tokens;
      first = p.starts[i];
      end = p.starts[i + 1];
    }
    if (first < 0 || first > end || end > p.n_tokens) {
      fine = false;
      first = 0;
      end = 0;
    }
    s.first = (int)first;
    s.count = (int)(end - first);
    if (s.length < 0 || s.length > ((long long)p.v.max_pages << p.v.page_shift)) {
      fine = false;
      s.length = 0;
    }
    if (s.count > s.length && (p.starts || s.length > 0)) fine = false;     // (the one token of an empty sequence sees nothing)
    if (!(fine && covered) && blockIdx.x == 0) kv_report(p.v, KV_INVALID);
    b->seq[i] = s;
    const int n = sched.row_tiles(s);
    b->before[i + 1] = n == 0 ? 0 : (n == 1 ? (long long)sched.range(s, 0).n * p.v.n_kv_heads : -1);
  }
  __syncthreads();
  // sequences of several row tiles: a warp each
  for (int i = threadIdx.x >> 5; i < p.n; i += blockDim.x >> 5) {
    if (b->before[i + 1] >= 0) continue;
    const KvSeq s = b->seq[i];
    const int n = sched.row_tiles(s), lane = threadIdx.x & 31;
    long long sum = 0;
    for (int rt = lane; rt < n; rt += 32) sum += sched.range(s, rt).n;
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(FULL_MASK, sum, d);
    __syncwarp();
    if (lane == 0) b->before[i + 1] = sum * p.v.n_kv_heads;
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    long long sum = 0;
    for (int i0 = 0; i0 < p.n; i0 += 32) {
      const int i = i0 + threadIdx.x;
      long long x = i < p.n ? b->before[i + 1] : 0;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const long long y = __shfl_up_sync(FULL_MASK, x, d);
        if ((int)threadIdx.x >= d) x += y;
      }
      if (i < p.n) b->before[i + 1] = sum + x;
      sum += __shfl_sync(FULL_MASK, x, 31);
    }
    if (threadIdx.x == 0) b->before[0] = 0;
  }
}

// One more piece of an item is written: by one thread, after a barrier that the writers have passed.  Returns how many were
// there before.  Release for the pieces of this CTA, acquire for those of the others.
__device__ __forceinline__ int kv_arrive(int* arrivals) {
  int before;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(arrivals) : "memory");
  return before;
}

// 64-bit division, which is a long sequence of instructions, only where 32 bits do not do.
__device__ __forceinline__ long long kv_div(long long a, long long b) {
  return (a >> 31) == 0 ? (long long)((unsigned)a / (unsigned)min(b, 0xffffffffll)) : a / b;
}

// Walks a CTA's stretch of the line, item by item.  The present item's key tiles within the stretch are
// [from, to); `left` tiles of the stretch begin with them.
template <int ROWS, int KEYS, int WHOLE>
struct KvWalk {
  KvSchedule<ROWS, KEYS> sched;
  int i, head, rt;                       // the item: sequence of the batch, kv head, row tile
  KvRange r;
  int from, to, left;
  long long end;                         // where the stretch ends
  long long base;                        // before cuts move, each CTA's stretch is `base` long, the first `extra` ones' one more
  int extra;

  __device__ KvWalk(const KvAttendParams& p, const KvBatch& b, int c, int grid) : sched(p, b) {
    const long long total = b.before[p.n];
    const int n_ctas = (int)min((long long)grid, total);     // no stretch is empty before its cuts move
    left = 0;
    if (c >= n_ctas) return;
    base = kv_div(total, n_ctas);
    extra = (int)(total - base * n_ctas);
    end = c + 1 == n_ctas ? total : cut(raw_begin(c + 1));
    const long long at = c == 0 ? 0 : cut(raw_begin(c));
    left = (int)(end - at);
    if (left == 0) return;
    locate(at);
    to = min(r.n, from + left);
  }
  __device__ __forceinline__ long long raw_begin(int c) const { return base * c + min(c, extra); }
  // Where the cut at key tile u of the line is made.
  __device__ __forceinline__ long long cut(long long u) {
    locate(u);
    if (r.n > min((long long)WHOLE, base)) return u;
    return 2 * from < r.n ? u - from : u - from + r.n;
  }
  // The item of key tile u, and `from` = its place in it.  Whole warps.
  __device__ __forceinline__ void locate(long long u) {
    const KvBatch& b = *sched.b;
    int lo = 0, hi = sched.p->n - 1;     // the last sequence that begins at or before u
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (b.before[mid] <= u) lo = mid;
      else hi = mid - 1;
    }
    i = lo;
    long long into = u - b.before[i];
    const int heads = sched.p->v.n_kv_heads;
    const long long per_head = kv_div(b.before[i + 1] - b.before[i], heads);
    head = (int)kv_div(into, per_head);
    into -= head * per_head;
    // the row tile that `into` lies in: the warp looks at 32 of them at a time
    const int n = sched.row_tiles(b.seq[i]);
    rt = 0;
    if (n > 1) {
      for (int rt0 = 0;; rt0 += 32) {
        const int mine = rt0 + (threadIdx.x & 31);
        long long upto = mine < n ? sched.range(b.seq[i], mine).n : 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const long long y = __shfl_up_sync(FULL_MASK, upto, d);
          if ((int)(threadIdx.x & 31) >= d) upto += y;
        }
        const unsigned past = __ballot_sync(FULL_MASK, upto > into);       // never empty in the last round
        if (past || rt0 + 32 >= n) {
          const int at_lane = past ? __ffs(past) - 1 : 31;
          rt = rt0 + at_lane;
          const long long before_it = __shfl_sync(FULL_MASK, upto, max(at_lane - 1, 0));
          into -= at_lane > 0 ? before_it : 0;
          break;
        }
        into -= __shfl_sync(FULL_MASK, upto, 31);
      }
    }
    r = sched.range(b.seq[i], rt);
    from = (int)into;
  }
  __device__ __forceinline__ bool done() const { return left == 0; }
  __device__ __forceinline__ bool whole() const { return from == 0 && to == r.n; }
  // On to the next item of the stretch.
  __device__ __forceinline__ void next() {
    left -= to - from;
    if (left == 0) return;
    if (++rt >= sched.row_tiles(sched.b->seq[i])) {
      rt = 0;
      if (++head >= sched.p->v.n_kv_heads) {
        head = 0;
        do ++i; while (sched.b->seq[i].count == 0);
      }
    }
    r = sched.range(sched.b->seq[i], rt);
    from = 0;
    to = min(r.n, left);
  }
  // The CTA whose stretch holds key tile u of an item that is cut: its own cuts have not moved, and those that
  // have stay on their side of it.
  __device__ __forceinline__ int cta_of(long long u) const {
    const long long longer = (base + 1) * extra;
    return u < longer ? (int)kv_div(u, base + 1) : extra + (int)kv_div(u - longer, base);
  }
  // The pieces of the present item lie with CTAs [first, first + n).  A CTA has two slots for partial results: for the
  // item that goes on into its stretch, and for the one that begins there and goes on past its end.
  struct Pieces {
    int first, n;
    __device__ __forceinline__ int slot(int c) const { return (first + c) * 2 + (c == 0 ? 1 : 0); }
  };
  __device__ __forceinline__ Pieces pieces() const {
    const long long u = end - left - from;             // first key tile of the item
    Pieces x;
    x.first = cta_of(u);
    x.n = cta_of(u + r.n - 1) - x.first + 1;
    return x;
  }
  __device__ __forceinline__ int my_slot(int c) const { return c * 2 + (from == 0 ? 1 : 0); }
};

}  // namespace icc
