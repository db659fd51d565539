// How a call over the states is divided among the CTAs.
//
// The chunks of all sequences, heads and value slices of a launch form one line, and each CTA takes an equal stretch of it.  A stretch may begin
// or end inside an item (a sequence, head and slice), whose state then comes from the CTAs before.  To leave nobody waiting, a CTA begins with
// what others wait for:
//   - the item that it begins and does not end: its chunks, from the stored state, and the state there is published (if the item goes on over
//     more than one other CTA, these wait for it at once: then first without results, and the chunks again with them);
//   - or, where its whole stretch lies inside one item, the sum that its chunks add to a state, without any results, is published;
// then it does the items that are its own, and last the rest of the item that it did not begin: the state there is put together from what the CTAs
// before it have published.
#pragma once
#include <stdint.h>

namespace icc {

constexpr int STATE_CHUNK = 64;           // tokens
constexpr int STATE_BATCH = 256;          // sequences of a launch
// Items of at most STATE_WHOLE chunks are not cut (8 sequences of 700 tokens, 32 heads of 128 x 128: 73 us, with 6 90; 5 sequences, 16 heads of 64 x 128:
// 31 and 51; 8 of 1,000 tokens 110, with 16 95, but one sequence, 4 heads of 64 x 64, 32 in place of 28), and no piece has fewer than STATE_LEAST (2: 75
// in place of 68 us for 8 sequences of 500 tokens).
constexpr int STATE_WHOLE = 12;
constexpr int STATE_LEAST = 3;

struct StateLine {
  int before[STATE_BATCH + 1];            // chunks of the sequences before this one
  int n, per_chunk;                       // sequences; items of a sequence (heads times slices)
  int parts;                              // CTAs
  int per;                                // chunks of a stretch
  // (the line has fewer than 2^31 chunks: state_items() sees to it)
  __host__ __device__ int length() const { return before[n] * per_chunk; }
  __host__ __device__ int chunks(int i) const { return before[i + 1] - before[i]; }
  // longest: chunks of the longest sequence
  __host__ __device__ void set_per(int longest) {
    per = (int)(((unsigned)length() + parts - 1) / parts);
    if (per >= STATE_LEAST) return;
    // (few chunks: items that are not cut may go one to a CTA)
    if (longest > STATE_WHOLE) per = STATE_LEAST;
    else if (per < 1) per = 1;
  }
  // The item that position x (below length()) lies in: its sequence, which of its items, and where that begins.
  struct At {
    int i, item, start;
  };
  __host__ __device__ At find(int x) const {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (before[mid] * per_chunk <= x) lo = mid;
      else hi = mid - 1;
    }
    // (sequences without chunks begin where the next one does: the last of them is found, which has some)
    const int first = before[lo] * per_chunk, c = chunks(lo), item = (x - first) / c;
    return {lo, item, first + item * c};
  }
  // Where the stretch of CTA b begins.
  __host__ __device__ int cut(int b) const {
    const int all = length();
    const long long at = (long long)per * b;
    if (at >= all) return all;
    const int x = (int)at;
    const At a = find(x);
    const int c = chunks(a.i), rest = x - a.start;
    if (c <= STATE_WHOLE || rest < STATE_LEAST) return a.start;
    if (c - rest < STATE_LEAST) return a.start + c;
    return x;
  }
};

// How many items of a sequence (heads times slices) a launch may have, so that the line of n sequences with so many tokens in all stays below
// 2^31 chunks.
inline int state_items(long long n_tokens, int n) {
  const long long chunks = n_tokens / STATE_CHUNK + n;
  return chunks ? (int)(0x7fffffffll / chunks < 0x7fffffffll ? 0x7fffffffll / chunks : 0x7fffffffll) : 0x7fffffff;
}

// A piece of a CTA's stretch.
struct StatePiece {
  enum : int { STORED = 0, NOTHING = 1, PUBLISHED = 2 };
  int i, item;              // sequence of the launch; head and slice
  int c0, c1;               // chunks of the item
  int from;                 // where its state comes from: STORED, NOTHING (zeros), or PUBLISHED by other CTAs
  int to;                   // where it goes: STORED, NOTHING (nowhere) or PUBLISHED
  int sum_only;             // no results
};

// A CTA's stretch: what others wait for, its own items, the rest of another's.
struct StatePlan {
  StatePiece first, again, last;          // none: c1 is 0
  int own_i, own_item, own_count;         // its own items: the first, and how many
  int begin, slot_first, item_start;      // of `last`: its place on the line, the CTA that begun its item, and where that begins
  __host__ __device__ void make(const StateLine& l, int b) {
    const int x0 = l.cut(b), x1 = l.cut(b + 1);
    first.c1 = again.c1 = last.c1 = own_i = own_item = own_count = begin = slot_first = item_start = 0;
    if (x0 >= x1) return;
    const StateLine::At a = l.find(x0), z = l.find(x1 - 1);
    const int end = a.start + l.chunks(a.i);          // of the item that x0 lies in
    const bool open = z.start + l.chunks(z.i) > x1;   // the last item goes on behind x1
    if (open) {
      const bool begun = z.start >= x0;
      first = {z.i, z.item, (begun ? z.start : x0) - z.start, x1 - z.start, begun ? StatePiece::STORED : StatePiece::NOTHING, StatePiece::PUBLISHED, !begun};
      if (begun && z.start + l.chunks(z.i) > l.cut(b + 2)) {
        again = {z.i, z.item, first.c0, first.c1, StatePiece::STORED, StatePiece::NOTHING, 0};
        first.sum_only = 1;
      }
    }
    int x = x0;
    own_i = a.i;
    own_item = a.item;
    if (a.start < x0) {
      last = {a.i, a.item, x0 - a.start, (end < x1 ? end : x1) - a.start, StatePiece::PUBLISHED, end <= x1 ? StatePiece::STORED : StatePiece::NOTHING, 0};
      begin = x0;
      item_start = a.start;
      slot_first = a.start / l.per < l.parts ? a.start / l.per : l.parts - 1;
      while (slot_first > 0 && l.cut(slot_first) > a.start) --slot_first;
      while (slot_first + 1 < b && l.cut(slot_first + 1) <= a.start) ++slot_first;
      x = end;
      if (x < x1) {
        const StateLine::At o = l.find(x);
        own_i = o.i;
        own_item = o.item;
      }
    }
    // items from x to where the open one begins
    const int own_end = open ? z.start : x1;
    if (x < own_end) {
      const StateLine::At e = l.find(own_end - 1);
      int sequences = 0;                              // that have chunks, from the first one's on
      for (int i = own_i; i < e.i; ++i) sequences += l.chunks(i) > 0;
      own_count = sequences * l.per_chunk + e.item - own_item + 1;
    }
  }
};

// The pieces, in the order in which they are done.
struct StateWalk {
  const StateLine* line;
  const StatePlan* plan;
  int step, i, item, left;
  __host__ __device__ StateWalk(const StateLine* l, const StatePlan* p) : line(l), plan(p), step(0), i(p->own_i), item(p->own_item), left(p->own_count) {}
  __host__ __device__ bool next(StatePiece* p) {
    if (step == 0) {
      step = 1;
      if (plan->first.c1) {
        *p = plan->first;
        return true;
      }
    }
    if (step == 1) {
      step = 2;
      if (plan->again.c1) {
        *p = plan->again;
        return true;
      }
    }
    if (left > 0) {
      *p = {i, item, 0, line->chunks(i), StatePiece::STORED, StatePiece::STORED, 0};
      if (--left > 0 && ++item == line->per_chunk) {
        item = 0;
        do ++i;
        while (line->chunks(i) == 0);
      }
      return true;
    }
    if (step == 2) {
      step = 3;
      if (plan->last.c1) {
        *p = plan->last;
        return true;
      }
    }
    return false;
  }
};

}  // namespace icc
