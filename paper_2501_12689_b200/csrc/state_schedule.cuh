// How a call over the states is divided among the CTAs.
//
// The chunks of all sequences, heads and value slices of a launch form one line, and each CTA takes an equal stretch of it.  A stretch may begin
// or end inside an item (a sequence, head and slice), whose state then comes from the CTAs before.  To leave nobody waiting, a CTA begins with
// what others wait for:
//   - the item that it begins and does not end: its chunks, from the stored state, and the state there is published;
//   - or, where its whole stretch lies inside one item, the sum that its chunks add to a state, without any results, is published;
// then it does the items that are its own, and last the rest of the item that it did not begin: the state there is put together from what the CTAs
// before it have published.
#pragma once
#include <stdint.h>

namespace icc {

constexpr int STATE_CHUNK = 64;           // tokens
constexpr int STATE_BATCH = 256;          // sequences of a launch
constexpr int STATE_WHOLE = 6;            // items of at most so many chunks are not cut,
constexpr int STATE_LEAST = 3;            // and no piece has fewer

struct StateLine {
  int before[STATE_BATCH + 1];            // chunks of the sequences before this one
  int n, per_chunk;                       // sequences; items of a sequence (heads times slices)
  int parts;                              // CTAs
  __host__ __device__ long long length() const { return (long long)before[n] * per_chunk; }
  __host__ __device__ int chunks(int i) const { return before[i + 1] - before[i]; }
  // The item that position x (below length()) lies in: its sequence, which of its items, and where that begins.
  struct At {
    int i, item;
    long long start;
  };
  __host__ __device__ At find(long long x) const {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((long long)before[mid] * per_chunk <= x) lo = mid;
      else hi = mid - 1;
    }
    // (sequences without chunks begin where the next one does: the last of them is found, which has some)
    const long long first = (long long)before[lo] * per_chunk;
    const int c = chunks(lo), item = (int)((x - first) / c);
    return {lo, item, first + (long long)item * c};
  }
  __host__ __device__ long long per() const {
    const long long p = (length() + parts - 1) / parts;
    return p < STATE_LEAST ? STATE_LEAST : p;
  }
  // A CTA about where position x lies.
  __host__ __device__ int near(long long x) const {
    const long long b = x / per();
    return b < parts ? (int)b : parts - 1;
  }
  // Where the stretch of CTA b begins.
  __host__ __device__ long long cut(int b) const {
    const long long all = length(), x = per() * b;
    if (x >= all) return all;
    const At a = find(x);
    const int c = chunks(a.i), rest = (int)(x - a.start);
    if (c <= STATE_WHOLE || rest < STATE_LEAST) return a.start;
    if (c - rest < STATE_LEAST) return a.start + c;
    return x;
  }
};

// A stretch's pieces, in the order in which they are done.
struct StatePiece {
  enum : int { STORED = 0, NOTHING = 1, PUBLISHED = 2 };
  int i, item;              // sequence of the launch; head and slice
  int c0, c1;               // chunks of the item
  int from;                 // where its state comes from: STORED, NOTHING (zeros) or PUBLISHED by the CTAs first .. own - 1
  int to;                   // where it goes: STORED, NOTHING (nowhere) or PUBLISHED
  int first;
  bool sum_only;            // no results
};

struct StateWalk {
  const StateLine* line;
  int own, step;
  long long x0, x1, x;      // the stretch; where its own items go on
  long long head_end;       // where the item ends that it did not begin; x0 if it begins one
  __host__ __device__ StateWalk(const StateLine* l, int b) : line(l), own(b), step(0) {
    x0 = l->cut(b);
    x1 = l->cut(b + 1);
    head_end = x0;
    if (x0 < x1) {
      const StateLine::At a = l->find(x0);
      if (a.start < x0) {
        const long long end = a.start + l->chunks(a.i);
        head_end = end < x1 ? end : x1;
      }
    }
    x = head_end;
  }
  __host__ __device__ bool next(StatePiece* p) {
    if (x0 >= x1) return false;
    if (step == 0) {                       // what others wait for
      step = 1;
      const StateLine::At a = line->find(x1 - 1);
      if (a.start + line->chunks(a.i) > x1) {
        const bool begun = a.start >= x0;
        *p = {a.i, a.item, (int)((begun ? a.start : x0) - a.start), (int)(x1 - a.start), begun ? StatePiece::STORED : StatePiece::NOTHING,
              StatePiece::PUBLISHED, own, !begun};
        return true;
      }
    }
    if (step == 1) {                       // its own
      if (x < x1) {
        const StateLine::At a = line->find(x);
        const int c = line->chunks(a.i);
        if (a.start + c <= x1) {
          *p = {a.i, a.item, 0, c, StatePiece::STORED, StatePiece::STORED, own, false};
          x = a.start + c;
          return true;
        }
      }
      step = 2;
    }
    if (step == 2 && head_end > x0) {      // the rest of another's
      step = 3;
      const StateLine::At a = line->find(x0);
      int first = line->near(a.start);
      while (first > 0 && line->cut(first) > a.start) --first;
      while (first + 1 < own && line->cut(first + 1) <= a.start) ++first;
      *p = {a.i, a.item, (int)(x0 - a.start), (int)(head_end - a.start), StatePiece::PUBLISHED,
            head_end == a.start + line->chunks(a.i) ? StatePiece::STORED : StatePiece::NOTHING, first, false};
      return true;
    }
    return false;
  }
};

}  // namespace icc
