// Log-probabilities of given tokens, entropy and the top alternatives of rows of logits, in one pass.
//
// A thread walks over its part of a row with a running maximum m of the logits x and the sums  s = sum 2^d  and  w = sum 2^d d,
// d = (x - m) scale log2(e):  at a new maximum m' both are rescaled, w <- f (w + s c), s <- f s, f = 2^c, c = (m - m') scale log2(e).  Then
// log_prob(t) = (x_t - m) scale - log s,  entropy = log s - log(2) w / s.  The difference is taken before the product: that of the largest logit is 0 and
// none is above it, however large the logits are.  (scale x rounded for the maximum and not for the difference would leave the product's rounding error,
// 10^30 for rows masked with the type's lowest value.)
// Every logit is read once, as 16-byte vectors, VECTORS of them at a time.  Per logit: one exponential (the special
// function units do 16 a cycle and SM: in 16 bits three quarters of their rate at the copy's bandwidth), and about six other
// instructions, pairs of floats at a time, where the bandwidth leaves room for eleven.  4,001 rows of 128,256 in bf16, in a graph: 163 us, 6.3 TB/s; with five
// alternatives 192, with twenty 211.  VECTORS and CTAS an SM: 6 and 4; 8 and 3 take 166, 200 and 227, 4 and 4 171, 198 and 216, 4 and 5 161, 200 and 216.
//
// Top alternatives: a lower bound of the row's n-th best is the n-th largest of the maxima of 64 groups of threads, as these are n different
// elements.  So all that the pass over the row does for them is to note the maximum of each thread's blocks (or of groups of them, in long
// rows).  At the end few blocks reach the bound, a little more than n; those are read again, and the elements that reach it go to a buffer of the
// warp, where the rank of each is the number of larger ones.  A buffer that fills up is taken into the warp's list of its 32 best keys (value,
// lowest index first), one a lane, sorted.  A warp's steps, a vector a lane, ascend in their indices, so an element equal to the list's
// last one never enters later.  (Sorted lists kept on the way instead: 512 us with five alternatives, 920 with twenty.)
//
// Rows are split over CTAs when there are few of them; the CTA that finishes last joins the pieces, in their order.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "kernels.h"
#include "kv.h"
#include "kv_mma.cuh"
#include "pipeline.cuh"
#include "score.h"

namespace icc {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int VECTORS = 6;                // 16-byte vectors of a thread's block
constexpr int CTAS = 4;                   // an SM
constexpr int GROUPS = 16;                // of a thread's blocks, each with its maximum
constexpr int BUFFER = 384;               // keys of a warp that have passed the bound: more than a step's 256, so that it is seldom emptied
static_assert(WARPS * BUFFER >= SCORE_MAX_SPLIT * SCORE_MAX_TOP, "the pieces' keys are joined there");
constexpr float LOG_OF_2 = 0.6931471805599453f;
constexpr float LEAST = -217.0f;          // 2^LEAST is 0 in fp32; keeps banned tokens' differences finite
constexpr float INF = __builtin_huge_valf();

enum : int { BF16 = 0, F16 = 1, F32 = 2 };

__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

template <int T>
struct Elements {
  static constexpr int SIZE = T == F32 ? 4 : 2, PER = 16 / SIZE;      // bytes, elements of a vector
  static constexpr uint32_t BANNED = T == F32 ? 0xff800000u : T == F16 ? 0xfc00fc00u : 0xff80ff80u;
  // Elements 2 i and 2 i + 1 of a vector.
  __device__ __forceinline__ static float2 pair(const uint4& v, int i) {
    const uint32_t* x = &v.x;
    if (T == F32) return make_float2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1]));
    if (T == F16) return __half22float2(*reinterpret_cast<const __half2*>(x + i));
    return make_float2(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u));
  }
  // Element e, which the compiler does not know.
  __device__ __forceinline__ static float any(const uint4& v, int e) {
    const int i = T == F32 ? e : e >> 1;
    const uint32_t x = i & 2 ? (i & 1 ? v.w : v.z) : (i & 1 ? v.y : v.x);
    if (T == F32) return __uint_as_float(x);
    const uint16_t h = (uint16_t)(e & 1 ? x >> 16 : x);
    return T == F16 ? __half2float(__ushort_as_half(h)) : __bfloat162float(__ushort_as_bfloat16(h));
  }
  // Largest element; NaN if there is one.
  __device__ __forceinline__ static float largest(const uint4& v) { return widest(larger(larger(v.x, v.y), larger(v.z, v.w))); }
  // The same by words, of one element or two.
  __device__ __forceinline__ static uint32_t larger(uint32_t a, uint32_t b) {
    if (T == F32) return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b)));
    uint32_t d;
    if (T == F16) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
  }
  __device__ __forceinline__ static float widest(uint32_t x) {
    if (T == F32) return __uint_as_float(x);
    const float2 m = T == F16 ? __half22float2(*reinterpret_cast<const __half2*>(&x)) : make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
    return max_nan(m.x, m.y);
  }
  __device__ __forceinline__ static float one(const unsigned char* row, int i) {
    if (T == F32) return reinterpret_cast<const float*>(row)[i];
    const uint16_t x = reinterpret_cast<const uint16_t*>(row)[i];
    return T == F16 ? __half2float(__ushort_as_half(x)) : __bfloat162float(__ushort_as_bfloat16(x));
  }
};

// Maximum and sums, by halves: even and odd elements are summed apart.  c: scale log2(e).
struct Sums {
  float top;                // -infinity: nothing yet
  uint64_t s, w;
  __device__ __forceinline__ Sums() : top(-INF), s(0), w(0) {}
  // Raise the maximum to cover x; returns what differences are taken against.
  __device__ __forceinline__ float raise(float x, float c) {
    const float now = max_nan(top, x), at = now == -INF ? 0.0f : now;
    const float d = fmaxf((top - at) * c, LEAST), f = exp2_fast(d);
    const uint64_t f2 = pair_of(f, f);
    w = mul_pairs(fma_pairs(s, pair_of(d, d), w), f2);
    s = mul_pairs(s, f2);
    top = now;
    return at;
  }
  __device__ __forceinline__ void add(uint64_t x2, uint64_t minus2, uint64_t c2) {
    float a, b;
    split_pair(mul_pairs(add_pairs(x2, minus2), c2), &a, &b);
    a = fmaxf(a, LEAST);
    b = fmaxf(b, LEAST);
    const uint64_t e = pair_of(exp2_fast(a), exp2_fast(b));
    s = add_pairs(s, e);
    w = fma_pairs(e, pair_of(a, b), w);
  }
};

struct Joined {
  float top, sum, weighted;
  __device__ __forceinline__ void join(const Joined& o, float c) {
    const float now = max_nan(top, o.top), at = now == -INF ? 0.0f : now;
    const float da = fmaxf((top - at) * c, LEAST), db = fmaxf((o.top - at) * c, LEAST), fa = exp2_fast(da), fb = exp2_fast(db);
    weighted = fa * (weighted + sum * da) + fb * (o.weighted + o.sum * db);
    sum = fa * sum + fb * o.sum;
    top = now;
  }
  __device__ __forceinline__ void over_warp(float c) {
#pragma unroll
    for (int x = 16; x; x >>= 1) {
      const Joined o{__shfl_xor_sync(FULL_MASK, top, x), __shfl_xor_sync(FULL_MASK, sum, x), __shfl_xor_sync(FULL_MASK, weighted, x)};
      join(o, c);
    }
  }
};

// The 32 best of two sets of 32 keys, one a lane, in descending order; the first set is in that order.
__device__ __noinline__ uint64_t merge_sorted(uint64_t sorted, uint64_t key, int lane) {
#pragma unroll
  for (int k = 2; k <= 32; k *= 2)
#pragma unroll
    for (int j = k / 2; j; j /= 2) {
      const uint64_t other = __shfl_xor_sync(FULL_MASK, key, j);
      if (((lane & k) == 0) == ((lane & j) == 0) ? other > key : other < key) key = other;
    }
  const uint64_t turned = __shfl_sync(FULL_MASK, key, 31 - lane);
  if (turned > sorted) sorted = turned;
#pragma unroll
  for (int j = 16; j; j /= 2) {
    const uint64_t other = __shfl_xor_sync(FULL_MASK, sorted, j);
    if ((lane & j) == 0 ? other > sorted : other < sorted) sorted = other;
  }
  return sorted;
}

// The warp's best keys, one a lane in descending order; the first n of them count.
struct TopList {
  uint64_t mine, last;      // last: the n-th, KEY_EMPTY until there are n
  __device__ __forceinline__ TopList() : mine(KEY_EMPTY), last(KEY_EMPTY) {}
  // What an element of a later step has to reach to enter: the next number after the last one's (NaN, which nothing reaches, after infinity).
  __device__ __forceinline__ float least() const { return last == KEY_EMPTY ? -INF : ord_to_score((uint32_t)(last >> 32) + 1); }
  // A key per lane, KEY_EMPTY for none.
  __device__ __forceinline__ void offer(uint64_t key, int n, int lane) {
    unsigned who = __ballot_sync(FULL_MASK, key > last);
    if (__popc(who) > 6) {  // some 20 exchanges between lanes, as in three to six insertions that wait for one another
      mine = merge_sorted(mine, key, lane);
      last = __shfl_sync(FULL_MASK, mine, n - 1);
      return;
    }
    while (who) {
      const uint64_t k = __shfl_sync(FULL_MASK, key, __ffs(who) - 1);
      const int at = __popc(__ballot_sync(FULL_MASK, mine > k));
      const uint64_t up = __shfl_up_sync(FULL_MASK, mine, 1);
      if (lane == at) mine = k;
      else if (lane > at) mine = up;
      last = __shfl_sync(FULL_MASK, mine, n - 1);
      who &= who - 1;
      who &= __ballot_sync(FULL_MASK, key > last);
    }
  }
};

// The n-th largest of the maxima of 64 groups of threads, without what is behind its first BITS bits.
template <int BITS>
__device__ __forceinline__ uint32_t nth_largest(const volatile uint32_t* words, int n, int lane) {
  uint32_t x[2] = {0, 0}, y = 0;
#pragma unroll
  for (int i = 0; i < WARPS; ++i) x[i & 1] = max(x[i & 1], words[i * 32 + lane]);
  static_assert(BITS % 2 == 0, "two bits a round: half as many rounds, each waiting for the last, as with one");
#pragma unroll 1
  for (int at = 30; at >= 32 - BITS; at -= 2) {
    uint32_t more = 0;
#pragma unroll
    for (uint32_t d = 1; d < 4; ++d) {
      const uint32_t t = y | d << at;
      more += __popc(__ballot_sync(FULL_MASK, x[0] >= t)) + __popc(__ballot_sync(FULL_MASK, x[1] >= t)) >= n;
    }
    y |= more << at;
  }
  return y;
}

template <int T, bool TOP>
__global__ void __launch_bounds__(THREADS, CTAS) score_kernel(const ScoreParams p) {
  using E = Elements<T>;
  __shared__ Joined of_warp[WARPS];
  __shared__ uint64_t passed[TOP ? WARPS * BUFFER : 1], keys[TOP ? THREADS : 1], best[SCORE_MAX_TOP];
  __shared__ float group_max[TOP ? GROUPS * THREADS : 1];
  __shared__ uint32_t maxima[THREADS];
  __shared__ int n_passed, last_one;
  grid_dep_launch_dependents();
  grid_dep_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = p.n_top;
  const int64_t row = blockIdx.x / p.split;
  const int piece = blockIdx.x - (int)row * p.split;
  const unsigned char* x = p.logits + row * p.row_stride * E::SIZE;
  // a row need not begin on a vector: single elements up to the first, and behind the last
  const int head = min(p.vocab, (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / E::SIZE);
  const int vectors = (p.vocab - head) / E::PER, tail = p.vocab - head - vectors * E::PER;
  const uint4* xv = reinterpret_cast<const uint4*>(x + head * E::SIZE);
  const int per = (vectors + p.split - 1) / p.split, v0 = min(vectors, per * piece), v1 = min(vectors, v0 + per);
  float largest = -INF, of_group = -INF, least = -INF;         // the thread's so far, its group's; what elements have to reach
  const float c = p.scale_log2;
  const uint64_t c2 = pair_of(c, c);
  // what the end needs, on its way from the start
  const int target = p.targets && warp == 0 ? p.targets[row] : -1;
  const float of_target = target >= 0 && target < p.vocab ? E::one(x, target) : 0.0f;
  Sums sums;
  TopList list;

  uint64_t* const mine_passed = passed + (TOP ? warp * BUFFER : 0);
  int count = 0;                                      // of the warp's keys there
  auto push = [&](uint32_t mask, auto key_of) {       // a bit for each element of the lane's that has passed
    for (unsigned who; (who = __ballot_sync(FULL_MASK, mask != 0)) != 0; count += __popc(who))
      if (mask) {
        mine_passed[count + __popc(who & ((1u << lane) - 1u))] = key_of(__ffs(mask) - 1);
        mask &= mask - 1;
      }
    __syncwarp();
  };
  auto take_in = [&]() {                              // what has passed, into the list
    for (int i = 0; i < count; i += 32) list.offer(i + lane < count ? mine_passed[i + lane] : KEY_EMPTY, n, lane);
    count = 0;
    __syncwarp();
  };
  // single elements, of the first warp's lanes
  auto single_value = [&](int i, int end) { return i < end ? E::one(x, i) : -INF; };
  auto single_sums = [&](float y) {
    const float at = sums.raise(y, c);
    sums.add(pair_of(y, -INF), pair_of(-at, -at), c2);
  };
  auto single_key = [&](float y, int i, int end) { push(i < end && y >= least, [&](int) { return make_key(y, i); }); };
  const bool has_head = piece == 0 && warp == 0 && head, has_tail = piece == p.split - 1 && warp == 0 && tail;
  float of_head = -INF, of_tail = -INF;
  if (has_head) single_sums(of_head = single_value(lane, head));
  if (has_tail) single_sums(of_tail = single_value(p.vocab - tail + lane, p.vocab));

  uint4 v[VECTORS];
  auto load = [&](int base) {
    const uint4* from = xv + base + tid;
    if (base + VECTORS * THREADS <= v1) {
#pragma unroll
      for (int j = 0; j < VECTORS; ++j) v[j] = ld_stream_16B(from + j * THREADS);
    } else {
#pragma unroll
      for (int j = 0; j < VECTORS; ++j)
        v[j] = base + j * THREADS + tid < v1 ? ld_stream_16B(from + j * THREADS) : make_uint4(E::BANNED, E::BANNED, E::BANNED, E::BANNED);
    }
  };
  const int blocks = (v1 - v0 + VECTORS * THREADS - 1) / (VECTORS * THREADS);
  int shift = 0;                                      // 2^shift blocks are a group
  while (blocks > GROUPS << shift) ++shift;
  for (int block = 0; block < blocks; ++block) {
    load(v0 + block * VECTORS * THREADS);
    uint32_t words[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      words[i] = (&v[0].x)[i];
#pragma unroll
      for (int j = 1; j < VECTORS; ++j) words[i] = E::larger(words[i], (&v[j].x)[i]);
    }
    const float all = E::widest(E::larger(E::larger(words[0], words[1]), E::larger(words[2], words[3])));
    if (TOP) {
      of_group = block & ((1 << shift) - 1) ? max_nan(of_group, all) : all;
      group_max[(block >> shift) * THREADS + tid] = of_group;
      largest = max_nan(largest, all);
    }
    const float at = sums.raise(all, c);
    const uint64_t minus2 = pair_of(-at, -at);
#pragma unroll
    for (int j = 0; j < VECTORS; ++j)
#pragma unroll
      for (int i = 0; i < E::PER / 2; ++i) {
        const float2 u = E::pair(v[j], i);
        sums.add(pair_of(u.x, u.y), minus2, c2);
      }
  }

  // the CTA's result
  float sa, sb, wa, wb;
  split_pair(sums.s, &sa, &sb);
  split_pair(sums.w, &wa, &wb);
  Joined mine{sums.top, sa + sb, wa + wb};
  mine.over_warp(c);
  if (lane == 0) of_warp[warp] = mine;
  if (TOP) {
    maxima[tid] = largest == largest ? score_to_ord(largest) : 0u;
    if (tid == 0) n_passed = 0;
    __syncthreads();
    least = fmaxf(ord_to_score(nth_largest<T == BF16 ? 16 : 20>(maxima, n, lane)), -INF);        // (NaN where less than n threads have something)
    if (has_head) single_key(of_head, lane, head);
    uint32_t mine_reach = 0;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) mine_reach |= (g << shift < blocks && group_max[g * THREADS + tid] >= least ? 1u : 0u) << g;
    for (uint32_t groups = __reduce_or_sync(FULL_MASK, mine_reach); groups; groups &= groups - 1) {
      const int first = (__ffs(groups) - 1) << shift;
      const bool reaches = mine_reach & groups & -groups;
      for (int block = first; block < min(blocks, first + (1 << shift)); ++block) {
        const int i0 = v0 + block * VECTORS * THREADS + tid;
#pragma unroll
        for (int j = 0; j < VECTORS; ++j)
          v[j] = reaches && i0 + j * THREADS < v1 ? ld_stream_16B(xv + i0 + j * THREADS) : make_uint4(E::BANNED, E::BANNED, E::BANNED, E::BANNED);
#pragma unroll
        for (int j = 0; j < VECTORS; ++j) {
          const bool some = reaches && i0 + j * THREADS < v1 && E::largest(v[j]) >= least;
          if (!__any_sync(FULL_MASK, some)) continue;
          uint32_t mask = 0;
#pragma unroll
          for (int e = 0; e < E::PER; ++e) {
            const float2 u = E::pair(v[j], e / 2);
            mask |= ((e & 1 ? u.y : u.x) >= least ? 1u : 0u) << e;
          }
          push(some ? mask : 0u, [&](int e) { return make_key(E::any(v[j], e), head + (i0 + j * THREADS) * E::PER + e); });
          if (count > BUFFER - 32 * E::PER) {
            take_in();
            least = max_nan(least, list.least());
          }
        }
      }
    }
    if (has_tail) single_key(of_tail, p.vocab - tail + lane, p.vocab);
    if (count > 32 || __any_sync(FULL_MASK, list.mine != KEY_EMPTY)) {
      take_in();
      count = __popc(__ballot_sync(FULL_MASK, lane < n && list.mine != KEY_EMPTY));
      if (lane < count) mine_passed[lane] = list.mine;
    }
    // all warps' keys, one behind the other
    int at = 0;
    if (lane == 0) at = atomicAdd(&n_passed, count);
    at = __shfl_sync(FULL_MASK, at, 0);
    if (lane < count) keys[at + lane] = mine_passed[lane];
  }
  __syncthreads();
  int found = 0;
  if (TOP) {                                          // a key a thread: its rank is the number of larger ones
    found = n_passed;
    if (tid < found) {
      const uint64_t key = keys[tid];
      int rank = 0;
#pragma unroll 8
      for (int k = 0; k < found; ++k) rank += keys[k] > key;
      if (rank < n) best[rank] = key;
    }
    if (found > 32) __syncthreads();
    if (found > n) found = n;
    __syncwarp();
  }
  if (warp != 0) return;
  mine = lane < WARPS ? of_warp[lane] : Joined{-INF, 0.0f, 0.0f};
  mine.over_warp(c);
  if (p.split > 1) {
    ScorePartial* to = p.partials + row * p.split + piece;
    if (lane == 0) {
      to->top = mine.top;
      to->sum = mine.sum;
      to->weighted = mine.weighted;
    }
    if (TOP && lane < n) to->keys[lane] = lane < found ? best[lane] : KEY_EMPTY;
    __threadfence();
    __syncwarp();
    if (lane == 0) {
      last_one = atomicAdd(p.arrivals + row, 1) == p.split - 1;
      if (last_one) p.arrivals[row] = 0;
    }
    __syncwarp();
    if (!last_one) return;
    __threadfence();
    const ScorePartial* all = p.partials + row * p.split;
    mine = Joined{-INF, 0.0f, 0.0f};
    if (lane < p.split) mine = Joined{__ldcg(&all[lane].top), __ldcg(&all[lane].sum), __ldcg(&all[lane].weighted)};
    mine.over_warp(c);
    if (TOP) {
#pragma unroll 8
      for (int i = 0; i < p.split; ++i)
        if (lane < n) passed[i * SCORE_MAX_TOP + lane] = __ldcg(&all[i].keys[lane]);
      __syncwarp();
      found = tournament_in_registers<1>(passed, SCORE_MAX_TOP, p.split, n, lane, best);
      __syncwarp();
    }
  }
  // the row's
  const float y_top = __fmul_rn(mine.top, p.scale);
  const bool none = !(y_top < INF), banned = y_top == -INF;
  const float log_sum = banned ? 0.0f : logf(mine.sum), top = banned ? 0.0f : mine.top, nan = __int_as_float(0x7fffffff);
  // (halves: the difference of two finite logits may leave fp32 where scale brings it back)
  auto log_prob = [&](float v) { return none ? nan : fmaf(0.5f * v - 0.5f * top, p.scale, -0.5f * log_sum) * 2.0f; };
  if (lane == 0 && p.entropy) p.entropy[row] = none ? nan : banned ? 0.0f : log_sum - LOG_OF_2 * (mine.weighted / mine.sum);
  if (lane == 0 && p.targets) {
    float r = 0.0f;
    if (target >= 0 && target < p.vocab) {
      r = log_prob(of_target);
    } else if (target != -1) {
      r = nan;
      report_status(p.host_status, KV_INVALID);
    }
    p.log_probs[row] = r;
  }
  if (TOP && lane < n) {
    const uint64_t k = lane < found ? best[lane] : KEY_EMPTY;
    p.top_ids[row * n + lane] = none || k == KEY_EMPTY ? -1 : (int)key_slot(k);
    p.top_log_probs[row * n + lane] = k == KEY_EMPTY ? nan : log_prob(key_score(k));
  }
}

template <int T>
cudaError_t launch(const ScoreParams& p, cudaStream_t st) {
  return launch_overlapped(p.n_top ? score_kernel<T, true> : score_kernel<T, false>, dim3((unsigned)(p.n_rows * p.split)), dim3(THREADS), 0, st, 1, p);
}

}  // namespace

cudaError_t score_launch(ScoreParams p, int dtype, int sm_count, cudaStream_t st) {
  // few rows are split until CTAS an SM have something to do, down to a block per thread
  const int64_t wanted = CTAS * sm_count / p.n_rows, blocks = (int64_t)p.vocab * (dtype == F32 ? 4 : 2) / (16 * VECTORS * THREADS);
  p.split = (int)(wanted < SCORE_MAX_SPLIT ? wanted : SCORE_MAX_SPLIT);
  if (p.split > blocks) p.split = (int)blocks;
  if (p.split < 1) p.split = 1;
  if (p.split > 1 && p.n_rows * p.split > SCORE_SLOTS) p.split = (int)(SCORE_SLOTS / p.n_rows) > 1 ? (int)(SCORE_SLOTS / p.n_rows) : 1;
  return dtype == F32 ? launch<F32>(p, st) : dtype == F16 ? launch<F16>(p, st) : launch<BF16>(p, st);
}

}  // namespace icc
