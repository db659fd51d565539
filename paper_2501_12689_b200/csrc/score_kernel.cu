// Log-probabilities of given tokens, entropy and the top alternatives of rows of logits, in one pass.
//
// A thread walks over its part of a row with a running maximum m and the sums  s = sum e^(y - m)  and  w = sum e^(y - m) (y - m):  at a new
// maximum m' both are rescaled, w <- f (w + s (m - m')), s <- f s, f = e^(m - m').  Then  log_prob(t) = y_t - m - log s,  entropy = log s - w / s.
// Every logit is read once, as 16-byte vectors, VECTORS of them under way while as many are worked on.  Per logit: one exponential (the special
// function units do 16 a cycle and SM: in 16 bits three quarters of their rate at the copy's bandwidth), and about six other
// instructions, pairs of floats at a time, where the bandwidth leaves room for eleven.
//
// Top alternatives: a warp keeps its 32 best keys (value, lowest index first) one a lane, sorted.  A block of elements is looked at more closely
// only if its maximum reaches the list: the largest known lower bound of the row's n-th best, shared by the CTA, starts as
// the n-th largest of the lanes' maxima over their first blocks, so that even then few elements pass.  A warp's steps, a vector a lane,
// ascend in their indices, so an element equal to the list's last one of an earlier step never enters.
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
constexpr int VECTORS = 4;                // 16-byte vectors of a thread's block
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LEAST = -150.0f;          // e^LEAST is 0 in fp32; keeps banned tokens' differences finite
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
  // Largest element; NaN if there is one.
  __device__ __forceinline__ static float largest(const uint4& v) {
    if (T == F32) return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)), max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
    if (T == F16) {
      const __half2* x = reinterpret_cast<const __half2*>(&v.x);
      const float2 m = __half22float2(__hmax2_nan(__hmax2_nan(x[0], x[1]), __hmax2_nan(x[2], x[3])));
      return max_nan(m.x, m.y);
    }
    const __nv_bfloat162* x = reinterpret_cast<const __nv_bfloat162*>(&v.x);
    const float2 m = __bfloat1622float2(__hmax2_nan(__hmax2_nan(x[0], x[1]), __hmax2_nan(x[2], x[3])));
    return max_nan(m.x, m.y);
  }
  __device__ __forceinline__ static float one(const unsigned char* row, int i) {
    if (T == F32) return reinterpret_cast<const float*>(row)[i];
    const uint16_t x = reinterpret_cast<const uint16_t*>(row)[i];
    return T == F16 ? __half2float(__ushort_as_half(x)) : __bfloat162float(__ushort_as_bfloat16(x));
  }
};

// Maximum and sums, by halves: even and odd elements are summed apart.
struct Sums {
  float top;                // -infinity: nothing yet
  uint64_t s, w;
  __device__ __forceinline__ Sums() : top(-INF), s(0), w(0) {}
  // Raise the maximum to cover y; returns what differences are taken against.
  __device__ __forceinline__ float raise(float y) {
    const float now = max_nan(top, y), at = now == -INF ? 0.0f : now;
    const float d = fmaxf(top - at, LEAST), f = exp2_fast(d * LOG2E);
    const uint64_t f2 = pair_of(f, f);
    w = mul_pairs(fma_pairs(s, pair_of(d, d), w), f2);
    s = mul_pairs(s, f2);
    top = now;
    return at;
  }
  __device__ __forceinline__ void add(uint64_t y2, uint64_t minus2) {
    float a, b;
    split_pair(add_pairs(y2, minus2), &a, &b);
    const uint64_t d = pair_of(fmaxf(a, LEAST), fmaxf(b, LEAST));
    split_pair(mul_pairs(d, pair_of(LOG2E, LOG2E)), &a, &b);
    const uint64_t e = pair_of(exp2_fast(a), exp2_fast(b));
    s = add_pairs(s, e);
    w = fma_pairs(e, d, w);
  }
};

struct Joined {
  float top, sum, weighted;
  __device__ __forceinline__ void join(const Joined& o) {
    const float now = max_nan(top, o.top), at = now == -INF ? 0.0f : now;
    const float da = fmaxf(top - at, LEAST), db = fmaxf(o.top - at, LEAST), fa = exp2_fast(da * LOG2E), fb = exp2_fast(db * LOG2E);
    weighted = fa * (weighted + sum * da) + fb * (o.weighted + o.sum * db);
    sum = fa * sum + fb * o.sum;
    top = now;
  }
  __device__ __forceinline__ void over_warp() {
#pragma unroll
    for (int x = 16; x; x >>= 1) {
      const Joined o{__shfl_xor_sync(FULL_MASK, top, x), __shfl_xor_sync(FULL_MASK, sum, x), __shfl_xor_sync(FULL_MASK, weighted, x)};
      join(o);
    }
  }
};

// The warp's best keys, one a lane in descending order; the first n of them count.
struct TopList {
  uint64_t mine, last;      // last: the n-th, KEY_EMPTY until there are n
  float above;              // its value
  __device__ __forceinline__ TopList() : mine(KEY_EMPTY), last(KEY_EMPTY), above(-INF) {}
  // Whether an element x may be among the row's n best; `bound`: a value that n elements of the row reach.
  __device__ __forceinline__ bool admits(float x, float bound) const { return x >= bound && (x > above || last == KEY_EMPTY); }
  // A key per lane, KEY_EMPTY for none.
  __device__ __forceinline__ void offer(uint64_t key, int n, int lane) {
    unsigned who = __ballot_sync(FULL_MASK, key > last);
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
    if (last != KEY_EMPTY) above = key_score(last);
  }
};

template <int T, bool TOP>
__global__ void __launch_bounds__(THREADS, 3) score_kernel(const ScoreParams p) {
  using E = Elements<T>;
  __shared__ Joined of_warp[WARPS];
  __shared__ uint64_t lists[SCORE_MAX_SPLIT * SCORE_MAX_TOP], best[SCORE_MAX_TOP];
  __shared__ uint32_t bound_word;
  __shared__ int last_one;
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
  if (TOP && tid == 0) bound_word = score_to_ord(-INF);
  if (TOP) __syncthreads();
  volatile uint32_t* bound_at = &bound_word;
  const uint64_t scale2 = pair_of(p.scale, p.scale);
  Sums sums;
  TopList list;

  auto single = [&](int i, bool there) {             // an element per lane
    const float v = there ? E::one(x, i) : -INF, y = __fmul_rn(v, p.scale), at = sums.raise(y);
    sums.add(pair_of(y, -INF), pair_of(-at, -at));
    if (TOP) list.offer(there && list.admits(v, ord_to_score(*bound_at)) ? make_key(v, i) : KEY_EMPTY, n, lane);
  };
  if (piece == 0 && warp == 0 && head) single(lane, lane < head);

  uint4 next[VECTORS];
  auto load = [&](int base) {
#pragma unroll
    for (int j = 0; j < VECTORS; ++j) {
      const int i = base + j * THREADS + tid;
      next[j] = i < v1 ? ld_stream_16B(xv + i) : make_uint4(E::BANNED, E::BANNED, E::BANNED, E::BANNED);
    }
  };
  load(v0);
  for (int base = v0; base < v1; base += VECTORS * THREADS) {
    uint4 v[VECTORS];
    float most[VECTORS], all = -INF;
#pragma unroll
    for (int j = 0; j < VECTORS; ++j) v[j] = next[j];
    load(base + VECTORS * THREADS);
#pragma unroll
    for (int j = 0; j < VECTORS; ++j) {
      most[j] = E::largest(v[j]);
      all = max_nan(all, most[j]);
    }
    const float at = sums.raise(__fmul_rn(all, p.scale));
    const uint64_t minus2 = pair_of(-at, -at);
#pragma unroll
    for (int j = 0; j < VECTORS; ++j)
#pragma unroll
      for (int i = 0; i < E::PER / 2; ++i) {
        const float2 u = E::pair(v[j], i);
        sums.add(mul_pairs(pair_of(u.x, u.y), scale2), minus2);
      }
    if (TOP) {
      if (base == v0) {
        // the n-th largest of the lanes' maxima: n elements reach it
        const uint32_t o = base + tid < v1 && all == all ? score_to_ord(all) : 0u;
        int rank = 0;
#pragma unroll 8
        for (int i = 0; i < 32; ++i) {
          const uint32_t other = __shfl_sync(FULL_MASK, o, i);
          rank += other > o || (other == o && i < lane);
        }
        if (rank == n - 1 && o) atomicMax(&bound_word, o);
        __syncwarp();
      }
      const float bound = ord_to_score(*bound_at);
      if (__any_sync(FULL_MASK, list.admits(all, bound))) {
#pragma unroll
        for (int j = 0; j < VECTORS; ++j) {
          if (!__any_sync(FULL_MASK, list.admits(most[j], bound))) continue;
          const int i = base + j * THREADS + tid;
          const TopList before = list;               // of lower indices all; among this step's own, the keys decide
#pragma unroll
          for (int e = 0; e < E::PER; ++e) {
            const float2 u = E::pair(v[j], e / 2);
            const float one = e & 1 ? u.y : u.x;
            list.offer(i < v1 && before.admits(one, bound) ? make_key(one, head + i * E::PER + e) : KEY_EMPTY, n, lane);
          }
        }
        if (lane == 0 && list.last != KEY_EMPTY) atomicMax(&bound_word, (uint32_t)(list.last >> 32));
      }
    }
  }
  if (piece == p.split - 1 && warp == 0 && tail) single(p.vocab - tail + lane, lane < tail);

  // the CTA's result
  float sa, sb, wa, wb;
  split_pair(sums.s, &sa, &sb);
  split_pair(sums.w, &wa, &wb);
  Joined mine{sums.top, sa + sb, wa + wb};
  mine.over_warp();
  if (lane == 0) of_warp[warp] = mine;
  if (TOP && lane < n) lists[warp * SCORE_MAX_TOP + lane] = list.mine;
  __syncthreads();
  if (warp != 0) return;
  mine = lane < WARPS ? of_warp[lane] : Joined{-INF, 0.0f, 0.0f};
  mine.over_warp();
  int found = 0;
  if (TOP) {
    found = tournament_in_registers<1>(lists, SCORE_MAX_TOP, WARPS, n, lane, best);
    __syncwarp();
  }
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
    mine.over_warp();
    if (TOP) {
      for (int i = 0; i < p.split; ++i)
        if (lane < n) lists[i * SCORE_MAX_TOP + lane] = __ldcg(&all[i].keys[lane]);
      __syncwarp();
      found = tournament_in_registers<1>(lists, SCORE_MAX_TOP, p.split, n, lane, best);
      __syncwarp();
    }
  }
  // the row's
  const bool none = !(mine.top < INF), banned = mine.top == -INF;
  const float log_sum = banned ? 0.0f : logf(mine.sum), top = banned ? 0.0f : mine.top, nan = __int_as_float(0x7fffffff);
  auto log_prob = [&](float v) { return none ? nan : __fmul_rn(v, p.scale) - top - log_sum; };
  if (lane == 0 && p.entropy) p.entropy[row] = none ? nan : banned ? 0.0f : log_sum - mine.weighted / mine.sum;
  if (lane == 0 && p.targets) {
    const int t = p.targets[row];
    float r = 0.0f;
    if (t >= 0 && t < p.vocab) {
      r = log_prob(E::one(x, t));
    } else if (t != -1) {
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
  // few rows are split until three CTAs an SM have something to do, down to a block per thread
  const int64_t wanted = (3 * sm_count + p.n_rows - 1) / p.n_rows, blocks = (int64_t)p.vocab * (dtype == F32 ? 4 : 2) / (16 * VECTORS * THREADS);
  p.split = (int)(wanted < SCORE_MAX_SPLIT ? wanted : SCORE_MAX_SPLIT);
  if (p.split > blocks) p.split = (int)blocks;
  if (p.split < 1) p.split = 1;
  if (p.split > 1 && p.n_rows * p.split > SCORE_SLOTS) p.split = (int)(SCORE_SLOTS / p.n_rows) > 1 ? (int)(SCORE_SLOTS / p.n_rows) : 1;
  return dtype == F32 ? launch<F32>(p, st) : dtype == F16 ? launch<F16>(p, st) : launch<BF16>(p, st);
}

}  // namespace icc
