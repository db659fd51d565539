// Rotary positions over the paged cache: new tokens' queries and keys turned on their way to attention and into the pages, and
// cached keys moved to other positions.
//
// Pair i of a row at position p turns by the angle p f_i:  (a, b) -> m (a cos - b sin, a sin + b cos).  The frequency is kept as a
// fraction of a turn, f_i / 2 pi modulo 1, in 64 bits after the point: p times it modulo 2^64 is the angle modulo a turn with an
// error of p 2^-65 turns, at any position, by one integer product.  (p f_i in 32-bit floats is 0.008 radians off at p = 131,072.)  The
// upper 32 bits of the product, as a signed number of half turns, go to sincospif, as a float: off by up to 2^-25 half turns.
//
// Nothing is computed to speak of; the bound is the bytes: each row read once and written once.  Sines and cosines are worked out once per
// token and CTA into shared memory, and a thread takes the same place in the rows of TOKENS tokens, so that their loads are
// under way together.  8 prompts of up to 6000 tokens, 32 query and 8 kv heads of 128: 132 us, 6.0 TB/s; keys moved in place: 111 us, 5.2 TB/s.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kernels.h"
#include "kv_mma.cuh"
#include "kv_pages.cuh"
#include "pipeline.cuh"

namespace icc {

namespace {

constexpr int THREADS = 256;
constexpr int PAIRS_MAX = 128;            // pairs of a row of 256 elements
// How a row is cut into the places that threads take.
//   HALVES     pairs (i, i + dim / 2), dim a multiple of 16: two vectors of 8 elements; one beyond dim
//   NEIGHBOURS pairs (2 i, 2 i + 1): one vector of 8 elements
//   ODD_HALVES pairs (i, i + dim / 2) that do not fall on vectors: one vector, its partners exchanged through shared memory within the warp
enum : int { HALVES = 0, NEIGHBOURS = 1, ODD_HALVES = 2 };

struct Places {
  int per_row, turned;                    // places of a row; those that turn
  int in_warp;                            // ODD_HALVES: rows of a warp
  __host__ __device__ Places(int kind, int head_dim, int dim) {
    turned = kind == HALVES ? dim / 16 : (dim + 7) / 8;
    per_row = kind == HALVES ? turned + (head_dim - dim) / 8 : head_dim / 8;
    in_warp = 32 / per_row;
  }
  // Rows that `threads` threads take at a time.
  __host__ __device__ int rows(int kind, int threads) const { return kind == ODD_HALVES ? threads / 32 * in_warp : threads / per_row; }
};

int kind_of(const KvRotary& r) { return r.neighbours ? NEIGHBOURS : r.dim % 16 == 0 ? HALVES : ODD_HALVES; }

// Where pair i's sine and cosine stand: as the threads read them, four at a time, without conflicts.
template <int KIND>
__device__ __forceinline__ int table_at(int i, int turned) {
  return KIND == HALVES ? ((i >> 2) & 1) * turned * 4 + (i >> 3) * 4 + (i & 3) : i;
}
// Sine and cosine of pair i at position pos, times the magnitude.
template <int KIND>
__device__ __forceinline__ void make_entry(const KvRotary& r, int i, long long pos, float magnitude, int turned, float* cosv, float* sinv) {
  float c, s;
  const int turn = (int)(((unsigned long long)pos * r.turn[i]) >> 32);        // in 2^-31 half turns
  sincospif((float)turn * 4.656612873077393e-10f, &s, &c);
  const int at = table_at<KIND>(i, turned);
  cosv[at] = c * magnitude;
  sinv[at] = s * magnitude;
}

// Streaming loads and stores of rows that may be turned in place (so not through the read-only path).
__device__ __forceinline__ uint4 ld_row(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
template <bool F16>
__device__ __forceinline__ float2 unpack2(uint32_t x) {
  if (F16) return __half22float2(*reinterpret_cast<const __half2*>(&x));
  return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}

// A thread's place in a row: one vector, or two.
template <bool F16, int KIND>
struct Piece {
  uint4 a, b;
  __device__ __forceinline__ static int first(int place, int turned, int dim) {
    return KIND == HALVES && place >= turned ? dim + 8 * (place - turned) : 8 * place;
  }
  __device__ __forceinline__ void load(const unsigned char* row, int place, int turned, int dim) {
    a = ld_row(row + 2 * first(place, turned, dim));
    if (KIND == HALVES && place < turned) b = ld_row(row + 2 * (8 * place + dim / 2));
  }
  __device__ __forceinline__ void store(unsigned char* row, int place, int turned, int dim) const {
    *reinterpret_cast<uint4*>(row + 2 * first(place, turned, dim)) = a;
    if (KIND == HALVES && place < turned) *reinterpret_cast<uint4*>(row + 2 * (8 * place + dim / 2)) = b;
  }
  // Computed in fp32 and rounded once.
  __device__ __forceinline__ void turn(int place, int turned, int dim, const float* cosv, const float* sinv) {
    if (KIND == HALVES) {
      uint32_t* x = &a.x;
      uint32_t* y = &b.x;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 c = reinterpret_cast<const float4*>(cosv)[h * turned + place], s = reinterpret_cast<const float4*>(sinv)[h * turned + place];
        const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 u = unpack2<F16>(x[2 * h + j]), w = unpack2<F16>(y[2 * h + j]);
          x[2 * h + j] = pack2<F16>(u.x * cs[2 * j] - w.x * sn[2 * j], u.y * cs[2 * j + 1] - w.y * sn[2 * j + 1]);
          y[2 * h + j] = pack2<F16>(u.x * sn[2 * j] + w.x * cs[2 * j], u.y * sn[2 * j + 1] + w.y * cs[2 * j + 1]);
        }
      }
    } else {
      const float4 c = reinterpret_cast<const float4*>(cosv)[place], s = reinterpret_cast<const float4*>(sinv)[place];
      const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
      uint32_t* x = &a.x;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (8 * place + 2 * j >= dim) break;          // what does not turn is not touched (an infinity times a sine of 0 is a NaN)
        const float2 u = unpack2<F16>(x[j]);
        x[j] = pack2<F16>(u.x * cs[j] - u.y * sn[j], u.x * sn[j] + u.y * cs[j]);
      }
    }
  }
  // ODD_HALVES, the whole warp together: `stage`, 32 vectors of shared memory, holds the warp's rows; `row` is this thread's first one.
  // on: this thread's row turns.
  __device__ __forceinline__ void turn_staged(int place, int per_row, int dim, uint4* stage, int lane, bool on, const float* cosv, const float* sinv) {
    __syncwarp();
    stage[lane] = a;
    __syncwarp();
    if (on) {
      const uint16_t* row = reinterpret_cast<const uint16_t*>(stage + lane - place);
      const int half = dim / 2;
      float out[8];
      const uint32_t* x = &a.x;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 u = unpack2<F16>(x[j]);
        out[2 * j] = u.x;
        out[2 * j + 1] = u.y;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int e = 8 * place + j;
        if (e < dim) {
          const int i = e < half ? e : e - half;
          const uint16_t other = row[e < half ? e + half : e - half];
          const float o = F16 ? __half2float(__ushort_as_half(other)) : __bfloat162float(__ushort_as_bfloat16(other));
          out[j] = e < half ? out[j] * cosv[i] - o * sinv[i] : o * sinv[i] + out[j] * cosv[i];
        }
      }
      uint32_t* y = &a.x;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (8 * place + 2 * j < dim) y[j] = pack2<F16>(out[2 * j], out[2 * j + 1]);
    }
  }
};

// This thread's place, and its row among the rows that the CTA takes at a time; -1: none.
template <int KIND>
__device__ __forceinline__ int my_row(const Places& at, int* place) {
  const int tid = threadIdx.x;
  const int x = KIND == ODD_HALVES ? tid & 31 : tid, r = x / at.per_row;
  *place = x - r * at.per_row;
  if (KIND == ODD_HALVES) return r < at.in_warp ? (tid >> 5) * at.in_warp + r : -1;
  return r < (int)blockDim.x / at.per_row ? r : -1;
}

__global__ void __launch_bounds__(THREADS) kv_rotate_check_kernel(const KvView v, const int* __restrict__ seqs, const int* __restrict__ starts, int n,
                                                                  int64_t n_tokens) {
  grid_dep_launch_dependents();
  grid_dep_wait();
  const int i = blockIdx.x * THREADS + threadIdx.x;
  if (*v.err != KV_OK || i >= n) return;
  if (!WriteSeq(v, seqs, starts, i, n, n_tokens).fine) kv_report(v, KV_INVALID);
}

// TOKENS tokens per CTA, of each of which blockIdx.y takes a part of the rows: queries, keys, values.  As for a write, a bad sequence
// anywhere means that nothing is stored: every CTA looks over all of them, or, of more than THREADS, a kernel before this one has.
template <bool F16, int KIND, int TOKENS, bool CHECKED>
__global__ void __launch_bounds__(THREADS) kv_rotate_kernel(const __grid_constant__ KvRotateParams p) {
  __shared__ float cosv[TOKENS][PAIRS_MAX], sinv[TOKENS][PAIRS_MAX];
  __shared__ unsigned char* place_of[TOKENS];      // of the key of head 0
  __shared__ int row_of[TOKENS], pos_of[TOKENS];
  __shared__ uint4 stage[KIND == ODD_HALVES ? THREADS : 1];
  const KvView& v = p.v;
  grid_dep_launch_dependents();
  grid_dep_wait();
  const int tid = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
  if (p.seqs) {
    // (other CTAs may report a bad table entry meanwhile: whether this one goes on is its threads' common decision)
    bool fine = *v.err == KV_OK;
    if (CHECKED) {
      const int64_t t = t0 + tid;
      if (fine && tid < TOKENS && t < p.n_tokens) {
        const WriteSeq seq(v, p.seqs, p.starts, p.starts ? owner_of(p.starts, p.n, (int)t) : (int)t, p.n, p.n_tokens);
        row_of[tid] = seq.s;
        pos_of[tid] = (int)(seq.length - seq.end + t);
      }
    } else if (tid < p.n) {
      const WriteSeq seq(v, p.seqs, p.starts, tid, p.n, p.n_tokens);
      fine &= seq.fine;
      if (fine)
        for (int64_t t = max(seq.begin, t0); t < min(seq.end, t0 + TOKENS); ++t) {
          row_of[t - t0] = seq.s;
          pos_of[t - t0] = (int)(seq.length - seq.end + t);
        }
    }
    if (!__syncthreads_and(fine)) {
      if (tid == 0) kv_report(v, KV_INVALID);
      return;
    }
    if (p.k && tid < TOKENS) place_of[tid] = t0 + tid < p.n_tokens ? token_place(v, p.layer, row_of[tid], pos_of[tid]) : nullptr;
  }
  const Places at(KIND, v.head_dim, p.r.dim);
  const int entries = p.r.dim / 2;
  for (int u = tid; u < TOKENS * entries; u += blockDim.x) {
    const int x = u / entries;
    if (t0 + x < p.n_tokens) {
      const long long pos = p.positions ? p.positions[t0 + x] : pos_of[x];
      make_entry<KIND>(p.r, u - x * entries, p.inverse ? -pos : pos, p.r.magnitude, at.turned, cosv[x], sinv[x]);
    }
  }
  __syncthreads();
  int place;
  const int mine = my_row<KIND>(at, &place);
  const int rows = p.n_heads + (p.k ? 2 * v.n_kv_heads : 0);
  const int per = (rows + gridDim.y - 1) / gridDim.y, end = min(rows, per * ((int)blockIdx.y + 1));
  const int step = at.rows(KIND, blockDim.x);
  const size_t block = ((size_t)v.head_dim * 2) << v.page_shift;      // bytes of one head's keys in a page
  const int left = (int)min((int64_t)TOKENS, p.n_tokens - t0);
  for (int r0 = per * blockIdx.y; r0 < end; r0 += step) {
    const int r = r0 + mine;
    const bool here = mine >= 0 && r < end;
    const bool query = r < p.n_heads, key = !query && r < p.n_heads + v.n_kv_heads;
    const int h = query ? r : key ? r - p.n_heads : r - p.n_heads - v.n_kv_heads;
    const unsigned char* from = query ? p.q + (t0 * p.q_token_stride + h * p.q_head_stride) * 2
                                      : (key ? p.k : p.val) + (t0 * p.kv_token_stride + h * p.kv_head_stride) * 2;
    const int64_t from_step = (query ? p.q_token_stride : p.kv_token_stride) * 2;
    Piece<F16, KIND> w[TOKENS];
    unsigned char* to[TOKENS];
#pragma unroll
    for (int x = 0; x < TOKENS; ++x) {
      to[x] = nullptr;
      if (here && x < left) {
        if (query) to[x] = p.out + ((t0 + x) * p.out_token_stride + h * p.out_head_stride) * 2;
        else if (place_of[x]) to[x] = place_of[x] + (size_t)(r - p.n_heads) * block;
      }
      if (to[x]) w[x].load(from + x * from_step, place, at.turned, p.r.dim);
    }
#pragma unroll
    for (int x = 0; x < TOKENS; ++x) {
      const bool turns = to[x] && (query || key) && place < at.turned;
      if (KIND == ODD_HALVES) w[x].turn_staged(place, at.per_row, p.r.dim, stage + (tid & ~31), tid & 31, turns, cosv[x], sinv[x]);
      else if (turns) w[x].turn(place, at.turned, p.r.dim, cosv[x], sinv[x]);
      if (to[x]) w[x].store(to[x], place, at.turned, p.r.dim);
    }
  }
}

// ---------------------------------------------------------------- shift
// Two or three steps: the plan (sequences, and where each one's pages begin in the list of all), by one CTA; that all pages are there and
// held once, spread over CTAs unless there are few; and the turning.  The last is left out if something was wrong.
constexpr int PLAN_THREADS = 1024;
constexpr int SMALL_SHIFT = 8192;         // table entries at most that the plan's CTA looks over itself

__device__ __forceinline__ bool entry_fine(const KvView& v, const int* seqs, int i, int col) {
  const int page = v.tables[(size_t)seqs[i] * v.max_pages + col];
  if ((unsigned)page < (unsigned)v.n_pages && v.refs[page] == 1) return true;
  kv_report(v, KV_INVALID);
  return false;
}

__global__ void __launch_bounds__(PLAN_THREADS) kv_shift_plan_kernel(const KvView v, const int* __restrict__ seqs, int n, int entries_too) {
  __shared__ unsigned sums[33];
  __shared__ int bad;
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (threadIdx.x == 0) {
    bad = 0;
    v.meta[0] = 0;
  }
  __syncthreads();
  if (*v.err != KV_OK) return;
  unsigned entries = 0;
  for (int i0 = 0; i0 < n; i0 += PLAN_THREADS) {
    const int i = i0 + threadIdx.x;
    unsigned mine = 0;
    if (i < n) {
      const int s = seqs[i];
      if (s < 0 || s >= v.max_seqs || atomicExch(&v.mark[s], 1) != 0 || !length_fits(v, v.lengths[s])) bad = 1;
      else mine = kv_pages_of(v.lengths[s], v.page_shift);
    }
    unsigned total;
    const unsigned before = block_scan(mine, sums, &total);
    if (i < n) v.begin[i] = (int)(entries + before);
    entries += total;       // (no sequence twice: at most the tables' entries, fewer than 2^31)
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += PLAN_THREADS) {
    const int s = seqs[i];
    if (s >= 0 && s < v.max_seqs) v.mark[s] = 0;
  }
  if (bad) {
    if (threadIdx.x == 0) kv_report(v, KV_INVALID);
    return;
  }
  bool fine = true;
  if (entries_too)
    for (int u = threadIdx.x; u < (int)entries; u += PLAN_THREADS) {
      const int i = owner_of(v.begin, n, u);
      fine &= entry_fine(v, seqs, i, u - v.begin[i]);
    }
  if (!__syncthreads_and(fine)) return;
  if (threadIdx.x == 0) {
    v.meta[0] = 1;
    v.meta[1] = (int)entries;
  }
}

__global__ void __launch_bounds__(THREADS) kv_shift_check_kernel(const KvView v, const int* __restrict__ seqs, int n) {
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (v.meta[0] == 0) return;
  const int entries = v.meta[1];
  for (int u = blockIdx.x * THREADS + threadIdx.x; u < entries; u += gridDim.x * THREADS) {
    const int i = owner_of(v.begin, n, u);
    entry_fine(v, seqs, i, u - v.begin[i]);
  }
}

// a / b, both positive: 64-bit division is slow.
__device__ __forceinline__ long long divided(long long a, int b) { return a >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b); }

// A unit of work is the keys of `layers` layers in one page.  A CTA's units are next to each other, so that it seldom needs another
// sequence's angles, and it works these out and looks up the next one's page while the rows of one are on their way.
constexpr int ROWS_AT_ONCE = 4;
template <bool F16, int KIND>
__global__ void __launch_bounds__(THREADS) kv_shift_kernel(const KvView v, const __grid_constant__ KvRotary rot, const int* __restrict__ seqs,
                                                           const int* __restrict__ by, int n, int layers) {
  __shared__ float cosv[PAIRS_MAX], sinv[PAIRS_MAX];
  __shared__ uint4 stage[KIND == ODD_HALVES ? THREADS : 1];
  grid_dep_launch_dependents();
  grid_dep_wait();
  if (v.meta[0] == 0 || *v.err != KV_OK) return;
  const int tid = threadIdx.x;
  const Places at(KIND, v.head_dim, rot.dim);
  const int table = rot.dim / 2, groups = (v.n_layers + layers - 1) / layers;
  const int of_layer = v.n_kv_heads << v.page_shift, slots = (1 << v.page_shift) - 1;
  int place;
  const int mine = my_row<KIND>(at, &place), step = at.rows(KIND, THREADS);
  const long long units = (long long)v.meta[1] * groups, per = divided(units + gridDim.x - 1, (int)gridDim.x),
                  u0 = per * blockIdx.x, u1 = min(units, u0 + per);
  struct Unit {
    int i, l0, tokens;
    unsigned char* page;
  } next;
  auto find = [&](long long u) {
    const int e = (int)divided(u, groups);
    next.l0 = (int)(u - (long long)e * groups) * layers;
    next.i = owner_of(v.begin, n, e);
    const int col = e - v.begin[next.i], s = seqs[next.i];
    next.tokens = min(v.lengths[s] - (col << v.page_shift), slots + 1);
    next.page = v.pool + (size_t)v.tables[(size_t)s * v.max_pages + col] * v.page_bytes;
  };
  if (u0 < u1) find(u0);
  int known = -1;                          // the sequence whose angles are in shared memory
  for (long long u = u0; u < u1; ++u) {
    const int i = next.i, l0 = next.l0, tokens = next.tokens;
    unsigned char* page = next.page;
    const int rows = min(layers, v.n_layers - l0) * of_layer;
    for (int r0 = 0; r0 < rows; r0 += ROWS_AT_ONCE * step) {
      Piece<F16, KIND> w[ROWS_AT_ONCE];
      unsigned char* to[ROWS_AT_ONCE];
#pragma unroll
      for (int x = 0; x < ROWS_AT_ONCE; ++x) {
        const int r = r0 + x * step + mine;
        to[x] = nullptr;
        if (mine >= 0 && r < rows && (r & slots) < tokens && place < at.turned) {
          const int l = r / of_layer;      // keys and values of a layer lie behind each other
          to[x] = page + ((size_t)(l0 + l) * of_layer + r) * v.head_dim * 2 + (size_t)l0 * of_layer * v.head_dim * 2;
          w[x].load(to[x], place, at.turned, rot.dim);
        }
      }
      if (r0 == 0) {
        if (i != known) {
          known = i;
          __syncthreads();
          const long long d = by[i];
          for (int x = tid; x < table; x += THREADS) make_entry<KIND>(rot, x, d, 1.0f, at.turned, cosv, sinv);
          __syncthreads();
        }
        if (u + 1 < u1) find(u + 1);
      }
#pragma unroll
      for (int x = 0; x < ROWS_AT_ONCE; ++x) {
        if (KIND == ODD_HALVES) w[x].turn_staged(place, at.per_row, rot.dim, stage + (tid & ~31), tid & 31, to[x] != nullptr, cosv, sinv);
        else if (to[x]) w[x].turn(place, at.turned, rot.dim, cosv, sinv);
        if (to[x]) w[x].store(to[x], place, at.turned, rot.dim);
      }
    }
  }
}

template <bool F16, int KIND>
cudaError_t rotate_launch(const KvRotateParams& p, int sm_count, int* launches, cudaStream_t st) {
  const bool checked = p.seqs && p.n > THREADS;
  *launches = checked ? 2 : 1;
  if (checked) {
    const cudaError_t e = launch_overlapped(kv_rotate_check_kernel, dim3((unsigned)((p.n + THREADS - 1) / THREADS)), dim3(THREADS), 0, st, 1, p.v, p.seqs,
                                            p.starts, p.n, p.n_tokens);
    if (e != cudaSuccess) return e;
  }
  const bool single = p.n_tokens <= 4 * sm_count;
  const int tokens = single ? 1 : 4;
  const int64_t ctas = (p.n_tokens + tokens - 1) / tokens;
  // threads: as many rows at a time as leave no thread idle in the last round
  const Places at(KIND, p.v.head_dim, p.r.dim);
  const int rows = p.n_heads + (p.k ? 2 * p.v.n_kv_heads : 0), most = at.rows(KIND, THREADS);
  // few tokens: their rows are spread over CTAs too
  int split = (rows + most - 1) / most;
  if (ctas * split > 2 * sm_count) split = (int)(2 * sm_count / ctas);
  if (split < 1) split = 1;
  const int per = (rows + split - 1) / split, rounds = (per + most - 1) / most, at_once = (per + rounds - 1) / rounds;
  int threads = KIND == ODD_HALVES ? (at_once + at.in_warp - 1) / at.in_warp * 32 : (at_once * at.per_row + 31) / 32 * 32;
  if (threads < 64 || (p.seqs && threads < THREADS && !checked && p.n > threads)) threads = THREADS;      // (a thread looks over a sequence)
  auto* kernel = single ? (checked ? kv_rotate_kernel<F16, KIND, 1, true> : kv_rotate_kernel<F16, KIND, 1, false>)
                        : (checked ? kv_rotate_kernel<F16, KIND, 4, true> : kv_rotate_kernel<F16, KIND, 4, false>);
  return launch_overlapped(kernel, dim3((unsigned)ctas, (unsigned)split), dim3((unsigned)threads), 0, st, 1, p);
}

template <bool F16, int KIND>
cudaError_t shift_launch(const KvView& v, const KvRotary& rot, const int* seqs, const int* by, int n, int sm_count, cudaStream_t st) {
  const int of_layer = v.n_kv_heads << v.page_shift;
  int layers = 128 / of_layer;             // about 128 rows to a unit
  if (layers < 1) layers = 1;
  if (layers > v.n_layers) layers = v.n_layers;
  // (8 CTAs an SM, in turns: 48 sequences of up to 701 tokens, 8 layers of 8 heads of 128: 111 us, 5.2 TB/s; 4 an SM: 124)
  const int64_t units = (int64_t)n * v.max_pages * ((v.n_layers + layers - 1) / layers), ctas = units < 8 * sm_count ? units : 8 * sm_count;
  return launch_overlapped(kv_shift_kernel<F16, KIND>, dim3((unsigned)ctas), dim3(THREADS), 0, st, 1, v, rot, seqs, by, n, layers);
}

}  // namespace

cudaError_t kv_rotate_launch(const KvRotateParams& p, bool f16, int sm_count, int* launches, cudaStream_t st) {
  const int kind = kind_of(p.r);
  auto* go = kind == HALVES ? (f16 ? rotate_launch<true, HALVES> : rotate_launch<false, HALVES>)
             : kind == NEIGHBOURS ? (f16 ? rotate_launch<true, NEIGHBOURS> : rotate_launch<false, NEIGHBOURS>)
                                  : (f16 ? rotate_launch<true, ODD_HALVES> : rotate_launch<false, ODD_HALVES>);
  return go(p, sm_count, launches, st);
}

cudaError_t kv_shift_launch(const KvView& v, const KvRotary& rot, const int* seqs, const int* by, int n, bool f16, int sm_count, int* launches,
                            cudaStream_t st) {
  const bool small = (long long)n * v.max_pages <= SMALL_SHIFT;
  *launches = small ? 2 : 3;
  cudaError_t e = launch_overlapped(kv_shift_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, 1, v, seqs, n, (int)small);
  if (e == cudaSuccess && !small) e = launch_overlapped(kv_shift_check_kernel, dim3((unsigned)(2 * sm_count)), dim3(THREADS), 0, st, 1, v, seqs, n);
  if (e != cudaSuccess) return e;
  const int kind = kind_of(rot);
  auto* go = kind == HALVES ? (f16 ? shift_launch<true, HALVES> : shift_launch<false, HALVES>)
             : kind == NEIGHBOURS ? (f16 ? shift_launch<true, NEIGHBOURS> : shift_launch<false, NEIGHBOURS>)
                                  : (f16 ? shift_launch<true, ODD_HALVES> : shift_launch<false, ODD_HALVES>);
  return go(v, rot, seqs, by, n, sm_count, st);
}

}  // namespace icc
