// Linear attention with a decay per head for many tokens: chunks of 64, on the tensor cores (tcgen05).
//
// With the state S in front of a chunk of n tokens (rows t, s = 0 .. n - 1), l = e^(-rate):
//     out_t = scale ( sum over s <= t of l^(t-s) (q_t . k_s) v_s  +  l^(t+1) q_t S )
//     S'    = l^n S + sum over s of k_s (l^(n-1-s) v_s)^T
// A CTA walks over the chunks of an item (sequence, head, 128 value columns).  S^T is held in fp32 in registers, a thread per value
// column.  Everything with the state's shape is transposed, so that what depends on the value column is a thread's own and all
// operands are taken as they lie:
//     P    = Q K^T       tokens x tokens     Q, K from shared memory (half of the 128 lanes are of no use)
//     O1^T = V^T P^T     values x tokens     V from shared memory; P weighted, rounded to 16 bits, by way of shared memory
//     O2^T = S^T Q^T     values x tokens     S^T rounded to 16 bits, in tensor memory
//     U^T  = W^T K       values x keys       W = l^(n-1-s) v_s in fp32, split into two or three 16-bit numbers, in tensor memory
// The scores and the copy of S that meets the queries are rounded to 16 bits once, as wide as the inputs are; the state itself is not: W's parts
// hold 24 (bf16) and 22 (fp16) bits.  U is not summed up in tensor memory over the chunks: a tensor core's fp32 sums are cut off, not
// rounded, and over 3,000 tokens of a slow decay the state came out 2e-6 too small.  Now a chunk's parts are summed from the least on, and
// the chunks by rounded additions: 2e-7.
// fp16 has little range, so there P is scaled by a power of two per token, and W and the copy of S per value column.  A column's
// factor is its thread's own, a token's goes through shared memory.
//
//   warps 0-3    results: out = scale (O1 + l^(t+1) O2), rounded and stored
//   warps 4-7    the state: loaded, copied for the queries, S <- l^n S + U, and stored in the end
//   warps 8-11   W
//   warps 12-13  P; warp 12 also loads K, V and Q into a ring of stages: boxes of tensor maps (where the strides allow none, 16-byte copies)
//   warp 14      issues the products U(c), O2(c)
//   warp 15      issues P(c + 1), O1(c)
// Two warps issue because a product takes one about 100 cycles, more than the tensor cores.  The rows of a sequence's last chunk that
// lie behind its end (another sequence's) are set to zeros in shared memory, by the warps of W.
// Bound: HBM, 1 KB a token and head of 128 x 128; a chunk is 64 KB, 2,750 cycles of an SM's share.  The products take 1,600, a chunk with all that waits
// for them 3,800: 8 prompts of 2,800 tokens, 32 heads of 128 x 128, in bf16: 219 us, 3.3 TB/s.  Loops are rolled where registers allow: the roles'
// code has to stay in the instruction caches, and warps still wait for instructions more than for any unit.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "kernels.h"
#include "kv_mma.cuh"
#include "state_check.cuh"
#include "state_schedule.cuh"
#include "tensor_core.cuh"

namespace icc {

namespace {

constexpr int C = STATE_CHUNK;
constexpr int THREADS = 512;
constexpr int MAX_STAGES = 6;
constexpr int OUT_BYTES = 4 * 32 * 64;
constexpr int ROW_CHUNK = C * 128;                    // bytes of 64 tokens' 64 elements
enum : int { W_OUT = 0, W_STATE = 4, W_VALUES = 8, W_SCORES = 12, W_STATE_PRODUCTS = 14, W_RESULT_PRODUCTS = 15 };
// Registers of the four warpgroups' threads; they are launched with 128.
constexpr int OUT_REGS = 96, STATE_REGS = 208, VALUE_REGS = 96, OTHER_REGS = 112;
static_assert(OUT_REGS + STATE_REGS + VALUE_REGS + OTHER_REGS <= 4 * 128, "what some have more, others have less");
// Columns of tensor memory.
constexpr uint32_t T_P = 0, T_O1 = 64, T_O2 = 128, T_COPY = 192, T_U = 256, T_W = 384;

template <bool F16>
constexpr int PARTS = F16 ? 2 : 3;                    // 16-bit numbers that hold one of W

// A head's powers of l.  What a chunk leaves of a state, l^64, rounded would be off the same way every time (1e-5 after 900 chunks of a slow decay), so the
// chunks take turns with the two floats next to it: what TURNS of them leave is right to half a step of one.
constexpr int FALL = C, TURN = 2 * C + 4, TURNS = 32;
struct Fall {
  float at[TURN + TURNS];                             // l^j at FALL + j, j = 0 .. 64, with zeros in front; the turns at TURN
};

struct Tail {
  StateLine line;
  union {                                             // (the check comes first)
    int starts[2 * STATE_BATCH];                      // of the call's tokens, and behind each where it ends
    uint32_t seen[STATE_MAX_SEQS / 32];
  };
  StatePlan plan;
  // published states that the last piece's is put together from: whose, and what is left of them after the chunks between
  int slots, slot_cta[KV_MAX_CTAS];
  float slot_weight[KV_MAX_CTAS];
  Fall fall[2];                                       // of a piece and the next one
  uint64_t fall_ready[2], fall_free[2];
  alignas(16) float token_scale[2][C];                      // fp16: what P's row was divided by, by the chunk's parity
  float lane_scale[2][128];                           // fp16: what W's column was multiplied by
  float copy_scale[2][128];                           // fp16: what the copy of S has to be multiplied by
  uint64_t full[MAX_STAGES], empty[MAX_STAGES];
  uint64_t w_ready[2], w_free[2];                     // of a chunk's halves
  uint64_t clean[MAX_STAGES];                         // of a stage with a sequence's last chunk: rows behind the end are zeros
  uint64_t p_full, p_ready, copy_ready, u_full, u_free, o1_full, o2_full, o_free, drain[2];
  uint64_t slots_read[MAX_STAGES];
  uint32_t tmem_base;
  int abort_flag, holds;
};

__device__ __forceinline__ float ld_shared(uint32_t addr) {
  float x;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(addr));
  return x;
}
// The power of two that brings the largest magnitude m (>= 0, finite) into [2^13, 2^14); 1 for 0.
__device__ __forceinline__ float lift_of(float m, int most) {
  if (m == 0.0f) return 1.0f;
  const int e = 13 - ((int)(__float_as_uint(m) >> 23) - 127);
  return __uint_as_float((uint32_t)(min(max(e, -100), most) + 127) << 23);
}
__device__ __forceinline__ float reciprocal_of_power(float p) { return __uint_as_float((254u << 23) - __float_as_uint(p)); }

// Where a role is in the ring of stages.
struct Ring {
  int stage, n_stages;
  uint32_t phase;
  __device__ __forceinline__ explicit Ring(int n) : stage(0), n_stages(n), phase(0) {}
  __device__ __forceinline__ void advance() {
    if (++stage == n_stages) {
      stage = 0;
      phase ^= 1u;
    }
  }
};

// A wait of a whole warp, in few instructions (the roles' code together has to stay in the instruction cache).  It ends after WAIT_LIMIT_CYCLES, about a
// second, which 32 bits of the clock count.
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  const uint32_t t0 = (uint32_t)clock();
#pragma unroll 1
  for (;;) {
    if (__all_sync(FULL_MASK, mbar_try_wait(bar, parity))) return true;
    if (__any_sync(FULL_MASK, *abort_flag != 0 || (uint32_t)clock() - t0 > (uint32_t)WAIT_LIMIT_CYCLES)) break;
  }
  *abort_flag = 1;
  return false;
}

template <bool F16>
__device__ __forceinline__ float2 pair16(uint32_t x) {
  return F16 ? __half22float2(*reinterpret_cast<const __half2*>(&x)) : make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}

// e^(-rate * steps): the exponent in 64 bits, as it would be rounded to 1e-6 in 32, and what is left of it below a power of two in 32.
__device__ __noinline__ float fall_of(float rate, int steps) {
  if (steps == 0) return 1.0f;                       // (also of an infinite rate)
  const double y = fmax(-(double)rate * steps * 1.4426950408889634, -200.0), whole = rint(y);
  return ldexpf(exp2f((float)(y - whole)), (int)whole);
}

// What chunk i, modulo TURNS, leaves of a state.
__device__ __noinline__ float turn_of(float rate, int i) {
  const double whole = exp(-(double)rate * C);
  const float near = (float)whole, rest = (float)(whole - (double)near);
  const float other = __uint_as_float(__float_as_uint(near) + (rest < 0.0f ? -1 : 1)), share = rest / (other - near);      // share: 0 .. 1 / 2
  return rintf((i + 1) * share) != rintf(i * share) ? other : near;
}

template <bool F16, int DK, int DV>
struct Sizes {
  static constexpr int K_BYTES = DK * ROW_CHUNK, V_BYTES = DV * ROW_CHUNK;
  static constexpr int STAGE = 2 * K_BYTES + V_BYTES;                  // Q, K, V
  static constexpr int SLOT_HALF = 64 * DV * 64;                       // floats: 64 key dimensions of a published state
  static constexpr int LANE_WARPS = 2 * DV;                            // of a role that has a thread per value column
};

template <bool F16, int DK, int DV>
__global__ void __launch_bounds__(THREADS, 1) state_chunk_kernel(const __grid_constant__ StateAttendParams p, const __grid_constant__ StateMaps maps,
                                                                 int n_stages) {
  using X = Sizes<F16, DK, DV>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* ring = smem_raw + (-smem_u32(smem_raw) & 1023u);      // (an offset: the compiler still knows whose memory this is)
  unsigned char* p_smem = ring + n_stages * X::STAGE;                  // P: 64 tokens of 128 bytes
  unsigned char* out_smem = p_smem + ROW_CHUNK;                        // results on their way out: 32 tokens of 32 columns a warp
  Tail* t = reinterpret_cast<Tail*>(out_smem + OUT_BYTES);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const StateView& v = p.v;
  if (p.least) {                                     // as a rule there is no sequence for this launch
    grid_dep_wait();
    bool some = false;
    for (int i = tid; i < p.n; i += THREADS) some |= p.ends[i] - p.starts[i] > p.least;
    if (!__syncthreads_or(some)) return;
  }
  if (tid == 0) {
    for (int s = 0; s < n_stages; ++s) {
      mbar_init(&t->full[s], 32);
      mbar_init(&t->empty[s], 2);                    // the two warps that issue products
      mbar_init(&t->slots_read[s], 2 * X::LANE_WARPS);
      mbar_init(&t->clean[s], X::LANE_WARPS);
    }
    mbar_init(&t->p_full, 1);
    mbar_init(&t->p_ready, 2);
    for (int h = 0; h < 2; ++h) {
      mbar_init(&t->w_ready[h], X::LANE_WARPS);
      mbar_init(&t->w_free[h], 1);
    }
    mbar_init(&t->copy_ready, X::LANE_WARPS);
    mbar_init(&t->u_full, 1);
    mbar_init(&t->u_free, X::LANE_WARPS);
    mbar_init(&t->o2_full, 1);
    mbar_init(&t->o1_full, 1);
    mbar_init(&t->o_free, X::LANE_WARPS);
    for (int h = 0; h < 2; ++h) {
      mbar_init(&t->fall_ready[h], 1);
      mbar_init(&t->fall_free[h], 3 * X::LANE_WARPS + 2);
    }
    mbar_init(&t->drain[0], 1);
    mbar_init(&t->drain[1], 1);
    t->abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == W_STATE_PRODUCTS) tmem_alloc(&t->tmem_base, 512);
  grid_dep_launch_dependents();
  grid_dep_wait();
  const bool holds = state_call_holds(p, t->seen);
  if (holds && warp == 0) {
    // chunks before each sequence
    int sum = 0, longest = 0;
    for (int i0 = 0; i0 < p.n; i0 += 32) {
      const int i = i0 + lane;
      const int from = i < p.n ? p.starts[i] : 0, to = i < p.n ? p.ends[i] : 0;
      if (i < p.n) {
        t->starts[2 * i] = from;
        t->starts[2 * i + 1] = to;
      }
      const int mine = to - from > p.least ? (int)(((unsigned)(to - from) + C - 1) / C) : 0;
      longest = max(longest, mine);
      int inc = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(FULL_MASK, inc, d);
        if (lane >= d) inc += y;
      }
      if (i < p.n) t->line.before[i + 1] = sum + inc;
      sum += __shfl_sync(FULL_MASK, inc, 31);
    }
    longest = __reduce_max_sync(FULL_MASK, longest);
    if (lane == 0) {
      t->line.before[0] = 0;
      t->line.n = p.n;
      t->line.per_chunk = p.n_items;
      t->line.parts = gridDim.x;
      t->line.set_per(longest);
      t->plan.make(t->line, blockIdx.x);
    }
    __syncwarp();
    int slots = 0;
    if (t->plan.last.c1)
      for (int j0 = t->plan.slot_first; j0 < (int)blockIdx.x; j0 += 32) {
        const int j = j0 + lane;
        const int to = j < (int)blockIdx.x ? t->line.cut(j + 1) : 0;
        const bool some = j < (int)blockIdx.x && t->line.cut(j) < to;
        const unsigned who = __ballot_sync(FULL_MASK, some);
        if (some) {
          const int at = slots + __popc(who & ((1u << lane) - 1u));
          t->slot_cta[at] = j;
          t->slot_weight[at] = fall_of(p.rates[(t->plan.last.item + p.first_item) / p.slices], C * (t->plan.begin - to));
        }
        slots += __popc(who);
      }
    if (lane == 0) t->slots = slots;
  } else if (!holds && tid == 0) {
    // nothing to do: a line without chunks
    t->line.before[0] = t->line.before[1] = 0;
    t->line.n = t->line.per_chunk = 1;
    t->line.parts = gridDim.x;
    t->line.set_per(0);
    t->plan.make(t->line, blockIdx.x);
    t->slots = 0;
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = t->tmem_base, lane_base = (uint32_t)((warp & 3) * 32) << 16;
  const uint32_t on = lane == 0;
  volatile int* abort_flag = &t->abort_flag;
  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (ok) ok = wait_for(bar, parity, abort_flag);
  };
  Ring at(n_stages);                                  // of the roles that follow the stages
  StateWalk walk(&t->line, &t->plan);
  StatePiece piece;
  // (one slice or two: value_dim is 256 at most)
  auto head_of = [&](const StatePiece& x) { return (x.item + p.first_item) >> (p.slices - 1); };
  auto slice_of = [&](const StatePiece& x) { return (x.item + p.first_item) & (p.slices - 1); };
  auto first_token = [&](const StatePiece& x) { return t->starts[2 * x.i]; };
  auto tokens_of = [&](const StatePiece& x) { return t->starts[2 * x.i + 1] - t->starts[2 * x.i]; };
  // Stages in front of a piece's chunks: the state that it begins with, or the published ones that this is put together from, 64 key dimensions each.
  auto states_of = [&](const StatePiece& x) { return x.from == StatePiece::PUBLISHED ? t->slots : x.from == StatePiece::STORED ? 1 : 0; };
  auto slots_of = [&](const StatePiece& x) { return DK * states_of(x); };
  auto tell = [&](uint64_t* bar) {
    __syncwarp();
    arrive_one(bar, on);
  };

  // The powers of its head's decay are worked out by warp 13, a piece ahead.
  int n_pieces = 0;
  auto next_piece = [&]() {
    if (!ok || !walk.next(&piece)) return false;
    wait(&t->fall_ready[n_pieces & 1], (n_pieces >> 1) & 1);
    return ok;
  };
  auto end_piece = [&]() {
    tell(&t->fall_free[n_pieces & 1]);
    ++n_pieces;
  };
  // products
  const int key_steps = (v.key_dim + 15) / 16;
  constexpr uint32_t CH = ROW_CHUNK >> 4, K_AT = X::K_BYTES >> 4, V_AT = 2 * X::K_BYTES >> 4;
  // Nothing issued is still running when tensor memory is released.
  auto drain = [&](uint64_t* bar) {
    commit_products(bar, on);
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, 0) && clock64() - t0 < WAIT_LIMIT_CYCLES) {
    }
  };

  // (one place for the warps of a warpgroup: the instruction is theirs together)
  if (warp >= W_SCORES) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
  if (warp == W_STATE_PRODUCTS) {
    // ------------------------------------------------------------ U, O2
    const uint32_t id_o2 = idesc(F16, C, false), id_u = idesc(F16, key_steps * 16, true);
    const uint64_t rows_desc = umma_desc_k_major_sw128(smem_u32(ring)), columns_desc = desc_mn_major_sw128(smem_u32(ring), ROW_CHUNK);
    uint32_t ph = 0, out_ph = 0, slots_ph = 0;        // of the barriers that turn once a chunk, and once a chunk with results
    while (ok && walk.next(&piece)) {
      for (int j = slots_of(piece); j > 0 && ok; --j) {      // stages that hold published states
        wait(&t->slots_read[at.stage], (slots_ph >> at.stage) & 1u);      // a stage's barrier turns at each such use
        slots_ph ^= 1u << at.stage;
        arrive_one(&t->empty[at.stage], on);
        at.advance();
      }
      for (int c = piece.c0; c < piece.c1 && ok; ++c) {
        const uint32_t stage = at.stage * (X::STAGE >> 4);
        wait(&t->full[at.stage], at.phase);
        wait(&t->u_free, ph ^ 1u);
        // U by halves of the chunk, so that W's next is made while the other half is used; of each the least parts first: what is cut off of a
        // sum is a part of what is there
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          wait(&t->w_ready[h], ph);
          if (!ok) break;
          if (h == 0 && !maps.there) fence_async_shared();         // the copies were ordinary writes
          tc_fence_after_sync();
          const uint64_t b = columns_desc + stage + K_AT + h * 256;
          const uint32_t a = tmem + T_W + h * 16;
#pragma unroll
          for (int w = PARTS<F16> - 1; w >= 0; --w)
#pragma unroll
            for (int k = 0; k < 2; ++k)               // 16 tokens further: 8 columns of W, 2048 bytes of K
              product_tmem(tmem + T_U, a + w * (C / 2) + k * 8, b + k * 128, id_u, h != 0 || w + 1 < PARTS<F16> || k != 0, on);
          commit_products(&t->w_free[h], on);
        }
        if (!ok) break;
        commit_products(&t->u_full, on);
        ph ^= 1u;
        if (!piece.sum_only) {
          wait(&t->copy_ready, out_ph);
          wait(&t->o_free, out_ph ^ 1u);
          out_ph ^= 1u;
          if (!ok) break;
          tc_fence_after_sync();
#pragma unroll
          for (int k = 0; k < DK * 4; ++k)
            product_tmem(tmem + T_O2, tmem + T_COPY + k * 8, rows_desc + stage + (k >> 2) * CH + (k & 3) * 2, id_o2, k != 0, k < key_steps ? on : 0u);
          commit_products(&t->o2_full, on);
        }
        commit_products(&t->empty[at.stage], on);
        at.advance();
      }
    }
    drain(&t->drain[0]);
  } else if (warp == W_RESULT_PRODUCTS) {
    // ------------------------------------------------------------ P, O1
    const uint32_t id_p = idesc(F16, C, false), id_o1 = idesc(F16, C, false, true);
    const uint64_t rows_desc = umma_desc_k_major_sw128(smem_u32(ring)), p_desc = umma_desc_k_major_sw128(smem_u32(p_smem)),
                   columns_desc = desc_mn_major_sw128(smem_u32(ring), ROW_CHUNK);
    uint32_t ph = 0, clean_ph = 0;
    int before = -1;                                  // the stage of the chunk whose P is under way
    // O1 of that chunk, as soon as its P is ready; and with that there is room for the next one's
    auto ready = [&]() {
      wait(&t->p_ready, ph);
      wait(&t->o_free, ph ^ 1u);
      ph ^= 1u;
      tc_fence_after_sync();
    };
    auto values = [&]() {
      const uint64_t a = columns_desc + before * (X::STAGE >> 4) + V_AT;
#pragma unroll
      for (int k = 0; k < C / 16; ++k) product_smem(tmem + T_O1, a + k * 128, p_desc + k * 2, id_o1, k != 0, on);
      commit_products(&t->o1_full, on);
      commit_products(&t->empty[before], on);
      before = -1;
    };
    while (ok && walk.next(&piece)) {
      const int count = tokens_of(piece);
      // (of stages that are not for this warp it says so when they are full, or it could lose count of the rounds)
      for (int j = slots_of(piece) + (piece.sum_only ? piece.c1 - piece.c0 : 0); j > 0 && ok; --j) {
        if (before >= 0) {
          ready();
          if (ok) values();
        }
        wait(&t->full[at.stage], at.phase);
        arrive_one(&t->empty[at.stage], on);
        at.advance();
      }
      for (int c = piece.c0; c < piece.c1 && ok && !piece.sum_only; ++c) {
        wait(&t->full[at.stage], at.phase);
        if (count < (c + 1) * C) {                    // rows behind the end have been cleared
          wait(&t->clean[at.stage], (clean_ph >> at.stage) & 1u);      // a stage's barrier turns at each such use
          clean_ph ^= 1u << at.stage;
        }
        if (before >= 0) ready();
        if (!ok) break;
        if (!maps.there) fence_async_shared();        // the copies were ordinary writes
        tc_fence_after_sync();
        const uint64_t a = rows_desc + at.stage * (X::STAGE >> 4), b = a + K_AT;
#pragma unroll
        for (int k = 0; k < DK * 4; ++k) {
          const uint32_t step = (k >> 2) * CH + (k & 3) * 2;
          product_smem(tmem + T_P, a + step, b + step, id_p, k != 0, k < key_steps ? on : 0u);
        }
        commit_products(&t->p_full, on);
        if (before >= 0) values();
        before = at.stage;
        at.advance();
      }
    }
    if (ok && before >= 0) {
      ready();
      if (ok) values();
    }
    drain(&t->drain[1]);
  } else if (warp >= W_SCORES) {
    // ------------------------------------------------------------ P, loads
    // 64 rows of up to CH chunks of 64 elements; what is not there becomes zeros
    auto rows = [&](unsigned char* to, const StateRows& r, int64_t token, int head, int column, int dim, int there, auto ch) {
      constexpr int CH = decltype(ch)::value, LANES = CH * 8, AT_ONCE = 32 / LANES;
      const int x = lane % LANES, sub = lane / LANES;
      const bool in = column + x * 8 < dim;
      const unsigned char* from = r.at + (token * r.token_stride + head * r.head_stride + (in ? column + x * 8 : 0)) * 2;
      const uint32_t dst = smem_u32(to) + (x >> 3) * ROW_CHUNK;
#pragma unroll 2
      for (int i = sub; i < C; i += AT_ONCE) {
        const bool here = in && i < there;
        cp_async_16(dst + i * 128 + (((x & 7) ^ (i & 7)) << 4), from + (i < there ? i : 0) * r.token_stride * 2, here);
      }
    };
    const std::integral_constant<int, DK> key_chunks;
    const std::integral_constant<int, DV> value_chunks;
    // What comes next into the ring: published states, 64 key dimensions at a time, and chunks.
    StateWalk load_walk = walk;
    StatePiece loading;
    bool more = warp == W_SCORES;
    int load_c = 0, load_end = 0, load_slot = 0, load_slots = 0, loads = 0;
    auto load_one = [&]() {
      while (more && load_slot >= load_slots && load_c >= load_end) {
        more = load_walk.next(&loading);
        if (!more) break;
        load_c = loading.c0;
        load_end = loading.c1;
        load_slot = 0;
        load_slots = slots_of(loading);
      }
      if (!more || !ok) return;
      wait(&t->empty[at.stage], at.phase ^ 1u);
      if (!ok) return;
      unsigned char* to = ring + at.stage * X::STAGE;
      uint64_t* bar = &t->full[at.stage];
      if (load_slot < load_slots) {
        const int of = states_of(loading), half = load_slot / of;
        if (loading.from == StatePiece::PUBLISHED) {
          const int j = t->slot_cta[load_slot - half * of];
          const long long t0 = clock64();
          bool told = true;
          while (told && ld_acquire_gpu(p.flags + j) != X::LANE_WARPS) told = !*abort_flag && clock64() - t0 < WAIT_LIMIT_CYCLES;
          ok = __all_sync(FULL_MASK, told);
          if (!ok) {
            *abort_flag = 1;
            return;
          }
          if (lane == 0) {
            asm volatile("fence.proxy.async;" ::: "memory");     // what is copied was written by ordinary stores
            mbar_arrive_expect_tx(bar, X::SLOT_HALF * 4);
            bulk_load(to, p.slots + (size_t)j * p.slot_floats + half * X::SLOT_HALF, X::SLOT_HALF * 4, bar);
          } else {
            mbar_arrive(bar);
          }
        } else {
          const int column = slice_of(loading) * 128, width = min(128, v.value_dim - column), there = min(64, v.key_dim - half * 64);
          const float* from = v.pool + (((size_t)p.seqs[loading.i] * v.n_layers + p.layer) * v.n_heads + head_of(loading)) * v.head_floats() +
                              (size_t)half * 64 * v.value_dim + column;
          if (lane == 0) mbar_arrive_expect_tx(bar, there * width * 4);
          __syncwarp();
          if (v.value_dim == DV * 64) {               // the rows lie as they have to: one copy (64 of them take 4,000 cycles to issue)
            if (lane == 0) bulk_load(to, from, there * (DV * 256), bar);
          } else {
            for (int r = lane; r < there; r += 32) bulk_load(to + r * (DV * 256), from + (size_t)r * v.value_dim, width * 4, bar);
          }
          if (lane != 0) mbar_arrive(bar);
        }
        __syncwarp();
        ++load_slot;
      } else {
        const int head = head_of(loading), column = slice_of(loading) * 128;
        const int64_t token = first_token(loading) + (int64_t)load_c * C;
        if (maps.there) {
          if (lane == 0) {
            const int y = (int)token, z = head;
            mbar_arrive_expect_tx(bar, (loading.sum_only ? DK + DV : 2 * DK + DV) * ROW_CHUNK);
#pragma unroll 1
            for (int x = 0; x < DK; ++x) {
              tma_load_3d(to + X::K_BYTES + x * ROW_CHUNK, &maps.k, x * 64, y, p.k.head_stride ? z : 0, bar);
              if (!loading.sum_only) tma_load_3d(to + x * ROW_CHUNK, &maps.q, x * 64, y, p.q.head_stride ? z : 0, bar);
            }
#pragma unroll 1
            for (int x = 0; x < DV; ++x) tma_load_3d(to + 2 * X::K_BYTES + x * ROW_CHUNK, &maps.val, column + x * 64, y, p.val.head_stride ? z : 0, bar);
          } else {
            mbar_arrive(bar);
          }
          __syncwarp();
        } else {
          const int there = min(C, tokens_of(loading) - load_c * C);
          rows(to + X::K_BYTES, p.k, token, head, 0, v.key_dim, there, key_chunks);
          rows(to + 2 * X::K_BYTES, p.val, token, head, column, v.value_dim, there, value_chunks);
          if (!loading.sum_only) rows(to, p.q, token, head, 0, v.key_dim, there, key_chunks);
          cp_async_arrive(bar);
        }
        ++load_c;
      }
      at.advance();
      ++loads;
    };
    const int row = tid - W_SCORES * 32;              // token of the chunk
    uint32_t ph = 0;
    const uint32_t to = smem_u32(p_smem) + row * 128;
    int served = 0;
    auto serve = [&]() {                              // the next piece's powers
      if (warp == W_SCORES || !ok || !load_walk.next(&loading)) return;
      const float rate = p.rates[head_of(loading)];
      wait(&t->fall_free[served & 1], ((served >> 1) & 1) ^ 1);
      for (int j = lane; j < TURN; j += 32) t->fall[served & 1].at[j] = j < FALL ? 0.0f : fall_of(rate, j - FALL);
      t->fall[served & 1].at[TURN + lane] = turn_of(rate, lane);
      tell(&t->fall_ready[served & 1]);
      ++served;
    };
    // Loads and powers are called for at one place, as their code is long: a load for each stage of the ring and then one more for each that has
    // been passed (the first one is kept back), powers two pieces ahead.
    int to_load = warp == W_SCORES ? n_stages : 0, to_serve = 2, to_pass = 0, c = 0, c1 = 0;
    bool begun = false, open = false;
    const float* fall = nullptr;
    auto passed = [&]() {
      if (warp == W_SCORES && begun) ++to_load;
      begun = true;
    };
    for (;;) {
#pragma unroll 1
      for (; to_load > 0; --to_load) load_one();
#pragma unroll 1
      for (; to_serve > 0; --to_serve) serve();
      if (!ok) break;
      if (to_pass > 0) {
        --to_pass;
        passed();
        continue;
      }
      if (c == c1) {
        if (open) end_piece();
        open = next_piece();
        if (!open) break;
        to_pass = slots_of(piece) + (piece.sum_only ? piece.c1 - piece.c0 : 0);
        c = piece.sum_only ? piece.c1 : piece.c0;
        c1 = piece.c1;
        fall = t->fall[n_pieces & 1].at + FALL + row;       // fall[-s]: l^(row - s), 0 for s > row
        continue;
      }
      wait(&t->p_full, ph);
      if (!ok) break;
      tc_fence_after_sync();
      float lift = 1.0f;
      if (F16) {
        float m = 0.0f;
#pragma unroll 1
        for (int h = 0; h < C; h += 32) {
          uint32_t x[32];
          tmem_ld_32x32(tmem + lane_base + T_P + h, x);
          tmem_ld_wait_for32(x);
#pragma unroll
          for (int s = 0; s < 32; ++s) m = fmaxf(m, fabsf(__uint_as_float(x[s]) * fall[-h - s]));
        }
        lift = lift_of(m, 100);
      }
      wait(&t->o1_full, ph ^ 1u);                   // the last chunk's has been used, and the factors of the one before
      if (!ok) break;
      if (F16) t->token_scale[ph][row] = reciprocal_of_power(lift);
#pragma unroll 1
      for (int h = 0; h < C; h += 32) {
        uint32_t x[32];
        tmem_ld_32x32(tmem + lane_base + T_P + h, x);
        tmem_ld_wait_for32(x);
#pragma unroll
        for (int s = 0; s < 32; ++s) {
          const float y = __uint_as_float(x[s]) * fall[-h - s];
          x[s] = __float_as_uint(F16 ? y * lift : y);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = pack2<F16>(__uint_as_float(x[8 * j + 2 * i]), __uint_as_float(x[8 * j + 2 * i + 1]));
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (((h / 8 + j) ^ (row & 7)) << 4)), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                       : "memory");
        }
      }
      ph ^= 1u;
      fence_async_shared();
      tc_fence_before_sync();
      tell(&t->p_ready);
      passed();
      if (c == piece.c0 && n_pieces > 0) to_serve = 1;
      ++c;
    }
    // what is in flight lands before the CTA leaves
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!ok)
      for (int j = max(0, loads - n_stages); j < loads; ++j) {
        const long long t0 = clock64();
        while (!mbar_try_wait(&t->full[j % n_stages], (uint32_t)((j / n_stages) & 1)) && clock64() - t0 < WAIT_LIMIT_CYCLES) {
        }
      }
  } else if (warp >= W_VALUES) {
    // ------------------------------------------------------------ W
    // A thread has the tokens 8 j + 2 (lane % 4) and the next, of the value columns lane / 4 + 8 i: as matrices come out of shared memory
    // transposed, and as tensor memory takes them.
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(VALUE_REGS));
    const int column0 = (warp - W_VALUES) * 32, pair = (lane & 3) * 2;
    // the address of a row of the matrix that this lane has to name: token lane % 8 of the first or second eight (lane / 16), columns of
    // the first or second eight (lane / 8 % 2)
    auto matrix_row = [&](int g) {
      const int eight = ((column0 & 63) >> 3) + 2 * g + ((lane >> 3) & 1);
      return (uint32_t)((column0 >> 6) * ROW_CHUNK + ((lane >> 4) * 8 + (lane & 7)) * 128 + ((eight ^ (lane & 7)) << 4));
    };
    const uint32_t from0 = smem_u32(ring) + 2 * X::K_BYTES, row_of[2] = {matrix_row(0), matrix_row(1)};
    uint32_t ph = 0;
    // (warps whose value columns there are none of have nothing to do)
    while ((warp & 3) < X::LANE_WARPS && next_piece()) {
      const int count = tokens_of(piece);
      // (stages that hold published states are not for these warps, but they follow them, or they could lose count of the rounds)
      for (int j = slots_of(piece); j > 0 && ok; --j) {
        wait(&t->full[at.stage], at.phase);
        tell(&t->slots_read[at.stage]);
        at.advance();
      }
      for (int c = piece.c0; c < piece.c1; ++c) {
        const float* weight = t->fall[n_pieces & 1].at + FALL + min(C, count - c * C) - 1 - pair;       // weight[-s]: l^(n-1-s-pair), 0 behind the end
        wait(&t->full[at.stage], at.phase);
        if (!ok) break;
        const uint32_t from = from0 + at.stage * X::STAGE;
        if (count < (c + 1) * C) {
          // rows behind the end: of V what this warp reads, of K a share.  (A weight of zero would not undo an infinity.)
          const int there = count - c * C;
          unsigned char* stage = ring + at.stage * X::STAGE + X::K_BYTES;
#pragma unroll 1
          for (int u = lane; u < (C - there) * 4; u += 32) {
            const int r = there + (u >> 2), x = column0 / 8 + (u & 3);
            *reinterpret_cast<uint4*>(stage + X::K_BYTES + (x >> 3) * ROW_CHUNK + r * 128 + ((x & 7) ^ (r & 7)) * 16) = make_uint4(0, 0, 0, 0);
          }
#pragma unroll 1
          for (int u = tid - W_VALUES * 32; u < (C - there) * DK * 8; u += X::LANE_WARPS * 32) {
            const int r = there + u / (DK * 8), x = u % (DK * 8);
            *reinterpret_cast<uint4*>(stage + (x >> 3) * ROW_CHUNK + r * 128 + (x & 7) * 16) = make_uint4(0, 0, 0, 0);
          }
          fence_async_shared();
          tell(&t->clean[at.stage]);
        }
        // (loops that are not unrolled: the roles' code together has to stay in the instruction cache.  Unrolled, warps waited for
        // instructions more than for anything else, and a chunk took 6,500 cycles.)
        float lift[4] = {1.0f, 1.0f, 1.0f, 1.0f};
        if (F16) {
          float m[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
          for (int s = 0; s < C; s += 16) {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              uint32_t raw[4];
              ldmatrix_x4_trans(raw, from + row_of[g] + s * 128);
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                const float2 y = pair16<F16>(raw[u]);
                const float* f = weight - s - (u >> 1) * 8;
                m[2 * g + (u & 1)] = fmaxf(m[2 * g + (u & 1)], fmaxf(fabsf(y.x * f[0]), fabsf(y.y * f[-1])));
              }
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            m[i] = fmaxf(m[i], __shfl_xor_sync(FULL_MASK, m[i], 1));
            lift[i] = lift_of(fmaxf(m[i], __shfl_xor_sync(FULL_MASK, m[i], 2)), 38);
          }
        }
#pragma unroll 1
        for (int x = 0; x < 4; ++x) {                 // halves of the chunk, and of these halves of the warp's value columns
          const int half = x >> 1, g = x & 1, s = half * 32;
          if (g == 0) {
            wait(&t->w_free[half], ph ^ 1u);          // the last chunk's has been used
            if (!ok) break;
            tc_fence_after_sync();
          }
          uint32_t raw[2][4], out[PARTS<F16>][8];
          const uint32_t matrix = from + (g ? row_of[1] : row_of[0]) + s * 128;
          ldmatrix_x4_trans(raw[0], matrix);
          ldmatrix_x4_trans(raw[1], matrix + 16 * 128);
          const uint64_t lift2[2] = {F16 ? pair_of(g ? lift[2] : lift[0], g ? lift[2] : lift[0]) : 0, F16 ? pair_of(g ? lift[3] : lift[1], g ? lift[3] : lift[1]) : 0};
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const float* f = weight - s - (u >> 1) * 8;
            const float2 y = pair16<F16>(raw[u >> 2][u & 3]);
            uint64_t x2 = mul_pairs(pair_of(y.x, y.y), pair_of(f[0], f[-1]));
            if (F16) x2 = mul_pairs(x2, lift2[u & 1]);
#pragma unroll
            for (int w = 0; w < PARTS<F16>; ++w) {
              float a, b;
              split_pair(x2, &a, &b);
              out[w][u] = pack2<F16>(a, b);
              if (w + 1 < PARTS<F16>) {               // what the rounding left over, exactly
                const float2 e = pair16<F16>(out[w][u]);
                x2 = fma_pairs(pair_of(e.x, e.y), pair_of(-1.0f, -1.0f), x2);
              }
            }
          }
#pragma unroll
          for (int w = 0; w < PARTS<F16>; ++w)
            tmem_st_16x16(tmem + lane_base + ((uint32_t)(g * 16) << 16) + T_W + w * (C / 2) + s / 2, out[w]);
          if (g == 1) {
            if (F16 && half == 1 && (lane & 3) == 0) {      // (the factors of the chunk before the last have been read)
#pragma unroll
              for (int i = 0; i < 4; ++i) t->lane_scale[ph][column0 + (lane >> 2) + 8 * i] = lift[i];
            }
            __syncwarp();
            tmem_st_wait();
            tc_fence_before_sync();
            tell(&t->w_ready[half]);
          }
        }
        if (!ok) break;
        ph ^= 1u;
        at.advance();
      }
      end_piece();
    }
  } else if (warp >= W_STATE) {
    // ------------------------------------------------------------ the state
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(STATE_REGS));
    if ((warp & 3) < X::LANE_WARPS) {
      const int column = tid - W_STATE * 32;
      uint32_t ph = 0, out_ph = 0;                    // chunks, and chunks with results, before this one
      const uint32_t u_at = tmem + lane_base + T_U, copy_at = tmem + lane_base + T_COPY;
      uint64_t s[DK * 32];                            // key dimensions in pairs
      bool to_tell = false;
      while (next_piece()) {
        const int count = tokens_of(piece), head = head_of(piece), global_column = slice_of(piece) * 128 + column;
        // the state in front of the piece
        const int states = states_of(piece);
        const bool published = piece.from == StatePiece::PUBLISHED;
#pragma unroll
        for (int h = 0; h < DK; ++h) {
#pragma unroll
          for (int k = 0; k < 32; ++k) s[h * 32 + k] = 0;
#pragma unroll 1
          for (int j = 0; j < states; ++j) {
            const float w = published ? t->slot_weight[j] : 1.0f;
            const int there = published ? 64 : v.key_dim - h * 64;
            wait(&t->full[at.stage], at.phase);
            if (!ok) break;
            const uint32_t from = smem_u32(ring) + at.stage * X::STAGE + column * 4;
            const uint64_t w2 = pair_of(w, w);
            // (code that runs once a piece comes from far away: the whole case has no more of it than it needs)
            if (there >= 64) {
#pragma unroll
              for (int k = 0; k < 64; k += 2)
                s[h * 32 + k / 2] = fma_pairs(w2, pair_of(ld_shared(from + k * (DV * 256)), ld_shared(from + (k + 1) * (DV * 256))), s[h * 32 + k / 2]);
            } else {
#pragma unroll
              for (int k = 0; k < 64; k += 2)         // (key_dim is even)
                if (k < there)
                  s[h * 32 + k / 2] = fma_pairs(w2, pair_of(ld_shared(from + k * (DV * 256)), ld_shared(from + (k + 1) * (DV * 256))), s[h * 32 + k / 2]);
            }
            tell(&t->slots_read[at.stage]);
            at.advance();
          }
        }
        if (!ok) break;
        if (to_tell) {
          // the state that was published last: now that what was stored has been read (another CTA writes there when it has ended the item)
          to_tell = false;
          __threadfence();
          __syncwarp();
          if (lane == 0) atomicAdd(p.flags + blockIdx.x, 1u);
        }
        for (int c = piece.c0; c < piece.c1; ++c, at.advance()) {
          if (!piece.sum_only) {
            float lift = 1.0f;
            if (F16) {
              float m = 0.0f;
#pragma unroll
              for (int k = 0; k < DK * 32; ++k) {
                float a, b;
                split_pair(s[k], &a, &b);
                m = fmaxf(m, fmaxf(fabsf(a), fabsf(b)));
              }
              lift = lift_of(m, 100);
            }
            wait(&t->o2_full, out_ph ^ 1u);           // the copy before has been used, and the results before that have their factors
            if (!ok) break;
            if (F16) t->copy_scale[out_ph][column] = reciprocal_of_power(lift);
#pragma unroll
            for (int h = 0; h < DK; ++h) {
              uint32_t w[32];
#pragma unroll
              for (int k = 0; k < 32; ++k) {
                float a, b;
                split_pair(F16 ? mul_pairs(s[h * 32 + k], pair_of(lift, lift)) : s[h * 32 + k], &a, &b);
                w[k] = pack2<F16>(a, b);
              }
              tmem_st_32x32(copy_at + h * 32, w);
            }
            tmem_st_wait();
            tc_fence_before_sync();
            tell(&t->copy_ready);
            out_ph ^= 1u;
          }
          const float decay = t->fall[n_pieces & 1].at[count - c * C < C ? FALL + count - c * C : TURN + (c & (TURNS - 1))];
          wait(&t->u_full, ph);
          if (!ok) break;
          tc_fence_after_sync();
          const float back = F16 ? reciprocal_of_power(t->lane_scale[ph][column]) : 1.0f;
#pragma unroll
          for (int h = 0; h < DK * 2; ++h) {
            uint32_t u[32];
            tmem_ld_32x32(u_at + h * 32, u);
            tmem_ld_wait_for32(u);
            if (h == DK * 2 - 1) {
              tc_fence_before_sync();
              tell(&t->u_free);
            }
            // (columns beyond key_dim rounded up to 16 are not written by the products)
#pragma unroll
            for (int k = 0; k < 32; k += 2)
              if (h * 32 + (k & ~15) < v.key_dim) {
                uint64_t y = pair_of(__uint_as_float(u[k]), __uint_as_float(u[k + 1]));
                if (F16) y = mul_pairs(y, pair_of(back, back));
                s[h * 16 + k / 2] = fma_pairs(pair_of(decay, decay), s[h * 16 + k / 2], y);
              }
          }
          ph ^= 1u;
        }
        if (!ok) break;
        end_piece();
        // the state behind it
        if (piece.to != StatePiece::NOTHING) {
          const bool publish = piece.to == StatePiece::PUBLISHED;
          const int stride = publish ? DV * 64 : v.value_dim, there = publish ? DK * 64 : v.key_dim;
          float* to = publish ? p.slots + (size_t)blockIdx.x * p.slot_floats + column
                              : v.pool + (((size_t)p.seqs[piece.i] * v.n_layers + p.layer) * v.n_heads + head) * v.head_floats() + global_column;
          const bool here = publish || global_column < v.value_dim;
          if (stride == DV * 64 && there == DK * 64) {
#pragma unroll
            for (int k = 0; k < DK * 64; k += 2) {
              float a, b;
              split_pair(s[k / 2], &a, &b);
              to[k * (DV * 64)] = a;
              to[(k + 1) * (DV * 64)] = b;
            }
          } else {
#pragma unroll
            for (int k = 0; k < DK * 64; k += 2) {
              float a, b;
              split_pair(s[k / 2], &a, &b);
              if (here && k < there) {
                to[0] = a;
                to[stride] = b;
              }
              to += 2 * stride;
            }
          }
          if (publish && t->plan.again.c1) {
            to_tell = true;
          } else if (publish) {
            __threadfence();
            __syncwarp();
            if (lane == 0) atomicAdd(p.flags + blockIdx.x, 1u);
          }
        }
      }
    }
  } else {
    // ------------------------------------------------------------ results
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OUT_REGS));
    // A thread has the tokens 8 j + 2 (lane % 4) and the next, of the value columns lane / 4 + 8 i; by way of shared memory they become a
    // token's vectors of 8 columns.
    const int pair = (lane & 3) * 2;
    uint32_t ph = 0;
    const uint32_t mine = smem_u32(out_smem) + warp * 32 * 64;
    const uint64_t scale2 = pair_of(p.scale, p.scale);
    auto place = [&](int token, int eight) { return mine + token * 64 + ((eight ^ ((token >> 1) & 3)) << 4); };
    while ((warp & 3) < X::LANE_WARPS && next_piece()) {
      if (piece.sum_only) {
        end_piece();
        continue;
      }
      const float* fall = t->fall[n_pieces & 1].at + FALL + 1 + pair;          // fall[t]: l^(t+pair+1)
      const int count = tokens_of(piece), first_column = slice_of(piece) * 128 + warp * 32;
      const int64_t token0 = first_token(piece);
      uint16_t* out = reinterpret_cast<uint16_t*>(const_cast<unsigned char*>(p.out.at)) + token0 * p.out.token_stride + head_of(piece) * p.out.head_stride +
                      first_column + (lane & 3) * 8;
      const bool here = first_column + (lane & 3) * 8 < v.value_dim;
      for (int c = piece.c0; c < piece.c1; ++c) {
        wait(&t->o1_full, ph);
        wait(&t->o2_full, ph);
        if (!ok) break;
        tc_fence_after_sync();
        const int there = here ? min(C, count - c * C) : 0;
        uint16_t* to = out + (int64_t)c * C * p.out.token_stride;
        auto flush = [&](int h) {                     // 32 tokens from shared memory to the result
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int row = i * 8 + (lane >> 2);
            uint4 y;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(y.x), "=r"(y.y), "=r"(y.z), "=r"(y.w) : "r"(place(row, lane & 3)));
            if (h * 32 + row < there) *reinterpret_cast<uint4*>(to + (h * 32 + row) * p.out.token_stride) = y;
          }
          __syncwarp();
        };
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {                 // 32 tokens
          uint32_t w[2][8];
#pragma unroll
          for (int g = 0; g < 2; ++g) {               // 16 value columns
            uint32_t a[16], b[16];
            const uint32_t from = tmem + lane_base + ((uint32_t)(g * 16) << 16) + h * 32;
            tmem_ld_16x32(from + T_O1, a);
            tmem_ld_16x32(from + T_O2, b);
            tmem_ld_wait_for16(a);
            tmem_ld_wait_for16(b);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float* f = fall + h * 32 + j * 8;
              const uint64_t fall2 = mul_pairs(pair_of(f[0], f[1]), scale2);
              const uint64_t one = F16 ? mul_pairs(*reinterpret_cast<const uint64_t*>(&t->token_scale[ph][h * 32 + j * 8 + pair]), scale2) : scale2;
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                const int x = 4 * j + 2 * r;
                uint64_t y = pair_of(__uint_as_float(b[x]), __uint_as_float(b[x + 1]));
                if (F16) {
                  const float copy = t->copy_scale[ph][warp * 32 + (lane >> 2) + 8 * (2 * g + r)];
                  y = mul_pairs(y, pair_of(copy, copy));
                }
                y = fma_pairs(fall2, y, mul_pairs(one, pair_of(__uint_as_float(a[x]), __uint_as_float(a[x + 1]))));
                float u, v;
                split_pair(y, &u, &v);
                w[g][2 * j + r] = pack2<F16>(u, v);
              }
            }
          }
          if (h == 1) {
            // all of the chunk's has been read, its factors too: the products of the next one wait for this
            tc_fence_before_sync();
            tell(&t->o_free);
            flush(0);
          }
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int j = 0; j < 4; j += 2)
              stmatrix_x4_trans(place(8 * (j + (lane >> 4)) + (lane & 7), g * 2 + ((lane >> 3) & 1)), w[g][2 * j], w[g][2 * j + 1], w[g][2 * j + 2],
                                w[g][2 * j + 3]);
        }
        flush(1);
        ph ^= 1u;
      }
      end_piece();
    }
  }
  if (!ok && lane == 0) state_report(v, KV_TIMEOUT);
  tc_fence_before_sync();
  __syncthreads();
  if (warp == W_STATE_PRODUCTS) tmem_dealloc(tmem, 512);
  // the last CTA leaves the flags as it found them
  if (holds && tid == 0) {
    __threadfence();
    if (atomicAdd(p.flags + gridDim.x, 1u) == gridDim.x - 1)
      for (int i = 0; i <= (int)gridDim.x; ++i) p.flags[i] = 0;
  }
}

template <bool F16, int DK, int DV>
constexpr int smem_bytes(int stages) { return 1024 + stages * Sizes<F16, DK, DV>::STAGE + ROW_CHUNK + OUT_BYTES + (int)sizeof(Tail); }

template <bool F16, int DK, int DV>
cudaError_t configure(int smem_optin) {
  return cudaFuncSetAttribute(state_chunk_kernel<F16, DK, DV>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin);
}

template <bool F16, int DK, int DV>
cudaError_t launch(const StateAttendParams& p, const StateMaps& maps, int sm_count, int smem_optin, cudaStream_t st) {
  int stages = MAX_STAGES;
  while (stages > 2 && smem_bytes<F16, DK, DV>(stages) > smem_optin) --stages;
  // A CTA with a part of an item waits for the states of all the parts before it and adds them up, so that beyond some number more parts cost more than
  // they give: with an item of M chunks, about sqrt(2 M) (30,000 tokens, one head of 128 x 128: 141 us; with sqrt(M) 142, with sqrt(4 M) 155, with an SM
  // each 314).  (Sequences of the mean length: what there is is not known here.)
  const int64_t chunks = (p.n_tokens - 1) / C + p.n_long, mean = (chunks + p.n_long - 1) / p.n_long;
  int64_t parts = 1;
  while (parts * parts < 2 * mean) ++parts;
  parts *= (int64_t)p.n_long * p.n_items;
  if (parts > sm_count) parts = sm_count;
  return launch_overlapped(state_chunk_kernel<F16, DK, DV>, dim3((unsigned)parts), dim3(THREADS), (size_t)smem_bytes<F16, DK, DV>(stages), st, 1, p, maps,
                           stages);
}

}  // namespace

size_t state_slot_floats(int key_dim, int value_dim) {
  return (size_t)(key_dim > 64 ? 128 : 64) * (value_dim > 64 ? 128 : 64);
}

cudaError_t state_chunk_configure(int smem_optin) {
  cudaError_t e = configure<false, 1, 1>(smem_optin);
  if (e == cudaSuccess) e = configure<false, 1, 2>(smem_optin);
  if (e == cudaSuccess) e = configure<false, 2, 1>(smem_optin);
  if (e == cudaSuccess) e = configure<false, 2, 2>(smem_optin);
  if (e == cudaSuccess) e = configure<true, 1, 1>(smem_optin);
  if (e == cudaSuccess) e = configure<true, 1, 2>(smem_optin);
  if (e == cudaSuccess) e = configure<true, 2, 1>(smem_optin);
  if (e == cudaSuccess) e = configure<true, 2, 2>(smem_optin);
  return e;
}

cudaError_t state_chunk_launch(StateAttendParams p, const StateMaps& maps, bool f16, int sm_count, int smem_optin, cudaStream_t st) {
  const bool k2 = p.v.key_dim > 64, v2 = p.v.value_dim > 64;
  auto* go = f16 ? (k2 ? (v2 ? launch<true, 2, 2> : launch<true, 2, 1>) : (v2 ? launch<true, 1, 2> : launch<true, 1, 1>))
                 : (k2 ? (v2 ? launch<false, 2, 2> : launch<false, 2, 1>) : (v2 ? launch<false, 1, 2> : launch<false, 1, 1>));
  return go(p, maps, sm_count, smem_optin, st);
}

}  // namespace icc
