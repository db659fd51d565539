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
//   warps 12-13  P
//   warp 14      issues the products: U(c), O2(c), O1(c), P(c + 1), ...
//   warp 15      loads of K, V and Q into a ring of stages: boxes of tensor maps; of a sequence's last, shorter chunk (and where the strides
//                allow no map) 16-byte copies, with zeros behind the end
//
// Bound: HBM, 1 KB a token and head of 128 x 128; a chunk is 64 KB, 2,750 cycles of an SM's share.  The products take 1,600.
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
enum : int { W_OUT = 0, W_STATE = 4, W_VALUES = 8, W_SCORES = 12, W_PRODUCTS = 14, W_LOADS = 15 };
// Registers of the four warpgroups' threads; they are launched with 128.
constexpr int OUT_REGS = 96, STATE_REGS = 208, VALUE_REGS = 96, OTHER_REGS = 112;
static_assert(OUT_REGS + STATE_REGS + VALUE_REGS + OTHER_REGS <= 4 * 128, "what some have more, others have less");
// Columns of tensor memory.
constexpr uint32_t T_P = 0, T_O1 = 64, T_O2 = 128, T_COPY = 192, T_U = 256, T_W = 384;

template <bool F16>
constexpr int PARTS = F16 ? 2 : 3;                    // 16-bit numbers that hold one of W

// A warp's powers of l.
constexpr int FALL = C;
struct Fall {
  float at[2 * C + 4];                                // l^j at FALL + j, j = 0 .. 64, with zeros in front
};

struct Tail {
  StateLine line;
  Fall fall[W_PRODUCTS];                              // of each warp that needs one
  alignas(16) float token_scale[2][C];                      // fp16: what P's row was divided by, by the chunk's parity
  float lane_scale[2][128];                           // fp16: what W's column was multiplied by
  float copy_scale[2][128];                           // fp16: what the copy of S has to be multiplied by
  uint64_t full[MAX_STAGES], empty[MAX_STAGES];
  uint64_t p_full, p_ready, w_ready, copy_ready, u_full, u_free, o2_done, o_full, o_free, drain;
  uint64_t slots_read[MAX_STAGES];
  uint32_t seen[STATE_MAX_SEQS / 32];
  uint32_t tmem_base;
  int abort_flag, holds;
};

// The power of two that brings the largest magnitude m (>= 0, finite) into [2^13, 2^14); 1 for 0.
__device__ __forceinline__ float lift_of(float m, int most) {
  if (m == 0.0f) return 1.0f;
  const int e = 13 - ((int)(__float_as_uint(m) >> 23) - 127);
  return __uint_as_float((uint32_t)(min(max(e, -100), most) + 127) << 23);
}
__device__ __forceinline__ float reciprocal_of_power(float p) { return __uint_as_float((254u << 23) - __float_as_uint(p)); }

template <bool F16>
__device__ __forceinline__ float2 pair16(uint32_t x) {
  return F16 ? __half22float2(*reinterpret_cast<const __half2*>(&x)) : make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
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
  if (tid == 0) {
    for (int s = 0; s < n_stages; ++s) {
      mbar_init(&t->full[s], 32);
      mbar_init(&t->empty[s], 1);
      mbar_init(&t->slots_read[s], 2 * X::LANE_WARPS);
    }
    mbar_init(&t->p_full, 1);
    mbar_init(&t->p_ready, 2);
    mbar_init(&t->w_ready, X::LANE_WARPS);
    mbar_init(&t->copy_ready, X::LANE_WARPS);
    mbar_init(&t->u_full, 1);
    mbar_init(&t->u_free, X::LANE_WARPS);
    mbar_init(&t->o2_done, 1);
    mbar_init(&t->o_full, 1);
    mbar_init(&t->o_free, X::LANE_WARPS);
    mbar_init(&t->drain, 1);
    t->abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == W_PRODUCTS) tmem_alloc(&t->tmem_base, 512);
  grid_dep_launch_dependents();
  grid_dep_wait();
  const bool holds = state_call_holds(p, t->seen);
  if (holds && warp == 0) {
    // chunks before each sequence
    int sum = 0;
    for (int i0 = 0; i0 < p.n; i0 += 32) {
      const int i = i0 + lane;
      const int mine = i < p.n ? (int)(((unsigned)(p.starts ? p.starts[i + 1] - p.starts[i] : 1) + C - 1) / C) : 0;
      int inc = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(FULL_MASK, inc, d);
        if (lane >= d) inc += y;
      }
      if (i < p.n) t->line.before[i + 1] = sum + inc;
      sum += __shfl_sync(FULL_MASK, inc, 31);
    }
    if (lane == 0) {
      t->line.before[0] = 0;
      t->line.n = p.n;
      t->line.per_chunk = v.n_heads * p.slices;
      t->line.parts = gridDim.x;
    }
  } else if (!holds && tid == 0) {
    // nothing to do: a line without chunks
    t->line.before[0] = t->line.before[1] = 0;
    t->line.n = t->line.per_chunk = 1;
    t->line.parts = gridDim.x;
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = t->tmem_base, lane_base = (uint32_t)((warp & 3) * 32) << 16;
  const uint32_t on = lane == 0;
  volatile int* abort_flag = &t->abort_flag;
  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (ok) ok = mbar_warp_wait(bar, parity, abort_flag);
  };
  StateWalk walk(&t->line, blockIdx.x);
  StatePiece piece;
  auto head_of = [&](const StatePiece& x) { return x.item / p.slices; };
  auto slice_of = [&](const StatePiece& x) { return x.item % p.slices; };
  auto first_token = [&](const StatePiece& x) { return p.starts ? p.starts[x.i] : p.first_seq + x.i; };
  auto tokens_of = [&](const StatePiece& x) { return p.starts ? p.starts[x.i + 1] - p.starts[x.i] : 1; };
  // How many published states a piece's own one is put together from.
  auto slots_of = [&](const StatePiece& x) {
    int n = 0;
    if (x.from == StatePiece::PUBLISHED)
      for (int j = x.first; j < (int)blockIdx.x; ++j) n += t->line.cut(j) < t->line.cut(j + 1);
    return n;
  };
  // This warp's powers of the head's decay.
  auto fill_falls = [&](const StatePiece& x) {
    Fall& f = t->fall[warp];
    const double rate = p.rates[head_of(x)];
    __syncwarp();
    for (int j = lane; j < 2 * C + 4; j += 32) f.at[j] = j < FALL ? 0.0f : j == FALL ? 1.0f : (float)exp(-rate * (j - FALL));
    __syncwarp();
  };
  auto tell = [&](uint64_t* bar) {
    __syncwarp();
    arrive_one(bar, on);
  };

  if (warp == W_LOADS) {
    // ------------------------------------------------------------ loads
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
    int n = 0;
    auto begin = [&]() {
      wait(&t->empty[n % n_stages], ((n / n_stages) & 1) ^ 1);
      return ring + (n % n_stages) * X::STAGE;
    };
    auto end = [&]() {
      cp_async_arrive(&t->full[n % n_stages]);
      ++n;
    };
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
    while (ok && walk.next(&piece)) {
      const int head = head_of(piece), count = tokens_of(piece);
      const int64_t token0 = first_token(piece);
      if (piece.from == StatePiece::PUBLISHED)
        for (int h = 0; h < DK && ok; ++h)
          for (int j = piece.first; j < (int)blockIdx.x && ok; ++j) {
            if (t->line.cut(j) == t->line.cut(j + 1)) continue;
            unsigned char* to = begin();
            if (!ok) break;
            const long long t0 = clock64();
            while (ok && ld_acquire_gpu(p.flags + j) != X::LANE_WARPS) {
              if (*abort_flag || clock64() - t0 > WAIT_LIMIT_CYCLES) ok = false;
            }
            ok = __all_sync(FULL_MASK, ok);
            if (!ok) {
              *abort_flag = 1;
              break;
            }
            const unsigned char* from = reinterpret_cast<const unsigned char*>(p.slots + (size_t)j * p.slot_floats + h * X::SLOT_HALF);
            for (int u = lane; u < X::SLOT_HALF / 4; u += 32) cp_async_16(smem_u32(to) + u * 16, from + u * 16, true);
            end();
          }
      for (int c = piece.c0; c < piece.c1 && ok; ++c) {
        unsigned char* to = begin();
        if (!ok) break;
        const int there = min(C, count - c * C);
        const int64_t token = token0 + (int64_t)c * C;
        if (there == C && maps.there) {
          uint64_t* bar = &t->full[n % n_stages];
          if (lane == 0) {
            const int y = (int)token;
            mbar_arrive_expect_tx(bar, (piece.sum_only ? DK + DV : 2 * DK + DV) * ROW_CHUNK);
#pragma unroll
            for (int x = 0; x < DK; ++x) tma_load_3d(to + X::K_BYTES + x * ROW_CHUNK, &maps.k, x * 64, y, p.k.head_stride ? head : 0, bar);
#pragma unroll
            for (int x = 0; x < DV; ++x)
              tma_load_3d(to + 2 * X::K_BYTES + x * ROW_CHUNK, &maps.val, slice_of(piece) * 128 + x * 64, y, p.val.head_stride ? head : 0, bar);
            if (!piece.sum_only)
#pragma unroll
              for (int x = 0; x < DK; ++x) tma_load_3d(to + x * ROW_CHUNK, &maps.q, x * 64, y, p.q.head_stride ? head : 0, bar);
          } else {
            mbar_arrive(bar);
          }
          __syncwarp();
          ++n;
          continue;
        }
        rows(to + X::K_BYTES, p.k, token, head, 0, v.key_dim, there, key_chunks);
        rows(to + 2 * X::K_BYTES, p.val, token, head, slice_of(piece) * 128, v.value_dim, there, value_chunks);
        if (!piece.sum_only) rows(to, p.q, token, head, 0, v.key_dim, there, key_chunks);
        end();
      }
    }
    // what is in flight lands before the CTA leaves
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!ok)
      for (int j = max(0, n - n_stages); j < n; ++j) {
        const long long t0 = clock64();
        while (!mbar_try_wait(&t->full[j % n_stages], (uint32_t)((j / n_stages) & 1)) && clock64() - t0 < WAIT_LIMIT_CYCLES) {
        }
      }
  } else if (warp == W_PRODUCTS) {
    // ------------------------------------------------------------ products
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
    const int key_steps = (v.key_dim + 15) / 16;
    const uint32_t id_p = idesc(F16, C, false), id_o1 = idesc(F16, C, false, true), id_o2 = idesc(F16, C, false), id_u = idesc(F16, key_steps * 16, true);
    const uint64_t rows_desc = umma_desc_k_major_sw128(smem_u32(ring)), p_desc = umma_desc_k_major_sw128(smem_u32(p_smem)),
                   columns_desc = desc_mn_major_sw128(smem_u32(ring), ROW_CHUNK);
    constexpr uint32_t CH = ROW_CHUNK >> 4, K_AT = X::K_BYTES >> 4, V_AT = 2 * X::K_BYTES >> 4;
    int n = 0;                                        // stages used before the present chunk's
    uint32_t sum_ph = 0, out_ph = 0, slots_ph = 0;    // of the barriers that turn once a chunk, and once a chunk with results
    bool scored = false;                              // the present chunk's P is under way
    auto at = [&](int stage) { return (uint32_t)((stage % n_stages) * (X::STAGE >> 4)); };
    auto loaded = [&](int stage, int there) {
      wait(&t->full[stage % n_stages], (stage / n_stages) & 1);
      if (!maps.there || there < C) fence_async_shared();       // the copies were ordinary writes
      tc_fence_after_sync();
    };
    auto scores = [&](int stage) {
      const uint64_t a = rows_desc + at(stage), b = a + K_AT;
      // (unrolled: a product whose operands have to be worked out first takes 130 cycles to issue)
#pragma unroll
      for (int k = 0; k < DK * 4; ++k) {
        const uint32_t step = (k >> 2) * CH + (k & 3) * 2;
        product_smem(tmem + T_P, a + step, b + step, id_p, k != 0, k < key_steps ? on : 0u);
      }
      commit_products(&t->p_full, on);
    };
    bool more = walk.next(&piece);
    int count = more ? tokens_of(piece) : 0;
    while (more && ok) {
      StateWalk after = walk;
      StatePiece next;
      const bool more_after = after.next(&next);
      const int count_after = more_after ? tokens_of(next) : 0;
      const int slots = DK * slots_of(piece);
      for (int j = 0; j < slots && ok; ++j) {         // stages that held published states
        wait(&t->slots_read[n % n_stages], (slots_ph >> (n % n_stages)) & 1u);      // a stage's barrier turns at each such use
        slots_ph ^= 1u << (n % n_stages);
        arrive_one(&t->empty[n % n_stages], on);
        ++n;
      }
      for (int c = piece.c0; c < piece.c1 && ok; ++c) {
        const uint32_t stage = at(n);
        if (!scored) loaded(n, count - c * C);
        if (!piece.sum_only && !scored && ok) scores(n);
        scored = false;
        wait(&t->w_ready, sum_ph);
        wait(&t->u_free, sum_ph ^ 1u);
        sum_ph ^= 1u;
        if (!ok) break;
        tc_fence_after_sync();
#pragma unroll 1
        for (int w = PARTS<F16> - 1; w >= 0; --w)     // the least parts first: what is cut off of a sum is a part of what is there
#pragma unroll
          for (int k = 0; k < C / 16; ++k)            // 16 tokens further: 8 columns of W, 2048 bytes of K
            product_tmem(tmem + T_U, tmem + T_W + w * (C / 2) + k * 8, columns_desc + stage + K_AT + k * 128, id_u, w + 1 < PARTS<F16> || k != 0, on);
        commit_products(&t->u_full, on);
        if (piece.sum_only) {
          commit_products(&t->empty[n % n_stages], on);
        } else {
          wait(&t->copy_ready, out_ph);
          wait(&t->o_free, out_ph ^ 1u);
          if (!ok) break;
          tc_fence_after_sync();
#pragma unroll
          for (int k = 0; k < DK * 4; ++k)
            product_tmem(tmem + T_O2, tmem + T_COPY + k * 8, rows_desc + stage + (k >> 2) * CH + (k & 3) * 2, id_o2, k != 0, k < key_steps ? on : 0u);
          commit_products(&t->o2_done, on);
          wait(&t->p_ready, out_ph);
          out_ph ^= 1u;
          if (!ok) break;
          tc_fence_after_sync();
#pragma unroll
          for (int k = 0; k < C / 16; ++k)
            product_smem(tmem + T_O1, columns_desc + stage + V_AT + k * 128, p_desc + k * 2, id_o1, k != 0, on);
          commit_products(&t->o_full, on);
          commit_products(&t->empty[n % n_stages], on);
        }
        ++n;
        // the next chunk's scores, unless published states lie between in the ring
        const bool last = c + 1 == piece.c1;
        if (last ? more_after && !next.sum_only && next.from != StatePiece::PUBLISHED : !piece.sum_only) {
          loaded(n, last ? count_after - next.c0 * C : count - (c + 1) * C);
          if (ok) scores(n);
          scored = true;
        }
      }
      walk = after;
      piece = next;
      count = count_after;
      more = more_after;
    }
    // nothing issued is still running when tensor memory is released
    commit_products(&t->drain, on);
    const long long t0 = clock64();
    while (!mbar_try_wait(&t->drain, 0) && clock64() - t0 < WAIT_LIMIT_CYCLES) {
    }
  } else if (warp >= W_SCORES) {
    // ------------------------------------------------------------ P
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
    const int row = tid - W_SCORES * 32;              // token of the chunk
    uint32_t ph = 0;
    const uint32_t to = smem_u32(p_smem) + row * 128;
    while (ok && walk.next(&piece)) {
      if (piece.sum_only) continue;
      fill_falls(piece);
      const float* fall = t->fall[warp].at + FALL + row;                // fall[-s]: l^(row - s), 0 for s > row
      for (int c = piece.c0; c < piece.c1; ++c) {
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
          t->token_scale[ph][row] = reciprocal_of_power(lift);
        }
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
    int n = 0;
    uint32_t ph = 0;
    // (warps whose value columns there are none of have nothing to do)
    while (ok && (warp & 3) < X::LANE_WARPS && walk.next(&piece)) {
      fill_falls(piece);
      const int count = tokens_of(piece);
      // (stages that hold published states are not for these warps, but they follow them, or they could lose count of the rounds)
      for (int j = DK * slots_of(piece); j > 0 && ok; --j, ++n) {
        wait(&t->full[n % n_stages], (n / n_stages) & 1);
        tell(&t->slots_read[n % n_stages]);
      }
      for (int c = piece.c0; c < piece.c1; ++c) {
        const float* weight = t->fall[warp].at + FALL + min(C, count - c * C) - 1 - pair;       // weight[-s]: l^(n-1-s-pair), 0 behind the end
        wait(&t->full[n % n_stages], (n / n_stages) & 1);
        if (!ok) break;
        const uint32_t from = from0 + (n % n_stages) * X::STAGE;
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
        wait(&t->u_full, ph ^ 1u);                    // the last chunk's W has been used, and the factors of the one before
        if (!ok) break;
        tc_fence_after_sync();
        if (F16 && (lane & 3) == 0) {
#pragma unroll
          for (int i = 0; i < 4; ++i) t->lane_scale[ph][column0 + (lane >> 2) + 8 * i] = lift[i];
        }
#pragma unroll 1
        for (int s = 0; s < C; s += 32) {
          float f[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = weight[-s - (j >> 1) * 8 - (j & 1)];
#pragma unroll
          for (int g = 0; g < 2; ++g) {               // 16 value columns
            uint32_t raw[2][4], out[PARTS<F16>][8];
            ldmatrix_x4_trans(raw[0], from + row_of[g] + s * 128);
            ldmatrix_x4_trans(raw[1], from + row_of[g] + (s + 16) * 128);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const float2 y = pair16<F16>(raw[u >> 2][u & 3]);
              float a = y.x * f[2 * (u >> 1)], b = y.y * f[2 * (u >> 1) + 1];
              if (F16) {
                a *= lift[2 * g + (u & 1)];
                b *= lift[2 * g + (u & 1)];
              }
#pragma unroll
              for (int w = 0; w < PARTS<F16>; ++w) {
                out[w][u] = pack2<F16>(a, b);
                const float2 e = pair16<F16>(out[w][u]);
                a -= e.x;
                b -= e.y;
              }
            }
#pragma unroll
            for (int w = 0; w < PARTS<F16>; ++w)
              tmem_st_16x16(tmem + lane_base + ((uint32_t)(g * 16) << 16) + T_W + w * (C / 2) + s / 2, out[w]);
          }
        }
        tmem_st_wait();
        tc_fence_before_sync();
        tell(&t->w_ready);
        ph ^= 1u;
        ++n;
      }
    }
  } else if (warp >= W_STATE) {
    // ------------------------------------------------------------ the state
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(STATE_REGS));
    if ((warp & 3) < X::LANE_WARPS) {
      const int column = tid - W_STATE * 32;
      int n = 0;
      uint32_t ph = 0, out_ph = 0;                    // chunks, and chunks with results, before this one
      const uint32_t u_at = tmem + lane_base + T_U, copy_at = tmem + lane_base + T_COPY;
      float s[DK * 64];
      while (ok && walk.next(&piece)) {
        fill_falls(piece);
        const int count = tokens_of(piece), head = head_of(piece), global_column = slice_of(piece) * 128 + column;
        const bool here = global_column < v.value_dim;
        float* stored = v.pool + (((size_t)p.seqs[piece.i] * v.n_layers + p.layer) * v.n_heads + head) * v.head_floats() + global_column;
        // the state in front of the piece
#pragma unroll
        for (int k = 0; k < DK * 64; ++k)
          s[k] = piece.from == StatePiece::STORED && here && k < v.key_dim ? stored[(size_t)k * v.value_dim] : 0.0f;
        if (piece.from == StatePiece::PUBLISHED) {
          const double rate = p.rates[head];
          const long long start = t->line.cut(blockIdx.x) - piece.c0;
#pragma unroll
          for (int h = 0; h < DK; ++h)
            for (int j = piece.first; j < (int)blockIdx.x; ++j) {
              const long long to = t->line.cut(j + 1);
              if (t->line.cut(j) == to) continue;
              const int chunks = piece.c0 - (int)(to - start);           // between its end and this piece
              const float w = chunks == 0 ? 1.0f : (float)exp(-rate * C * chunks);
              wait(&t->full[n % n_stages], (n / n_stages) & 1);
              if (!ok) break;
              const float* from = reinterpret_cast<const float*>(ring + (n % n_stages) * X::STAGE) + column;
#pragma unroll
              for (int k = 0; k < 64; ++k) s[h * 64 + k] = fmaf(w, from[k * DV * 64], s[h * 64 + k]);
              tell(&t->slots_read[n % n_stages]);
              ++n;
            }
        }
        for (int c = piece.c0; c < piece.c1; ++c, ++n) {
          if (!piece.sum_only) {
            float lift = 1.0f;
            if (F16) {
              float m = 0.0f;
#pragma unroll
              for (int k = 0; k < DK * 64; ++k) m = fmaxf(m, fabsf(s[k]));
              lift = lift_of(m, 100);
            }
            wait(&t->o2_done, out_ph ^ 1u);           // the copy before has been used, and the results before that have their factors
            if (!ok) break;
            if (F16) t->copy_scale[out_ph][column] = reciprocal_of_power(lift);
#pragma unroll
            for (int h = 0; h < DK; ++h) {
              uint32_t w[32];
#pragma unroll
              for (int k = 0; k < 32; ++k) w[k] = pack2<F16>(s[h * 64 + 2 * k] * lift, s[h * 64 + 2 * k + 1] * lift);
              tmem_st_32x32(copy_at + h * 32, w);
            }
            tmem_st_wait();
            tc_fence_before_sync();
            tell(&t->copy_ready);
            out_ph ^= 1u;
          }
          const float decay = t->fall[warp].at[FALL + min(C, count - c * C)];
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
            for (int k = 0; k < 32; ++k)
              if (h * 32 + (k & ~15) < v.key_dim) s[h * 32 + k] = fmaf(decay, s[h * 32 + k], F16 ? __uint_as_float(u[k]) * back : __uint_as_float(u[k]));
          }
          ph ^= 1u;
        }
        if (!ok) break;
        // the state behind it
        if (piece.to == StatePiece::STORED) {
#pragma unroll
          for (int k = 0; k < DK * 64; ++k)
            if (here && k < v.key_dim) stored[(size_t)k * v.value_dim] = s[k];
        } else if (piece.to == StatePiece::PUBLISHED) {
          float* slot = p.slots + (size_t)blockIdx.x * p.slot_floats + column;
#pragma unroll
          for (int k = 0; k < DK * 64; ++k) slot[k * (DV * 64)] = s[k];
          __threadfence();
          __syncwarp();
          if (lane == 0) atomicAdd(p.flags + blockIdx.x, 1u);
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
    auto place = [&](int token, int eight) { return mine + token * 64 + ((eight ^ ((token >> 1) & 3)) << 4); };
    while (ok && (warp & 3) < X::LANE_WARPS && walk.next(&piece)) {
      if (piece.sum_only) continue;
      fill_falls(piece);
      const float* fall = t->fall[warp].at + FALL + 1 + pair;          // fall[t]: l^(t+pair+1)
      const int count = tokens_of(piece), first_column = slice_of(piece) * 128 + warp * 32;
      const int64_t token0 = first_token(piece);
      uint16_t* out = reinterpret_cast<uint16_t*>(const_cast<unsigned char*>(p.out.at)) + token0 * p.out.token_stride + head_of(piece) * p.out.head_stride +
                      first_column + (lane & 3) * 8;
      const bool here = first_column + (lane & 3) * 8 < v.value_dim;
      for (int c = piece.c0; c < piece.c1; ++c) {
        wait(&t->o_full, ph);
        if (!ok) break;
        tc_fence_after_sync();
        const int there = here ? min(C, count - c * C) : 0;
        uint16_t* to = out + (int64_t)c * C * p.out.token_stride;
        float copy[4];
        if (F16)
#pragma unroll
          for (int i = 0; i < 4; ++i) copy[i] = t->copy_scale[ph][warp * 32 + (lane >> 2) + 8 * i];
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {                 // 32 tokens
          float f[8];
          float2 one[4];
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = p.scale * fall[h * 32 + (j >> 1) * 8 + (j & 1)];
          if (F16)
#pragma unroll
            for (int j = 0; j < 4; ++j) one[j] = *reinterpret_cast<const float2*>(&t->token_scale[ph][h * 32 + j * 8 + pair]);
#pragma unroll
          for (int g = 0; g < 2; ++g) {               // 16 value columns
            uint32_t a[16], b[16], w[8];
            const uint32_t from = tmem + lane_base + ((uint32_t)(g * 16) << 16) + h * 32;
            tmem_ld_16x32(from + T_O1, a);
            tmem_ld_16x32(from + T_O2, b);
            tmem_ld_wait_for16(a);
            tmem_ld_wait_for16(b);
            if (g == 1 && h == 1) {
              tc_fence_before_sync();
              tell(&t->o_free);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                float y[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                  float o = p.scale;
                  if (F16) o *= x ? one[j].y : one[j].x;
                  y[x] = fmaf(F16 ? f[j * 2 + x] * copy[2 * g + r] : f[j * 2 + x], __uint_as_float(b[4 * j + 2 * r + x]),
                              o * __uint_as_float(a[4 * j + 2 * r + x]));
                }
                w[2 * j + r] = pack2<F16>(y[0], y[1]);
              }
#pragma unroll
            for (int j = 0; j < 4; j += 2)
              stmatrix_x4_trans(place(8 * (j + (lane >> 4)) + (lane & 7), g * 2 + ((lane >> 3) & 1)), w[2 * j], w[2 * j + 1], w[2 * j + 2], w[2 * j + 3]);
          }
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int row = i * 8 + (lane >> 2);
            uint4 w;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(place(row, lane & 3)));
            if (h * 32 + row < there) *reinterpret_cast<uint4*>(to + (h * 32 + row) * p.out.token_stride) = w;
          }
          __syncwarp();
        }
        ph ^= 1u;
      }
    }
  }
  if (!ok && lane == 0) state_report(v, KV_TIMEOUT);
  tc_fence_before_sync();
  __syncthreads();
  if (warp == W_PRODUCTS) tmem_dealloc(tmem, 512);
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
  return launch_overlapped(state_chunk_kernel<F16, DK, DV>, dim3((unsigned)sm_count), dim3(THREADS), (size_t)smem_bytes<F16, DK, DV>(stages), st, 1, p, maps,
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
  p.slices = (p.v.value_dim + 127) / 128;
  auto* go = f16 ? (k2 ? (v2 ? launch<true, 2, 2> : launch<true, 2, 1>) : (v2 ? launch<true, 1, 2> : launch<true, 1, 1>))
                 : (k2 ? (v2 ? launch<false, 2, 2> : launch<false, 2, 1>) : (v2 ? launch<false, 1, 2> : launch<false, 1, 1>));
  return go(p, maps, sm_count, smem_optin, st);
}

}  // namespace icc
