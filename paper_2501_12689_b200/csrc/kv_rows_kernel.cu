// Attention over the paged cache for more than 16 query rows per sequence and kv head and a head_dim of 129 to 256,
// which the tensor-memory kernel (kv_extend_kernel.cu) has no room for.
//
// One CTA per SM; an item is 32 query rows (tokens times query heads of a kv head).  A producer warp fetches 64-key
// tiles, one tensor-map box per page, 64-element column chunk and keys/values, into a ring of shared-memory
// stages (128-byte swizzle, so that the fragment loads below have no bank conflicts) and looks up page
// numbers two tiles ahead.  Eight warps consume: two 16-row tiles of the query times four key groups (halves of
// a tile, even and odd tiles).  Scores and weighted values are m16n8k16 products with fp32 accumulation; each
// warp keeps its own running maximum and sum and its own accumulator for its keys, which are merged once
// per item through shared memory.  With 32 rows per fetched key and value it is bound by the fetches from L2 and by
// these products in about equal parts.
//
// The weights are rounded to the cache's 16-bit type for the second product.  To lose nothing by that
// they are split in two such numbers (high part, remainder), twice the second product's instructions.
#include <type_traits>

#include "kernels.h"
#include "kv_mma.cuh"
#include "kv_schedule.cuh"
#include "pipeline.cuh"

namespace icc {

namespace {

constexpr int KEYS = 64;                 // keys per tile
constexpr int WARPS = 8;                 // consumer warps
constexpr int Q_WARPS = 3;               // warps that fetch query rows
constexpr int THREADS = WARPS * 32 + 32 + Q_WARPS * 32;
// Registers: launched with 168 a thread (the most that 384 threads can have); the producers' warpgroup gives
// part of its share to the two that hold accumulators.  384 x 168 = 256 x 216 + 128 x 72.
constexpr int PRODUCER_REGS = 72, CONSUMER_REGS = 216;
constexpr int MAX_STAGES = 12;
constexpr int WHOLE = 16;                // items of at most so many tiles are not cut (kv_schedule.cuh): 20 prompts of up to 600
                                         // tokens, head_dim 256, 1380 us cut everywhere, 1358 so

struct RowsTail {
  uint64_t full[MAX_STAGES], empty[MAX_STAGES], q_full, q_empty;
  float m[WARPS][16], l[WARPS][16];      // per consumer warp: its rows' maxima and sums
  float scale[64];                       // factors of the final step
  int abort_flag, last;
  KvBatch batch;
};

__host__ __device__ constexpr int stage_bytes(int dch) { return 2 * dch * KEYS * 128; }
__host__ __device__ constexpr int merge_stride(int dch) { return dch * 64 + 8; }    // floats; rows 8 banks apart: the quads of a fragment row spread out
__host__ __device__ constexpr int merge_bytes(int dch, int rt) { return 16 * rt * merge_stride(dch) * 4; }
__host__ __device__ constexpr int q_pitch(int dch) { return dch * 128 + 16; }           // bytes of a query row in shared memory
__host__ __device__ constexpr int q_bytes(int dch, int rt) { return 16 * rt * q_pitch(dch); }
int rows_smem(int dch, int rt, int stages) {
  return 1024 + stages * stage_bytes(dch) + merge_bytes(dch, rt) + q_bytes(dch, rt) + (int)sizeof(RowsTail);
}

template <int I, int N, typename F>
__device__ __forceinline__ void static_for(F f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<I + 1, N>(f);
  }
}
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

template <bool F16, int DCH, int RT>
__global__ void __launch_bounds__(THREADS, 1) kv_rows_kernel(const KvAttendParams p, const __grid_constant__ CUtensorMap tmap, int n_stages) {
  constexpr int ROWS = 16 * RT;
  constexpr int KG = WARPS / RT;                     // key groups: SLICES of a tile, times even and odd tiles
  constexpr int SLICES = KG / 2;
  constexpr int STEPS = KEYS / 16 / SLICES;          // 16-key steps of a warp in a tile
  constexpr int CHUNK = KEYS * 128;                  // bytes of one 64-element column chunk of a tile
  constexpr int KV_BYTES = DCH * CHUNK;              // keys of a tile; the values follow
  constexpr int STAGE = 2 * KV_BYTES;
  constexpr int PITCH = merge_stride(DCH);
  extern __shared__ unsigned char smem_raw[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* merge = reinterpret_cast<float*>(ring + n_stages * STAGE);
  unsigned char* q_smem = reinterpret_cast<unsigned char*>(merge) + merge_bytes(DCH, RT);
  RowsTail* t = reinterpret_cast<RowsTail*>(q_smem + q_bytes(DCH, RT));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const KvView& v = p.v;
  if (tid == 0) {
    for (int s = 0; s < n_stages; ++s) {
      mbar_init(&t->full[s], 1);
      mbar_init(&t->empty[s], WARPS / 2);
    }
    mbar_init(&t->q_full, Q_WARPS);
    mbar_init(&t->q_empty, WARPS);
    t->abort_flag = 0;
    mbar_fence_init();
    prefetch_tmap(&tmap);
  }
  grid_dep_launch_dependents();
  grid_dep_wait();   // queries, tables and pages come from earlier kernels in the stream
  kv_load_batch<ROWS, KEYS>(p, &t->batch);
  __syncthreads();
  KvWalk<ROWS, KEYS, WHOLE> walk(p, t->batch, blockIdx.x, gridDim.x);
  if (walk.done()) return;

  if (warp >= WARPS) {
    // ------------------------------------------------------------ producer
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PRODUCER_REGS));
    if (warp > WARPS) {
      // ---------------------------------------------------------- query rows: an item's are fetched while the one before it is worked on
      constexpr int PIECES = DCH * 8;                        // 16-byte pieces of a row
      uint32_t ph = 1;
      for (; !walk.done(); walk.next(), ph ^= 1u) {
        const KvSeq& seq = t->batch.seq[walk.i];
        const int rows = seq.count * p.group - walk.rt * ROWS;
        if (!mbar_wait(&t->q_empty, ph, &t->abort_flag)) {
          if (lane == 0) kv_report(v, KV_TIMEOUT);
          break;
        }
#pragma unroll 4
        for (int u = (warp - WARPS - 1) * 32 + lane; u < ROWS * PIECES; u += Q_WARPS * 32) {
          const int r = u / PIECES, piece = u - r * PIECES;
          uint4 w = make_uint4(0, 0, 0, 0);
          if (r < rows && piece * 8 < v.head_dim) {
            const int rr = walk.rt * ROWS + r, tok = kv_token_of(p, rr), hq = walk.head * p.group + (rr - tok * p.group);
            w = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p.q) + (int64_t)(seq.first + tok) * p.q_token_stride +
                                                (int64_t)hq * p.q_head_stride + piece * 8);
          }
          *reinterpret_cast<uint4*>(q_smem + r * q_pitch(DCH) + piece * 16) = w;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&t->q_full);
      }
      return;
    }
    const int per_tile = max(1, KEYS >> v.page_shift);     // pages of a tile
    const int box_rows = min(KEYS, 1 << v.page_shift);
    const uint32_t box_bytes = (uint32_t)box_rows * 128;
    const int page_rows = (v.n_layers * 2 * v.n_kv_heads) << v.page_shift;   // rows of the tensor map per page
    // What this lane loads of the next tile: its page (-1: nothing) and the first row in it.  The page number is
    // looked at only when the tile is issued, three tiles later, so that nothing waits for the table here.
    struct Ahead {
      int page, row;
    };
    const int n_tiles = walk.left;
    int k = walk.from;
    bool more = true;
    auto look = [&]() {
      Ahead a{-1, 0};
      if (more) {
        const KvSeq& s = t->batch.seq[walk.i];
        const int key0 = walk.r.tile(k) * KEYS;
        const int entry = (key0 >> v.page_shift) + lane;
        if (lane < per_tile && entry < kv_pages_of(s.length, v.page_shift)) a.page = v.tables[(size_t)s.slot * v.max_pages + entry];
        a.row = ((p.layer * 2 * v.n_kv_heads + walk.head) << v.page_shift) + (key0 & ((1 << v.page_shift) - 1));
        if (++k >= walk.to) {
          walk.next();
          more = !walk.done();
          if (more) k = walk.from;
        }
      }
      return a;
    };
    const int to_values = v.n_kv_heads << v.page_shift;
    Ahead a0 = look(), a1 = look(), a2 = look();
    int s = 0, lt = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (; lt < n_tiles; ++lt) {
      ok = mbar_wait(&t->empty[s], ph ^ 1u, &t->abort_flag);
      ok = __all_sync(FULL_MASK, ok);
      if (!ok) break;
      const bool mine = (unsigned)a0.page < (unsigned)v.n_pages;
      const unsigned who = __ballot_sync(FULL_MASK, mine);
      if (a0.page != -1 && !mine) kv_report(v, KV_INVALID);      // a borrowed table's entry that names no page
      if (lane == 0) mbar_arrive_expect_tx(&t->full[s], (uint32_t)__popc(who) * 2 * DCH * box_bytes);
      __syncwarp();
      if (mine) {
        const int y0 = a0.page * page_rows + a0.row;
        unsigned char* dst = ring + s * STAGE + lane * box_bytes;
#pragma unroll
        for (int c = 0; c < DCH; ++c) tma_load_2d(dst + c * CHUNK, &tmap, c * 64, y0, &t->full[s]);
#pragma unroll
        for (int c = 0; c < DCH; ++c) tma_load_2d(dst + KV_BYTES + c * CHUNK, &tmap, c * 64, y0 + to_values, &t->full[s]);
      }
      a0 = a1;
      a1 = a2;
      a2 = look();
      if (++s == n_stages) {
        s = 0;
        ph ^= 1u;
      }
    }
    if (!ok) {
      if (lane == 0) {
        kv_report(v, KV_TIMEOUT);
        // what is in flight lands before the CTA leaves
        for (int j = max(0, lt - n_stages); j < lt; ++j) {
          const long long t0 = clock64();
          while (!mbar_try_wait(&t->full[j % n_stages], (uint32_t)((j / n_stages) & 1)) && clock64() - t0 < WAIT_LIMIT_CYCLES) {
          }
        }
      }
    }
    return;
  }

  // -------------------------------------------------------------- consumers
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(CONSUMER_REGS));
  const int rtile = warp % RT, kg = warp / RT;       // 16-row tile and key group
  const int half = kg / SLICES, slice = kg % SLICES; // even or odd tiles, and where in them
  const int key_in_tile = slice * (STEPS * 16);
  const uint32_t ring_addr = smem_u32(ring);
  const int qr = lane >> 2, qc = (lane & 3) * 2;     // row and column pair of this thread in a fragment
  // ldmatrix: lane l gives the address of row (l & 7) of matrix l >> 3
  //   keys: matrices (keys 0-7, dims 0-7), (keys 0-7, dims 8-15), (keys 8-15, dims 0-7), (keys 8-15, dims 8-15)
  const int k_row = key_in_tile + (lane & 7) + ((lane >> 4) << 3), k_col = (lane >> 3) & 1;
  //   values, transposed: (keys 0-7, dims 0-7), (keys 8-15, dims 0-7), (keys 0-7, dims 8-15), (keys 8-15, dims 8-15)
  const int v_row = key_in_tile + (lane & 7) + (((lane >> 3) & 1) << 3), v_col = lane >> 4;
  //   queries: matrices (rows 0-7, dims 0-7), (rows 8-15, dims 0-7), (rows 0-7, dims 8-15), (rows 8-15, dims 8-15)
  const uint32_t q_addr = smem_u32(q_smem) + (rtile * 16 + (lane & 7) + (((lane >> 3) & 1) << 3)) * q_pitch(DCH) + (lane >> 4) * 16;
  int lt = 0, s = 0;                                 // tiles seen, and their stage and parity
  uint32_t ph = 0, q_ph = 0;
  bool ok = true;

  for (; !walk.done(); walk.next()) {
    const KvSeq seq = t->batch.seq[walk.i];
    const int rows = seq.count * p.group - walk.rt * ROWS;        // rows of this tile, if below ROWS
    int pos[2];                                                   // positions of this thread's two rows; -1 = no row
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int r = rtile * 16 + qr + x * 8;
      pos[x] = r < rows ? seq.length - seq.count + kv_token_of(p, walk.rt * ROWS + r) : -1;
    }
    uint32_t q[DCH * 4][4];
    if (ok) ok = mbar_wait(&t->q_full, q_ph, &t->abort_flag);
    q_ph ^= 1u;
#pragma unroll
    for (int c = 0; c < DCH * 4; ++c)
      ldmatrix_x4(q[c], q_addr + c * 32);
    __syncwarp();
    if (lane == 0) mbar_arrive(&t->q_empty);
    // positions of the first and last row of the warp's 16
    int lowest = 0x7fffffff, highest = -1;
    {
      const int r0 = rtile * 16, r1 = min(r0 + 16, rows) - 1;
      if (r0 < rows) {
        lowest = seq.length - seq.count + kv_token_of(p, walk.rt * ROWS + r0);
        highest = seq.length - seq.count + kv_token_of(p, walk.rt * ROWS + r1);
      }
    }
    float o[DCH * 8][4];
#pragma unroll
    for (int c = 0; c < DCH * 8; ++c)
#pragma unroll
      for (int x = 0; x < 4; ++x) o[c][x] = 0.0f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};

    const int to = walk.to;
    for (int k = walk.from; k < to; ++k, ++lt) {
      if ((lt & 1) == half) {
        if (ok) ok = mbar_wait(&t->full[s], ph, &t->abort_flag);
        const int key0 = walk.r.tile(k) * KEYS + key_in_tile;
        const uint32_t kbase = ring_addr + s * STAGE + k_row * 128, vbase = ring_addr + s * STAGE + KV_BYTES + v_row * 128;
        float sc[STEPS][2][4];
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
#pragma unroll
          for (int x = 0; x < 4; ++x) sc[st][0][x] = sc[st][1][x] = 0.0f;
#pragma unroll
          for (int c = 0; c < DCH * 4; ++c) {
            uint32_t b[4];
            ldmatrix_x4(b, kbase + (c >> 2) * CHUNK + st * 2048 + (((((c & 3) << 1) | k_col) ^ (k_row & 7)) << 4));
            mma16816<F16>(sc[st][0], q[c], b[0], b[1]);
            mma16816<F16>(sc[st][1], q[c], b[2], b[3]);
          }
        }
        // all of the warp's keys seen by all of its rows?
        const int last = key0 + STEPS * 16 - 1;
        const bool clear = last <= lowest && highest >= 0 && (!p.window || key0 > highest - p.window || last < p.sinks);
        float top[2] = {m[0], m[1]};
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
#pragma unroll
          for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              float y = sc[st][nt][x] * p.scale_log2;
              if (!clear) {
                const int j = key0 + st * 16 + nt * 8 + qc + (x & 1), pr = pos[x >> 1];
                const bool seen = j <= pr && (!p.window || j > pr - p.window || j < p.sinks);
                y = seen ? y : -INFINITY;
              }
              sc[st][nt][x] = y;
              top[x >> 1] = fmaxf(top[x >> 1], y);
            }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          top[x] = fmaxf(top[x], __shfl_xor_sync(FULL_MASK, top[x], 1));
          top[x] = fmaxf(top[x], __shfl_xor_sync(FULL_MASK, top[x], 2));
        }
        if (__any_sync(FULL_MASK, top[0] > m[0] || top[1] > m[1])) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float shrink = m[x] == -INFINITY ? 0.0f : exp2_fast(m[x] - top[x]);
            m[x] = top[x];
            l[x] *= shrink;
#pragma unroll
            for (int c = 0; c < DCH * 8; ++c) {
              o[c][2 * x] *= shrink;
              o[c][2 * x + 1] *= shrink;
            }
          }
        }
        // (a NaN score is no maximum; it reaches the sum and the result through its weight)
        const float base[2] = {m[0] == -INFINITY ? 0.0f : m[0], m[1] == -INFINITY ? 0.0f : m[1]};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              sc[st][nt][x] = exp2_fast(sc[st][nt][x] - base[x >> 1]);
              l[x >> 1] += sc[st][nt][x];
            }
            split2<F16>(sc[st][nt][0], sc[st][nt][1], &hi[2 * nt], &lo[2 * nt]);
            split2<F16>(sc[st][nt][2], sc[st][nt][3], &hi[2 * nt + 1], &lo[2 * nt + 1]);
          }
          // values of keys that none of the rows sees count as zeros, whatever they hold
          uint32_t keep[2] = {~0u, ~0u};
          if (!clear) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int j = key0 + st * 16 + qc + x * 8;
              keep[x] = 0;
              if (j <= highest && (!p.window || j > lowest - p.window || j < p.sinks)) keep[x] |= 0xffffu;
              if (j + 1 <= highest && (!p.window || j + 1 > lowest - p.window || j + 1 < p.sinks)) keep[x] |= 0xffff0000u;
            }
          }
#pragma unroll
          for (int c = 0; c < DCH * 4; ++c) {
            uint32_t b[4];
            ldmatrix_x4_trans(b, vbase + (c >> 2) * CHUNK + st * 2048 + (((((c & 3) << 1) | v_col) ^ (v_row & 7)) << 4));
            b[0] &= keep[0];
            b[1] &= keep[1];
            b[2] &= keep[0];
            b[3] &= keep[1];
            mma16816<F16>(o[2 * c], hi, b[0], b[1]);
            mma16816<F16>(o[2 * c], lo, b[0], b[1]);
            mma16816<F16>(o[2 * c + 1], hi, b[2], b[3]);
            mma16816<F16>(o[2 * c + 1], lo, b[2], b[3]);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&t->empty[s]);
      }
      if (++s == n_stages) {
        s = 0;
        ph ^= 1u;
      }
    }

    // ---- merge the key groups: common maximum per row, then the accumulators column group by column group
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      l[x] += __shfl_xor_sync(FULL_MASK, l[x], 1);
      l[x] += __shfl_xor_sync(FULL_MASK, l[x], 2);
    }
    if ((lane & 3) == 0) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        t->m[warp][qr + 8 * x] = m[x];
        t->l[warp][qr + 8 * x] = l[x];
      }
    }
    consumers_sync();
    float big[2], sum[2], part[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      big[x] = -INFINITY;
#pragma unroll
      for (int g = 0; g < KG; ++g) big[x] = fmaxf(big[x], t->m[g * RT + rtile][qr + 8 * x]);
      const float b0 = big[x] == -INFINITY ? 0.0f : big[x];
      sum[x] = 0.0f;
#pragma unroll
      for (int g = 0; g < KG; ++g) sum[x] += t->l[g * RT + rtile][qr + 8 * x] * exp2_fast(t->m[g * RT + rtile][qr + 8 * x] - b0);
      part[x] = exp2_fast(m[x] - b0);
    }
    // round r: group kg adds its columns of part (kg + r) mod KG, so that all warps work and none collide
    constexpr int CT = DCH * 8 / KG;                 // 8-column tiles per part
#pragma unroll 1
    for (int r = 0; r < KG; ++r) {
      static_for<0, KG>([&](auto part_no) {
        constexpr int c0 = decltype(part_no)::value;
        if (((kg + r) & (KG - 1)) == c0) {
          asm volatile("" ::"n"(c0));                // keeps the branches apart: merged, they would index registers at run time
#pragma unroll
          for (int c = c0 * CT; c < (c0 + 1) * CT; ++c)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float2* at = reinterpret_cast<float2*>(merge + (rtile * 16 + qr + 8 * x) * PITCH + c * 8 + qc);
              float2 w = make_float2(o[c][2 * x] * part[x], o[c][2 * x + 1] * part[x]);
              if (r > 0) {
                const float2 have = *at;
                w.x += have.x;
                w.y += have.y;
              }
              *at = w;
            }
        }
      });
      if (r == 0 && kg == 0 && (lane & 3) == 0) {
#pragma unroll
        for (int x = 0; x < 2; ++x) t->scale[rtile * 16 + qr + 8 * x] = sum[x];
      }
      consumers_sync();
    }
    if (kg == 0 && (lane & 3) == 0) {                // the rows' common maxima, for a partial result (read after the next barrier)
#pragma unroll
      for (int x = 0; x < 2; ++x) t->m[warp][qr + 8 * x] = big[x];
    }

    const bool whole = walk.whole();
    float* slot = p.partials + (size_t)walk.my_slot(blockIdx.x) * p.partial_floats;
    const int live = min(rows, ROWS);
    auto put = [&](int r, int d, float a, float b) {              // two values of one row of the result
      const int rr = walk.rt * ROWS + r, tok = kv_token_of(p, rr), hq = walk.head * p.group + (rr - tok * p.group);
      uint16_t* to16 = reinterpret_cast<uint16_t*>(p.out) + (int64_t)(seq.first + tok) * p.out_token_stride + (int64_t)hq * p.out_head_stride + d;
      *reinterpret_cast<uint32_t*>(to16) = pack2<F16>(a, b);
    };
    if (whole) {
      for (int r = warp; r < live; r += WARPS) {
        const float total = t->scale[r], inv = total == 0.0f ? 0.0f : 1.0f / total;
        for (int d = lane * 2; d < v.head_dim; d += 64) {
          const float2 w = *reinterpret_cast<const float2*>(merge + r * PITCH + d);
          put(r, d, w.x * inv, w.y * inv);
        }
      }
    } else {
      consumers_sync();
      // layout of a partial result: ROWS maxima, ROWS sums, ROWS x 64 * DCH values
      for (int r = warp; r < live; r += WARPS) {
        if (lane == 0) {
          slot[r] = t->m[r >> 4][r & 15];
          slot[ROWS + r] = t->scale[r];
        }
        for (int d = lane * 2; d < v.head_dim; d += 64)
          *reinterpret_cast<float2*>(slot + 2 * ROWS + r * (DCH * 64) + d) = *reinterpret_cast<const float2*>(merge + r * PITCH + d);
      }
      consumers_sync();
      const auto pieces = walk.pieces();
      const int n_parts = pieces.n;
      if (tid == 0) {
        t->last = kv_arrive(&p.arrivals[pieces.first]) == n_parts - 1;
        if (t->last) p.arrivals[pieces.first] = 0;   // ready for the next launch
      }
      consumers_sync();
      if (t->last) {
        // Join the pieces, in the order of the CTAs: a warp per row, lanes along the row, JOIN loads in
        // flight per lane (the pieces come from L2, a microsecond away).
        constexpr int VPL = (DCH + 1) / 2;           // 16-byte vectors of a row per lane
        constexpr int SIDE = DCH == 1 ? 2 : 1;       // pieces side by side in a warp
        constexpr int JOIN = 16 / VPL;
        auto part_at = [&](int c) { return p.partials + (size_t)pieces.slot(c) * p.partial_floats; };
        const int side = SIDE == 2 ? lane >> 4 : 0, col = (SIDE == 2 ? lane & 15 : lane) * 4;
        for (int r = warp; r < live; r += WARPS) {
          float w[KV_MAX_CTAS / 32], total = 0.0f, top = -INFINITY;
#pragma unroll
          for (int x = 0; x < KV_MAX_CTAS / 32; ++x) w[x] = x * 32 + lane < n_parts ? __ldcg(part_at(x * 32 + lane) + r) : -INFINITY;
#pragma unroll
          for (int x = 0; x < KV_MAX_CTAS / 32; ++x) top = fmaxf(top, w[x]);
#pragma unroll
          for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL_MASK, top, d));
          const float b0 = top == -INFINITY ? 0.0f : top;
#pragma unroll
          for (int x = 0; x < KV_MAX_CTAS / 32; ++x) {
            w[x] = exp2_fast(w[x] - b0);
            if (x * 32 + lane < n_parts) total += w[x] * __ldcg(part_at(x * 32 + lane) + ROWS + r);
          }
          float4 acc[VPL];
#pragma unroll
          for (int x = 0; x < VPL; ++x) acc[x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
          for (int x = 0; x < KV_MAX_CTAS / 32; ++x) {
            for (int cb = 0; cb < 32 && x * 32 + cb < n_parts; cb += JOIN * SIDE) {
              float4 y[JOIN][VPL];
#pragma unroll
              for (int u = 0; u < JOIN; ++u)
#pragma unroll
                for (int z = 0; z < VPL; ++z) {
                  const int c = x * 32 + cb + u * SIDE + side, d = z * 128 + col;
                  y[u][z] = (c < n_parts && d < v.head_dim) ? __ldcg(reinterpret_cast<const float4*>(part_at(c) + 2 * ROWS + r * (DCH * 64) + d))
                                                            : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                }
#pragma unroll
              for (int u = 0; u < JOIN; ++u) {
                const float wc = __shfl_sync(FULL_MASK, w[x], (cb + u * SIDE + side) & 31);
#pragma unroll
                for (int z = 0; z < VPL; ++z) {
                  acc[z].x += wc * y[u][z].x;
                  acc[z].y += wc * y[u][z].y;
                  acc[z].z += wc * y[u][z].z;
                  acc[z].w += wc * y[u][z].w;
                }
              }
            }
          }
#pragma unroll
          for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(FULL_MASK, total, d);
          if (SIDE == 2) {
            acc[0].x += __shfl_xor_sync(FULL_MASK, acc[0].x, 16);
            acc[0].y += __shfl_xor_sync(FULL_MASK, acc[0].y, 16);
            acc[0].z += __shfl_xor_sync(FULL_MASK, acc[0].z, 16);
            acc[0].w += __shfl_xor_sync(FULL_MASK, acc[0].w, 16);
          }
          const float inv = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
          for (int z = 0; z < VPL; ++z) {
            const int d = z * 128 + col;
            if (side == 0 && d < v.head_dim) {
              put(r, d, acc[z].x * inv, acc[z].y * inv);
              put(r, d + 2, acc[z].z * inv, acc[z].w * inv);
            }
          }
        }
      }
    }
  }
  if (!ok && lane == 0) kv_report(v, KV_TIMEOUT);
}

template <bool F16, int DCH>
cudaError_t launch_one(const KvAttendParams& p, const CUtensorMap& tmap, int sm_count, int smem_optin, cudaStream_t st) {
  // An even number of stages, so that a stage always belongs to the same half of the consumers: a warp that met
  // a stage's barrier at every other round only could not tell a round's parity from that of two rounds before.
  int stages = 2;
  while (stages + 2 <= MAX_STAGES && rows_smem(DCH, 2, stages + 2) <= smem_optin) stages += 2;
  return launch_overlapped(kv_rows_kernel<F16, DCH, 2>, dim3(sm_count), dim3(THREADS), rows_smem(DCH, 2, stages), st, 1, p, tmap, stages);
}

}  // namespace

cudaError_t kv_rows_configure(int smem_optin) {
  cudaError_t e = cudaFuncSetAttribute(kv_rows_kernel<false, 3, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kv_rows_kernel<false, 4, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kv_rows_kernel<true, 3, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kv_rows_kernel<true, 4, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin);
  return e;
}

size_t kv_rows_partial_floats(int head_dim) { return (size_t)32 * (2 + (head_dim + 63) / 64 * 64); }

cudaError_t kv_rows_launch(const KvAttendParams& p, const CUtensorMap& tmap, bool f16, int sm_count, int smem_optin, cudaStream_t st) {
  if (p.v.head_dim <= 192) return f16 ? launch_one<true, 3>(p, tmap, sm_count, smem_optin, st) : launch_one<false, 3>(p, tmap, sm_count, smem_optin, st);
  return f16 ? launch_one<true, 4>(p, tmap, sm_count, smem_optin, st) : launch_one<false, 4>(p, tmap, sm_count, smem_optin, st);
}

}  // namespace icc
