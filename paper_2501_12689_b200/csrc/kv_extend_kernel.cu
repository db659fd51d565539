// Attention over the paged cache for many query rows: prompts, on the tensor cores (tcgen05), head_dim <= 128.
//
// An item is 256 rows of one sequence and kv head (tokens times query heads of the kv head), two tiles A and
// B of 128 that share every key and value fetched.  Per 128-key tile and row tile there are two products,
// S = Q K^T and O += P V, of 128 x 128 x head_dim each, with S, P and O in tensor memory (512 columns: S_A, S_B,
// O_A, O_B; P, 16 bit, takes the first 64 columns of its S).  The same work needs 128 x 128 exponentials, for
// which the special-function units take as long as the tensor cores do for the products (2,048 cycles
// each for both row tiles); neither may wait for the other.  Hence the two row tiles: while one's scores are turned
// into weights, the tensor cores work for the other one.
//
//   warps 0-3, 4-7   softmax of row tile A, B: a thread owns a row (a tensor-memory lane)
//   warp 8           loads of keys and values: one tensor-map box per page (or 64 rows) and 64-element chunk
//   warp 9           issues the products: PV_A(j), S_A(j+1), PV_B(j), S_B(j+1), ...
//   warps 10, 11     query rows of the next item, into the swizzled layout of the left operand
//
// A row's maximum is only raised when it is exceeded by more than 2^8: O is rescaled a few times per item and not
// per tile, and weights of up to 256 are as exact as those up to 1.  Weights are rounded to the cache's
// 16-bit type (the tensor cores take both operands in one type); their sum is taken before the rounding.
#include "kernels.h"
#include "kv_mma.cuh"
#include "kv_schedule.cuh"
#include "pipeline.cuh"

namespace icc {

namespace {

constexpr int KEYS = 128;                // keys per tile
constexpr int ROWS = 256;                // rows per item
constexpr int SOFTMAX_WARPS = 8;
constexpr int THREADS = 384;
constexpr int MAX_SLOTS = 8;             // of the key/value ring
// Registers: launched with 168 a thread; the softmax warpgroups take from the third: 384 x 168 = 256 x 216 + 128 x 72.
constexpr int OTHER_REGS = 72, SOFTMAX_REGS = 216;
constexpr float RAISE = 8.0f;            // how far (log2) a row's scores may exceed its maximum before O is rescaled
constexpr int AHEAD = 3;                 // batches of page numbers under way

struct ExtendTail {
  uint64_t full[MAX_SLOTS], empty[MAX_SLOTS], q_full, q_empty;
  uint64_t s_full[2], p_full[2], o_full[2], drain;
  uint32_t tmem_base;
  int abort_flag, last[2];
  KvBatch batch;
};

__host__ __device__ constexpr int slot_bytes(int dch) { return dch * KEYS * 128; }
int extend_smem(int dch, int slots) { return 1024 + ROWS * dch * 128 + slots * slot_bytes(dch) + (int)sizeof(ExtendTail); }

// Instruction descriptor: A and B 16-bit floats of one type, fp32 accumulator, M = 128.
__host__ __device__ constexpr uint32_t idesc(bool f16, int n, bool b_mn_major) {
  return (1u << 4) | (f16 ? 0u : (1u << 7) | (1u << 10)) | (b_mn_major ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}
// Operand whose rows (keys) are the summed dimension: 64-element chunks of the other one `chunk` bytes apart, groups of
// eight rows 1024 bytes apart, 128-byte swizzle.
__device__ __forceinline__ uint64_t desc_mn_major_sw128(uint32_t smem_addr, uint32_t chunk) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr & 0x3ffffu) >> 4);
  d |= (uint64_t)(chunk >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
// D[tmem] (+)= A[tmem] * B[smem], issued by one thread.
__device__ __forceinline__ void umma_from_tmem(uint32_t tmem_d, uint32_t tmem_a, uint64_t desc_b, uint32_t id, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "}\n" ::"r"(tmem_d),
      "r"(tmem_a), "l"(desc_b), "r"(id), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st_32x32(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
      "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]),
      "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// As tmem_ld_wait, for 32 registers that are about to be used.
__device__ __forceinline__ void tmem_ld_wait_for32(uint32_t* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                 "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]),
                 "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]),
                 "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
               :
               : "memory");
}
// Generic writes to shared memory become visible to the tensor cores and copies.
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void cp_async_16(uint32_t smem_dst, const void* src, bool there) {
  const int bytes = there ? 16 : 0;      // the rest is filled with zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// The lowest n bits, n <= 0: none, n >= 32: all.
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : (n >= 32 ? ~0u : (1u << n) - 1u); }
__device__ __forceinline__ void warpgroup_sync(int which) {
  if (which == 0) asm volatile("bar.sync 1, 128;" ::: "memory");
  else asm volatile("bar.sync 2, 128;" ::: "memory");
}

template <bool F16, int DCH>
__global__ void __launch_bounds__(THREADS, 1) kv_extend_kernel(const KvAttendParams p, const __grid_constant__ CUtensorMap tmap, int n_slots) {
  constexpr int DIM = DCH * 64;                      // head_dim, padded
  constexpr int CHUNK = KEYS * 128;                  // bytes of a 64-element column chunk of 128 rows
  constexpr int SLOT = slot_bytes(DCH);
  constexpr int Q_TILE = DCH * CHUNK;                // bytes of a row tile of the query
  constexpr uint32_t TMEM_O = 256;                   // first column of O_A; S_A at 0, S_B at 128, O_B at 256 + 128
  extern __shared__ unsigned char smem_raw[];
  unsigned char* q_smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* ring = q_smem + 2 * Q_TILE;
  ExtendTail* t = reinterpret_cast<ExtendTail*>(ring + n_slots * SLOT);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const KvView& v = p.v;
  if (tid == 0) {
    for (int s = 0; s < n_slots; ++s) {
      mbar_init(&t->full[s], 1);
      mbar_init(&t->empty[s], 1);
    }
    mbar_init(&t->q_full, 2);
    mbar_init(&t->q_empty, 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(&t->s_full[x], 1);
      mbar_init(&t->p_full[x], 4);
      mbar_init(&t->o_full[x], 1);
    }
    mbar_init(&t->drain, 1);
    t->abort_flag = 0;
    mbar_fence_init();
    prefetch_tmap(&tmap);
  }
  if (warp == 9) tmem_alloc(&t->tmem_base, 512);
  grid_dep_launch_dependents();
  grid_dep_wait();   // queries, tables and pages come from earlier kernels in the stream
  kv_load_batch<ROWS, KEYS>(p, &t->batch);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = t->tmem_base;
  KvWalk<ROWS, KEYS> walk(p, t->batch, blockIdx.x, gridDim.x);

  if (warp >= SOFTMAX_WARPS) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
    if (warp == 8) {
      // ---------------------------------------------------------- keys and values
      const int per_tile = max(1, KEYS >> v.page_shift);         // pages of a tile
      const int per_batch = 32 / per_tile;
      const int box_rows = min(64, 1 << v.page_shift), boxes = KEYS / box_rows;
      const uint32_t box_bytes = (uint32_t)box_rows * 128;
      const int page_mask = (1 << v.page_shift) - 1;
      const int page_rows = (v.n_layers * 2 * v.n_kv_heads) << v.page_shift;
      const int to_values = v.n_kv_heads << v.page_shift;
      struct Batch {
        int page;           // this lane's page number, -1 = none
        int key, n, row;    // first key, tiles, first row of the head in a page
      };
      int k = walk.from;
      auto look = [&]() {
        Batch b{-1, 0, 0, 0};
        if (!walk.done()) {
          const KvSeq& s = t->batch.seq[walk.i];
          const int stop = k < walk.r.sink_tiles ? min(walk.to, walk.r.sink_tiles) : walk.to;
          b.key = walk.r.tile(k) * KEYS;
          b.n = min(stop - k, per_batch);
          b.row = (p.layer * 2 * v.n_kv_heads + walk.head) << v.page_shift;
          const int entry = (b.key >> v.page_shift) + lane;
          if (entry < kv_pages_of(s.length, v.page_shift)) b.page = v.tables[(size_t)s.slot * v.max_pages + entry];
          k += b.n;
          if (k >= walk.to) {
            walk.next();
            k = walk.from;
          }
        }
        return b;
      };
      int left = walk.left, s = 0, n = 0;
      uint32_t ph = 0;
      bool ok = true;
      Batch ahead[AHEAD];
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) ahead[x] = look();
      while (left > 0 && ok) {
        const Batch b = ahead[0];
#pragma unroll
        for (int x = 0; x + 1 < AHEAD; ++x) ahead[x] = ahead[x + 1];
        ahead[AHEAD - 1] = look();
        left -= b.n;
        const bool exists = (unsigned)b.page < (unsigned)v.n_pages;
        if (b.page != -1 && !exists) kv_report(v, KV_INVALID);
        const int y_page = exists ? b.page * page_rows + b.row : -1;
        const int e0 = b.key >> v.page_shift;
        for (int j = 0; j < b.n && ok; ++j) {
          const int key = b.key + j * KEYS + lane * box_rows;    // first key of this lane's box
          int y = __shfl_sync(FULL_MASK, y_page, ((key >> v.page_shift) - e0) & 31);
          if (lane >= boxes) y = -1;
          const unsigned who = __ballot_sync(FULL_MASK, y >= 0);
          if (y >= 0) y += key & page_mask;
          for (int values = 0; values < 2; ++values) {
            ok = __all_sync(FULL_MASK, mbar_wait(&t->empty[s], ph ^ 1u, &t->abort_flag));
            if (!ok) break;
            if (lane == 0) mbar_arrive_expect_tx(&t->full[s], (uint32_t)__popc(who) * DCH * box_bytes);
            __syncwarp();
            if (y >= 0) {
              unsigned char* dst = ring + s * SLOT + lane * box_bytes;
#pragma unroll
              for (int c = 0; c < DCH; ++c) tma_load_2d(dst + c * CHUNK, &tmap, c * 64, y + values * to_values, &t->full[s]);
            }
            ++n;
            if (++s == n_slots) {
              s = 0;
              ph ^= 1u;
            }
          }
        }
      }
      if (!ok && lane == 0) {
        kv_report(v, KV_TIMEOUT);
        for (int j = max(0, n - n_slots); j < n; ++j) {          // what is in flight lands before the CTA leaves
          const long long t0 = clock64();
          while (!mbar_try_wait(&t->full[j % n_slots], (uint32_t)((j / n_slots) & 1)) && clock64() - t0 < WAIT_LIMIT_CYCLES) {
          }
        }
      }
    } else if (warp == 9) {
      // ---------------------------------------------------------- products
      constexpr uint32_t id_s = idesc(F16, KEYS, false), id_o = idesc(F16, DIM, true);
      const uint32_t q_addr = smem_u32(q_smem), ring_addr = smem_u32(ring);
      int s = 0;                                     // next slot of the ring
      uint32_t ph = 0, q_ph = 0, p_ph[2] = {0, 0};
      bool ok = true;
      auto advance = [&]() {
        if (++s == n_slots) {
          s = 0;
          ph ^= 1u;
        }
      };
      auto scores = [&](int x, int slot) {           // S_x = Q_x K^T
#pragma unroll
        for (int c = 0; c < DCH; ++c) {
          const uint64_t da = umma_desc_k_major_sw128(q_addr + x * Q_TILE + c * CHUNK), db = umma_desc_k_major_sw128(ring_addr + slot * SLOT + c * CHUNK);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) umma_bf16(tmem + x * 128, da + kk * 2, db + kk * 2, id_s, (c | kk) != 0 ? 1u : 0u);
        }
        umma_commit(&t->s_full[x]);
      };
      auto values = [&](int x, int slot, bool add) { // O_x (+)= P_x V
        const uint64_t db = desc_mn_major_sw128(ring_addr + slot * SLOT, CHUNK);
#pragma unroll
        for (int kk = 0; kk < KEYS / 16; ++kk)       // 16 keys further: 8 columns of P, 2048 bytes of V
          umma_from_tmem(tmem + TMEM_O + x * 128, tmem + x * 128 + kk * 8, db + kk * 128, id_o, (add || kk != 0) ? 1u : 0u);
      };
      for (; !walk.done() && ok; walk.next()) {
        const KvSeq& seq = t->batch.seq[walk.i];
        const bool two = seq.count * p.group - walk.rt * ROWS > 128;
        // what the call's tokens of this sequence see: keys below `sinks` and from `first_seen` on
        const int first_seen = p.window ? max(0, seq.length - seq.count - p.window + 1) : 0;
        ok = mbar_wait(&t->q_full, q_ph, &t->abort_flag) && mbar_wait(&t->full[s], ph, &t->abort_flag);
        q_ph ^= 1u;
        if (!__all_sync(FULL_MASK, ok)) {
          ok = false;
          break;
        }
        tc_fence_after_sync();
        if (lane == 0) {
          scores(0, s);
          if (two) scores(1, s);
          umma_commit(&t->empty[s]);
          if (walk.from + 1 == walk.to) umma_commit(&t->q_empty);
        }
        __syncwarp();
        advance();
        for (int k = walk.from; k < walk.to; ++k) {
          const bool more = k + 1 < walk.to;
          const int sv = s;
          ok = __all_sync(FULL_MASK, mbar_wait(&t->full[s], ph, &t->abort_flag));
          if (!ok) break;
          advance();
          // Values of keys that no token of the call sees count as zeros, whatever is there (slots past the
          // end, tokens that have left the window): a weight of zero would not undo an infinity or a NaN.
          const int key0 = walk.r.tile(k) * KEYS;
          const int gap = max(key0, p.sinks), gap_end = min(key0 + KEYS, first_seen), tail = max(key0, seq.length);
          if (gap < gap_end || tail < key0 + KEYS) {
            constexpr int PIECES = DCH * 8;
            for (int u = lane; u < KEYS * PIECES; u += 32) {
              const int r = u / PIECES, j = key0 + r, piece = u % PIECES;
              if ((j >= gap && j < gap_end) || j >= tail)
                *reinterpret_cast<uint4*>(ring + sv * SLOT + (piece >> 3) * CHUNK + r * 128 + (piece & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_async_shared();
            __syncwarp();
          }
          if (more) {
            ok = __all_sync(FULL_MASK, mbar_wait(&t->full[s], ph, &t->abort_flag));
            if (!ok) break;
          }
          for (int x = 0; x < (two ? 2 : 1) && ok; ++x) {
            ok = __all_sync(FULL_MASK, mbar_wait(&t->p_full[x], p_ph[x], &t->abort_flag));
            if (!ok) break;
            p_ph[x] ^= 1u;
            tc_fence_after_sync();
            if (lane == 0) {
              values(x, sv, k > walk.from);
              if (more) scores(x, s);
              else umma_commit(&t->o_full[x]);
            }
            __syncwarp();
          }
          if (!ok) break;
          if (lane == 0) {
            umma_commit(&t->empty[sv]);
            if (more) umma_commit(&t->empty[s]);
            if (k + 2 == walk.to) umma_commit(&t->q_empty);      // the last scores of the item are under way
          }
          __syncwarp();
          if (more) advance();
        }
      }
      if (lane == 0) {
        // nothing issued is still running when tensor memory is released
        umma_commit(&t->drain);
        const long long t0 = clock64();
        while (!mbar_try_wait(&t->drain, 0) && clock64() - t0 < WAIT_LIMIT_CYCLES) {
        }
        if (!ok) kv_report(v, KV_TIMEOUT);
      }
    } else {
      // ---------------------------------------------------------- query rows
      constexpr int PIECES = DCH * 8;
      const uint32_t q_addr = smem_u32(q_smem);
      uint32_t ph = 1;
      for (; !walk.done(); walk.next(), ph ^= 1u) {
        const KvSeq& seq = t->batch.seq[walk.i];
        const int rows = min(ROWS, seq.count * p.group - walk.rt * ROWS);
        if (!mbar_wait(&t->q_empty, ph, &t->abort_flag)) {
          if (lane == 0) kv_report(v, KV_TIMEOUT);
          break;
        }
        const int fill = rows > 128 ? 256 : 128;     // the rest of a tile is zeros
        const int first = (warp - 10) * 32 + lane, piece = first % PIECES;     // a thread's pieces are in one column
        const bool column = piece * 8 < v.head_dim;
        const uint16_t* base = reinterpret_cast<const uint16_t*>(p.q) + (int64_t)seq.first * p.q_token_stride +
                               (int64_t)walk.head * p.group * p.q_head_stride + (column ? piece * 8 : 0);
#pragma unroll 4
        for (int r = first / PIECES; r < fill; r += 64 / PIECES) {
          const bool there = r < rows && column;
          const int rr = walk.rt * ROWS + (there ? r : 0), tok = kv_token_of(p, rr);
          const uint16_t* from = base + (int64_t)tok * p.q_token_stride + (int64_t)(rr - tok * p.group) * p.q_head_stride;
          cp_async_16(q_addr + (r >> 7) * Q_TILE + (piece >> 3) * CHUNK + (r & 127) * 128 + (((piece & 7) ^ (r & 7)) << 4), from, there);
        }
        cp_async_wait_all();
        fence_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(&t->q_full);
      }
    }
  } else {
    // ------------------------------------------------------------ softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFTMAX_REGS));
    const int x = warp >> 2, row = tid & 127;        // row tile, and row (tensor-memory lane) of this thread
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lane_base + x * 128, o_addr = tmem + lane_base + TMEM_O + x * 128;
    uint32_t s_ph = 0, o_ph = 0;
    bool ok = true;
    for (; !walk.done(); walk.next()) {
      const KvSeq seq = t->batch.seq[walk.i];
      const int rows = seq.count * p.group - walk.rt * ROWS - x * 128;        // of this row tile, if below 128
      if (rows <= 0) continue;
      const bool live = row < rows;
      // a row that is not there goes along with the last one that is, and is not written
      const int rr = walk.rt * ROWS + x * 128 + min(row, rows - 1), tok = kv_token_of(p, rr), hq = walk.head * p.group + (rr - tok * p.group);
      const int pos = seq.length - seq.count + tok;
      const int lowest = __shfl_sync(FULL_MASK, pos, 0), highest = __shfl_sync(FULL_MASK, pos, 31);     // of the warp's rows
      float m = -INFINITY, l = 0.0f;
      for (int k = walk.from; k < walk.to; ++k) {
        if (ok) ok = mbar_wait(&t->s_full[x], s_ph, &t->abort_flag);
        s_ph ^= 1u;
        __syncwarp();
        tc_fence_after_sync();
        uint32_t va[64], vb[64];
        tmem_ld_32x64(s_addr, va);
        tmem_ld_32x64(s_addr + 64, vb);
        tmem_ld_wait_for(va);
        tmem_ld_wait_for(vb);
        const int key0 = walk.r.tile(k) * KEYS, last = key0 + KEYS - 1;
        const bool clear = last <= lowest && (!p.window || key0 > highest - p.window || last < p.sinks);
        float scale = p.scale_log2;
        if (!clear) {
          // one bit per key: at or before the row's position, and in its window or a sink
          uint32_t seen[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int j = key0 + y * 32;
            seen[y] = bits_below(pos - j + 1);
            if (p.window) seen[y] &= ~bits_below(pos - p.window + 1 - j) | bits_below(p.sinks - j);
          }
#pragma unroll
          for (int i = 0; i < 64; ++i) {
            va[i] = (seen[i >> 5] >> (i & 31)) & 1u ? __float_as_uint(__uint_as_float(va[i]) * scale) : 0xff800000u;
            vb[i] = (seen[2 + (i >> 5)] >> (i & 31)) & 1u ? __float_as_uint(__uint_as_float(vb[i]) * scale) : 0xff800000u;
          }
          scale = 1.0f;
        }
        float top;
        if (scale >= 0.0f) {
          float g[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < 64; i += 4) {
#pragma unroll
            for (int y = 0; y < 4; ++y) g[y] = fmax3(g[y], __uint_as_float(va[i + y]), __uint_as_float(vb[i + y]));
          }
          top = fmaxf(fmax3(g[0], g[1], g[2]), g[3]) * scale;
        } else {
          float g = INFINITY;
#pragma unroll
          for (int i = 0; i < 64; ++i) g = fminf(g, fminf(__uint_as_float(va[i]), __uint_as_float(vb[i])));
          top = g * scale;
        }
        const bool raise = top > m + RAISE || (m == -INFINITY && top > -INFINITY);
        if (__any_sync(FULL_MASK, raise)) {
          const float now = raise ? top : m;
          const float shrink = raise ? (m == -INFINITY ? 0.0f : exp2_fast(m - now)) : 1.0f;
          m = now;
          l *= shrink;
          if (k > walk.from) {                       // S(k) is complete, and with it everything issued before it: PV(k - 1) too
#pragma unroll 1
            for (int c = 0; c < DIM; c += 32) {
              uint32_t o[32];
              tmem_ld_32x32(o_addr + c, o);
              tmem_ld_wait_for32(o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * shrink);
              tmem_st_32x32(o_addr + c, o);
            }
          }
        }
        const float base = m == -INFINITY ? 0.0f : m;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        uint32_t w[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const float a = exp2_fast(fmaf(__uint_as_float(va[2 * i]), scale, -base)), b = exp2_fast(fmaf(__uint_as_float(va[2 * i + 1]), scale, -base));
          sum[(2 * i) & 3] += a;
          sum[(2 * i + 1) & 3] += b;
          w[i] = pack2<F16>(a, b);
        }
        tmem_st_32x32(s_addr, w);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const float a = exp2_fast(fmaf(__uint_as_float(vb[2 * i]), scale, -base)), b = exp2_fast(fmaf(__uint_as_float(vb[2 * i + 1]), scale, -base));
          sum[(2 * i) & 3] += a;
          sum[(2 * i + 1) & 3] += b;
          w[i] = pack2<F16>(a, b);
        }
        tmem_st_32x32(s_addr + 32, w);
        tmem_st_wait();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&t->p_full[x]);
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
      // ---- the result, or a piece of it
      if (ok) ok = mbar_wait(&t->o_full[x], o_ph, &t->abort_flag);
      o_ph ^= 1u;
      __syncwarp();
      tc_fence_after_sync();
      uint16_t* to = reinterpret_cast<uint16_t*>(p.out) + (int64_t)(seq.first + tok) * p.out_token_stride + (int64_t)hq * p.out_head_stride;
      if (walk.whole()) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll 1
        for (int c = 0; c < DIM; c += 32) {
          uint32_t o[32];
          tmem_ld_32x32(o_addr + c, o);
          tmem_ld_wait_for32(o);
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            uint4 w;
            w.x = pack2<F16>(__uint_as_float(o[i]) * inv, __uint_as_float(o[i + 1]) * inv);
            w.y = pack2<F16>(__uint_as_float(o[i + 2]) * inv, __uint_as_float(o[i + 3]) * inv);
            w.z = pack2<F16>(__uint_as_float(o[i + 4]) * inv, __uint_as_float(o[i + 5]) * inv);
            w.w = pack2<F16>(__uint_as_float(o[i + 6]) * inv, __uint_as_float(o[i + 7]) * inv);
            if (live && c + i < v.head_dim) *reinterpret_cast<uint4*>(to + c + i) = w;
          }
        }
        tc_fence_before_sync();
      } else {
        // layout of a piece: 256 maxima, 256 sums, then four columns of all rows at a time
        const int r = x * 128 + row;
        float* slot = p.partials + (size_t)walk.my_slot(blockIdx.x) * p.partial_floats;
        slot[r] = m;
        slot[ROWS + r] = l;
#pragma unroll 1
        for (int c = 0; c < DIM; c += 32) {
          uint32_t o[32];
          tmem_ld_32x32(o_addr + c, o);
          tmem_ld_wait_for32(o);
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            *reinterpret_cast<uint4*>(slot + 2 * ROWS + ((c + i) / 4 * ROWS + r) * 4) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
        }
        tc_fence_before_sync();
        __threadfence();
        warpgroup_sync(x);
        const auto pieces = walk.pieces();
        if (row == 0) {
          int* arrivals = p.arrivals + pieces.first * 2 + x;
          const int arrived = atomicAdd(arrivals, 1);
          t->last[x] = arrived == pieces.n - 1;
          if (t->last[x]) *arrivals = 0;             // ready for the next launch
          __threadfence();
        }
        warpgroup_sync(x);
        if (t->last[x]) {                            // join the pieces, in the order of the CTAs
          float top = -INFINITY, total = 0.0f;
          for (int c = 0; c < pieces.n; ++c) top = fmaxf(top, __ldcg(p.partials + (size_t)pieces.slot(c) * p.partial_floats + r));
          if (top == -INFINITY) top = 0.0f;
          for (int c = 0; c < pieces.n; ++c) {
            const float* from = p.partials + (size_t)pieces.slot(c) * p.partial_floats + r;
            total += exp2_fast(__ldcg(from) - top) * __ldcg(from + ROWS);
          }
          const float inv = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll 1
          for (int c32 = 0; c32 < DIM; c32 += 32) {
            float4 acc[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 2
            for (int c = 0; c < pieces.n; ++c) {
              const float* from = p.partials + (size_t)pieces.slot(c) * p.partial_floats;
              const float w = exp2_fast(__ldcg(from + r) - top) * inv;
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float4 y = __ldcg(reinterpret_cast<const float4*>(from + 2 * ROWS + ((c32 / 4 + i) * ROWS + r) * 4));
                acc[i].x += w * y.x;
                acc[i].y += w * y.y;
                acc[i].z += w * y.z;
                acc[i].w += w * y.w;
              }
            }
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
              uint4 w;
              w.x = pack2<F16>(acc[i].x, acc[i].y);
              w.y = pack2<F16>(acc[i].z, acc[i].w);
              w.z = pack2<F16>(acc[i + 1].x, acc[i + 1].y);
              w.w = pack2<F16>(acc[i + 1].z, acc[i + 1].w);
              if (live && c32 + i * 4 < v.head_dim) *reinterpret_cast<uint4*>(to + c32 + i * 4) = w;
            }
          }
        }
      }
    }
    if (!ok && lane == 0) kv_report(v, KV_TIMEOUT);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

template <bool F16, int DCH>
cudaError_t launch_one(const KvAttendParams& p, const CUtensorMap& tmap, int sm_count, int smem_optin, cudaStream_t st) {
  int slots = 2;
  while (slots < MAX_SLOTS && extend_smem(DCH, slots + 1) <= smem_optin) ++slots;
  return launch_overlapped(kv_extend_kernel<F16, DCH>, dim3(sm_count), dim3(THREADS), extend_smem(DCH, slots), st, 1, p, tmap, slots);
}

}  // namespace

cudaError_t kv_extend_configure(int smem_optin) {
  cudaError_t e = cudaFuncSetAttribute(kv_extend_kernel<false, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kv_extend_kernel<false, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kv_extend_kernel<true, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kv_extend_kernel<true, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin);
  return e;
}

size_t kv_extend_partial_floats(int head_dim) { return head_dim <= 128 ? (size_t)ROWS * (2 + (head_dim + 63) / 64 * 64) : 0; }

cudaError_t kv_extend_launch(const KvAttendParams& p, const CUtensorMap& tmap, bool f16, int sm_count, int smem_optin, cudaStream_t st) {
  if (p.v.head_dim <= 64)
    return f16 ? launch_one<true, 1>(p, tmap, sm_count, smem_optin, st) : launch_one<false, 1>(p, tmap, sm_count, smem_optin, st);
  return f16 ? launch_one<true, 2>(p, tmap, sm_count, smem_optin, st) : launch_one<false, 2>(p, tmap, sm_count, smem_optin, st);
}

}  // namespace icc
