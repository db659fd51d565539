// Attention over the paged cache for at most 16 query rows per sequence and kv head: decoding, one token with up
// to 16 query heads per kv head (or a few tokens with fewer).
//
// What bounds it is the read of the cache: each key and value is read once and used 8 or 16 times.  So the
// kernel is built around the loads.  One CTA per SM.  A producer warp fetches 64-key tiles into a ring of
// shared-memory stages, one tensor-map box per page, 64-element column chunk and keys/values (128-byte
// swizzle: the fragment loads below are free of bank conflicts), with the page numbers looked up three
// batches ahead.  Eight warps consume: even and odd tiles go to different halves of them, and a warp
// takes 16 keys of its tile.  Keys and values are the left operand of m16n8k16 products, so that the rows
// (8 or 16 of them) are the short side: scores^T = K q^T, out^T = V^T p^T.  A warp keeps the running maximum and
// sum of its own keys and its own out^T; they are merged once per item through shared memory.
//
// The weights are rounded to the cache's 16-bit type for the second product.  They are split in two such numbers (high
// part and remainder), 16 bits of each weight in bf16: a few more products, which are not the bound.  fp16 has 22 bits, but
// no step finer than 2^-24; so there all weights carry a factor of 2^LIFT, which cancels in the division by their sum.
// Without it, keys 10 nats below the maximum were down to 11 bits and those 17.3 nats below it had no weight at all, however many
// they were.  With it that is so 20 and 27.7 nats below, where the result itself comes to the end of fp16.
//
// Measured: 64 sequences of 900 to 8192 tokens, 32 query and 8 kv heads, head_dim 128 (1.2 GB of keys and values):
// 212 to 217 us, 5.5 to 5.65 TB/s, 85 to 87 % of a copy's rate.  One sequence of 131,071 tokens, 4 kv heads: 57 us, 4.7 TB/s; of these
// about 3 us pass before the first load, 6 us at the join of its pieces, and the SMs' loads end 9 us apart.  One token
// of a short sequence: 8.7 us a call, 5.6 us of them on the GPU, launch and the chain table - page - keys - sum.
#include "kernels.h"
#include "kv_mma.cuh"
#include "kv_schedule.cuh"
#include "pipeline.cuh"

namespace icc {

namespace {

constexpr int KEYS = 64;                 // keys per tile
constexpr int WARPS = 8;                 // consumer warps
constexpr int Q_WARPS = 3;               // warps that fetch query rows
constexpr int THREADS = (WARPS + 1 + Q_WARPS) * 32;
constexpr int MAX_STAGES = 12;
constexpr int AHEAD = 3;                 // batches of page numbers under way
constexpr int WHOLE = 16;                // items of at most so many tiles are not cut (kv_schedule.cuh).  Cut everywhere | 8 | 16 | 32:
                                         // a window of 1024, 33 sequences 53 | 49 | 47 | 47 us; of 2095, 35 sequences 64 | 65 | 59 | 61 us

template <bool F16>
constexpr float LIFT = F16 ? 15.0f : 0.0f;          // the largest weight is 2^LIFT (fp16 ends below 2^16)

template <int ROWS>
struct DecodeTail {
  uint64_t full[MAX_STAGES], empty[MAX_STAGES], q_full, q_empty;
  float m[WARPS][ROWS], l[WARPS][ROWS];  // per consumer warp: its rows' maxima and sums
  alignas(16) float big[ROWS], total[ROWS];   // of all of them
  int abort_flag, last;
  KvBatch batch;
};

// Warps whose out^T is in the merge buffer at a time: 16 KB of it at most.
__host__ __device__ constexpr int merge_warps(int dch, int rows) {
  return dch * rows <= 8 ? 8 : (dch * rows <= 16 ? 4 : (dch * rows <= 32 ? 2 : 1));
}
__host__ __device__ constexpr int merge_bytes(int dch, int rows) { return merge_warps(dch, rows) * dch * 64 * rows * 4; }
__host__ __device__ constexpr int q_pitch(int dch) { return dch * 128 + 16; }     // bytes of a query row in shared memory
template <int DCH, int ROWS>
constexpr int decode_smem(int stages) {
  return 1024 + stages * 2 * DCH * KEYS * 128 + merge_bytes(DCH, ROWS) + ROWS * q_pitch(DCH) + (int)sizeof(DecodeTail<ROWS>);
}

__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

template <bool F16, int DCH, int NB>
__global__ void __launch_bounds__(THREADS, 1) kv_decode_kernel(const KvAttendParams p, const __grid_constant__ CUtensorMap tmap, int n_stages) {
  constexpr int ROWS = 8 * NB;
  constexpr int CHUNK = KEYS * 128;                  // bytes of one 64-element column chunk of a tile
  constexpr int KV_BYTES = DCH * CHUNK;              // keys of a tile; the values follow
  constexpr int STAGE = 2 * KV_BYTES;
  constexpr int MERGE = merge_warps(DCH, ROWS);
  constexpr int VECS = (DCH * 64 * ROWS / 4 + WARPS * 32 - 1) / (WARPS * 32);     // float4s of out^T per consumer thread
  constexpr bool Q_IN_REGISTERS = DCH <= 2;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* merge = reinterpret_cast<float*>(ring + n_stages * STAGE);
  unsigned char* q_smem = reinterpret_cast<unsigned char*>(merge) + merge_bytes(DCH, ROWS);
  DecodeTail<ROWS>* t = reinterpret_cast<DecodeTail<ROWS>*>(q_smem + ROWS * q_pitch(DCH));
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

  if (warp == WARPS) {
    // ------------------------------------------------------------ producer
    const int per_tile = max(1, KEYS >> v.page_shift);           // pages of a tile
    const int per_batch = 32 / per_tile;                         // tiles whose page numbers one load of the warp brings
    const uint32_t box_bytes = (uint32_t)min(KEYS, 1 << v.page_shift) * 128;
    const int page_mask = (1 << v.page_shift) - 1;
    const int page_rows = (v.n_layers * 2 * v.n_kv_heads) << v.page_shift;     // rows of the tensor map per page
    const int to_values = v.n_kv_heads << v.page_shift;
    // A batch: tiles of one item that follow each other.  The lanes' page numbers are looked at only when the
    // batch is issued, so that nothing waits for the table before that.
    struct Batch {
      int page;             // this lane's page number,
      bool owned;           // if there is one
      int key, n, row;      // first key, tiles, first row of the head in a page
    };
    int k = walk.from;
    auto look = [&]() {
      Batch b{0, false, 0, 0, 0};
      if (!walk.done()) {
        const KvSeq& s = t->batch.seq[walk.i];
        const int stop = k < walk.r.sink_tiles ? min(walk.to, walk.r.sink_tiles) : walk.to;
        b.key = walk.r.tile(k) * KEYS;
        b.n = min(stop - k, per_batch);
        b.row = (p.layer * 2 * v.n_kv_heads + walk.head) << v.page_shift;
        const int entry = (b.key >> v.page_shift) + lane;
        b.owned = entry < kv_pages_of(s.length, v.page_shift);
        if (b.owned) b.page = v.tables[(size_t)s.slot * v.max_pages + entry];
        k += b.n;
        if (k >= walk.to) {
          walk.next();
          k = walk.from;
        }
      }
      return b;
    };
    int left = walk.left, s = 0, lt = 0;
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
      const bool exists = b.owned && (unsigned)b.page < (unsigned)v.n_pages;
      if (b.owned && !exists) kv_report(v, KV_INVALID);     // a borrowed table's entry that names no page
      const int y_page = exists ? b.page * page_rows + b.row : -1;
      const int e0 = b.key >> v.page_shift;
      for (int j = 0; j < b.n; ++j) {
        ok = __all_sync(FULL_MASK, mbar_wait(&t->empty[s], ph ^ 1u, &t->abort_flag));
        if (!ok) break;
        const int key = b.key + j * KEYS;
        int y = __shfl_sync(FULL_MASK, y_page, ((key >> v.page_shift) - e0 + lane) & 31);
        if (lane >= per_tile) y = -1;
        const unsigned who = __ballot_sync(FULL_MASK, y >= 0);
        if (lane == 0) mbar_arrive_expect_tx(&t->full[s], (uint32_t)__popc(who) * 2 * DCH * box_bytes);
        __syncwarp();
        if (y >= 0) {
          y += key & page_mask;
          unsigned char* dst = ring + s * STAGE + lane * box_bytes;
#pragma unroll
          for (int c = 0; c < DCH; ++c) tma_load_2d(dst + c * CHUNK, &tmap, c * 64, y, &t->full[s]);
#pragma unroll
          for (int c = 0; c < DCH; ++c) tma_load_2d(dst + KV_BYTES + c * CHUNK, &tmap, c * 64, y + to_values, &t->full[s]);
        }
        ++lt;
        if (++s == n_stages) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
    if (!ok && lane == 0) {
      kv_report(v, KV_TIMEOUT);
      // what is in flight lands before the CTA leaves
      for (int j = max(0, lt - n_stages); j < lt; ++j) {
        const long long t0 = clock64();
        while (!mbar_try_wait(&t->full[j % n_stages], (uint32_t)((j / n_stages) & 1)) && clock64() - t0 < WAIT_LIMIT_CYCLES) {
        }
      }
    }
    return;
  }
  if (warp > WARPS) {
    // ------------------------------------------------------------ query rows: an item's are fetched while the one before it is worked on
    constexpr int PIECES = DCH * 8;                              // 16-byte pieces of a row
    uint32_t ph = 1;
    for (; !walk.done(); walk.next(), ph ^= 1u) {
      const KvSeq& seq = t->batch.seq[walk.i];
      const int rows = seq.count * p.group - walk.rt * ROWS;
      if (!mbar_wait(&t->q_empty, ph, &t->abort_flag)) {
        if (lane == 0) kv_report(v, KV_TIMEOUT);
        break;
      }
#pragma unroll 2
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

  // -------------------------------------------------------------- consumers
  const int half = warp >> 2, key_in_tile = (warp & 3) * 16;
  const uint32_t ring_addr = smem_u32(ring);
  const int fr = lane >> 2, fc = (lane & 3) * 2;     // row and column pair of this thread in a fragment
  // ldmatrix: lane l gives the address of row (l & 7) of matrix l >> 3
  //   keys: matrices (keys 0-7, dims 0-7), (keys 8-15, dims 0-7), (keys 0-7, dims 8-15), (keys 8-15, dims 8-15)
  const int k_row = key_in_tile + (lane & 7) + (((lane >> 3) & 1) << 3), k_col = lane >> 4;
  //   values, transposed: (keys 0-7, dims 0-7), (keys 0-7, dims 8-15), (keys 8-15, dims 0-7), (keys 8-15, dims 8-15)
  const int v_row = key_in_tile + (lane & 7) + ((lane >> 4) << 3), v_col = (lane >> 3) & 1;
  //   queries: (rows 0-7, dims 0-7), (dims 8-15), (dims 16-23), (dims 24-31)
  const uint32_t q_addr = smem_u32(q_smem) + (lane & 7) * q_pitch(DCH) + (lane >> 3) * 16;
  int lt = 0, s = 0;                                 // tiles seen, and their stage and parity
  uint32_t ph = 0, q_ph = 0;
  bool ok = true;

  for (; !walk.done(); walk.next()) {
    const KvSeq seq = t->batch.seq[walk.i];
    const int rows = seq.count * p.group - walk.rt * ROWS;        // rows of this tile, if below ROWS
    const int first_pos = seq.length - seq.count;
    int pos[NB][2];                                               // positions of this thread's rows; -1 = no row
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = b * 8 + fc + x;
        pos[b][x] = r < rows ? first_pos + kv_token_of(p, walk.rt * ROWS + r) : -1;
      }
    const int live = min(rows, ROWS);
    const int lowest = first_pos + kv_token_of(p, walk.rt * ROWS), highest = first_pos + kv_token_of(p, walk.rt * ROWS + live - 1);
    uint32_t q[Q_IN_REGISTERS ? DCH * 2 : 1][NB][4];              // two 16-element steps each
    if (ok) ok = mbar_wait(&t->q_full, q_ph, &t->abort_flag);
    q_ph ^= 1u;
    if (Q_IN_REGISTERS) {
#pragma unroll
      for (int c = 0; c < DCH * 2; ++c)
#pragma unroll
        for (int b = 0; b < NB; ++b) ldmatrix_x4(q[c][b], q_addr + b * 8 * q_pitch(DCH) + c * 64);
      __syncwarp();
      if (lane == 0) mbar_arrive(&t->q_empty);
    }
    float o[DCH * 4][NB][4];
#pragma unroll
    for (int c = 0; c < DCH * 4; ++c)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[c][b][x] = 0.0f;
    float m[NB][2], l[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        m[b][x] = -INFINITY;
        l[b][x] = 0.0f;
      }

    for (int k = walk.from; k < walk.to; ++k, ++lt) {
      if ((lt & 1) == half) {
        if (ok) ok = mbar_wait(&t->full[s], ph, &t->abort_flag);
        const int key0 = walk.r.tile(k) * KEYS + key_in_tile;
        const uint32_t kbase = ring_addr + s * STAGE + k_row * 128, vbase = ring_addr + s * STAGE + KV_BYTES + v_row * 128;
        float sc[NB][4], sd[NB][4];                  // two chains of products
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int x = 0; x < 4; ++x) sc[b][x] = sd[b][x] = 0.0f;
#pragma unroll
        for (int c = 0; c < DCH * 2; ++c) {
          uint32_t a0[4], a1[4], qq[NB][4];
          const uint32_t at = kbase + (c >> 1) * CHUNK;
          ldmatrix_x4(a0, at + (((((c & 1) << 2) | k_col) ^ (k_row & 7)) << 4));
          ldmatrix_x4(a1, at + (((((c & 1) << 2) | 2 | k_col) ^ (k_row & 7)) << 4));
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            if (Q_IN_REGISTERS) {
#pragma unroll
              for (int x = 0; x < 4; ++x) qq[b][x] = q[c][b][x];
            } else {
              ldmatrix_x4(qq[b], q_addr + b * 8 * q_pitch(DCH) + c * 64);
            }
            mma16816<F16>(sc[b], a0, qq[b][0], qq[b][1]);
            mma16816<F16>(sd[b], a1, qq[b][2], qq[b][3]);
          }
        }
        // all of the warp's keys seen by all rows?
        const int last = key0 + 15;
        const bool clear = live == ROWS && last <= lowest && (!p.window || key0 > highest - p.window || last < p.sinks);
        float top[NB][2];
        bool grows = false;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            float y = (sc[b][x] + sd[b][x]) * p.scale_log2;
            if (!clear) {
              const int j = key0 + fr + (x >> 1) * 8, pr = pos[b][x & 1];
              const bool seen = j <= pr && (!p.window || j > pr - p.window || j < p.sinks);
              y = seen ? y : -INFINITY;
            }
            sc[b][x] = y;
          }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            top[b][x] = fmaxf(sc[b][x], sc[b][2 + x]);
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) top[b][x] = fmaxf(top[b][x], __shfl_xor_sync(FULL_MASK, top[b][x], d));
            grows |= top[b][x] > m[b][x];
          }
        }
        if (__any_sync(FULL_MASK, grows)) {
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const float now = fmaxf(m[b][x], top[b][x]);
              const float shrink = m[b][x] == -INFINITY ? 0.0f : exp2_fast(m[b][x] - now);
              m[b][x] = now;
              l[b][x] *= shrink;
#pragma unroll
              for (int c = 0; c < DCH * 4; ++c) {
                o[c][b][x] *= shrink;
                o[c][b][2 + x] *= shrink;
              }
            }
        }
        // (a NaN score is no maximum; it reaches the sum and the result through its weight)
        uint32_t hi[NB][2], lo[NB][2];               // p^T, keys by rows
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float base = (m[b][x & 1] == -INFINITY ? 0.0f : m[b][x & 1]) - LIFT<F16>;
            sc[b][x] = exp2_fast(sc[b][x] - base);
            l[b][x & 1] += sc[b][x];
          }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            split2<F16>(sc[b][2 * x], sc[b][2 * x + 1], &hi[b][x], &lo[b][x]);
            hi[b][x] = movmatrix_trans(hi[b][x]);
            lo[b][x] = movmatrix_trans(lo[b][x]);
          }
        }
        // values of keys that none of the rows sees count as zeros, whatever they hold
        uint32_t keep[2] = {~0u, ~0u};
        if (!clear) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int j = key0 + fc + x * 8;
            keep[x] = 0;
            if (j <= highest && (!p.window || j > lowest - p.window || j < p.sinks)) keep[x] |= 0xffffu;
            if (j + 1 <= highest && (!p.window || j + 1 > lowest - p.window || j + 1 < p.sinks)) keep[x] |= 0xffff0000u;
          }
        }
#pragma unroll
        for (int c = 0; c < DCH * 4; ++c) {
          uint32_t a[4];
          ldmatrix_x4_trans(a, vbase + (c >> 2) * CHUNK + (((((c & 3) << 1) | v_col) ^ (v_row & 7)) << 4));
          a[0] &= keep[0];
          a[1] &= keep[0];
          a[2] &= keep[1];
          a[3] &= keep[1];
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            mma16816<F16>(o[c][b], a, hi[b][0], hi[b][1]);
            mma16816<F16>(o[c][b], a, lo[b][0], lo[b][1]);
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
    if (!Q_IN_REGISTERS) {
      __syncwarp();
      if (lane == 0) mbar_arrive(&t->q_empty);
    }

    // ---- merge the warps: common maximum and sum per row, then out^T
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[b][x] += __shfl_xor_sync(FULL_MASK, l[b][x], d);
        if (fr == 0) {
          t->m[warp][b * 8 + fc + x] = m[b][x];
          t->l[warp][b * 8 + fc + x] = l[b][x];
        }
      }
    consumers_sync();
    float part[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = b * 8 + fc + x;
        float big = -INFINITY;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) big = fmaxf(big, t->m[w][r]);
        const float b0 = big == -INFINITY ? 0.0f : big;
        part[b][x] = exp2_fast(m[b][x] - b0);
        if (warp == 0 && fr == 0) {
          float sum = 0.0f;
#pragma unroll
          for (int w = 0; w < WARPS; ++w) sum += t->l[w][r] * exp2_fast(t->m[w][r] - b0);
          t->big[r] = big;
          t->total[r] = sum;
        }
      }
    // buffers of out^T [dims][ROWS], one per warp modulo MERGE
    float* mine = merge + (warp % MERGE) * (DCH * 64 * ROWS) + fr * ROWS + fc;
#pragma unroll 1
    for (int round = 0; round < WARPS / MERGE; ++round) {
      if (warp / MERGE == round) {
#pragma unroll
        for (int c = 0; c < DCH * 4; ++c)
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float2* at = reinterpret_cast<float2*>(mine + (c * 16 + x * 8) * ROWS + b * 8);
              float2 w = make_float2(o[c][b][2 * x] * part[b][0], o[c][b][2 * x + 1] * part[b][1]);
              if (WARPS > MERGE && round > 0) {
                w.x += at->x;
                w.y += at->y;
              }
              *at = w;
            }
      }
      consumers_sync();
    }
    float4 sum[VECS];                                // four rows of one dim each, in the order of the buffer
    const bool whole = walk.whole();
    float* slot = p.partials + (size_t)walk.my_slot(blockIdx.x) * p.partial_floats;
    auto put = [&](int f, const float4& y) {         // four rows of one dim of the result
      const int d = f * 4 / ROWS, r0 = f * 4 % ROWS;
      if (d >= v.head_dim) return;
      const float e[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int r = r0 + x;
        if (r >= live) break;
        const int rr = walk.rt * ROWS + r, tok = kv_token_of(p, rr), hq = walk.head * p.group + (rr - tok * p.group);
        reinterpret_cast<uint16_t*>(p.out)[(int64_t)(seq.first + tok) * p.out_token_stride + (int64_t)hq * p.out_head_stride + d] = round16<F16>(e[x]);
      }
    };
#pragma unroll
    for (int x = 0; x < VECS; ++x) {
      const int f = x * WARPS * 32 + tid;
      sum[x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (f < DCH * 64 * ROWS / 4) {
#pragma unroll
        for (int w = 0; w < MERGE; ++w) {
          const float4 y = *reinterpret_cast<const float4*>(merge + w * (DCH * 64 * ROWS) + f * 4);
          sum[x].x += y.x;
          sum[x].y += y.y;
          sum[x].z += y.z;
          sum[x].w += y.w;
        }
        if (whole) {
          const float* tot = t->total + f * 4 % ROWS;
          const float4 z = make_float4(sum[x].x * (tot[0] == 0.0f ? 0.0f : 1.0f / tot[0]), sum[x].y * (tot[1] == 0.0f ? 0.0f : 1.0f / tot[1]),
                                       sum[x].z * (tot[2] == 0.0f ? 0.0f : 1.0f / tot[2]), sum[x].w * (tot[3] == 0.0f ? 0.0f : 1.0f / tot[3]));
          put(f, z);
        } else {
          // layout of a piece: ROWS maxima, ROWS sums, out^T
          *reinterpret_cast<float4*>(slot + 2 * ROWS + f * 4) = sum[x];
        }
      }
    }
    if (!whole) {
      if (tid < ROWS) {
        slot[tid] = t->big[tid];
        slot[ROWS + tid] = t->total[tid];
      }
      consumers_sync();
      const auto pieces = walk.pieces();
      if (tid == 0) {
        t->last = kv_arrive(&p.arrivals[pieces.first]) == pieces.n - 1;
        if (t->last) p.arrivals[pieces.first] = 0;   // ready for the next launch
      }
      consumers_sync();
      if (t->last) {
        // Join the pieces in the order of the CTAs.  They come from L2, a microsecond away: maxima, sums and the
        // first values are asked for at once, and FLIGHT loads are in flight per thread.
        constexpr int FLIGHT = 24 / VECS, CHUNKS = KV_MAX_CTAS / 32;
        float4 y[FLIGHT][VECS];
        auto fetch = [&](int c0) {
#pragma unroll
          for (int u = 0; u < FLIGHT; ++u)
#pragma unroll
            for (int x = 0; x < VECS; ++x) {
              const int f = x * WARPS * 32 + tid;
              y[u][x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
              if (c0 + u < pieces.n && f < DCH * 64 * ROWS / 4)
                y[u][x] = __ldcg(reinterpret_cast<const float4*>(p.partials + (size_t)pieces.slot(c0 + u) * p.partial_floats + 2 * ROWS + f * 4));
            }
        };
        float pm[NB][CHUNKS], pl[NB][CHUNKS];        // warp w: rows w and w + 8; lanes: pieces
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int x = 0; x < CHUNKS; ++x) {
            pm[b][x] = -INFINITY;
            pl[b][x] = 0.0f;
            if (x * 32 + lane < pieces.n) {
              const float* from = p.partials + (size_t)pieces.slot(x * 32 + lane) * p.partial_floats + b * 8 + warp;
              pm[b][x] = __ldcg(from);
              pl[b][x] = __ldcg(from + ROWS);
            }
          }
        fetch(0);
        float* weight = merge;                       // [pieces][ROWS]
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const int r = b * 8 + warp;
          float top = -INFINITY, sum_l = 0.0f;
#pragma unroll
          for (int x = 0; x < CHUNKS; ++x) top = fmaxf(top, pm[b][x]);
#pragma unroll
          for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL_MASK, top, d));
          if (top == -INFINITY) top = 0.0f;
#pragma unroll
          for (int x = 0; x < CHUNKS; ++x) {
            const float w = exp2_fast(pm[b][x] - top);
            if (x * 32 + lane < pieces.n) weight[(x * 32 + lane) * ROWS + r] = w;
            sum_l += w * pl[b][x];
          }
#pragma unroll
          for (int d = 16; d; d >>= 1) sum_l += __shfl_xor_sync(FULL_MASK, sum_l, d);
          if (lane == 0) t->total[r] = sum_l == 0.0f ? 0.0f : 1.0f / sum_l;
        }
        consumers_sync();
#pragma unroll
        for (int x = 0; x < VECS; ++x) sum[x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int c0 = 0;;) {
#pragma unroll
          for (int u = 0; u < FLIGHT; ++u)
#pragma unroll
            for (int x = 0; x < VECS; ++x) {
              if (c0 + u >= pieces.n) break;
              const float4 w = *reinterpret_cast<const float4*>(weight + (c0 + u) * ROWS + (x * WARPS * 32 + tid) * 4 % ROWS);
              sum[x].x += w.x * y[u][x].x;
              sum[x].y += w.y * y[u][x].y;
              sum[x].z += w.z * y[u][x].z;
              sum[x].w += w.w * y[u][x].w;
            }
          c0 += FLIGHT;
          if (c0 >= pieces.n) break;
          fetch(c0);
        }
#pragma unroll
        for (int x = 0; x < VECS; ++x) {
          const int f = x * WARPS * 32 + tid;
          const float4 w = *reinterpret_cast<const float4*>(t->total + f * 4 % ROWS);
          if (f < DCH * 64 * ROWS / 4) put(f, make_float4(sum[x].x * w.x, sum[x].y * w.y, sum[x].z * w.z, sum[x].w * w.w));
        }
        consumers_sync();                            // the weights have been read: the buffer is free again
      }
    }
  }
  if (!ok && lane == 0) kv_report(v, KV_TIMEOUT);
}

template <bool F16, int DCH, int NB>
cudaError_t configure_one(int smem_optin) {
  return cudaFuncSetAttribute(kv_decode_kernel<F16, DCH, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin);
}

template <bool F16, int DCH, int NB>
cudaError_t launch_one(const KvAttendParams& p, const CUtensorMap& tmap, int sm_count, int smem_optin, cudaStream_t st) {
  // An even number of stages, so that a stage always belongs to the same half of the consumers: a warp that met
  // a stage's barrier at every other round only could not tell a round's parity from that of two rounds before.
  int stages = 2;
  while (stages + 2 <= MAX_STAGES && decode_smem<DCH, 8 * NB>(stages + 2) <= smem_optin) stages += 2;
  return launch_overlapped(kv_decode_kernel<F16, DCH, NB>, dim3(sm_count), dim3(THREADS), decode_smem<DCH, 8 * NB>(stages), st, 1, p, tmap, stages);
}

template <bool F16>
cudaError_t launch_dch(const KvAttendParams& p, const CUtensorMap& tmap, bool two, int sm_count, int smem_optin, cudaStream_t st) {
  switch ((p.v.head_dim + 63) / 64) {
    case 1: return two ? launch_one<F16, 1, 2>(p, tmap, sm_count, smem_optin, st) : launch_one<F16, 1, 1>(p, tmap, sm_count, smem_optin, st);
    case 2: return two ? launch_one<F16, 2, 2>(p, tmap, sm_count, smem_optin, st) : launch_one<F16, 2, 1>(p, tmap, sm_count, smem_optin, st);
    case 3: return two ? launch_one<F16, 3, 2>(p, tmap, sm_count, smem_optin, st) : launch_one<F16, 3, 1>(p, tmap, sm_count, smem_optin, st);
    default: return two ? launch_one<F16, 4, 2>(p, tmap, sm_count, smem_optin, st) : launch_one<F16, 4, 1>(p, tmap, sm_count, smem_optin, st);
  }
}

template <bool F16>
cudaError_t configure_all(int smem_optin) {
  cudaError_t e = configure_one<F16, 1, 1>(smem_optin);
  if (e == cudaSuccess) e = configure_one<F16, 1, 2>(smem_optin);
  if (e == cudaSuccess) e = configure_one<F16, 2, 1>(smem_optin);
  if (e == cudaSuccess) e = configure_one<F16, 2, 2>(smem_optin);
  if (e == cudaSuccess) e = configure_one<F16, 3, 1>(smem_optin);
  if (e == cudaSuccess) e = configure_one<F16, 3, 2>(smem_optin);
  if (e == cudaSuccess) e = configure_one<F16, 4, 1>(smem_optin);
  if (e == cudaSuccess) e = configure_one<F16, 4, 2>(smem_optin);
  return e;
}

}  // namespace

cudaError_t kv_decode_configure(int smem_optin) {
  const cudaError_t e = configure_all<false>(smem_optin);
  return e == cudaSuccess ? configure_all<true>(smem_optin) : e;
}

cudaError_t kv_decode_launch(const KvAttendParams& p, const CUtensorMap& tmap, bool f16, bool two, int sm_count, int smem_optin, cudaStream_t st) {
  return f16 ? launch_dch<true>(p, tmap, two, sm_count, smem_optin, st) : launch_dch<false>(p, tmap, two, sm_count, smem_optin, st);
}

}  // namespace icc
