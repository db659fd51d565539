// Attention over the paged cache for many query rows: prompts, on the tensor cores (tcgen05).
//
// Up to a head_dim of 128 an item is 256 rows of one sequence and kv head (tokens times query heads of the kv head), two row tiles A and
// B of 128 that share every key and value fetched.  Per 64 keys (a unit) and row tile there are two products,
// S = Q K^T and O += P V, with S, P and O in tensor memory (512 columns: two units' S of A and of B, O_A, O_B; a
// unit's P, 16 bit, takes the first half of its S).  The same work needs 128 x 64 exponentials, for which the
// special-function units take as long as the tensor cores do for the products, so neither may wait for the
// other: two row tiles in flight, and of each the scores of the next unit while the present one's become
// weights.  (Units of 128 keys fit only once per row tile; then a row tile's chain softmax - PV - S is exposed:
// 4,300 cycles for both row tiles and 128 keys, of which the tensor cores work 2,048.)  The price is that
// S with 64 columns is bound by shared memory: 48 cycles a product where the tensor cores need 32.
//
// Of a head_dim of 129 to 256, O_A alone takes 256 columns, and there is one row tile to an item.  Its products (1,280
// cycles for 64 keys at 256) take as long as those of two row tiles at 128, but the softmax is one warp's chain of
// latencies per scheduler, which is what bounds it: tensor cores 31 % busy, special-function units 16 %, L2 22 %.
//
//   warps 0-3, 4-7   softmax of row tile A, B: a thread owns a row (a tensor-memory lane), and copies the row's
//                    query into the swizzled layout of the left operand, an item ahead
//   warp 8           loads of keys and values, 128 (64) of each a slot: one tensor-map box per page (or 64 rows) and
//                    64-element chunk
//   warps 9, 10      issue the products of row tile A, B: PV(u), S(u + 2), ...
//   warp 11          zeros in place of values that nobody sees; tells the softmax warps what the next items are
//
// A row's maximum is only raised when it is exceeded by more than 2^8: O is rescaled a few times per item and not
// per unit, and weights of up to 256 are as exact as those up to 1.  Weights are rounded to the cache's
// 16-bit type (the tensor cores take both operands in one type), once: the second number that the decode kernel adds to it would
// double the products with the values, half of what the tensor cores do here.  Their sum is taken before the rounding.
//
// Measured, 32 query and 8 kv heads: 8 prompts of up to 4096 tokens, head_dim 128: 0.73 ms, 0.93 PFLOP/s, by itself behind a cold
// L2 (0.86 ms in a row of launches, where the power limit lowers the clock); one prompt of 16384 tokens 2.05 ms, 1.07 PFLOP/s; a
// window of 1024 over one sequence of 12,289 tokens 138 us; four requests of up to 57 tokens behind up to 6,000 38 us; head_dim
// 256: 20 prompts of 10 to 600 tokens 204 us.  (For wide heads a kernel of 32 rows an item on warp-level products took five to six
// times as long on two such cases, and 32 against 29 us for the smallest, so that there is no kernel of that kind.)
// What bounds it: no unit.  64 keys of both row tiles take 1,760 cycles, where their exponentials are 1,024 and their products
// 1,280; tensor pipe and special-function units are half busy each.  It is the order of the steps (scores, maximum, turn,
// exponentials, store), and the change of items (4,600 cycles).
#include "kernels.h"
#include "kv_mma.cuh"
#include "kv_schedule.cuh"
#include "pipeline.cuh"

namespace icc {

namespace {

constexpr int SOFTMAX_WARPS = 8;
constexpr int THREADS = 384;
constexpr int MAX_SLOTS = 8;             // of the key/value ring
// Registers: launched with 168 a thread; the softmax warpgroups take from the third: 384 x 168 = 256 x 216 + 128 x 72.
constexpr int OTHER_REGS = 72, SOFTMAX_REGS = 216;
constexpr float RAISE = 8.0f;            // how far (log2) a row's scores may exceed its maximum before O is rescaled
// fp16 has no step finer than 2^-24 and ends below 2^16: there all weights carry a factor of 2^LIFT, which cancels in the division by
// their sum.  They keep 11 bits down to 14.5 nats below the maximum and vanish 22 nats below it (without the factor: 9.7 and 17.3).
// A smaller RAISE would leave room for a larger factor: 6 and 9, 1.4 nats more, cost 5 % of 8 prompts of up to 4096 tokens, 4 and 11 25 %.
template <bool F16>
constexpr float LIFT = F16 ? 7.0f : 0.0f;
constexpr int AHEAD = 3;                 // batches of page numbers under way
constexpr int WHOLE_KEYS = 1024;         // items of at most so many keys are not cut (kv_schedule.cuh).  Cut everywhere | 640 | 1024 | 1536:
                                         // 40 prompts of up to 1000 tokens 221 | 213 | 213 | 211 us; the window of 1024 143 | 143 | 143 | 152 us

// What follows from the head_dim, in chunks of 64.
template <int DCH>
struct Shape {
  static constexpr int TILES = DCH <= 2 ? 2 : 1;               // row tiles of an item
  static constexpr int KEYS = DCH <= 2 ? 128 : 64;             // keys per tile (a slot of the ring), in units of 64
  static constexpr int ROWS = TILES * 128;                     // rows per item
  static constexpr int CHUNK = KEYS * 128, Q_CHUNK = 128 * 128;        // bytes of a 64-element column chunk of keys, of a row tile
  static constexpr int SLOT = DCH * CHUNK, Q_TILE = DCH * Q_CHUNK;
  using Walk = KvWalk<ROWS, KEYS, WHOLE_KEYS / KEYS>;
};

// What the softmax warps need to know of an item: worked out by warp 11, ITEMS ahead at most.
constexpr int ITEMS = 8;
struct alignas(16) Item {
  int more;                              // 0: there are no more
  int rows;                              // query rows from the item's first one to the sequence's last
  int row0, first_pos;                   // first row; position of the call's first token of the sequence
  int q_first, head0;                    // that token's row of q; first query head
  int from, to, sink_tiles, first_tile;  // key tiles, as in KvWalk and KvRange
  int whole, my_slot;                    // 0: a piece of an item, and where the partial result goes
  int piece_first, pieces;               // which CTAs have the others (KvWalk::Pieces)
  int unused[2];
};

struct ExtendTail {
  Item item[ITEMS];
  uint64_t item_full[ITEMS], item_empty[ITEMS];
  uint64_t group_sync[2];                // the four warps of a row tile (with a limit, as all waits here)
  uint64_t full[MAX_SLOTS], empty[MAX_SLOTS], clean[MAX_SLOTS];
  uint64_t q_full[2], s_full[2][2], p_full[2][2], o_last[2], o_full[2], drain[2];     // per row tile (and unit of a tile)
  uint32_t tmem_base;
  int abort_flag, last[2], left[SOFTMAX_WARPS];
  float zero;
  KvBatch batch;
};

template <int DCH>
int extend_smem(int slots) { return 1024 + Shape<DCH>::TILES * Shape<DCH>::Q_TILE + slots * Shape<DCH>::SLOT + (int)sizeof(ExtendTail); }

// Instruction descriptor: A and B 16-bit floats of one type, fp32 accumulator, M = 128.
__host__ __device__ constexpr uint32_t idesc(bool f16, int n, bool b_mn_major) {
  return (1u << 4) | (f16 ? 0u : (1u << 7) | (1u << 10)) | (b_mn_major ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}
constexpr uint32_t NEGATE_A = 1u << 13;
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
// Products and their completion, executed by a whole warp and issued by the one lane whose `on` is not 0, so that the
// warp never has to leave for a branch of one lane.
__device__ __forceinline__ void product_smem(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t id, uint32_t accumulate, uint32_t on) {
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "setp.ne.b32 q, %5, 0;\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
      "}\n" ::"r"(tmem_d),
      "l"(desc_a), "l"(desc_b), "r"(id), "r"(accumulate), "r"(on)
      : "memory");
}
// The left operand in tensor memory.
__device__ __forceinline__ void product_tmem(uint32_t tmem_d, uint32_t tmem_a, uint64_t desc_b, uint32_t id, uint32_t accumulate, uint32_t on) {
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "setp.ne.b32 q, %5, 0;\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "}\n" ::"r"(tmem_d),
      "r"(tmem_a), "l"(desc_b), "r"(id), "r"(accumulate), "r"(on)
      : "memory");
}
__device__ __forceinline__ void commit_products(uint64_t* bar, uint32_t on) {
  asm volatile(
      "{\n"
      ".reg .pred q;\n"
      "setp.ne.b32 q, %1, 0;\n"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n"
      "}\n" ::"r"(smem_u32(bar)),
      "r"(on)
      : "memory");
}
__device__ __forceinline__ void arrive_one(uint64_t* bar, uint32_t on) {
  asm volatile(
      "{\n"
      ".reg .pred q;\n"
      "setp.ne.b32 q, %1, 0;\n"
      "@q mbarrier.arrive.shared::cta.b64 _, [%0];\n"
      "}\n" ::"r"(smem_u32(bar)),
      "r"(on)
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
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// A wait of a whole warp.  All lanes ask together: a lane that waits by itself, inside a branch, wakes up to 200 cycles
// later (measured: 54 against 70 to 240 cycles from the arrival).
__device__ __forceinline__ bool mbar_warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(FULL_MASK, mbar_wait(bar, parity, abort_flag)) != 0;
}
// The lowest n bits, n <= 0: none, n >= 32: all.
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : (n >= 32 ? ~0u : (1u << n) - 1u); }
// Turns between warp w of row tile A and warp w + 4 of B, on the hardware's barriers (110 cycles a turn quicker than a
// barrier in shared memory): 3 .. 6 call A's warp, 7 .. 10 B's.
__device__ __forceinline__ void turn_wait(int warp) { asm volatile("bar.sync %0, 64;" ::"r"(3 + warp) : "memory"); }
__device__ __forceinline__ void turn_pass(int warp) { asm volatile("bar.arrive %0, 64;" ::"r"(3 + (warp ^ 4)) : "memory"); }

// ---------------------------------------------------------------- pairs of floats in one instruction
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ void split_pair(uint64_t x, float* a, float* b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(*a), "=f"(*b) : "l"(x)); }
__device__ __forceinline__ uint64_t fma_pairs(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add_pairs(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// Weights 2^(scale s - base) of 64 scores, packed to the cache's type; their sum is added to sum2.
template <bool F16>
__device__ __forceinline__ void weights(const uint32_t (&s)[64], uint64_t scale2, uint64_t base2, uint64_t (&sum2)[2], uint32_t (&w)[32]) {
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const uint64_t x2 = fma_pairs(pair_of(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), scale2, base2);
    float a, b;
    split_pair(x2, &a, &b);
    a = exp2_fast(a);
    b = exp2_fast(b);
    sum2[i & 1] = add_pairs(sum2[i & 1], pair_of(a, b));
    w[i] = pack2<F16>(a, b);
  }
}

// 16 columns of a thread's row to the result: 32 bytes at a time where the address allows (a whole sector per lane; halves
// of sectors from different instructions cost as many passes as whole ones).
template <bool F16>
__device__ __forceinline__ void store_row(uint16_t* to, int column, int head_dim, const uint32_t (&w)[8]) {
  uint16_t* at = to + column;
  if (column + 16 <= head_dim && (reinterpret_cast<uintptr_t>(at) & 31) == 0) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                 "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
    if (column < head_dim) *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
    if (column + 8 < head_dim) *reinterpret_cast<uint4*>(at + 8) = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// Keys that no token of the call sees: between the sinks and the first token's window, and past the end (slots of
// the last page without tokens).  Whatever stands there must not reach a product: a weight of zero would not undo an
// infinity or a NaN.
struct Hidden {
  int sinks, first_seen, length;
  __device__ __forceinline__ Hidden(const KvAttendParams& p, const KvSeq& s)
      : sinks(p.sinks), first_seen(p.window ? max(0, s.length - s.count - p.window + 1) : 0), length(s.length) {}
  __device__ __forceinline__ bool is(int key) const { return (key >= sinks && key < first_seen) || key >= length; }
  __device__ __forceinline__ bool any(int key0, int keys) const {          // among the keys of a tile
    return max(key0, sinks) < min(key0 + keys, first_seen) || key0 + keys > length;
  }
};

template <bool F16, int DCH>
__global__ void __launch_bounds__(THREADS, 1) kv_extend_kernel(const KvAttendParams p, const __grid_constant__ CUtensorMap tmap, int n_slots) {
  constexpr int DIM = DCH * 64;                      // head_dim, padded
  using X = Shape<DCH>;
  using Walk = typename X::Walk;
  constexpr int TILES = X::TILES, KEYS = X::KEYS, ROWS = X::ROWS, CHUNK = X::CHUNK, Q_CHUNK = X::Q_CHUNK, SLOT = X::SLOT, Q_TILE = X::Q_TILE;
  constexpr int UNITS = KEYS / 64;                   // of a tile
  constexpr int AT_HAND = DCH <= 2 ? DCH : 1;        // chunks of a result in a thread's registers
  constexpr uint32_t TMEM_O = 256;                   // first column of O_A; S of A's units at 0 and 64, of B's at 128 and 192, O_B at 256 + 128
  extern __shared__ unsigned char smem_raw[];
  unsigned char* q_smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* ring = q_smem + TILES * Q_TILE;
  ExtendTail* t = reinterpret_cast<ExtendTail*>(ring + n_slots * SLOT);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const KvView& v = p.v;
  if (tid == 0) {
    for (int s = 0; s < n_slots; ++s) {
      mbar_init(&t->full[s], 1);
      mbar_init(&t->empty[s], TILES + (s & 1));      // the row tiles; and warp 11 for values, which take the odd slots
      mbar_init(&t->clean[s], 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&t->q_full[x], 128);
      for (int h = 0; h < 2; ++h) {
        mbar_init(&t->s_full[x][h], 1);
        mbar_init(&t->p_full[x][h], 4);
      }
      mbar_init(&t->o_last[x], 1);
      mbar_init(&t->group_sync[x], 4);
      mbar_init(&t->o_full[x], 1);
      mbar_init(&t->drain[x], 1);
    }
    t->abort_flag = 0;
    t->zero = 0.0f;
    for (int i = 0; i < ITEMS; ++i) {
      mbar_init(&t->item_full[i], 1);
      mbar_init(&t->item_empty[i], 4 * TILES);
    }
    for (int w = 0; w < SOFTMAX_WARPS; ++w) t->left[w] = 0;
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
  Walk walk(p, t->batch, blockIdx.x, gridDim.x);

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
        int page;           // this lane's page number,
        bool owned;         // if there is one
        int key, n, row;    // first key, tiles, first row of the head in a page
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
        const bool exists = b.owned && (unsigned)b.page < (unsigned)v.n_pages;
        if (b.owned && !exists) kv_report(v, KV_INVALID);
        const int y_page = exists ? b.page * page_rows + b.row : -1;
        const int e0 = b.key >> v.page_shift;
        for (int j = 0; j < b.n && ok; ++j) {
          const int key = b.key + j * KEYS + lane * box_rows;    // first key of this lane's box
          int y = __shfl_sync(FULL_MASK, y_page, ((key >> v.page_shift) - e0) & 31);
          if (lane >= boxes) y = -1;
          const unsigned who = __ballot_sync(FULL_MASK, y >= 0);
          if (y >= 0) y += key & page_mask;
          for (int values = 0; values < 2; ++values) {
            ok = mbar_warp_wait(&t->empty[s], ph ^ 1u, &t->abort_flag);
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
    } else if (warp <= 10) {
      // ---------------------------------------------------------- products
      if (warp - 9 < TILES) {
        // (a negative scale: the product with -Q, and the scale's magnitude)
        const uint32_t id_s = idesc(F16, 64, false) | (p.scale_log2 < 0.0f ? NEGATE_A : 0u);
        constexpr uint32_t id_o = idesc(F16, DIM, true);
        const int x = warp - 9;                      // row tile
        const uint32_t on = lane == 0;
        const uint32_t s_at = tmem + x * 128, o_at = tmem + TMEM_O + x * 128;
        const uint64_t q_desc = umma_desc_k_major_sw128(smem_u32(q_smem) + x * Q_TILE), k_desc = umma_desc_k_major_sw128(smem_u32(ring)),
                       v_desc = desc_mn_major_sw128(smem_u32(ring), CHUNK);
        uint32_t q_ph = 0, p_ph = 0, clean_ph = 0;
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_warp_wait(bar, parity, &t->abort_flag); };
        auto scores = [&](int slot, int part, int half) {        // S = Q K^T, 64 of the keys, into one of the two places for S
          const uint64_t db = k_desc + (slot * (SLOT >> 4) + part * (64 * 128 >> 4));
#pragma unroll
          for (int c = 0; c < DCH; ++c)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              product_smem(s_at + half * 64, q_desc + (c * (Q_CHUNK >> 4) + kk * 2), db + (c * (CHUNK >> 4) + kk * 2), id_s,
                           (c | kk) != 0 ? 1u : 0u, on);
          commit_products(&t->s_full[x][half], on);
        };
        auto values = [&](int slot, int part, int half, bool add) {        // O (+)= P V, 64 of the keys
          const uint64_t db = v_desc + (slot * (SLOT >> 4) + part * (64 * 128 >> 4));
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)             // 16 keys further: 8 columns of P, 2048 bytes of V
            product_tmem(o_at, s_at + half * 64 + kk * 8, db + kk * 128, id_o, (add || kk != 0) ? 1u : 0u, on);
        };
        // A slot is free when both row tiles are done with it; one that has no rows in the item says so at once.
        auto done_with = [&](int slot, bool mine) {
          if (mine) commit_products(&t->empty[slot], on);
          else arrive_one(&t->empty[slot], on);
        };
        if constexpr (UNITS == 2) {
          int s = 0;                                 // next slot of the ring
          uint32_t ph = 0;
          auto advance = [&]() {
            if (++s == n_slots) {
              s = 0;
              ph ^= 1u;
            }
          };
          for (; !walk.done() && ok; walk.next()) {
            const KvSeq& seq = t->batch.seq[walk.i];
            const int rows = seq.count * p.group - walk.rt * ROWS, n = walk.to - walk.from;
            const bool mine = rows > x * 128;
            const Hidden hidden(p, seq);
            ok = wait(&t->full[s], ph);
            if (mine && ok) {
              ok = wait(&t->q_full[x], q_ph);
              q_ph ^= 1u;
              fence_async_shared();                    // the query's copies were ordinary writes
              tc_fence_after_sync();
              if (ok) {
                scores(s, 0, 0);
                scores(s, 1, 1);
              }
            }
            if (!ok) break;
            done_with(s, mine);
            advance();
            for (int j = 0; j < n; ++j) {
              const bool more = j + 1 < n;
              const int sv = s;
              const bool cleaned = hidden.any(walk.r.tile(walk.from + j) * KEYS, KEYS);
              ok = wait(&t->full[s], ph);
              if (ok && cleaned) {
                ok = wait(&t->clean[sv], (clean_ph >> sv) & 1u);   // a slot's barrier turns at each use that is cleaned
                clean_ph ^= 1u << sv;
              }
              if (!ok) break;
              advance();
              if (mine) {
                ok = wait(&t->p_full[x][0], p_ph);
                if (!ok) break;
                tc_fence_after_sync();
                values(sv, 0, 0, j > 0);
                if (!more) commit_products(&t->o_last[x], on);
              }
              if (more) ok = wait(&t->full[s], ph);
              if (mine && ok) {
                if (more) scores(s, 0, 0);
                ok = wait(&t->p_full[x][1], p_ph);
                p_ph ^= 1u;
                if (!ok) break;
                tc_fence_after_sync();
                values(sv, 1, 1, true);
                done_with(sv, true);
                if (more) scores(s, 1, 1);
                else commit_products(&t->o_full[x], on);
              }
              if (!ok) break;
              if (!mine) done_with(sv, false);
              if (more) {
                done_with(s, mine);
                advance();
              }
            }
          }
        } else {
          // One row tile, a unit a slot: S(0), S(1), PV(0), S(2), PV(1), ...  Keys and values are taken at their own paces.
          int ks = 0, vs = 1;
          uint32_t k_ph = 0, v_ph = 0;
          auto advance = [&](int& s, uint32_t& ph) {
            if ((s += 2) >= n_slots) {
              s -= n_slots;
              ph ^= 1u;
            }
          };
          auto next_scores = [&](int half) {
            ok = wait(&t->full[ks], k_ph);
            if (!ok) return;
            scores(ks, 0, half);
            done_with(ks, true);
            advance(ks, k_ph);
          };
          for (; !walk.done() && ok; walk.next()) {
            const Hidden hidden(p, t->batch.seq[walk.i]);
            const int n = walk.to - walk.from;
            ok = wait(&t->q_full[0], q_ph);
            q_ph ^= 1u;
            if (!ok) break;
            fence_async_shared();                    // the query's copies were ordinary writes
            tc_fence_after_sync();
            next_scores(0);
            if (ok && n > 1) next_scores(1);
            for (int u = 0; u < n && ok; ++u) {
              const int half = u & 1;
              ok = wait(&t->full[vs], v_ph);
              if (ok && hidden.any(walk.r.tile(walk.from + u) * KEYS, KEYS)) {
                ok = wait(&t->clean[vs], (clean_ph >> vs) & 1u);   // a slot's barrier turns at each use that is cleaned
                clean_ph ^= 1u << vs;
              }
              if (ok) ok = wait(&t->p_full[0][half], (p_ph >> half) & 1u);
              p_ph ^= 1u << half;
              if (!ok) break;
              tc_fence_after_sync();
              values(vs, 0, half, u > 0);
              done_with(vs, true);
              advance(vs, v_ph);
              if (u == max(n - 2, 0)) commit_products(&t->o_last[0], on);
              if (u == n - 1) commit_products(&t->o_full[0], on);
              if (u + 2 < n) next_scores(half);
            }
          }
        }
        // nothing issued is still running when tensor memory is released
        commit_products(&t->drain[x], on);
        const long long t0 = clock64();
        while (!mbar_try_wait(&t->drain[x], 0) && clock64() - t0 < WAIT_LIMIT_CYCLES) {
        }
        if (!ok && lane == 0) kv_report(v, KV_TIMEOUT);
      }
    } else {
      // ---------------------------------------------------------- values that no token of the call sees count as zeros
      // (it looks at every tile and has a say in its slot's release, or it could lose count of the rounds)
      int s = 1, n_items = 0;
      uint32_t ph = 0;
      bool ok = true;
      auto publish = [&](const Walk& w) {
        const int at = n_items % ITEMS;
        if (ok) ok = mbar_warp_wait(&t->item_empty[at], ((n_items / ITEMS) & 1) ^ 1, &t->abort_flag);
        if (lane == 0) {
          Item d = {};
          if (!w.done()) {
            const KvSeq& seq = t->batch.seq[w.i];
            d.more = 1;
            d.row0 = w.rt * ROWS;
            d.rows = seq.count * p.group - d.row0;
            d.first_pos = seq.length - seq.count;
            d.q_first = seq.first;
            d.head0 = w.head * p.group;
            d.from = w.from;
            d.to = w.to;
            d.sink_tiles = w.r.sink_tiles;
            d.first_tile = w.r.first;
            d.whole = w.whole();
            if (!d.whole) {
              const auto pieces = w.pieces();
              d.my_slot = w.my_slot(blockIdx.x);
              d.piece_first = pieces.first;
              d.pieces = pieces.n;
            }
          }
          t->item[at] = d;
          mbar_arrive(&t->item_full[at]);
        }
        __syncwarp();
        ++n_items;
      };
      publish(walk);
      while (!walk.done() && ok) {
        Walk after = walk;
        after.next();
        publish(after);
        const Hidden hidden(p, t->batch.seq[walk.i]);
        for (int k = walk.from; k < walk.to; ++k) {
          const int key0 = walk.r.tile(k) * KEYS;
          ok = mbar_warp_wait(&t->full[s], ph, &t->abort_flag);
          if (!ok) break;
          if (hidden.any(key0, KEYS)) {
            constexpr int PIECES = DCH * 8;
            for (int u = lane; u < KEYS * PIECES; u += 32) {
              const int r = u / PIECES, piece = u % PIECES;
              if (hidden.is(key0 + r))
                *reinterpret_cast<uint4*>(ring + s * SLOT + (piece >> 3) * CHUNK + r * 128 + (piece & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(&t->clean[s]);
          }
          if (lane == 0) mbar_arrive(&t->empty[s]);
          if ((s += 2) >= n_slots) {
            s = 1;
            ph ^= 1u;
          }
        }
        walk = after;
      }
      if (!ok && lane == 0) kv_report(v, KV_TIMEOUT);
    }
  } else if (warp < 4 * TILES) {
    // ------------------------------------------------------------ softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFTMAX_REGS));
    const int x = warp >> 2, row = tid & 127;        // row tile, and row (tensor-memory lane) of this thread
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lane_base + x * 128, o_addr = tmem + lane_base + TMEM_O + x * 128;
    // A scale of zero must not make NaN of the minus infinity that stands for a hidden key.
    const float scale = fmaxf(fabsf(p.scale_log2), 1e-30f);
    const uint32_t on = lane == 0;
    uint32_t s_ph = 0, o_ph = 0, sync_ph = 0;
    bool ok = true;
    int n_items = 0;
    auto read_item = [&]() {
      const int at = n_items % ITEMS;
      if (ok) ok = mbar_warp_wait(&t->item_full[at], (n_items / ITEMS) & 1, &t->abort_flag);
      Item d = t->item[at];
      if (!ok) d.more = 0;
      return d;
    };
    auto next_item = [&]() {                         // the present one's place may be used again
      __syncwarp();
      if (lane == 0) mbar_arrive(&t->item_empty[n_items % ITEMS]);
      ++n_items;
    };
    // A row that is not there goes along with the last one that is, and is not written.
    auto row_of = [&](const Item& d) { return d.row0 + x * 128 + min(row, d.rows - x * 128 - 1); };
    auto fetch_q = [&](const Item& d) {              // a warp's 32 rows, LANES lanes along a row
      constexpr int LANES = DCH * 8, AT_ONCE = 32 / LANES;       // (of three chunks: 24 lanes, the rest have nothing to do)
      const int rr = row_of(d), tok = kv_token_of(p, rr);
      const uint16_t* mine = reinterpret_cast<const uint16_t*>(p.q) + (int64_t)(d.q_first + tok) * p.q_token_stride +
                             (int64_t)(d.head0 + (rr - tok * p.group)) * p.q_head_stride;
      const int piece = lane % LANES, sub = lane / LANES;
      const bool there = piece * 8 < v.head_dim;
      const uint32_t to = smem_u32(q_smem) + x * Q_TILE + (piece >> 3) * Q_CHUNK;
#pragma unroll 4
      for (int i = 0; i < 32; i += AT_ONCE) {
        const uint16_t* from = reinterpret_cast<const uint16_t*>(__shfl_sync(FULL_MASK, reinterpret_cast<unsigned long long>(mine), i + sub));
        const int r = (warp & 3) * 32 + i + sub;
        if (sub < AT_ONCE) cp_async_16(to + r * 128 + (((piece & 7) ^ (r & 7)) << 4), from + (there ? piece * 8 : 0), there);
      }
      cp_async_arrive(&t->q_full[x]);                // when this thread's copies have landed
    };
    auto group_sync = [&]() {
      __syncwarp();
      arrive_one(&t->group_sync[x], on);
      if (ok) ok = mbar_warp_wait(&t->group_sync[x], sync_ph, &t->abort_flag);
      sync_ph ^= 1u;
    };
    bool fetched = false;
    Item item = read_item();
    while (item.more) {
      if (item.rows <= x * 128) {                    // none of this row tile's rows
        next_item();
        item = read_item();
        continue;
      }
      if (!fetched) fetch_q(item);
      fetched = false;
      Item after = {};
      const bool live = row < item.rows - x * 128;
      const int rr = row_of(item), tok = kv_token_of(p, rr), hq = item.head0 + (rr - tok * p.group);
      const int pos = item.first_pos + tok;
      const int lowest = __shfl_sync(FULL_MASK, pos, 0), highest = __shfl_sync(FULL_MASK, pos, 31);     // of the warp's rows
      float m = -INFINITY, l = 0.0f;
      const int units = UNITS * (item.to - item.from);
      // The two row tiles' warps on one scheduler take turns with their exponentials: at the same time they would
      // both have them, and then both load scores and look for maxima while the special-function unit has
      // nothing to do.  A begins; what B passes on after its last unit of an item would be one too many.
      const bool paired = TILES == 2 && item.rows > 128;
      if (paired && x == 1) turn_pass(warp);
      bool last_seen = false;
      for (int u = 0; u < units; ++u) {
        const int half = u & 1;
        if (ok) ok = mbar_warp_wait(&t->s_full[x][half], (s_ph >> half) & 1u, &t->abort_flag);
        __syncwarp();
        tc_fence_after_sync();
        uint32_t va[64];
        tmem_ld_32x64(s_addr + half * 64, va);
        if (u + 1 == units) {                        // the item's last scores are there: its query is no longer read
          next_item();
          after = read_item();
          fetched = after.more && after.rows > x * 128;
          if (fetched) fetch_q(after);
        }
        const int k = item.from + u / UNITS;
        const int key0 = (k < item.sink_tiles ? k : item.first_tile + (k - item.sink_tiles)) * KEYS + u % UNITS * 64, last = key0 + 63;
        const bool clear = last <= lowest && (!p.window || key0 > highest - p.window || last < p.sinks);
        tmem_ld_wait_for(va);
        if (!clear) {
          // Hidden keys become minus infinity.  One bit per key: at or before the row's position, and in its window
          // or a sink.
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const int j = key0 + y * 32;
            uint32_t seen = bits_below(pos - j + 1);
            if (p.window) seen &= ~bits_below(pos - p.window + 1 - j) | bits_below(p.sinks - j);
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!(seen & (1u << i))) va[y * 32 + i] = 0xff800000u;
          }
        }
        float g[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 64; i += 8) {
#pragma unroll
          for (int y = 0; y < 4; ++y) g[y] = fmax3(g[y], __uint_as_float(va[i + 2 * y]), __uint_as_float(va[i + 2 * y + 1]));
        }
        const float top = fmaxf(fmax3(g[0], g[1], g[2]), g[3]) * scale;
        const bool raise = top > m + RAISE || (m == -INFINITY && top > -INFINITY);
        if (__any_sync(FULL_MASK, raise)) {
          const float now = raise ? top : m;
          const float shrink = raise ? (m == -INFINITY ? 0.0f : exp2_fast(m - now)) : 1.0f;
          m = now;
          l *= shrink;
          if (u > 0) {
            // All products into O so far have to be complete: those before the scores of unit u + 1 are when these
            // are there; for the last unit there is a barrier of its own.
            if (ok) {
              if (u + 1 < units) {
                ok = mbar_warp_wait(&t->s_full[x][half ^ 1], (s_ph >> (half ^ 1)) & 1u, &t->abort_flag);
              } else {
                ok = mbar_warp_wait(&t->o_last[x], o_ph, &t->abort_flag);
                last_seen = true;
              }
            }
            tc_fence_after_sync();
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
        float base = (m == -INFINITY ? 0.0f : m) - LIFT<F16>;
        if (paired) {
          // (the zero that is read behind the wait keeps the exponentials behind it too: nothing else would; on
          // the other side the store of the weights does)
          turn_wait(warp);
          base -= *reinterpret_cast<volatile float*>(&t->zero);
        }
        const uint64_t scale2 = pair_of(scale, scale), base2 = pair_of(-base, -base);
        uint64_t sum2[2] = {0, 0};
        uint32_t w[32];
        weights<F16>(va, scale2, base2, sum2, w);
        tmem_st_32x32(s_addr + half * 64, w);
        if (paired && (x == 0 || u + 1 < units)) turn_pass(warp);
        tmem_st_wait();
        tc_fence_before_sync();
        __syncwarp();
        arrive_one(&t->p_full[x][half], on);
        float sa, sb;
        split_pair(add_pairs(sum2[0], sum2[1]), &sa, &sb);
        l += sa + sb;
        s_ph ^= 1u << half;
      }
      if (!last_seen && ok) ok = mbar_warp_wait(&t->o_last[x], o_ph, &t->abort_flag);      // (keeps count of its rounds)
      // ---- the result, or a piece of it
      if (ok) ok = mbar_warp_wait(&t->o_full[x], o_ph, &t->abort_flag);
      o_ph ^= 1u;
      __syncwarp();
      tc_fence_after_sync();
      uint16_t* to = reinterpret_cast<uint16_t*>(p.out) + (int64_t)(item.q_first + tok) * p.out_token_stride + (int64_t)hq * p.out_head_stride;
      if (item.whole) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        uint32_t o[AT_HAND][64];
#pragma unroll
        for (int c = 0; c < AT_HAND; ++c) tmem_ld_32x64(o_addr + c * 64, o[c]);
#pragma unroll
        for (int c = 0; c < DCH; ++c) {
          if (c >= AT_HAND) tmem_ld_32x64(o_addr + c * 64, o[c % AT_HAND]);
          tmem_ld_wait_for(o[c % AT_HAND]);
#pragma unroll
          for (int i = 0; i < 64; i += 16) {
            uint32_t w[8];
#pragma unroll
            for (int y = 0; y < 8; ++y) w[y] = pack2<F16>(__uint_as_float(o[c % AT_HAND][i + 2 * y]) * inv, __uint_as_float(o[c % AT_HAND][i + 2 * y + 1]) * inv);
            if (live) store_row<F16>(to, c * 64 + i, v.head_dim, w);
          }
        }
        tc_fence_before_sync();
      } else {
        // layout of a piece: its rows' maxima, their sums, then four columns of all rows at a time (rows that are not there
        // are left out)
        const int r = x * 128 + row;
        float* slot = p.partials + (size_t)item.my_slot * p.partial_floats;
        if (live) {
          slot[r] = m;
          slot[ROWS + r] = l;
        }
        uint32_t o[AT_HAND][64];
#pragma unroll
        for (int c = 0; c < AT_HAND; ++c) tmem_ld_32x64(o_addr + c * 64, o[c]);
#pragma unroll
        for (int c = 0; c < DCH; ++c) {
          if (c >= AT_HAND) tmem_ld_32x64(o_addr + c * 64, o[c % AT_HAND]);
          tmem_ld_wait_for(o[c % AT_HAND]);
          if (live) {
#pragma unroll
            for (int i = 0; i < 64; i += 4)
              *reinterpret_cast<uint4*>(slot + 2 * ROWS + ((c * 64 + i) / 4 * ROWS + r) * 4) = make_uint4(o[c % AT_HAND][i], o[c % AT_HAND][i + 1], o[c % AT_HAND][i + 2], o[c % AT_HAND][i + 3]);
          }
        }
        tc_fence_before_sync();
        const typename Walk::Pieces pieces{item.piece_first, item.pieces};
        group_sync();
        if (row == 0) {
          int* arrivals = p.arrivals + pieces.first * 2 + x;
          t->last[x] = kv_arrive(arrivals) == pieces.n - 1;
          if (t->last[x]) *arrivals = 0;             // ready for the next launch
        }
        group_sync();
        if (t->last[x]) {
          // Join the pieces, in the order of the CTAs: a row per thread, FLIGHT pieces' loads of eight columns' groups
          // under way at a time (they come from L2, a microsecond away).  Written to be short: code that runs once
          // costs its own way from memory, and a version that spread few rows over all threads was slower for it.
          if (live) {                                // (whole batches of loads, the last piece again where there are fewer)
            float top = -INFINITY, total = 0.0f;
#pragma unroll 1
            for (int c0 = 0; c0 < pieces.n; c0 += 8) {
              float pm[8], pl[8];
#pragma unroll
              for (int c = 0; c < 8; ++c) {
                const float* from = p.partials + (size_t)pieces.slot(min(c0 + c, pieces.n - 1)) * p.partial_floats + r;
                pm[c] = __ldcg(from);
                pl[c] = c0 + c < pieces.n ? __ldcg(from + ROWS) : 0.0f;
              }
              float now = top;
#pragma unroll
              for (int c = 0; c < 8; ++c) now = fmaxf(now, pm[c]);
              const float base = now == -INFINITY ? 0.0f : now;
              total *= exp2_fast(top - base);
              top = now;
#pragma unroll
              for (int c = 0; c < 8; ++c) total += exp2_fast(pm[c] - base) * pl[c];
            }
            if (top == -INFINITY) top = 0.0f;
            const float inv = total == 0.0f ? 0.0f : 1.0f / total;
            constexpr int FLIGHT = 4;
#pragma unroll 1
            for (int c32 = 0; c32 < DIM; c32 += 32) {
              float4 acc[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) acc[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
              for (int c0 = 0; c0 < pieces.n; c0 += FLIGHT) {
                float4 y[FLIGHT][8];
                float w[FLIGHT];
#pragma unroll
                for (int c = 0; c < FLIGHT; ++c) {
                  const float* from = p.partials + (size_t)pieces.slot(c0 + c) * p.partial_floats;
                  w[c] = -INFINITY;
#pragma unroll
                  for (int i = 0; i < 8; ++i) y[c][i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                  if (c0 + c < pieces.n) {
                    w[c] = __ldcg(from + r);
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[c][i] = __ldcg(reinterpret_cast<const float4*>(from + 2 * ROWS + ((c32 / 4 + i) * ROWS + r) * 4));
                  }
                }
#pragma unroll
                for (int c = 0; c < FLIGHT; ++c) {
                  const float f = exp2_fast(w[c] - top) * inv;
#pragma unroll
                  for (int i = 0; i < 8; ++i) {
                    acc[i].x += f * y[c][i].x;
                    acc[i].y += f * y[c][i].y;
                    acc[i].z += f * y[c][i].z;
                    acc[i].w += f * y[c][i].w;
                  }
                }
              }
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                uint32_t w[8];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                  w[2 * y] = pack2<F16>(acc[4 * i + y].x, acc[4 * i + y].y);
                  w[2 * y + 1] = pack2<F16>(acc[4 * i + y].z, acc[4 * i + y].w);
                }
                store_row<F16>(to, c32 + 16 * i, v.head_dim, w);
              }
            }
          }
        }
      }
      item = after;
    }
    // A warp that leaves early, because a wait ran out, must not leave its partner in a turn that nobody passes on: it
    // passes turns on until the partner has left too (whose other waits have limits).
    __syncwarp();
    if (lane == 0) *reinterpret_cast<volatile int*>(&t->left[warp]) = 1;
    if (!ok && lane == 0) kv_report(v, KV_TIMEOUT);
    if (!ok && TILES == 2) {
      const long long t0 = clock64();
      while (__all_sync(FULL_MASK, *reinterpret_cast<volatile int*>(&t->left[warp ^ 4]) == 0 && clock64() - t0 < 8 * WAIT_LIMIT_CYCLES)) {
        turn_pass(warp);
        __nanosleep(1000);
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

template <bool F16, int DCH>
struct Launch {
  static constexpr auto kernel = kv_extend_kernel<F16, DCH>;
  static cudaError_t configure(int smem_optin) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin); }
  static cudaError_t run(const KvAttendParams& p, const CUtensorMap& tmap, int sm_count, int smem_optin, cudaStream_t st) {
    int slots = 2;                                   // an even number: keys take the even slots, values the odd ones
    while (slots + 2 <= MAX_SLOTS && extend_smem<DCH>(slots + 2) <= smem_optin) slots += 2;
    return launch_overlapped(kernel, dim3(sm_count), dim3(THREADS), extend_smem<DCH>(slots), st, 1, p, tmap, slots);
  }
};

// f(Launch<type, chunks>()) for a head_dim.
template <bool F16, typename F>
cudaError_t for_dim(int head_dim, F f) {
  if (head_dim <= 64) return f(Launch<F16, 1>());
  if (head_dim <= 128) return f(Launch<F16, 2>());
  if (head_dim <= 192) return f(Launch<F16, 3>());
  return f(Launch<F16, 4>());
}

}  // namespace

cudaError_t kv_extend_configure(int smem_optin) {
  cudaError_t e = cudaSuccess;
  auto configure = [&](auto launch) { return launch.configure(smem_optin); };
  for (int head_dim = 64; head_dim <= 256 && e == cudaSuccess; head_dim += 64) {
    e = for_dim<false>(head_dim, configure);
    if (e == cudaSuccess) e = for_dim<true>(head_dim, configure);
  }
  return e;
}

size_t kv_extend_partial_floats(int head_dim) { return (size_t)(head_dim <= 128 ? 256 : 128) * (2 + (head_dim + 63) / 64 * 64); }

cudaError_t kv_extend_launch(const KvAttendParams& p, const CUtensorMap& tmap, bool f16, int sm_count, int smem_optin, cudaStream_t st) {
  auto run = [&](auto launch) { return launch.run(p, tmap, sm_count, smem_optin, st); };
  return f16 ? for_dim<true>(p.v.head_dim, run) : for_dim<false>(p.v.head_dim, run);
}

}  // namespace icc
