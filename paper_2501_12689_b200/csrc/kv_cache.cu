// Host side of the C ABI declared in include/ic_kv.h: argument checking, buffer ownership and kernel
// sequencing of the paged key-value cache.
#include <math.h>
#include <string.h>

#include <mutex>
#include <new>

#include "../../include/ic_kv.h"
#include "host_util.h"
#include "kv.h"

using icc::DeviceGuard;
using icc::fail;
using icc::is_device_ptr;

struct ic_kv {
  icc::KvView v;
  int device = 0;
  int sm_count = 0;
  int smem_optin = 0;
  bool f16 = false;
  cudaStream_t stream = nullptr;
  void* own_pool = nullptr;
  void* own_books = nullptr;       // tables, lengths and refs that were not lent
  void* own_workspace = nullptr;
  int* h_status = nullptr;
  int64_t launches = 0;
  CUtensorMap tmap;                // the pool, row by row
  float* partials = nullptr;       // in the workspace: pieces of attention split over a cache's length
  int* arrivals = nullptr;
  size_t partial_floats = 0;
};

namespace {

// Mapped host words for the handles' errors.  Allocating pinned memory takes longer than everything else in a
// creation, so a block of words serves many handles of the process; blocks are never given back.
struct StatusBlock {
  static constexpr int WORDS = 1024;
  int* words = nullptr;
  bool used[WORDS] = {};
  StatusBlock* next = nullptr;
};
std::mutex g_status_mutex;
StatusBlock* g_status_blocks = nullptr;

int* take_status_word() {
  std::lock_guard<std::mutex> lock(g_status_mutex);
  for (StatusBlock* b = g_status_blocks;; b = b->next) {
    if (!b) {
      void* p = nullptr;
      b = new (std::nothrow) StatusBlock;
      if (!b || cudaHostAlloc(&p, StatusBlock::WORDS * sizeof(int), cudaHostAllocMapped | cudaHostAllocPortable) != cudaSuccess) {
        cudaGetLastError();
        delete b;
        return nullptr;
      }
      b->words = static_cast<int*>(p);
      b->next = g_status_blocks;
      g_status_blocks = b;
    }
    for (int i = 0; i < StatusBlock::WORDS; ++i)
      if (!b->used[i]) {
        b->used[i] = true;
        b->words[i] = 0;
        return b->words + i;
      }
  }
}
void give_status_word(int* w) {
  std::lock_guard<std::mutex> lock(g_status_mutex);
  for (StatusBlock* b = g_status_blocks; b; b = b->next)
    if (w >= b->words && w < b->words + StatusBlock::WORDS) b->used[w - b->words] = false;
}

// The kernels' shared-memory limits, once per device.
cudaError_t configure_kernels(int dev, int smem) {
  static std::mutex mutex;
  static bool done[64] = {};
  std::lock_guard<std::mutex> lock(mutex);
  if (dev < 64 && done[dev]) return cudaSuccess;
  cudaError_t e = icc::kv_pages_configure(smem);
  if (e == cudaSuccess) e = icc::kv_decode_configure(smem);
  if (e == cudaSuccess) e = icc::kv_extend_configure(smem);
  if (e == cudaSuccess && dev < 64) done[dev] = true;
  return e;
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

int check_opts(const ic_kv_opts_t* o) {
  if (o->dtype != IC_KV_BF16 && o->dtype != IC_KV_F16) return fail(IC_ERR_INVALID, "unknown dtype %d", o->dtype);
  if (o->head_dim < 8 || o->head_dim > IC_KV_MAX_HEAD_DIM || o->head_dim % 8)
    return fail(IC_ERR_INVALID, "head_dim %d must be a multiple of 8 in [8, %d]", o->head_dim, IC_KV_MAX_HEAD_DIM);
  if (o->page_size < 8 || o->page_size > IC_KV_MAX_PAGE || (o->page_size & (o->page_size - 1)))
    return fail(IC_ERR_INVALID, "page_size %d must be a power of two in [8, %d]", o->page_size, IC_KV_MAX_PAGE);
  if (o->n_layers < 1 || o->n_kv_heads < 1 || o->n_kv_heads > 1024 || o->n_layers > 1024)
    return fail(IC_ERR_INVALID, "n_layers %d and n_kv_heads %d must be in [1, 1024]", o->n_layers, o->n_kv_heads);
  if (o->n_pages < 1) return fail(IC_ERR_INVALID, "n_pages %d must be positive", o->n_pages);
  if (o->max_seqs < 1 || o->max_seqs > IC_KV_MAX_SEQS) return fail(IC_ERR_INVALID, "max_seqs %d must be in [1, %d]", o->max_seqs, IC_KV_MAX_SEQS);
  // a position is a 32-bit number, and so is an index of the page tables
  if (o->max_pages < 1 || (int64_t)o->max_pages * o->page_size > 0x7fffffffll || (int64_t)o->max_pages * o->max_seqs > 0x7fffffffll)
    return fail(IC_ERR_INVALID, "max_pages %d: a row must hold fewer than 2^31 tokens and the tables fewer than 2^31 entries", o->max_pages);
  // rows of head_dim elements are what the tensor maps count, in 32 bits
  const double rows = (double)o->n_pages * o->n_layers * 2.0 * o->n_kv_heads * o->page_size;
  if (rows > 2147483647.0) return fail(IC_ERR_UNSUPPORTED, "a pool of %.0f rows (pages x layers x 2 x heads x page_size) exceeds 2^31 - 1", rows);
  return IC_OK;
}

// Pieces of the workspace, in order; `kv` (may be null) gets their addresses.
size_t carve(const ic_kv_opts_t* o, unsigned char* base, ic_kv* kv) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* p = base ? base + off : nullptr;
    off += up256(bytes);
    return p;
  };
  auto ints = [&](size_t n) { return reinterpret_cast<int*>(take(n * 4)); };
  int* err = ints(64);
  int* arrivals = ints(2 * icc::KV_MAX_CTAS);
  int* mark = ints(o->max_seqs);
  int* had = ints(o->max_seqs);
  int* upto = ints(o->max_seqs);
  int* shared = ints(o->max_seqs);
  int* begin = ints(o->max_seqs);
  int* fresh = ints(o->n_pages);
  int2* jobs = reinterpret_cast<int2*>(take((size_t)o->n_pages * 8));
  int* staged = ints((size_t)o->max_seqs * o->max_pages);
  const size_t partial_floats = icc::kv_extend_partial_floats(o->head_dim);      // (the decode kernel's pieces are smaller)
  float* partials = reinterpret_cast<float*>(take(2 * icc::KV_MAX_CTAS * partial_floats * 4));
  if (kv) {
    icc::KvView* at = &kv->v;
    kv->arrivals = arrivals;
    kv->partials = partials;
    kv->partial_floats = partial_floats;
    at->err = err;
    at->meta = err + 32;
    at->mark = mark;
    at->had = had;
    at->upto = upto;
    at->shared = shared;
    at->begin = begin;
    at->fresh = fresh;
    at->jobs = jobs;
    at->staged = staged;
  }
  return off;
}
// The words at the head of the workspace that start out as zeros, and that a kernel which gave up may leave otherwise:
// error, plan, arrivals, marks.
size_t zero_bytes(int max_seqs) { return 256 + up256(2 * icc::KV_MAX_CTAS * 4) + up256((size_t)max_seqs * 4); }

int read_opts(const ic_kv_opts_t* opts, ic_kv_opts_t* o) {
  memset(o, 0, sizeof *o);
  if (!opts) return fail(IC_ERR_INVALID, "NULL options");
  if (opts->struct_size < sizeof(uint32_t) || opts->struct_size > sizeof *o)
    return fail(IC_ERR_INVALID, "opts.struct_size %u not understood (this build: %zu)", opts->struct_size, sizeof *o);
  memcpy(o, opts, opts->struct_size);
  return check_opts(o);
}

int reported(int code) {
  switch (code) {
    case icc::KV_FULL: return fail(IC_ERR_FULL, "an earlier call found too few free pages or a full table row and changed nothing; call ic_kv_sync to clear");
    case icc::KV_INVALID: return fail(IC_ERR_INVALID, "an earlier call was given a bad sequence, count or start on the device; call ic_kv_sync to clear");
    default: return fail(IC_ERR_TIMEOUT, "an earlier kernel gave up on a bounded wait (code %d); call ic_kv_sync to clear", code);
  }
}

int check_handle(ic_kv* kv) {
  if (!kv) return fail(IC_ERR_INVALID, "NULL handle");
  const int code = *reinterpret_cast<volatile int*>(kv->h_status);
  return code == icc::KV_OK ? IC_OK : reported(code);
}

int check_rows(const ic_kv* kv, const void* p, int64_t token_stride, int64_t head_stride, const char* what) {
  if (!p || !is_device_ptr(p, kv->device)) return fail(IC_ERR_INVALID, "%s must be a device pointer on device %d", what, kv->device);
  constexpr int64_t most = 1ll << 46;      // more than an address has, and times 65535 heads a 63-bit number
  if ((reinterpret_cast<uintptr_t>(p) & 15) || token_stride % 8 || head_stride % 8 || token_stride < 0 || head_stride < 0 || token_stride > most ||
      head_stride > most)
    return fail(IC_ERR_INVALID, "%s must be 16-byte aligned, its strides (%lld, %lld) non-negative multiples of 8 elements", what,
                (long long)token_stride, (long long)head_stride);
  return IC_OK;
}

// Rows of `length` elements at t * token_stride + h * head_stride, t < tokens, h < heads: do two of them share an element?
bool rows_overlap(int64_t tokens, int64_t heads, int64_t token_stride, int64_t head_stride, int64_t length) {
  if (tokens > 1 && token_stride < length) return true;
  if (heads > 1 && head_stride < length) return true;
  if (tokens <= 1 || heads <= 1) return false;
  // one within the other, as in a tensor of tokens and heads in either order
  if ((token_stride - length) / head_stride >= heads - 1 || (head_stride - length) / token_stride >= tokens - 1) return false;
  // otherwise: a head h further on is d tokens back, give or take less than a row
  for (int64_t h = 1; h < heads; ++h) {
    const int64_t d = h * head_stride / token_stride, rest = h * head_stride - d * token_stride;
    if (d < tokens && d > 0 && rest < length) return true;
    if (d + 1 < tokens && token_stride - rest < length) return true;
  }
  return false;
}

int check_list(const ic_kv* kv, const int32_t* p, const char* what) {
  if (!p || !is_device_ptr(p, kv->device) || (reinterpret_cast<uintptr_t>(p) & 3))
    return fail(IC_ERR_INVALID, "%s must be a device array on device %d", what, kv->device);
  return IC_OK;
}

int check_n(const ic_kv* kv, int32_t n) {
  if (n < 0 || n > kv->v.max_seqs) return fail(IC_ERR_INVALID, "n = %d outside [0, max_seqs = %d]", n, kv->v.max_seqs);
  return IC_OK;
}

// The pool as rows of head_dim elements; a box is 64 elements (128 bytes, swizzled) of the rows of a page, at
// most 64 of them; what lies beyond head_dim reads as zero.
int encode_pool(ic_kv* kv) {
  cudaDriverEntryPointQueryResult qres;
  void* fn = nullptr;
  const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
  if (e != cudaSuccess || qres != cudaDriverEntryPointSuccess || !fn) {
    cudaGetLastError();
    return fail(IC_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  }
  const icc::KvView& v = kv->v;
  const int page = 1 << v.page_shift;
  cuuint64_t dims[2] = {(cuuint64_t)v.head_dim, (cuuint64_t)v.n_pages * v.n_layers * 2 * v.n_kv_heads * page};
  cuuint64_t strides[1] = {(cuuint64_t)v.head_dim * 2};
  cuuint32_t box[2] = {64, (cuuint32_t)(page < 64 ? page : 64)};
  cuuint32_t estr[2] = {1, 1};
  const CUresult r = reinterpret_cast<icc::EncodeTiledFn>(fn)(
      &kv->tmap, kv->f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, v.pool, dims, strides, box, estr,
      CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? IC_OK : fail(IC_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
}

int launched(ic_kv* kv, cudaError_t e, int n, const char* what) {
  if (e != cudaSuccess) return fail(IC_ERR_CUDA, "%s launch failed: %s", what, cudaGetErrorString(e));
  kv->launches += n;
  return IC_OK;
}

}  // namespace

extern "C" {

size_t ic_kv_workspace_bytes(const ic_kv_opts_t* opts) {
  ic_kv_opts_t o;
  if (read_opts(opts, &o) != IC_OK) return 0;
  return carve(&o, nullptr, nullptr);
}

ic_kv_t* ic_kv_create(const ic_kv_opts_t* opts) {
  ic_kv_opts_t o;
  if (read_opts(opts, &o) != IC_OK) return nullptr;
  int ndev = 0;
  cudaError_t e = cudaGetDeviceCount(&ndev);
  if (e != cudaSuccess || ndev == 0) {
    cudaGetLastError();
    fail(IC_ERR_CUDA, "no usable CUDA device (%s); this library has no CPU fallback", e != cudaSuccess ? cudaGetErrorString(e) : "device count is 0");
    return nullptr;
  }
  int dev = o.device;
  if (dev < 0 && cudaGetDevice(&dev) != cudaSuccess) {
    fail(IC_ERR_CUDA, "cudaGetDevice failed");
    return nullptr;
  }
  if (dev >= ndev) {
    fail(IC_ERR_INVALID, "device %d does not exist (%d devices)", dev, ndev);
    return nullptr;
  }
  DeviceGuard guard(dev);
  int major = 0, minor = 0, sms = 0, smem = 0;
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&smem, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev) != cudaSuccess) {
    cudaGetLastError();
    fail(IC_ERR_CUDA, "reading the device's attributes failed");
    return nullptr;
  }
  if (major != 10 || sms > icc::KV_MAX_CTAS) {
    fail(IC_ERR_UNSUPPORTED, "device %d is sm_%d%d with %d multiprocessors; this library is built for sm_100a only", dev, major, minor, sms);
    return nullptr;
  }
  ic_kv* kv = new (std::nothrow) ic_kv();
  if (!kv) {
    fail(IC_ERR_NOMEM, "host allocation failed");
    return nullptr;
  }
  memset(&kv->v, 0, sizeof kv->v);
  kv->device = dev;
  kv->sm_count = sms;
  kv->smem_optin = smem;
  kv->f16 = o.dtype == IC_KV_F16;
  kv->stream = static_cast<cudaStream_t>(o.stream);
  icc::KvView& v = kv->v;
  v.n_pages = o.n_pages;
  v.n_layers = o.n_layers;
  v.n_kv_heads = o.n_kv_heads;
  v.head_dim = o.head_dim;
  v.max_seqs = o.max_seqs;
  v.max_pages = o.max_pages;
  while ((1 << v.page_shift) < o.page_size) ++v.page_shift;
  v.page_bytes = (size_t)o.n_layers * 2 * o.n_kv_heads * o.page_size * o.head_dim * 2;

  bool ok = true;
  auto lent = [&](const void* p, uintptr_t align, const char* what) {
    if (is_device_ptr(p, dev) && (reinterpret_cast<uintptr_t>(p) & (align - 1)) == 0) return true;
    fail(IC_ERR_INVALID, "opts.%s must be a %d-byte aligned device pointer on device %d", what, (int)align, dev);
    return false;
  };
  auto allocate = [&](void** p, size_t bytes, size_t clear, const char* what) {
    e = cudaMalloc(p, bytes);
    if (e == cudaSuccess && clear) e = cudaMemsetAsync(*p, 0, clear, kv->stream);
    if (e == cudaSuccess) return true;
    cudaGetLastError();
    fail(IC_ERR_NOMEM, "cudaMalloc of %zu bytes for the %s failed: %s", bytes, what, cudaGetErrorString(e));
    return false;
  };
  // the pool
  if (o.pool) ok = lent(o.pool, 256, "pool");
  else ok = allocate(&kv->own_pool, v.page_bytes * o.n_pages, 0, "pool");
  v.pool = static_cast<unsigned char*>(o.pool ? o.pool : kv->own_pool);
  // the books: those that were not lent share one allocation
  const size_t tb = up256((size_t)o.max_seqs * o.max_pages * 4), lb = up256((size_t)o.max_seqs * 4), rb = up256((size_t)o.n_pages * 4);
  if (ok && o.tables) ok = lent(o.tables, 16, "tables");
  if (ok && o.lengths) ok = lent(o.lengths, 16, "lengths");
  if (ok && o.refs) ok = lent(o.refs, 16, "refs");
  const size_t books = (o.tables ? 0 : tb) + (o.lengths ? 0 : lb) + (o.refs ? 0 : rb);
  if (ok && books) ok = allocate(&kv->own_books, books, books, "page tables");
  if (ok) {
    unsigned char* b = static_cast<unsigned char*>(kv->own_books);
    auto place = [&](int32_t* given, size_t bytes) {
      if (given) return static_cast<int*>(given);
      int* p = reinterpret_cast<int*>(b);
      b += bytes;
      return p;
    };
    v.tables = place(o.tables, tb);
    v.lengths = place(o.lengths, lb);
    v.refs = place(o.refs, rb);
  }
  // scratch
  const size_t need = carve(&o, nullptr, nullptr), clear = zero_bytes(o.max_seqs);
  if (ok && o.workspace) {
    ok = lent(o.workspace, 256, "workspace");
    if (ok && o.workspace_bytes < need) {
      fail(IC_ERR_NOMEM, "opts.workspace holds %zu bytes, %zu are needed", o.workspace_bytes, need);
      ok = false;
    }
    if (ok && (cudaMemsetAsync(o.workspace, 0, clear, kv->stream) != cudaSuccess)) {
      cudaGetLastError();
      fail(IC_ERR_CUDA, "clearing the head of opts.workspace failed");
      ok = false;
    }
  } else if (ok) {
    ok = allocate(&kv->own_workspace, need, clear, "workspace");
  }
  if (ok) carve(&o, static_cast<unsigned char*>(o.workspace ? o.workspace : kv->own_workspace), kv);
  if (ok) {
    kv->h_status = take_status_word();
    e = kv->h_status ? cudaHostGetDevicePointer(reinterpret_cast<void**>(&v.host_status), kv->h_status, 0) : cudaErrorMemoryAllocation;
    if (e == cudaSuccess) e = configure_kernels(dev, smem);
    if (e != cudaSuccess) {
      cudaGetLastError();
      fail(IC_ERR_CUDA, "setting up the cache failed: %s", cudaGetErrorString(e));
      ok = false;
    }
  }
  if (ok) ok = encode_pool(kv) == IC_OK;
  if (!ok) {
    char keep[512];
    strncpy(keep, ic_cache_last_error(), sizeof keep - 1);
    keep[sizeof keep - 1] = 0;
    ic_kv_destroy(kv);
    fail(IC_ERR_CUDA, "%s", keep);
    return nullptr;
  }
  return kv;
}

void ic_kv_destroy(ic_kv_t* kv) {
  if (!kv) return;
  DeviceGuard guard(kv->device);
  cudaStreamSynchronize(kv->stream);
  if (kv->own_pool) cudaFree(kv->own_pool);
  if (kv->own_books) cudaFree(kv->own_books);
  if (kv->own_workspace) cudaFree(kv->own_workspace);
  if (kv->h_status) give_status_word(kv->h_status);
  delete kv;
}

int ic_kv_reserve(ic_kv_t* kv, const int32_t* seqs, const int32_t* counts, int32_t n) {
  int rc = check_handle(kv);
  if (rc == IC_OK) rc = check_n(kv, n);
  if (rc != IC_OK || n == 0) return rc;
  if ((rc = check_list(kv, seqs, "seqs")) != IC_OK || (rc = check_list(kv, counts, "counts")) != IC_OK) return rc;
  DeviceGuard guard(kv->device);
  return launched(kv, icc::kv_reserve_launch(kv->v, seqs, counts, n, kv->stream), 1, "reserve");
}

int ic_kv_write(ic_kv_t* kv, int32_t layer, const void* k, const void* v, int64_t token_stride, int64_t head_stride,
                const int32_t* seqs, const int32_t* starts, int32_t n, int64_t n_tokens) {
  int rc = check_handle(kv);
  if (rc == IC_OK) rc = check_n(kv, n);
  if (rc != IC_OK) return rc;
  if (layer < 0 || layer >= kv->v.n_layers) return fail(IC_ERR_INVALID, "layer %d outside [0, %d)", layer, kv->v.n_layers);
  if (n_tokens < 0 || n_tokens > 0x7fffffffll || (!starts && n_tokens != n))
    return fail(IC_ERR_INVALID, "n_tokens = %lld does not fit n = %d", (long long)n_tokens, n);
  if (n == 0 && n_tokens > 0) return fail(IC_ERR_INVALID, "tokens without sequences");
  if (n_tokens == 0) return IC_OK;
  if ((rc = check_rows(kv, k, token_stride, head_stride, "k")) != IC_OK || (rc = check_rows(kv, v, token_stride, head_stride, "v")) != IC_OK ||
      (rc = check_list(kv, seqs, "seqs")) != IC_OK || (starts && (rc = check_list(kv, starts, "starts")) != IC_OK))
    return rc;
  DeviceGuard guard(kv->device);
  int launches = 0;
  const cudaError_t e =
      icc::kv_write_launch(kv->v, layer, k, v, token_stride, head_stride, seqs, starts, n, n_tokens, kv->sm_count, &launches, kv->stream);
  return launched(kv, e, launches, "write");
}

int ic_kv_attend(ic_kv_t* kv, const ic_kv_attend_t* args) {
  int rc = check_handle(kv);
  if (rc != IC_OK) return rc;
  if (!args) return fail(IC_ERR_INVALID, "NULL arguments");
  ic_kv_attend_t a;
  memset(&a, 0, sizeof a);
  if (args->struct_size < sizeof(uint32_t) || args->struct_size > sizeof a)
    return fail(IC_ERR_INVALID, "struct_size %u not understood (this build: %zu)", args->struct_size, sizeof a);
  memcpy(&a, args, args->struct_size);
  if (a.n < 0 || a.n > IC_KV_MAX_SEQS) return fail(IC_ERR_INVALID, "n = %d outside [0, %d]", a.n, IC_KV_MAX_SEQS);
  if (a.layer < 0 || a.layer >= kv->v.n_layers) return fail(IC_ERR_INVALID, "layer %d outside [0, %d)", a.layer, kv->v.n_layers);
  if (a.n_heads < 1 || a.n_heads % kv->v.n_kv_heads || a.n_heads > 65535)
    return fail(IC_ERR_INVALID, "n_heads %d must be a multiple of n_kv_heads %d, at most 65535", a.n_heads, kv->v.n_kv_heads);
  if (a.window < 0 || a.sinks < 0) return fail(IC_ERR_INVALID, "window %d and sinks %d must not be negative", a.window, a.sinks);
  const float scale_log2 = a.scale * 1.4426950408889634f;
  if (!isfinite(scale_log2)) return fail(IC_ERR_INVALID, "scale %g, and scale * log2(e), must be finite", a.scale);
  if (a.n_tokens < 0 || a.n_tokens > 0x7fffffffll / a.n_heads || (!a.starts && a.n_tokens != a.n))
    return fail(IC_ERR_INVALID, "n_tokens = %lld does not fit n = %d and n_heads = %d", (long long)a.n_tokens, a.n, a.n_heads);
  if (a.n == 0 && a.n_tokens > 0) return fail(IC_ERR_INVALID, "tokens without sequences");
  if (a.n_tokens == 0) return IC_OK;
  if ((rc = check_rows(kv, a.q, a.q_token_stride, a.q_head_stride, "q")) != IC_OK ||
      (rc = check_rows(kv, a.out, a.out_token_stride, a.out_head_stride, "out")) != IC_OK ||
      (rc = check_list(kv, a.seqs, "seqs")) != IC_OK || (a.starts && (rc = check_list(kv, a.starts, "starts")) != IC_OK))
    return rc;
  if (rows_overlap(a.n_tokens, a.n_heads, a.out_token_stride, a.out_head_stride, kv->v.head_dim))
    return fail(IC_ERR_INVALID, "rows of out overlap with strides (%lld, %lld)", (long long)a.out_token_stride, (long long)a.out_head_stride);
  icc::KvAttendParams p;
  p.v = kv->v;
  p.q = static_cast<const unsigned char*>(a.q);
  p.out = static_cast<unsigned char*>(a.out);
  p.q_token_stride = a.q_token_stride;
  p.q_head_stride = a.q_head_stride;
  p.out_token_stride = a.out_token_stride;
  p.out_head_stride = a.out_head_stride;
  p.seqs = a.seqs;
  p.starts = a.starts;
  p.n = p.n_seqs = a.n;
  p.n_heads = a.n_heads;
  p.group = a.n_heads / kv->v.n_kv_heads;
  // division by the group as a product: with 2^b >= group, ceil(2^(31 + b) / group) is exact for 31-bit numerators
  int bits = 0;
  while ((1ll << bits) < p.group) ++bits;
  p.group_shift = 31 + bits;
  p.group_magic = (unsigned)(((1ull << p.group_shift) + p.group - 1) / p.group);
  p.layer = a.layer;
  p.n_tokens = a.n_tokens;
  p.window = a.window;
  p.sinks = a.window ? a.sinks : 0;
  p.scale_log2 = scale_log2;
  p.partials = kv->partials;
  p.arrivals = kv->arrivals;
  p.partial_floats = kv->partial_floats;
  DeviceGuard guard(kv->device);
  const int64_t rows = (a.n_tokens + a.n - 1) / a.n * p.group;      // query rows of a sequence and kv head, on average
  for (int off = 0; off < a.n && rc == IC_OK; off += icc::KV_BATCH) {
    p.first_seq = off;
    p.seqs = a.seqs + off;
    p.starts = a.starts ? a.starts + off : nullptr;
    p.n = a.n - off < icc::KV_BATCH ? a.n - off : icc::KV_BATCH;
    cudaError_t e;
    // Few rows are bound by the read of the cache, many by products and exponentials.  16 rows by either kernel, decode | extend, us:
    // 64 sequences of up to 8192 tokens, 2 kv heads, head_dim 64: 59 | 76, 128: 86 | 88, 256: 190 | 147;
    // one of 131,071, 1 kv head, 64: 44 | 102, 128: 53 | 174, 256: 86 | 269; four of up to 300, 128: 18 | 20, 256: 29 | 27.
    if (rows <= 16) e = icc::kv_decode_launch(p, kv->tmap, kv->f16, rows > 8, kv->sm_count, kv->smem_optin, kv->stream);
    else e = icc::kv_extend_launch(p, kv->tmap, kv->f16, kv->sm_count, kv->smem_optin, kv->stream);
    rc = launched(kv, e, 1, "attention");
  }
  return rc;
}

int ic_kv_fork(ic_kv_t* kv, const int32_t* parents, const int32_t* children, const int32_t* upto, int32_t n, int32_t copy) {
  int rc = check_handle(kv);
  if (rc == IC_OK) rc = check_n(kv, n);
  if (rc != IC_OK || n == 0) return rc;
  if ((rc = check_list(kv, parents, "parents")) != IC_OK || (rc = check_list(kv, children, "children")) != IC_OK ||
      (upto && (rc = check_list(kv, upto, "upto")) != IC_OK))
    return rc;
  DeviceGuard guard(kv->device);
  int launches = 0;
  const cudaError_t e = icc::kv_fork_launch(kv->v, parents, children, upto, n, copy != 0, kv->sm_count, &launches, kv->stream);
  return launched(kv, e, launches, "fork");
}

int ic_kv_free(ic_kv_t* kv, const int32_t* seqs, int32_t n) {
  int rc = check_handle(kv);
  if (rc != IC_OK) return rc;
  if (n < 0) return fail(IC_ERR_INVALID, "n = %d is negative", n);
  if (n == 0) return IC_OK;
  if ((rc = check_list(kv, seqs, "seqs")) != IC_OK) return rc;
  DeviceGuard guard(kv->device);
  return launched(kv, icc::kv_free_launch(kv->v, seqs, n, kv->sm_count, kv->stream), 1, "free");
}

int ic_kv_compact(ic_kv_t* kv) {
  int rc = check_handle(kv);
  if (rc != IC_OK) return rc;
  DeviceGuard guard(kv->device);
  int launches = 0;
  const cudaError_t e = icc::kv_compact_launch(kv->v, kv->sm_count, &launches, kv->stream);
  return launched(kv, e, launches, "compact");
}

int ic_kv_sync(ic_kv_t* kv) {
  if (!kv) return fail(IC_ERR_INVALID, "NULL handle");
  DeviceGuard guard(kv->device);
  cudaError_t e = cudaStreamSynchronize(kv->stream);
  if (e != cudaSuccess) return fail(IC_ERR_CUDA, "stream sync failed: %s", cudaGetErrorString(e));
  const int code = *reinterpret_cast<volatile int*>(kv->h_status);
  if (code == icc::KV_OK) return IC_OK;
  *kv->h_status = 0;
  e = cudaMemsetAsync(kv->v.err, 0, zero_bytes(kv->v.max_seqs), kv->stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(kv->stream);
  if (e != cudaSuccess) return fail(IC_ERR_CUDA, "clearing the error failed: %s", cudaGetErrorString(e));
  return reported(code);
}

int ic_kv_set_stream(ic_kv_t* kv, void* cuda_stream) {
  if (!kv) return fail(IC_ERR_INVALID, "NULL handle");
  kv->stream = static_cast<cudaStream_t>(cuda_stream);
  return IC_OK;
}

int64_t ic_kv_launch_count(const ic_kv_t* kv) { return kv ? kv->launches : IC_ERR_INVALID; }

}  // extern "C"
