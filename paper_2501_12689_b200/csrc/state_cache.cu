// Host side of the C ABI declared in include/ic_state.h: argument checking, buffer ownership and kernel
// sequencing of the state cache.
#include <math.h>
#include <string.h>

#include <mutex>
#include <new>

#include "../../include/ic_state.h"
#include "host_util.h"
#include "kv.h"
#include "state.h"
#include "state_schedule.cuh"

using icc::DeviceGuard;
using icc::fail;
using icc::is_device_ptr;

struct ic_state {
  icc::StateView v;
  int device = 0, sm_count = 0, smem_optin = 0;
  bool f16 = false;
  cudaStream_t stream = nullptr;
  void* own_pool = nullptr;
  void* own_workspace = nullptr;
  int* h_status = nullptr;
  int64_t launches = 0;
};

namespace {

static_assert(IC_STATE_MAX_SEQS == icc::STATE_MAX_SEQS, "the checks have a bit for each");
// The head of the workspace: error and plan, then the flags of published states.  Zeros to begin with, and again after an error.
constexpr size_t FLAGS = 256, WORDS = FLAGS + 1024;
static_assert((icc::KV_MAX_CTAS + 1) * 4 <= WORDS - FLAGS, "a flag for each CTA, and their count");
static_assert(icc::STATE_CHECK_THREADS <= icc::STATE_BATCH, "calls of more sequences than a launch takes are checked before");

cudaError_t configure_kernels(int dev, int smem) {
  static std::mutex mutex;
  static bool done[64] = {};
  std::lock_guard<std::mutex> lock(mutex);
  if (dev < 64 && done[dev]) return cudaSuccess;
  cudaError_t e = icc::state_configure(smem);
  if (e == cudaSuccess) e = icc::state_chunk_configure(smem);
  if (e == cudaSuccess && dev < 64) done[dev] = true;
  return e;
}

int read_opts(const ic_state_opts_t* opts, ic_state_opts_t* o) {
  memset(o, 0, sizeof *o);
  if (!opts) return fail(IC_ERR_INVALID, "NULL options");
  if (opts->struct_size < sizeof(uint32_t) || opts->struct_size > sizeof *o)
    return fail(IC_ERR_INVALID, "opts.struct_size %u not understood (this build: %zu)", opts->struct_size, sizeof *o);
  memcpy(o, opts, opts->struct_size);
  if (o->dtype != IC_STATE_BF16 && o->dtype != IC_STATE_F16) return fail(IC_ERR_INVALID, "unknown dtype %d", o->dtype);
  if (o->n_layers < 1 || o->n_layers > 1024 || o->n_heads < 1 || o->n_heads > icc::STATE_MAX_HEADS)
    return fail(IC_ERR_INVALID, "n_layers %d and n_heads %d must be in [1, 1024]", o->n_layers, o->n_heads);
  if (o->key_dim < 8 || o->key_dim > IC_STATE_MAX_KEY_DIM || o->key_dim % 8)
    return fail(IC_ERR_INVALID, "key_dim %d must be a multiple of 8 in [8, %d]", o->key_dim, IC_STATE_MAX_KEY_DIM);
  if (o->value_dim < 8 || o->value_dim > IC_STATE_MAX_VALUE_DIM || o->value_dim % 8)
    return fail(IC_ERR_INVALID, "value_dim %d must be a multiple of 8 in [8, %d]", o->value_dim, IC_STATE_MAX_VALUE_DIM);
  if (o->max_seqs < 1 || o->max_seqs > IC_STATE_MAX_SEQS) return fail(IC_ERR_INVALID, "max_seqs %d must be in [1, %d]", o->max_seqs, IC_STATE_MAX_SEQS);
  return IC_OK;
}

// The mean says little of the longest, and one token after the other takes as long as the longest sequence has tokens.  So in calls of more than DIVIDED_FROM
// tokens that go token by token, sequences of more than STEP_MOST are left to a launch of the chunks behind it.  As a rule that finds none and costs 1.3
// to 3 us (64 sequences of 2 tokens, 32 heads of 128 x 128: 65 us, without it 63; 17 of 4, 4 heads of 64 x 64: 6.8 and 5.5); with 255 single tokens and
// one sequence of 1,500 it takes 281 us, token by token 2,296; 31 and one of 352, 4 heads of 64 x 64: 23 and 192.  Where the two meet: 31 single tokens and one
// sequence of 24, 32, 64 on those 4 heads 16, 21, 38 us token by token, the last divided 14; 255 and one of 33, 64, 128 on 32 heads 227, 273, 365 and 244 to 246.
constexpr int STEP_MOST = 32, DIVIDED_FROM = 64;
size_t list_bytes(int max_seqs) { return ((size_t)max_seqs * 3 * 4 + 255) & ~(size_t)255; }

size_t workspace_need(const ic_state_opts_t& o) {
  return WORDS + list_bytes(o.max_seqs) + icc::KV_MAX_CTAS * icc::state_slot_floats(o.key_dim, o.value_dim) * 4;
}

int reported(int code) {
  if (code == icc::KV_INVALID)
    return fail(IC_ERR_INVALID, "an earlier call was given a bad sequence, start or rate on the device; call ic_state_sync to clear");
  return fail(IC_ERR_TIMEOUT, "an earlier kernel gave up on a bounded wait (code %d); call ic_state_sync to clear", code);
}

int check_handle(ic_state* s) {
  if (!s) return fail(IC_ERR_INVALID, "NULL handle");
  const int code = *reinterpret_cast<volatile int*>(s->h_status);
  return code == icc::KV_OK ? IC_OK : reported(code);
}

int check_rows(const ic_state* s, const void* p, int64_t token_stride, int64_t head_stride, const char* what) {
  if (!p || !is_device_ptr(p, s->device)) return fail(IC_ERR_INVALID, "%s must be a device pointer on device %d", what, s->device);
  constexpr int64_t most = 1ll << 46;
  if ((reinterpret_cast<uintptr_t>(p) & 15) || token_stride % 8 || head_stride % 8 || token_stride < 0 || head_stride < 0 || token_stride > most ||
      head_stride > most)
    return fail(IC_ERR_INVALID, "%s must be 16-byte aligned, its strides (%lld, %lld) non-negative multiples of 8 elements", what,
                (long long)token_stride, (long long)head_stride);
  return IC_OK;
}

int check_list(const ic_state* s, const void* p, const char* what) {
  if (!p || !is_device_ptr(p, s->device) || (reinterpret_cast<uintptr_t>(p) & 3))
    return fail(IC_ERR_INVALID, "%s must be a device array on device %d", what, s->device);
  return IC_OK;
}

int check_n(const ic_state* s, int32_t n) {
  if (n < 0 || n > s->v.max_seqs) return fail(IC_ERR_INVALID, "n = %d outside [0, max_seqs = %d]", n, s->v.max_seqs);
  return IC_OK;
}

// Rows of tokens and heads as a tensor map, if their strides allow one (a shared row, a stride of 0, does only among the heads).
bool encode_rows(const ic_state* s, const icc::StateRows& r, int dim, int64_t tokens, CUtensorMap* map) {
  static const icc::EncodeTiledFn encode = [] {
    cudaDriverEntryPointQueryResult found;
    void* fn = nullptr;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      fn = nullptr;
    }
    return reinterpret_cast<icc::EncodeTiledFn>(fn);
  }();
  const bool shared = r.head_stride == 0;
  const int64_t token_bytes = r.token_stride * 2, head_bytes = shared ? (int64_t)dim * 2 : r.head_stride * 2;
  if (!encode || token_bytes < (int64_t)dim * 2 || head_bytes < (int64_t)dim * 2 || token_bytes >= 1ll << 40 || head_bytes >= 1ll << 40) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)tokens, shared ? 1u : (cuuint64_t)s->v.n_heads};
  const cuuint64_t strides[2] = {(cuuint64_t)token_bytes, (cuuint64_t)head_bytes};
  const cuuint32_t box[3] = {64, icc::STATE_CHUNK, 1}, steps[3] = {1, 1, 1};
  return encode(map, s->f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<unsigned char*>(r.at), dims, strides, box,
                steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int launched(ic_state* s, cudaError_t e, int n, const char* what) {
  if (e != cudaSuccess) return fail(IC_ERR_CUDA, "%s launch failed: %s", what, cudaGetErrorString(e));
  s->launches += n;
  return IC_OK;
}

}  // namespace

extern "C" {

size_t ic_state_workspace_bytes(const ic_state_opts_t* opts) {
  ic_state_opts_t o;
  return read_opts(opts, &o) == IC_OK ? workspace_need(o) : 0;
}

ic_state_t* ic_state_create(const ic_state_opts_t* opts) {
  ic_state_opts_t o;
  if (read_opts(opts, &o) != IC_OK) return nullptr;
  int dev = 0, sms = 0, smem = 0;
  if (icc::usable_device(o.device, &dev, &sms, &smem) != IC_OK) return nullptr;
  DeviceGuard guard(dev);
  const size_t need = workspace_need(o);
  auto lent = [&](const void* p, const char* what) {
    if (!p || (is_device_ptr(p, dev) && (reinterpret_cast<uintptr_t>(p) & 255) == 0)) return true;
    fail(IC_ERR_INVALID, "opts.%s must be a 256-byte aligned device pointer on device %d", what, dev);
    return false;
  };
  if (!lent(o.pool, "pool") || !lent(o.workspace, "workspace")) return nullptr;
  if (o.workspace && o.workspace_bytes < need) {
    fail(IC_ERR_NOMEM, "opts.workspace holds %zu bytes, %zu are needed", o.workspace_bytes, need);
    return nullptr;
  }
  ic_state* s = new (std::nothrow) ic_state();
  if (!s) {
    fail(IC_ERR_NOMEM, "host allocation failed");
    return nullptr;
  }
  memset(&s->v, 0, sizeof s->v);
  s->device = dev;
  s->sm_count = sms;
  s->smem_optin = smem;
  s->f16 = o.dtype == IC_STATE_F16;
  s->stream = static_cast<cudaStream_t>(o.stream);
  icc::StateView& v = s->v;
  v.n_layers = o.n_layers;
  v.n_heads = o.n_heads;
  v.key_dim = o.key_dim;
  v.value_dim = o.value_dim;
  v.max_seqs = o.max_seqs;
  cudaError_t e = cudaSuccess;
  const size_t pool_bytes = v.seq_floats() * 4 * o.max_seqs;
  if (!o.pool) {
    e = cudaMalloc(&s->own_pool, pool_bytes);
    if (e == cudaSuccess) e = cudaMemsetAsync(s->own_pool, 0, pool_bytes, s->stream);
  }
  v.pool = o.pool ? o.pool : static_cast<float*>(s->own_pool);
  if (e == cudaSuccess && !o.workspace) e = cudaMalloc(&s->own_workspace, need);
  v.err = static_cast<int*>(o.workspace ? o.workspace : s->own_workspace);
  v.meta = v.err + 32;
  if (e == cudaSuccess) e = cudaMemsetAsync(v.err, 0, WORDS, s->stream);
  if (e == cudaSuccess && !(s->h_status = icc::take_status_word())) e = cudaErrorMemoryAllocation;
  if (e == cudaSuccess) e = cudaHostGetDevicePointer(reinterpret_cast<void**>(&v.host_status), s->h_status, 0);
  if (e == cudaSuccess) e = configure_kernels(dev, smem);
  if (e != cudaSuccess) {
    cudaGetLastError();
    ic_state_destroy(s);
    fail(e == cudaErrorMemoryAllocation ? IC_ERR_NOMEM : IC_ERR_CUDA, "setting up the states (a pool of %zu bytes) failed: %s", pool_bytes,
         cudaGetErrorString(e));
    return nullptr;
  }
  return s;
}

void ic_state_destroy(ic_state_t* s) {
  if (!s) return;
  DeviceGuard guard(s->device);
  cudaStreamSynchronize(s->stream);
  if (s->own_pool) cudaFree(s->own_pool);
  if (s->own_workspace) cudaFree(s->own_workspace);
  if (s->h_status) icc::give_status_word(s->h_status);
  delete s;
}

int ic_state_attend(ic_state_t* s, const ic_state_attend_t* args) {
  int rc = check_handle(s);
  if (rc != IC_OK) return rc;
  if (!args) return fail(IC_ERR_INVALID, "NULL arguments");
  ic_state_attend_t a;
  memset(&a, 0, sizeof a);
  if (args->struct_size < sizeof(uint32_t) || args->struct_size > sizeof a)
    return fail(IC_ERR_INVALID, "struct_size %u not understood (this build: %zu)", args->struct_size, sizeof a);
  memcpy(&a, args, args->struct_size);
  if ((rc = check_n(s, a.n)) != IC_OK) return rc;
  if (a.layer < 0 || a.layer >= s->v.n_layers) return fail(IC_ERR_INVALID, "layer %d outside [0, %d)", a.layer, s->v.n_layers);
  if (!isfinite(a.scale)) return fail(IC_ERR_INVALID, "scale %g must be finite", a.scale);
  if (a.n_tokens < 0 || a.n_tokens > 0x7fffffffll || (!a.starts && a.n_tokens != a.n))
    return fail(IC_ERR_INVALID, "n_tokens = %lld does not fit n = %d", (long long)a.n_tokens, a.n);
  if (a.n == 0 && a.n_tokens > 0) return fail(IC_ERR_INVALID, "tokens without sequences");
  if (a.n_tokens == 0) return IC_OK;
  if ((rc = check_rows(s, a.q, a.q_token_stride, a.q_head_stride, "q")) != IC_OK ||
      (rc = check_rows(s, a.k, a.k_token_stride, a.k_head_stride, "k")) != IC_OK ||
      (rc = check_rows(s, a.v, a.v_token_stride, a.v_head_stride, "v")) != IC_OK ||
      (rc = check_rows(s, a.out, a.out_token_stride, a.out_head_stride, "out")) != IC_OK ||
      (rc = check_list(s, a.rates, "rates")) != IC_OK || (rc = check_list(s, a.seqs, "seqs")) != IC_OK ||
      (a.starts && (rc = check_list(s, a.starts, "starts")) != IC_OK))
    return rc;
  if (icc::rows_overlap(a.n_tokens, s->v.n_heads, a.out_token_stride, a.out_head_stride, s->v.value_dim))
    return fail(IC_ERR_INVALID, "rows of out overlap with strides (%lld, %lld)", (long long)a.out_token_stride, (long long)a.out_head_stride);
  icc::StateAttendParams p;
  p.v = s->v;
  p.q = {static_cast<const unsigned char*>(a.q), a.q_token_stride, a.q_head_stride};
  p.k = {static_cast<const unsigned char*>(a.k), a.k_token_stride, a.k_head_stride};
  p.val = {static_cast<const unsigned char*>(a.v), a.v_token_stride, a.v_head_stride};
  p.out = {static_cast<const unsigned char*>(a.out), a.out_token_stride, a.out_head_stride};
  p.rates = a.rates;
  p.seqs = a.seqs;
  p.starts = a.starts;
  p.n = a.n;
  p.layer = a.layer;
  p.checked = a.n > icc::STATE_CHECK_THREADS;
  p.n_tokens = a.n_tokens;
  p.scale = a.scale;
  // Token by token or in chunks: up to 64 tokens a sequence, chunks take 9 to 23 us while there are few states, and a token 0.5 to 1.7 us (1 sequence, 4 heads
  // of 64 x 64: 9.4 us against 8.8 for 12 tokens, 11.0 for 16; 32 heads of 128 x 128: 12.7 against 13.5 and 16.8); with an SM's share of two and more
  // they are bound by the states and by their sums (8 such sequences: 23 us against 23 for 8, 29 for 12; 64 of them: 111 against 85 for 4, 128 for 8).
  const int few = (int64_t)a.n * s->v.n_heads > s->sm_count ? 7 : 12;
  const bool by_token = a.n_tokens <= few * (int64_t)a.n, divided = by_token && a.starts && a.n_tokens > DIVIDED_FROM;
  p.most = divided ? STEP_MOST : 0x7fffffff;
  p.least = divided ? STEP_MOST : 0;
  // sequences for the chunks, at most
  const int n = divided && a.n_tokens / (STEP_MOST + 1) < a.n ? (int)(a.n_tokens / (STEP_MOST + 1)) : a.n;
  p.long_ones = reinterpret_cast<int*>(reinterpret_cast<unsigned char*>(s->v.err) + WORDS);
  p.n_long = divided ? n : 0;
  DeviceGuard guard(s->device);
  if (p.checked && (rc = launched(s, icc::state_check_launch(p, s->stream), 1, "check")) != IC_OK) return rc;
  p.slices = (s->v.value_dim + 127) / 128;
  p.flags = reinterpret_cast<unsigned*>(reinterpret_cast<unsigned char*>(s->v.err) + FLAGS);
  p.slots = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(s->v.err) + WORDS + list_bytes(s->v.max_seqs));
  p.slot_floats = icc::state_slot_floats(s->v.key_dim, s->v.value_dim);
  if (by_token) rc = launched(s, icc::state_step_launch(p, s->f16, s->sm_count, s->stream), 1, "state");
  if (rc != IC_OK || (by_token && !divided)) return rc;
  // (a call without starts has a token a sequence and does not come here)
  const int32_t *seqs = a.seqs, *starts = a.starts, *ends = a.starts + 1;
  int among = a.n;                  // sequences that the launches look through
  if (divided && p.checked) {       // the check has picked them
    seqs = p.long_ones;
    starts = p.long_ones + s->v.max_seqs;
    ends = p.long_ones + 2 * s->v.max_seqs;
    among = n;
  }
  p.checked |= by_token;
  icc::StateMaps maps;
  maps.there = encode_rows(s, p.q, s->v.key_dim, a.n_tokens, &maps.q) && encode_rows(s, p.k, s->v.key_dim, a.n_tokens, &maps.k) &&
               encode_rows(s, p.val, s->v.value_dim, a.n_tokens, &maps.val);
  for (int off = 0; off < among && rc == IC_OK; off += icc::STATE_BATCH) {
    p.seqs = seqs + off;
    p.starts = starts + off;
    p.ends = ends + off;
    p.n = among - off < icc::STATE_BATCH ? among - off : icc::STATE_BATCH;
    p.n_long = p.n < n ? p.n : n;
    const int items = s->v.n_heads * ((s->v.value_dim + 127) / 128), most = icc::state_items(a.n_tokens, p.n);
    for (p.first_item = 0; p.first_item < items && rc == IC_OK; p.first_item += most) {
      p.n_items = items - p.first_item < most ? items - p.first_item : most;
      rc = launched(s, icc::state_chunk_launch(p, maps, s->f16, s->sm_count, s->smem_optin, s->stream), 1, "state");
    }
  }
  return rc;
}

int ic_state_fork(ic_state_t* s, const int32_t* parents, const int32_t* children, int32_t n) {
  int rc = check_handle(s);
  if (rc == IC_OK) rc = check_n(s, n);
  if (rc != IC_OK || n == 0) return rc;
  if ((rc = check_list(s, parents, "parents")) != IC_OK || (rc = check_list(s, children, "children")) != IC_OK) return rc;
  DeviceGuard guard(s->device);
  int launches = 0;
  const cudaError_t e = icc::state_fork_launch(s->v, parents, children, n, s->sm_count, &launches, s->stream);
  return launched(s, e, launches, "fork");
}

int ic_state_clear(ic_state_t* s, const int32_t* seqs, int32_t n) {
  int rc = check_handle(s);
  if (rc != IC_OK) return rc;
  if (n < 0) return fail(IC_ERR_INVALID, "n = %d is negative", n);
  if (n == 0) return IC_OK;
  if ((rc = check_list(s, seqs, "seqs")) != IC_OK) return rc;
  DeviceGuard guard(s->device);
  return launched(s, icc::state_clear_launch(s->v, seqs, n, s->sm_count, s->stream), 1, "clear");
}

int ic_state_sync(ic_state_t* s) {
  if (!s) return fail(IC_ERR_INVALID, "NULL handle");
  DeviceGuard guard(s->device);
  cudaError_t e = cudaStreamSynchronize(s->stream);
  if (e != cudaSuccess) return fail(IC_ERR_CUDA, "stream sync failed: %s", cudaGetErrorString(e));
  const int code = *reinterpret_cast<volatile int*>(s->h_status);
  if (code == icc::KV_OK) return IC_OK;
  *s->h_status = icc::KV_OK;
  e = cudaMemsetAsync(s->v.err, 0, WORDS, s->stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s->stream);
  if (e != cudaSuccess) return fail(IC_ERR_CUDA, "clearing the error failed: %s", cudaGetErrorString(e));
  return reported(code);
}

int ic_state_set_stream(ic_state_t* s, void* cuda_stream) {
  if (!s) return fail(IC_ERR_INVALID, "NULL handle");
  s->stream = static_cast<cudaStream_t>(cuda_stream);
  return IC_OK;
}

int64_t ic_state_launch_count(const ic_state_t* s) { return s ? s->launches : IC_ERR_INVALID; }

}  // extern "C"
