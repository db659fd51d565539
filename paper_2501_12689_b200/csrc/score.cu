// Host side of the C ABI declared in include/ic_score.h: argument checking, buffer ownership and the launch.
#include <math.h>
#include <string.h>

#include <new>

#include "../../include/ic_score.h"
#include "host_util.h"
#include "kv.h"
#include "score.h"

using icc::DeviceGuard;
using icc::fail;
using icc::is_device_ptr;

struct ic_score {
  int device = 0, sm_count = 0, dtype = 0, vocab = 0;
  cudaStream_t stream = nullptr;
  void* own_workspace = nullptr;
  icc::ScorePartial* partials = nullptr;
  int* arrivals = nullptr;
  int* h_status = nullptr;
  int* d_status = nullptr;
  int64_t launches = 0;
};

namespace {

constexpr size_t ARRIVALS = icc::SCORE_SLOTS * sizeof(int), WORKSPACE = ARRIVALS + icc::SCORE_SLOTS * sizeof(icc::ScorePartial);
static_assert(IC_SCORE_MAX_TOP == icc::SCORE_MAX_TOP, "the lists hold a key a lane");

int read_opts(const ic_score_opts_t* opts, ic_score_opts_t* o) {
  memset(o, 0, sizeof *o);
  if (!opts) return fail(IC_ERR_INVALID, "NULL options");
  if (opts->struct_size < sizeof(uint32_t) || opts->struct_size > sizeof *o)
    return fail(IC_ERR_INVALID, "opts.struct_size %u not understood (this build: %zu)", opts->struct_size, sizeof *o);
  memcpy(o, opts, opts->struct_size);
  if (o->dtype < IC_SCORE_BF16 || o->dtype > IC_SCORE_F32) return fail(IC_ERR_INVALID, "unknown dtype %d", o->dtype);
  if (o->vocab < 1 || o->vocab > IC_SCORE_MAX_VOCAB) return fail(IC_ERR_INVALID, "vocab %d must be in [1, %d]", o->vocab, IC_SCORE_MAX_VOCAB);
  return IC_OK;
}

int check_handle(ic_score* s) {
  if (!s) return fail(IC_ERR_INVALID, "NULL handle");
  if (*reinterpret_cast<volatile int*>(s->h_status) == icc::KV_OK) return IC_OK;
  return fail(IC_ERR_INVALID, "an earlier call was given a target outside the vocabulary; call ic_score_sync to clear");
}

int check_array(const ic_score* s, const void* p, size_t size, const char* what) {
  if (!p || !is_device_ptr(p, s->device) || reinterpret_cast<uintptr_t>(p) % size)
    return fail(IC_ERR_INVALID, "%s must be a device array on device %d", what, s->device);
  return IC_OK;
}

}  // namespace

extern "C" {

size_t ic_score_workspace_bytes(const ic_score_opts_t* opts) {
  ic_score_opts_t o;
  return read_opts(opts, &o) == IC_OK ? WORKSPACE : 0;
}

ic_score_t* ic_score_create(const ic_score_opts_t* opts) {
  ic_score_opts_t o;
  if (read_opts(opts, &o) != IC_OK) return nullptr;
  int dev = 0, sms = 0, smem = 0;
  if (icc::usable_device(o.device, &dev, &sms, &smem) != IC_OK) return nullptr;
  DeviceGuard guard(dev);
  unsigned char* work = static_cast<unsigned char*>(o.workspace);
  if (work && (!is_device_ptr(work, dev) || (reinterpret_cast<uintptr_t>(work) & 255))) {
    fail(IC_ERR_INVALID, "opts.workspace must be a 256-byte aligned device pointer on device %d", dev);
    return nullptr;
  }
  if (work && o.workspace_bytes < WORKSPACE) {
    fail(IC_ERR_NOMEM, "opts.workspace holds %zu bytes, %zu are needed", o.workspace_bytes, WORKSPACE);
    return nullptr;
  }
  ic_score* s = new (std::nothrow) ic_score();
  if (!s) {
    fail(IC_ERR_NOMEM, "host allocation failed");
    return nullptr;
  }
  s->device = dev;
  s->sm_count = sms;
  s->dtype = o.dtype;
  s->vocab = o.vocab;
  s->stream = static_cast<cudaStream_t>(o.stream);
  cudaError_t e = work ? cudaSuccess : cudaMalloc(&s->own_workspace, WORKSPACE);
  if (!work) work = static_cast<unsigned char*>(s->own_workspace);
  s->arrivals = reinterpret_cast<int*>(work);
  s->partials = reinterpret_cast<icc::ScorePartial*>(work + ARRIVALS);
  if (e == cudaSuccess) e = cudaMemsetAsync(work, 0, ARRIVALS, s->stream);
  if (e == cudaSuccess && !(s->h_status = icc::take_status_word())) e = cudaErrorMemoryAllocation;
  if (e == cudaSuccess) e = cudaHostGetDevicePointer(reinterpret_cast<void**>(&s->d_status), s->h_status, 0);
  if (e != cudaSuccess) {
    cudaGetLastError();
    ic_score_destroy(s);
    fail(e == cudaErrorMemoryAllocation ? IC_ERR_NOMEM : IC_ERR_CUDA, "setting up the scores failed: %s", cudaGetErrorString(e));
    return nullptr;
  }
  return s;
}

void ic_score_destroy(ic_score_t* s) {
  if (!s) return;
  DeviceGuard guard(s->device);
  cudaStreamSynchronize(s->stream);
  if (s->own_workspace) cudaFree(s->own_workspace);
  if (s->h_status) icc::give_status_word(s->h_status);
  delete s;
}

int ic_score_tokens(ic_score_t* s, const ic_score_args_t* args) {
  int rc = check_handle(s);
  if (rc != IC_OK) return rc;
  if (!args) return fail(IC_ERR_INVALID, "NULL arguments");
  ic_score_args_t a;
  memset(&a, 0, sizeof a);
  if (args->struct_size < sizeof(uint32_t) || args->struct_size > sizeof a)
    return fail(IC_ERR_INVALID, "struct_size %u not understood (this build: %zu)", args->struct_size, sizeof a);
  memcpy(&a, args, args->struct_size);
  if (a.n_top < 0 || a.n_top > IC_SCORE_MAX_TOP || a.n_top > s->vocab)
    return fail(IC_ERR_INVALID, "n_top %d must be in [0, %d] and at most vocab %d", a.n_top, IC_SCORE_MAX_TOP, s->vocab);
  if (a.n_rows < 0 || a.n_rows > 1 << 26) return fail(IC_ERR_INVALID, "n_rows = %lld outside [0, 2^26]", (long long)a.n_rows);
  const float scale_log2 = (float)((double)a.scale * 1.4426950408889634);
  if (!isfinite(a.scale) || a.scale <= 0.0f || !isfinite(scale_log2))
    return fail(IC_ERR_INVALID, "scale %g must be above 0 and finite, also times log2(e)", a.scale);
  if (a.row_stride < 0 || a.row_stride > 1ll << 36) return fail(IC_ERR_INVALID, "row_stride %lld must not be negative", (long long)a.row_stride);
  if (a.n_rows == 0) return IC_OK;
  if (!a.targets && !a.entropy && !a.n_top) return fail(IC_ERR_INVALID, "nothing is asked for");
  if ((rc = check_array(s, a.logits, s->dtype == IC_SCORE_F32 ? 4 : 2, "logits")) != IC_OK ||
      (a.targets && ((rc = check_array(s, a.targets, 4, "targets")) != IC_OK || (rc = check_array(s, a.log_probs, 4, "log_probs")) != IC_OK)) ||
      (a.entropy && (rc = check_array(s, a.entropy, 4, "entropy")) != IC_OK) ||
      (a.n_top && ((rc = check_array(s, a.top_ids, 4, "top_ids")) != IC_OK || (rc = check_array(s, a.top_log_probs, 4, "top_log_probs")) != IC_OK)))
    return rc;
  icc::ScoreParams p;
  p.logits = static_cast<const unsigned char*>(a.logits);
  p.row_stride = a.row_stride;
  p.n_rows = a.n_rows;
  p.targets = a.targets;
  p.log_probs = a.log_probs;
  p.entropy = a.entropy;
  p.top_ids = a.top_ids;
  p.top_log_probs = a.top_log_probs;
  p.vocab = s->vocab;
  p.n_top = a.n_top;
  p.split = 1;
  p.scale = a.scale;
  p.scale_log2 = scale_log2;
  p.partials = s->partials;
  p.arrivals = s->arrivals;
  p.host_status = s->d_status;
  DeviceGuard guard(s->device);
  const cudaError_t e = icc::score_launch(p, s->dtype, s->sm_count, s->stream);
  if (e != cudaSuccess) return fail(IC_ERR_CUDA, "score launch failed: %s", cudaGetErrorString(e));
  s->launches += 1;
  return IC_OK;
}

int ic_score_sync(ic_score_t* s) {
  if (!s) return fail(IC_ERR_INVALID, "NULL handle");
  DeviceGuard guard(s->device);
  const cudaError_t e = cudaStreamSynchronize(s->stream);
  if (e != cudaSuccess) return fail(IC_ERR_CUDA, "stream sync failed: %s", cudaGetErrorString(e));
  const int rc = check_handle(s);
  *s->h_status = icc::KV_OK;
  return rc;
}

int ic_score_set_stream(ic_score_t* s, void* cuda_stream) {
  if (!s) return fail(IC_ERR_INVALID, "NULL handle");
  s->stream = static_cast<cudaStream_t>(cuda_stream);
  return IC_OK;
}

int64_t ic_score_launch_count(const ic_score_t* s) { return s ? s->launches : IC_ERR_INVALID; }

}  // extern "C"
