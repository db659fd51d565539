// Host-side helpers shared by the C entry points of the retrieval cache and of the paged cache.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

namespace icc {

// Record the message behind ic_cache_last_error() for the calling thread and return `code`.
int fail(int code, const char* fmt, ...);

struct DeviceGuard {
  int prev = -1;
  bool changed = false;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) changed = (cudaSetDevice(dev) == cudaSuccess);
  }
  ~DeviceGuard() {
    if (changed) cudaSetDevice(prev);
  }
};

inline bool is_device_ptr(const void* p, int device) {
  cudaPointerAttributes a;
  if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  if (a.type == cudaMemoryTypeManaged) return true;
  return a.type == cudaMemoryTypeDevice && a.device == device;
}

// Rows of `length` elements at t * token_stride + h * head_stride, t < tokens, h < heads: do two of them share an element?
inline bool rows_overlap(int64_t tokens, int64_t heads, int64_t token_stride, int64_t head_stride, int64_t length) {
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

// A mapped host word for a handle's error, zero; nullptr if there is no memory.
int* take_status_word();
void give_status_word(int* w);

// The device that a handle is made for (wanted < 0: the current one), if this library runs on it: IC_OK, or the error's code.
int usable_device(int wanted, int* dev, int* sms, int* smem);

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

}  // namespace icc
