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
