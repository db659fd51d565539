// What the C entry points of the paged cache, of the token scores and of the states share: error words, the check of the device.
#include "host_util.h"

#include <mutex>
#include <new>

#include "../../include/ic_cache.h"
#include "kv.h"

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

}  // namespace

namespace icc {

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

int usable_device(int wanted, int* dev, int* sms, int* smem) {
  int ndev = 0;
  const cudaError_t e = cudaGetDeviceCount(&ndev);
  if (e != cudaSuccess || ndev == 0) {
    cudaGetLastError();
    return fail(IC_ERR_CUDA, "no usable CUDA device (%s); this library has no CPU fallback", e != cudaSuccess ? cudaGetErrorString(e) : "device count is 0");
  }
  *dev = wanted;
  if (*dev < 0 && cudaGetDevice(dev) != cudaSuccess) return fail(IC_ERR_CUDA, "cudaGetDevice failed");
  if (*dev >= ndev) return fail(IC_ERR_INVALID, "device %d does not exist (%d devices)", *dev, ndev);
  int major = 0, minor = 0;
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, *dev) != cudaSuccess ||
      cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *dev) != cudaSuccess ||
      cudaDeviceGetAttribute(smem, cudaDevAttrMaxSharedMemoryPerBlockOptin, *dev) != cudaSuccess) {
    cudaGetLastError();
    return fail(IC_ERR_CUDA, "reading the device's attributes failed");
  }
  if (major != 10 || *sms > KV_MAX_CTAS)
    return fail(IC_ERR_UNSUPPORTED, "device %d is sm_%d%d with %d multiprocessors; this library is built for sm_100a only", *dev, major, minor, *sms);
  return 0;
}

}  // namespace icc
