// The paged cache of request histories: what a handle names, and what the attention kernels over it are given.
#pragma once
#include <cuda.h>

#include "rocs_internal.h"

struct rocs_cache {
  rocs_dtype_t dtype;
  int32_t layers, n_pages, page, H_kv, dh;
  void *K, *V;
  int64_t ld_layer, ld_page, ld_token, ld_head;  // elements
  int32_t n_slots, width;
  int32_t *table, *lens, *refs;
};

namespace rocs {

int kernel_path();  // of rocs_set_path

// Pages, slots, and slots or tiles of a call at most: a block that goes over them some thousands at a time ends in 32 bits.
constexpr int32_t kMostCounted = 0x7fffffff - 8192;

// SMs of the current device, asked for once per device.
inline int sms_of_device() {
  static std::atomic<int> known[64];
  int dev = 0, n = 148;
  if (cudaGetDevice(&dev) != cudaSuccess) return n;
  if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) != 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 148;
  if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

#ifdef __CUDACC__
__device__ __forceinline__ int32_t pages_for(int32_t positions, int32_t page) { return (positions + page - 1) / page; }
#endif

}  // namespace rocs
