// What the model-side operators share: argument checks of a C entry and small device helpers.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "toploc_model.h"

namespace toploc_model {

inline bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

inline int element_bytes(int32_t dtype) {
  return dtype == TOPLOC_DTYPE_BF16 ? 2 : dtype == TOPLOC_DTYPE_FP32 ? 4 : 0;
}

// The current device is a B200 (compute capability 10.x); its SM count on request.
inline int check_device(int* sm_count = nullptr) {
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess)
    return TOPLOC_ERR_CUDA;
  if (major != 10) return TOPLOC_ERR_ARCH;
  if (sm_count && cudaDeviceGetAttribute(sm_count, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return TOPLOC_ERR_CUDA;
  return TOPLOC_OK;
}

// Lets a kernel have `bytes` of shared memory, the most that any of its launches takes, on the current device; once per
// kernel and device (a bit of `done` each).  Not this launch's bytes: the limit is the kernel's, and a thread that set a
// smaller one between another thread's call and launch would make that launch fail.
inline int allow_shared(const void* kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return TOPLOC_ERR_CUDA;
  const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return TOPLOC_OK;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess)
    return TOPLOC_ERR_CUDA;
  done.fetch_or(bit, std::memory_order_relaxed);
  return TOPLOC_OK;
}

inline int launched() { return cudaGetLastError() == cudaSuccess ? TOPLOC_OK : TOPLOC_ERR_CUDA; }

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Two fp32 values rounded to nearest-even bf16, the first in the lower half.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void store_as(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_as(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

}  // namespace toploc_model
