// Opt-in to large dynamic shared memory, remembered per device and kernel.  Internal; included by s3gd_api.cu.
#pragma once

#include <cuda_runtime.h>
#include <pthread.h>

namespace s3gd {

// `done`: bytes opted in so far, one per device.  Sizes may differ from call to call (small matrices take what they need), so
// the attribute and the record change together under a lock: otherwise a smaller size could be set after a larger one whose
// record is written last, and every later launch of the larger size would fail.  The lock is only taken until the largest
// size has been seen.  (A pthread mutex does not throw.)
inline cudaError_t raise_dynamic_smem(const void* func, int bytes, int* done, int devices) {
  static pthread_mutex_t lock = PTHREAD_MUTEX_INITIALIZER;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= devices) return cudaFuncSetAttribute(func, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (__atomic_load_n(&done[dev], __ATOMIC_ACQUIRE) >= bytes) return cudaSuccess;
  pthread_mutex_lock(&lock);
  if (done[dev] < bytes) {
    e = cudaFuncSetAttribute(func, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) __atomic_store_n(&done[dev], bytes, __ATOMIC_RELEASE);
  }
  pthread_mutex_unlock(&lock);
  return e;
}

}  // namespace s3gd
