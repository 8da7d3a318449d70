// Shared by the operators on a language model's parameters (orthogonalised updates, embedding table):
// element types, strided matrices, small helpers.  Internal; the public interface is include/s3gd.h.
#pragma once

#include <cuda_bf16.h>

#include "s3gd_common.cuh"

namespace s3gd {

inline bool is_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline size_t dtype_bytes(int dt) {
  switch (dt) {
    case S3GD_F32: case S3GD_I32: return 4;
    case S3GD_BF16: return 2;
    case S3GD_I8: return 1;
    case S3GD_I64: return 8;
  }
  return 0;
}

#ifdef __CUDACC__
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(int8_t v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
#endif

}  // namespace s3gd
