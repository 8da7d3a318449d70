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

inline bool is_real(int dt) { return dt == S3GD_F32 || dt == S3GD_BF16; }
inline bool is_index(int dt) { return dt == S3GD_I32 || dt == S3GD_I64; }

#ifdef __CUDACC__
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(int8_t v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// ------------------------------------------------------------------ access of kVec neighbouring entries
template <typename T, int kVec>
struct alignas((kVec * sizeof(T) > 16 ? 16 : kVec * sizeof(T))) Pack { T v[kVec]; };

template <typename T, int kVec>
__device__ __forceinline__ void store_pack(T* p, const float* v) {
  Pack<T, kVec> o;
#pragma unroll
  for (int e = 0; e < kVec; ++e) o.v[e] = from_f32<T>(v[e]);
  *reinterpret_cast<Pack<T, kVec>*>(p) = o;
}

// kVec neighbouring entries as 32-bit floats, and back (rounded to nearest); 16-bit entries two at a time
template <typename T, int kVec>
__device__ __forceinline__ void load_floats(const T* p, float* v) {
  if constexpr (sizeof(T) == 2 && kVec % 2 == 0) {
    const Pack<uint32_t, kVec / 2> o = *reinterpret_cast<const Pack<uint32_t, kVec / 2>*>(p);
#pragma unroll
    for (int i = 0; i < kVec / 2; ++i) {
      v[2 * i] = __uint_as_float(o.v[i] << 16);
      v[2 * i + 1] = __uint_as_float(o.v[i] & 0xffff0000u);
    }
  } else {
    const Pack<T, kVec> o = *reinterpret_cast<const Pack<T, kVec>*>(p);
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = to_f32(o.v[e]);
  }
}
template <typename T, int kVec>
__device__ __forceinline__ void store_floats(T* p, const float* v) {
  if constexpr (sizeof(T) == 2 && kVec % 2 == 0) {
    Pack<__nv_bfloat162, kVec / 2> o;
#pragma unroll
    for (int i = 0; i < kVec / 2; ++i) o.v[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<Pack<__nv_bfloat162, kVec / 2>*>(p) = o;
  } else {
    store_pack<T, kVec>(p, v);
  }
}

// the widest access that base and distances allow, no wider than what keeps 32 lanes busy on `dim` columns
inline int widest(uint64_t dim) {
  int v = 8;
  while (v > 1 && (dim % v != 0 || dim < 32u * v)) v /= 2;
  return v;
}
inline int allowed(int v, const void* p, int dtype, int64_t stride_a, int64_t stride_b) {
  const size_t size = dtype_bytes(dtype);
  while (v > 1 && (!is_aligned(p, v * size < 16 ? v * size : 16) || stride_a % v != 0 || stride_b % v != 0)) v /= 2;
  return v;
}

// f is called with a value of the element type, or with the number as a type
template <typename F>
cudaError_t by_real(int dt, F f) { return dt == S3GD_F32 ? f(float()) : f(__nv_bfloat16()); }
template <typename F>
cudaError_t by_index(int dt, F f) { return dt == S3GD_I32 ? f(int32_t()) : f(int64_t()); }
template <int kN> struct Width { static constexpr int value = kN; };
template <typename F>
cudaError_t by_width(int v, F f) { return v == 8 ? f(Width<8>()) : v == 4 ? f(Width<4>()) : v == 2 ? f(Width<2>()) : f(Width<1>()); }
#endif

}  // namespace s3gd
