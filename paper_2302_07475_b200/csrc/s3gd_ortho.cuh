// What the kernels of the orthogonalised updates share.  Internal.
#pragma once

#include <cuda_fp16.h>

#include "s3gd_ops.cuh"

namespace s3gd {

// X is held times 2^10, S = X X^T times 2^12, B = b S + c S^2 times 2^10: with singular values up to 2 and |B| up to 24 the
// largest entries stay under fp16's 65504, and the entries of an 8192-wide X_0 (about 1e-4) lie far above its subnormals.
constexpr float kScaleX = 1024.f, kScaleS = 4096.f, kScaleB = 1024.f;
constexpr float kMaxSingular = 2.f, kMaxPoly = 24.f;

// one matrix batch of the caller's as the kernels see it
struct Mat {
  char* p;
  long long row, batch;                   // strides in elements
};

// where the last product goes: p <- value, or (update) p <- keep * p - rate * value
struct Store {
  Mat to;
  int dtype;
  bool transpose, update, wide;           // wide: rows and base allow four entries in one access
  float keep, rate;
};

struct OrthoPlan {
  int batch;
  uint64_t rows, cols;
  int m, n;                               // shorter and longer side: X is [m x n]
  int ldx, lds;                           // row lengths of the 16-bit matrices
  int norm_blocks;
  size_t off_hdr, off_norm, off_x, off_y, off_s, off_b, total;   // each matrix: [batch][two pieces][m][ld]
};

struct OrthoRequest {
  Mat g, v;
  int g_dtype;
  bool has_v;
  float mu;
  int nesterov;
  Store out;
  int steps, split;
  float a, b, c, eps;
};

// For how many of the first steps X is held in two pieces: where the products take two, and in steps whose products the
// caller wants of one piece for the a X term alone, in all but the last two.  The products of one-piece operands lose little
// where singular values are small (B is of second order in them), while X itself must keep them through the steps that raise
// them: with a part of rank 16 ten times above the rest and no split step the result is off by 5e-4 this way, 3.6e-3 with X in
// one piece, and 1e-3 with X in one piece but two split steps.  In the last steps the rounding of X in both terms cancels in
// part, so one piece is as good there.
inline int carried_steps(int steps, int split) {
  const int c = steps > 3 ? steps - 2 : 1;
  return c > split ? c : split;
}

#ifdef __CUDACC__
// X_0 = u / (|u| + eps), times 2^10, as (u pre) inv.  2^10 over a norm below 2^-118 would not fit fp32, and one over 2^136
// would lose bits in its subnormals: such matrices are first moved by a power of two, which changes no bit of theirs.
struct Normaliser {
  float pre, inv;
  __device__ __forceinline__ Normaliser(double norm, float eps) {
    const double d = norm + (double)eps;
    pre = d < 0x1p-96 ? 0x1p96f : d > 0x1p96 ? 0x1p-96f : 1.f;
    inv = (float)((double)kScaleX / (d * (double)pre));
  }
  __device__ __forceinline__ float operator()(float u) const { return __fmul_rn(__fmul_rn(u, pre), inv); }
};
// a value as two fp16 pieces, 22 bits together
__device__ __forceinline__ void split_half(float v, __half* hi, __half* lo) {
  *hi = __float2half_rn(v);
  *lo = __float2half_rn(v - __half2float(*hi));
}

// eight neighbouring entries of a swizzled row as floats, from one or two pieces
__device__ __forceinline__ void read8(const char* hi, const char* lo, int off, bool two, float* x) {
  const uint4 h4 = *reinterpret_cast<const uint4*>(hi + off);
  const __half2* h = reinterpret_cast<const __half2*>(&h4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = __half22float2(h[e]);
    x[2 * e] = f.x; x[2 * e + 1] = f.y;
  }
  if (!two) return;
  const uint4 l4 = *reinterpret_cast<const uint4*>(lo + off);
  const __half2* l = reinterpret_cast<const __half2*>(&l4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = __half22float2(l[e]);
    x[2 * e] += f.x; x[2 * e + 1] += f.y;
  }
}
// the two pieces of eight entries, two entries to a word
__device__ __forceinline__ void split8(const float* x, bool two, uint32_t* hi, uint32_t* lo) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __half2 h = __floats2half2_rn(x[2 * e], x[2 * e + 1]);
    hi[e] = *reinterpret_cast<const uint32_t*>(&h);
    if (!two) continue;
    const float2 f = __half22float2(h);
    const __half2 l = __floats2half2_rn(x[2 * e] - f.x, x[2 * e + 1] - f.y);
    lo[e] = *reinterpret_cast<const uint32_t*>(&l);
  }
}

// The caller's entry after the last product
template <typename T>
__device__ __forceinline__ T stored(const Store& s, T old, float v) {
  return from_f32<T>(s.update ? __fmaf_rn(-s.rate, v, __fmul_rn(s.keep, to_f32(old))) : v);
}
template <typename T> struct alignas(4 * sizeof(T)) Four { T v[4]; };

// Eight neighbouring entries of row i of X to the caller's matrix: along its row, or down its column where it is transposed
template <typename T>
__device__ __forceinline__ void put8(const Store& s, int mat, int i, int j0, int m, int n, const float* x) {
  if (i >= m) return;
  T* base = reinterpret_cast<T*>(s.to.p) + (size_t)mat * s.to.batch;
  if (s.wide && !s.transpose && j0 + 8 <= n) {
    Four<T>* p = reinterpret_cast<Four<T>*>(base + (size_t)i * s.to.row + j0);
    Four<T> o[2] = {};
    if (s.update) { o[0] = p[0]; o[1] = p[1]; }
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e / 4].v[e % 4] = stored(s, o[e / 4].v[e % 4], x[e]);
    p[0] = o[0]; p[1] = o[1];
    return;
  }
  const size_t step = s.transpose ? s.to.row : 1;
  base += s.transpose ? (size_t)j0 * s.to.row + i : (size_t)i * s.to.row + j0;
  T old[8] = {};
  if (s.update)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (j0 + e < n) old[e] = base[e * step];
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (j0 + e < n) base[e * step] = stored(s, old[e], x[e]);
}

// up to four neighbouring entries of a row as floats
template <typename T>
__device__ __forceinline__ void get4(const T* p, bool wide, int64_t left, float* x) {
  if (wide && left >= 4) {
    const Four<T> f = *reinterpret_cast<const Four<T>*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = to_f32(f.v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = e < left ? to_f32(p[e]) : 0.f;
  }
}
__device__ __forceinline__ void put4(float* p, bool wide, int64_t left, const float* x) {
  if (wide && left >= 4) *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  else
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[e] = x[e];
}
#endif

// X_0 lies in off_x; enqueues all products, the last of which writes R.out
cudaError_t launch_products(const OrthoPlan& P, const OrthoRequest& R, char* ws, cudaStream_t st);
// Matrices that one CTA holds: everything in one launch
bool is_small(const OrthoPlan& P);
cudaError_t launch_small(const OrthoPlan& P, const OrthoRequest& R, char* ws, cudaStream_t st);

}  // namespace s3gd
