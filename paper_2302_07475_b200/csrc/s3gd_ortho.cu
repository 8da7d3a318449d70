// Orthogonalised updates: momentum, Newton-Schulz products, update of the matrices (see include/s3gd.h).
#include <math.h>

#include "s3gd_ops.cuh"

namespace s3gd {
namespace {

constexpr int kPrepThreads = 256;
constexpr int kMaxNormBlocks = 512;       // partial sums of squares per matrix
constexpr float kMaxSingular = 2.f, kMaxPoly = 24.f;

// one matrix batch as the kernels see it
struct Mat {
  char* p;
  long long row, batch;                   // strides in elements
};

struct OrthoPlan {
  int batch;
  uint64_t rows, cols, m, n;              // m = shorter side, n = longer: X is [m x n]
  int norm_blocks;
  size_t off_hdr, off_norm, off_x, off_y, off_s, off_b, total;
};

bool make_plan(int batch, uint64_t rows, uint64_t cols, OrthoPlan* P) {
  if (batch < 1 || batch > 65535 || rows == 0 || cols == 0 || rows >= (1u << 24) || cols >= (1u << 24)) return false;
  P->batch = batch; P->rows = rows; P->cols = cols;
  P->m = rows < cols ? rows : cols;
  P->n = rows < cols ? cols : rows;
  const uint64_t want = (rows * cols + 4095) / 4096, share = (uint64_t)(kMaxNormBlocks + batch - 1) / batch;
  P->norm_blocks = (int)(want < share ? want : share);
  size_t off = 0;
  P->off_hdr = off;   off = align_up(off + kHdrWords * sizeof(uint32_t), 256);
  P->off_norm = off;  off = align_up(off + (size_t)batch * P->norm_blocks * sizeof(double), 256);
  P->off_x = off;     off = align_up(off + (size_t)batch * P->m * P->n * 4, 256);
  P->off_y = off;     off = align_up(off + (size_t)batch * P->m * P->n * 4, 256);
  P->off_s = off;     off = align_up(off + (size_t)batch * P->m * P->m * 4, 256);
  P->off_b = off;     off = align_up(off + (size_t)batch * P->m * P->m * 4, 256);
  P->total = off;
  return true;
}

__device__ __forceinline__ double block_sum(double v, double* warp_sums) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lane_id() == 0) warp_sums[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) v += warp_sums[w];   // the same order in every thread
  __syncthreads();
  return v;
}

// v <- mu v + g, and the sum of squares of u, in 64 bits (no overflow for any finite fp32 input).
template <typename G>
__global__ void momentum_norm_kernel(Mat g, Mat v, bool has_v, uint64_t rows, uint64_t cols, float mu, int nesterov,
                                     double* partial) {
  __shared__ double warp_sums[kPrepThreads / 32];
  const G* gp = reinterpret_cast<const G*>(g.p) + (size_t)blockIdx.y * g.batch;
  float* vp = reinterpret_cast<float*>(v.p) + (has_v ? (size_t)blockIdx.y * v.batch : 0);
  const uint64_t segs = (cols + 127) / 128, warps = (uint64_t)gridDim.x * (kPrepThreads / 32);
  double sum = 0.0;
  for (uint64_t s = (uint64_t)blockIdx.x * (kPrepThreads / 32) + (threadIdx.x >> 5); s < segs * rows; s += warps) {
    const uint64_t r = s / segs, c0 = (s % segs) * 128;
    for (uint64_t c = c0 + lane_id(); c < cols && c < c0 + 128; c += 32) {
      float u = to_f32(gp[r * g.row + c]);
      if (has_v) {
        const float nv = __fadd_rn(__fmul_rn(mu, vp[r * v.row + c]), u);
        vp[r * v.row + c] = nv;
        u = nesterov ? __fadd_rn(u, __fmul_rn(mu, nv)) : nv;
      }
      sum += (double)u * (double)u;
    }
  }
  sum = block_sum(sum, warp_sums);
  if (threadIdx.x == 0) partial[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

// X_0 = u / (|u| + eps), transposed where the matrix is tall
template <typename G>
__global__ void normalise_kernel(Mat g, Mat v, bool has_v, uint64_t rows, uint64_t cols, float mu, int nesterov, float eps,
                                 const double* partial, int norm_blocks, float* x) {
  __shared__ double warp_sums[kPrepThreads / 32];
  const G* gp = reinterpret_cast<const G*>(g.p) + (size_t)blockIdx.y * g.batch;
  const float* vp = reinterpret_cast<const float*>(v.p) + (has_v ? (size_t)blockIdx.y * v.batch : 0);
  double s = 0.0;
  for (int i = threadIdx.x; i < norm_blocks; i += kPrepThreads) s += partial[(size_t)blockIdx.y * norm_blocks + i];
  const float inv = (float)(1.0 / (sqrt(block_sum(s, warp_sums)) + (double)eps));
  x += (size_t)blockIdx.y * rows * cols;
  for (uint64_t e = (uint64_t)blockIdx.x * kPrepThreads + threadIdx.x; e < rows * cols; e += (uint64_t)gridDim.x * kPrepThreads) {
    const uint64_t r = e / cols, c = e % cols;
    float u = to_f32(gp[r * g.row + c]);
    if (has_v) {
      const float nv = vp[r * v.row + c];
      u = nesterov ? __fadd_rn(u, __fmul_rn(mu, nv)) : nv;
    }
    x[rows > cols ? c * rows + r : e] = u * inv;
  }
}

// C = ca * Add + cb * P Q (Q transposed where kNT): 64 x 64 tiles, 4 x 4 entries per thread.
struct Store {
  char* p;                 // user matrix of the last product; NULL: C
  int dtype;
  long long row, batch;
  bool transpose, update;  // update: p <- keep * p - rate * value
  float keep, rate;
};
template <bool kNT>
__global__ void __launch_bounds__(256) simple_product_kernel(const float* P, const float* Q, const float* Add, float* C, int m, int n, int k,
                                                             float ca, float cb, Store st) {
  __shared__ float ps[16][65], qs[16][65];
  const size_t b = blockIdx.z;
  P += b * m * k; Q += b * (size_t)k * n;
  const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64, ti = threadIdx.x / 16, tj = threadIdx.x % 16;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < k; k0 += 16) {
    for (int e = threadIdx.x; e < 64 * 16; e += 256) {
      const int r = e / 16, kk = e % 16;
      ps[kk][r] = i0 + r < m && k0 + kk < k ? P[(size_t)(i0 + r) * k + k0 + kk] : 0.f;
      if (kNT) {
        qs[kk][r] = j0 + r < n && k0 + kk < k ? Q[(size_t)(j0 + r) * k + k0 + kk] : 0.f;
      } else {
        const int kr = e / 64, c = e % 64;
        qs[kr][c] = j0 + c < n && k0 + kr < k ? Q[(size_t)(k0 + kr) * n + j0 + c] : 0.f;
      }
    }
    __syncthreads();
    float part[4][4] = {};                 // sums in two levels: a long row's squares lose less than in one chain
    for (int kk = 0; kk < 16; ++kk)
      for (int a = 0; a < 4; ++a)
        for (int c = 0; c < 4; ++c) part[a][c] += ps[kk][ti * 4 + a] * qs[kk][tj * 4 + c];
    for (int a = 0; a < 4; ++a)
      for (int c = 0; c < 4; ++c) acc[a][c] += part[a][c];
    __syncthreads();
  }
  for (int a = 0; a < 4; ++a)
    for (int c = 0; c < 4; ++c) {
      const int i = i0 + ti * 4 + a, j = j0 + tj * 4 + c;
      if (i >= m || j >= n) continue;
      const size_t at = b * m * n + (size_t)i * n + j;
      const float val = __fmaf_rn(ca, Add ? Add[at] : 0.f, __fmul_rn(cb, acc[a][c]));
      if (st.p == nullptr) { C[at] = val; continue; }
      const size_t to = b * st.batch + (st.transpose ? (size_t)j * st.row + i : (size_t)i * st.row + j);
      if (st.dtype == S3GD_F32) {
        float* o = reinterpret_cast<float*>(st.p) + to;
        *o = st.update ? __fmaf_rn(-st.rate, val, __fmul_rn(st.keep, *o)) : val;
      } else {
        __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(st.p) + to;
        *o = __float2bfloat16_rn(st.update ? __fmaf_rn(-st.rate, val, __fmul_rn(st.keep, __bfloat162float(*o))) : val);
      }
    }
}

bool mat_ok(const s3gd_matrix* a, int batch, uint64_t cols, bool written) {
  return a != nullptr && a->data != nullptr && dtype_bytes(a->dtype) != 0 && is_aligned(a->data, dtype_bytes(a->dtype)) &&
         a->row_stride >= (int64_t)cols && a->batch_stride >= 0 && !(written && batch > 1 && a->batch_stride < (int64_t)cols);
}

// Does every singular value in [0, 1] stay within what the 16-bit forms hold?
bool poly_ok(int steps, float a, float b, float c, float eps) {
  if (steps < 1 || steps > 32 || !isfinite(a) || !isfinite(b) || !isfinite(c) || !isfinite(eps) || eps < 0.f) return false;
  for (int i = 0; i <= 1024; ++i) {
    double s = i / 1024.0;
    for (int k = 0; k < steps; ++k) {
      const double q = b * s * s + c * s * s * s * s;
      if (!(fabs(q) <= kMaxPoly)) return false;
      s = s * (a + q);
      if (!(fabs(s) <= kMaxSingular)) return false;
    }
  }
  return true;
}

struct Request {
  Mat g, v;
  int g_dtype;
  bool has_v;
  float mu; int nesterov;
  Store out;
  int steps, split;
  float a, b, c, eps;
};

template <typename G>
cudaError_t prepare(const OrthoPlan& P, const Request& R, char* ws, cudaStream_t st) {
  double* partial = reinterpret_cast<double*>(ws + P.off_norm);
  count_launch(2);
  momentum_norm_kernel<G><<<dim3(P.norm_blocks, P.batch), kPrepThreads, 0, st>>>(R.g, R.v, R.has_v, P.rows, P.cols, R.mu, R.nesterov, partial);
  const uint64_t blocks = (P.rows * P.cols + 1023) / 1024;
  normalise_kernel<G><<<dim3((unsigned)(blocks < 4096 ? blocks : 4096), P.batch), kPrepThreads, 0, st>>>(
      R.g, R.v, R.has_v, P.rows, P.cols, R.mu, R.nesterov, R.eps, partial, P.norm_blocks, reinterpret_cast<float*>(ws + P.off_x));
  return cudaGetLastError();
}

cudaError_t run(const OrthoPlan& P, const Request& R, char* ws, cudaStream_t st) {
  cudaError_t e = cudaMemsetAsync(ws + P.off_hdr, 0, kHdrWords * sizeof(uint32_t), st);
  if (e != cudaSuccess) return e;
  e = R.g_dtype == S3GD_F32 ? prepare<float>(P, R, ws, st) : R.g_dtype == S3GD_BF16 ? prepare<__nv_bfloat16>(P, R, ws, st) : prepare<int8_t>(P, R, ws, st);
  if (e != cudaSuccess) return e;
  float* x = reinterpret_cast<float*>(ws + P.off_x);
  float* y = reinterpret_cast<float*>(ws + P.off_y);
  float* s = reinterpret_cast<float*>(ws + P.off_s);
  float* q = reinterpret_cast<float*>(ws + P.off_b);
  const int m = (int)P.m, n = (int)P.n;
  const dim3 sq((m + 63) / 64, (m + 63) / 64, P.batch), wide((n + 63) / 64, (m + 63) / 64, P.batch);
  Store none = {};
  count_launch(3 * R.steps);
  for (int k = 0; k < R.steps; ++k) {
    simple_product_kernel<true><<<sq, 256, 0, st>>>(x, x, nullptr, s, m, m, n, 0.f, 1.f, none);
    simple_product_kernel<true><<<sq, 256, 0, st>>>(s, s, s, q, m, m, m, R.b, R.c, none);
    simple_product_kernel<false><<<wide, 256, 0, st>>>(q, x, x, y, m, n, m, R.a, 1.f, k + 1 == R.steps ? R.out : none);
    float* t = x; x = y; y = t;
  }
  return cudaGetLastError();
}

s3gd_status common_checks(const s3gd_matrix* g, int batch, uint64_t rows, uint64_t cols, int steps, float a, float b, float c, float eps,
                          int split_steps, OrthoPlan* P) {
  if (!make_plan(batch, rows, cols, P) || !mat_ok(g, batch, cols, false)) return S3GD_ERR_INVALID_ARG;
  if (g->dtype != S3GD_F32 && g->dtype != S3GD_BF16 && g->dtype != S3GD_I8) return S3GD_ERR_INVALID_ARG;
  if (!poly_ok(steps, a, b, c, eps) || split_steps < -1 || split_steps > steps) return S3GD_ERR_INVALID_ARG;
  return S3GD_OK;
}

Mat as_mat(const s3gd_matrix* a) { return {static_cast<char*>(a->data), (long long)a->row_stride, (long long)a->batch_stride}; }

int split_rule(int split_steps, int steps, int dtype) {
  if (split_steps >= 0) return split_steps;
  return dtype == S3GD_F32 ? steps : (steps < 2 ? steps : 2);
}

}  // namespace
}  // namespace s3gd

using namespace s3gd;

extern "C" size_t s3gd_orthogonalise_workspace_bytes(int batch, uint64_t rows, uint64_t cols) {
  OrthoPlan P;
  return make_plan(batch, rows, cols, &P) ? P.total : 0;
}

extern "C" s3gd_status s3gd_orthogonalise(const s3gd_matrix* g, const s3gd_matrix* out, int batch, uint64_t rows, uint64_t cols, int steps,
                                          float a, float b, float c, float eps, int split_steps, void* ws, size_t ws_bytes,
                                          void* stream) {
  OrthoPlan P;
  s3gd_status s = common_checks(g, batch, rows, cols, steps, a, b, c, eps, split_steps, &P);
  if (s != S3GD_OK) return s;
  if (!mat_ok(out, batch, cols, true) || (out->dtype != S3GD_F32 && out->dtype != S3GD_BF16)) return S3GD_ERR_INVALID_ARG;
  if (ws == nullptr || ws_bytes < P.total || !is_aligned(ws, 256)) return S3GD_ERR_WORKSPACE;
  Request R = {};
  R.g = as_mat(g); R.g_dtype = g->dtype;
  R.out = {static_cast<char*>(out->data), out->dtype, (long long)out->row_stride, (long long)out->batch_stride, rows > cols, false, 0.f, 0.f};
  R.steps = steps; R.split = split_rule(split_steps, steps, out->dtype);
  R.a = a; R.b = b; R.c = c; R.eps = eps;
  return run(P, R, static_cast<char*>(ws), static_cast<cudaStream_t>(stream)) == cudaSuccess ? S3GD_OK : S3GD_ERR_CUDA;
}

extern "C" s3gd_status s3gd_step_ortho(const s3gd_matrix* x, const s3gd_matrix* opt_v, const s3gd_matrix* g, int batch, uint64_t rows,
                                       uint64_t cols, float mu, int nesterov, float lr, float weight_decay, float scale, int steps,
                                       float a, float b, float c, float eps, int split_steps, void* ws, size_t ws_bytes, void* stream) {
  OrthoPlan P;
  s3gd_status s = common_checks(g, batch, rows, cols, steps, a, b, c, eps, split_steps, &P);
  if (s != S3GD_OK) return s;
  if (!mat_ok(x, batch, cols, true) || (x->dtype != S3GD_F32 && x->dtype != S3GD_BF16)) return S3GD_ERR_INVALID_ARG;
  if (opt_v != nullptr && (!mat_ok(opt_v, batch, cols, true) || opt_v->dtype != S3GD_F32)) return S3GD_ERR_INVALID_ARG;
  if (ws == nullptr || ws_bytes < P.total || !is_aligned(ws, 256)) return S3GD_ERR_WORKSPACE;
  Request R = {};
  R.g = as_mat(g); R.g_dtype = g->dtype;
  R.has_v = opt_v != nullptr;
  if (R.has_v) R.v = as_mat(opt_v);
  R.mu = mu; R.nesterov = nesterov;
  R.out = {static_cast<char*>(x->data), x->dtype, (long long)x->row_stride, (long long)x->batch_stride, rows > cols, true,
           1.f - lr * weight_decay, lr * scale};
  R.steps = steps; R.split = split_rule(split_steps, steps, x->dtype);
  R.a = a; R.b = b; R.c = c; R.eps = eps;
  return run(P, R, static_cast<char*>(ws), static_cast<cudaStream_t>(stream)) == cudaSuccess ? S3GD_OK : S3GD_ERR_CUDA;
}
