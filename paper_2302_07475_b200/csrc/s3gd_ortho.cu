// Orthogonalised updates: argument checks, momentum, norm and the first 16-bit matrix (see include/s3gd.h).
// Two passes over the gradient, because the norm must be known before anything can be rounded to 16 bits: momentum and sum of
// squares (32 us for 4 x 2048 x 2048 with bf16 gradients: 168 MB, 26 us at 6.5 TB/s), then u over the norm as fp16 pieces
// (50 us; its blocks live too briefly to keep more loads under way).
#include <math.h>

#include "s3gd_ortho.cuh"

namespace s3gd {
namespace {

constexpr int kPrepThreads = 256;
constexpr int kMaxNormBlocks = 512;       // partial sums of squares per matrix

bool make_plan(int batch, uint64_t rows, uint64_t cols, OrthoPlan* P) {
  if (batch < 1 || batch > 65535 || rows == 0 || cols == 0 || rows >= (1u << 24) || cols >= (1u << 24)) return false;
  if ((double)batch * (double)rows * (double)cols > 1e12 || (double)batch * (double)(rows < cols ? rows : cols) > 1e9) return false;
  P->batch = batch; P->rows = rows; P->cols = cols;
  P->m = (int)(rows < cols ? rows : cols);
  P->n = (int)(rows < cols ? cols : rows);
  P->ldx = (P->n + 7) / 8 * 8;            // TMA wants rows that start on 16 bytes
  P->lds = (P->m + 7) / 8 * 8;
  const uint64_t want = (rows * cols + 4095) / 4096, share = (uint64_t)(kMaxNormBlocks + batch - 1) / batch;
  P->norm_blocks = (int)(want < share ? want : share);
  const size_t x_bytes = (size_t)batch * 2 * P->m * P->ldx * 2, s_bytes = (size_t)batch * 2 * P->m * P->lds * 2;
  size_t off = 0;
  P->off_hdr = off;   off = align_up(off + kHdrWords * sizeof(uint32_t), 256);
  P->off_norm = off;  off = align_up(off + (size_t)batch * P->norm_blocks * sizeof(double), 256);
  P->off_x = off;     off = align_up(off + x_bytes, 256);
  P->off_y = off;     off = align_up(off + x_bytes, 256);
  P->off_s = off;     off = align_up(off + s_bytes, 256);
  P->off_b = off;     off = align_up(off + s_bytes, 256);
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

// v <- mu v + g, and the sum of squares of u, in 64 bits (no overflow for any finite fp32 input).  The matrix counts as one row
// where its rows follow one another.  Four times four entries per lane are under way.
template <typename G>
__global__ void __launch_bounds__(kPrepThreads) momentum_norm_kernel(Mat g, Mat v, bool has_v, bool g_wide, bool v_wide, uint64_t rows,
                                                                     uint64_t cols, float mu, int nesterov, double* partial, uint32_t* hdr) {
  __shared__ double warp_sums[kPrepThreads / 32];
  constexpr int kSeg = 512;
  grid_dependency_wait();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < kHdrWords) hdr[threadIdx.x] = 0;
  const G* gp = reinterpret_cast<const G*>(g.p) + (size_t)blockIdx.y * g.batch;
  float* vp = reinterpret_cast<float*>(v.p) + (has_v ? (size_t)blockIdx.y * v.batch : 0);
  const uint64_t segs = (cols + kSeg - 1) / kSeg, warps = (uint64_t)gridDim.x * (kPrepThreads / 32);
  double sum = 0.0;
  for (uint64_t s = (uint64_t)blockIdx.x * (kPrepThreads / 32) + (threadIdx.x >> 5); s < segs * rows; s += warps) {
    const uint64_t r = s / segs, c0 = (s % segs) * kSeg + lane_id() * 4;
    const G* gr = gp + r * g.row;
    float* vr = vp + (has_v ? r * v.row : 0);
    float u[4][4], old[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint64_t c = c0 + k * 128;
      get4(gr + c, g_wide, (int64_t)cols - (int64_t)c, u[k]);
      if (has_v) get4(vr + c, v_wide, (int64_t)cols - (int64_t)c, old[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint64_t c = c0 + k * 128;
      if (has_v) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          old[k][x] = __fadd_rn(__fmul_rn(mu, old[k][x]), u[k][x]);
          u[k][x] = nesterov ? __fadd_rn(u[k][x], __fmul_rn(mu, old[k][x])) : old[k][x];   // beside the matrix: zero
        }
        put4(vr + c, v_wide, (int64_t)cols - (int64_t)c, old[k]);
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) sum += (double)u[k][x] * (double)u[k][x];
    }
  }
  sum = block_sum(sum, warp_sums);
  if (threadIdx.x == 0) partial[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

// X_0 = u / (|u| + eps) in two fp16 pieces, transposed where the matrix is tall: 64 x 64 tiles through shared memory
template <typename G>
__global__ void __launch_bounds__(kPrepThreads) normalise_kernel(Mat g, Mat v, bool has_v, bool g_wide, bool v_wide, uint64_t rows, uint64_t cols,
                                                                 float mu, int nesterov, float eps, const double* partial, int norm_blocks,
                                                                 __half* x, int m, int n, int ldx) {
  __shared__ double warp_sums[kPrepThreads / 32];
  __shared__ float tile[64][65];
  const size_t b = blockIdx.z;
  const G* gp = reinterpret_cast<const G*>(g.p) + b * g.batch;
  const float* vp = reinterpret_cast<const float*>(v.p) + (has_v ? b * v.batch : 0);
  const bool tall = rows > cols;
  const uint64_t i0 = (uint64_t)blockIdx.y * 64, j0 = (uint64_t)blockIdx.x * 64;    // of X
  const uint64_t r0 = tall ? j0 : i0, c0 = (tall ? i0 : j0) + (threadIdx.x & 15) * 4;   // of the matrix
  grid_dependency_wait();
  float u[4][4], old[4][4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint64_t r = r0 + k * 16 + (threadIdx.x >> 4);
    const int64_t left = r < rows ? (int64_t)cols - (int64_t)c0 : 0;
    const bool from_v = has_v && !nesterov;
    if (!from_v) get4(gp + r * g.row + c0, g_wide, left, u[k]);
    if (has_v) get4(vp + r * v.row + c0, v_wide, left, from_v ? u[k] : old[k]);
  }
  double s = 0.0;
  for (int i = threadIdx.x; i < norm_blocks; i += kPrepThreads) s += partial[b * norm_blocks + i];
  const Normaliser normalised(sqrt(block_sum(s, warp_sums)), eps);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int dr = k * 16 + (threadIdx.x >> 4), dc = (threadIdx.x & 15) * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float w = has_v && nesterov ? __fadd_rn(u[k][e], __fmul_rn(mu, old[k][e])) : u[k][e];
      tile[tall ? dc + e : dr][tall ? dr : dc + e] = normalised(w);
    }
  }
  __syncthreads();
  __half* hi_row = x + b * 2 * m * (size_t)ldx;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int di = k * 32 + (threadIdx.x >> 3), dj = (threadIdx.x & 7) * 8;
    if (i0 + di >= (uint64_t)m || j0 + dj >= (uint64_t)ldx) continue;               // ldx is a multiple of eight
    float w[8];
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = tile[di][dj + e];
    split8(w, true, hi, lo);
    const size_t at = (i0 + di) * ldx + j0 + dj;
    *reinterpret_cast<uint4*>(hi_row + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(hi_row + (size_t)m * ldx + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
}

bool mat_ok(const s3gd_matrix* a, int batch, uint64_t cols, bool written) {
  return a != nullptr && a->data != nullptr && dtype_bytes(a->dtype) != 0 && is_aligned(a->data, dtype_bytes(a->dtype)) &&
         a->row_stride >= (int64_t)cols && a->batch_stride >= 0 && !(written && batch > 1 && a->batch_stride < (int64_t)cols);
}

// Follows the interval that the singular values of [0, 1] reach: the image of an interval that holds 0 under p(s) = s (a + q),
// q = b s^2 + c s^4, is one again, with its ends at p of the old ends or where p' = a + 3 b t + 5 c t^2 = 0 (t = s^2).  `widen`
// stretches it before each step.  Does it stay within max_s, and q within max_q?
bool orbit_stays(int steps, double a, double b, double c, double widen, double max_s, double max_q) {
  double zeros[2];
  int n = 0;
  const double square = 9.0 * b * b - 20.0 * a * c;
  if (square >= 0.0) {
    const double h = -0.5 * (3.0 * b + copysign(sqrt(square), b));
    if (c != 0.0 && h / (5.0 * c) > 0.0) zeros[n++] = sqrt(h / (5.0 * c));
    if (h != 0.0 && a / h > 0.0) zeros[n++] = sqrt(a / h);
  }
  double lo = 0.0, hi = 1.0;
  for (int k = 0; k < steps; ++k) {
    lo *= 1.0 + widen; hi *= 1.0 + widen;
    const double t_end = fmax(lo * lo, hi * hi), t_mid = c != 0.0 ? -b / (2.0 * c) : -1.0;
    auto q = [&](double t) { return t * (b + c * t); };
    if (!(fabs(q(t_end)) <= max_q) || (t_mid > 0.0 && t_mid < t_end && !(fabs(q(t_mid)) <= max_q))) return false;
    double next_lo = 0.0, next_hi = 0.0;
    auto reach = [&](double s) {
      const double p = s * (a + q(s * s));
      next_lo = fmin(next_lo, p); next_hi = fmax(next_hi, p);
      return fabs(p) <= max_s;
    };
    bool ok = reach(lo) && reach(hi);
    for (int i = 0; i < n; ++i) ok = ok && (zeros[i] > hi || reach(zeros[i])) && (-zeros[i] < lo || reach(-zeros[i]));
    if (!ok) return false;
    lo = next_lo; hi = next_hi;
  }
  return true;
}

// Does every singular value in [0, 1] stay within what the 16-bit forms hold?  Once exactly, and once with room for the rounding
// of one-piece operands, which takes a value out of the range of coefficients that the first question lets through where p is
// steep (4 of 8538 sets drawn at random); the forms hold values up to 3.9 and q up to 63.  0.3 us; a grid of 1025 values took 17 us
// for five steps and missed narrow gaps.
bool poly_ok(int steps, float a, float b, float c, float eps) {
  if (steps < 1 || steps > 32 || !isfinite(a) || !isfinite(b) || !isfinite(c) || !isfinite(eps) || eps < 0.f) return false;
  return orbit_stays(steps, a, b, c, 0.0, kMaxSingular, kMaxPoly) &&
         orbit_stays(steps, a, b, c, 0x1p-9, 1.125 * kMaxSingular, 1.125 * kMaxPoly);
}

bool wide_rows(const Mat& a, int dtype, int batch) {
  return is_aligned(a.p, 4 * dtype_bytes(dtype)) && a.row % 4 == 0 && (batch == 1 || a.batch % 4 == 0);
}

template <typename G>
cudaError_t prepare(const OrthoPlan& P, const OrthoRequest& R, char* ws, cudaStream_t st) {
  double* partial = reinterpret_cast<double*>(ws + P.off_norm);
  const bool g_wide = wide_rows(R.g, R.g_dtype, P.batch), v_wide = R.has_v && wide_rows(R.v, S3GD_F32, P.batch);
  const bool one_row = R.g.row == (long long)P.cols && (!R.has_v || R.v.row == (long long)P.cols);
  count_launch(2);
  cudaError_t e = launch_after(momentum_norm_kernel<G>, dim3(P.norm_blocks, P.batch), dim3(kPrepThreads), 0, st, R.g, R.v, R.has_v, g_wide, v_wide,
                               one_row ? (uint64_t)1 : P.rows, one_row ? P.rows * P.cols : P.cols, R.mu, R.nesterov, partial,
                               reinterpret_cast<uint32_t*>(ws + P.off_hdr));
  if (e != cudaSuccess) return e;
  return launch_after(normalise_kernel<G>, dim3((P.n + 63) / 64, (P.m + 63) / 64, P.batch), dim3(kPrepThreads), 0, st, R.g, R.v, R.has_v, g_wide,
                      v_wide, P.rows, P.cols, R.mu, R.nesterov, R.eps, partial, P.norm_blocks, reinterpret_cast<__half*>(ws + P.off_x), P.m, P.n,
                      P.ldx);
}

cudaError_t run(const OrthoPlan& P, const OrthoRequest& R, char* ws, cudaStream_t st) {
  if (is_small(P)) return launch_small(P, R, ws, st);
  cudaError_t e = R.g_dtype == S3GD_F32 ? prepare<float>(P, R, ws, st) : R.g_dtype == S3GD_BF16 ? prepare<__nv_bfloat16>(P, R, ws, st)
                                                                                             : prepare<int8_t>(P, R, ws, st);
  return e == cudaSuccess ? launch_products(P, R, ws, st) : e;
}

Store as_store(const s3gd_matrix* a, int batch, bool transpose, bool update, float keep, float rate) {
  const size_t four = 4 * dtype_bytes(a->dtype);
  const bool wide = is_aligned(a->data, four) && a->row_stride % 4 == 0 && (batch == 1 || a->batch_stride % 4 == 0);
  return {{static_cast<char*>(a->data), (long long)a->row_stride, (long long)a->batch_stride}, a->dtype, transpose, update, wide, keep, rate};
}

s3gd_status common_checks(const s3gd_matrix* g, int batch, uint64_t rows, uint64_t cols, int steps, float a, float b, float c, float eps,
                          int split_steps, OrthoPlan* P) {
  if (!make_plan(batch, rows, cols, P) || !mat_ok(g, batch, cols, false)) return S3GD_ERR_INVALID_ARG;
  if (g->dtype != S3GD_F32 && g->dtype != S3GD_BF16 && g->dtype != S3GD_I8) return S3GD_ERR_INVALID_ARG;
  if (!poly_ok(steps, a, b, c, eps) || split_steps < -1 || split_steps > steps) return S3GD_ERR_INVALID_ARG;
  return S3GD_OK;
}

Mat as_mat(const s3gd_matrix* a) { return {static_cast<char*>(a->data), (long long)a->row_stride, (long long)a->batch_stride}; }

// Two pieces in every product unless the caller asks for fewer, whatever the result's type: a bf16 result is then the fp32
// one rounded once (1.7e-3 from the definition, all of it rounding; with one piece 2.0e-3 to 2.3e-3).
int split_rule(int split_steps, int steps) { return split_steps >= 0 ? split_steps : steps; }

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
  OrthoRequest R = {};
  R.g = as_mat(g); R.g_dtype = g->dtype;
  R.out = as_store(out, batch, rows > cols, false, 0.f, 0.f);
  R.steps = steps; R.split = split_rule(split_steps, steps);
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
  OrthoRequest R = {};
  R.g = as_mat(g); R.g_dtype = g->dtype;
  R.has_v = opt_v != nullptr;
  if (R.has_v) R.v = as_mat(opt_v);
  R.mu = mu; R.nesterov = nesterov;
  R.out = as_store(x, batch, rows > cols, true, 1.f - lr * weight_decay, lr * scale);
  R.steps = steps; R.split = split_rule(split_steps, steps);
  R.a = a; R.b = b; R.c = c; R.eps = eps;
  return run(P, R, static_cast<char*>(ws), static_cast<cudaStream_t>(stream)) == cudaSuccess ? S3GD_OK : S3GD_ERR_CUDA;
}
