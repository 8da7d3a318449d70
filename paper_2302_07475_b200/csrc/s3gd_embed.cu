// Embedding table: scaled lookup, and the gradient of M workers written into their rows (see include/s3gd.h).
#include "s3gd_ops.cuh"

namespace s3gd {
namespace {

constexpr int kThreads = 256;

template <typename W, typename I, typename O>
__global__ void lookup_kernel(const W* table, long long table_stride, uint64_t vocab, uint32_t dim, const I* ids, uint64_t n, float scale,
                              O* out, long long out_stride, uint32_t* bad) {
  for (uint64_t t = blockIdx.x; t < n; t += gridDim.x) {
    const long long id = (long long)ids[t];
    const bool there = id >= 0 && (uint64_t)id < vocab;
    if (id >= 0 && !there && bad != nullptr && threadIdx.x == 0) atomicAdd(bad, 1u);
    for (uint32_t j = threadIdx.x; j < dim; j += kThreads)
      out[t * out_stride + j] = there ? from_f32<O>(__fmul_rn(scale, to_f32(table[id * table_stride + j]))) : from_f32<O>(0.f);
  }
}

template <typename O>
__global__ void zero_rows_kernel(O* grads, long long stride, uint64_t n) {
  O* row = grads + (size_t)blockIdx.y * stride;
  for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (uint64_t)gridDim.x * kThreads) row[i] = from_f32<O>(0.f);
}

// One CTA per token and 256 columns: the first token of its id sums all of them, in ascending order.
template <typename D, typename I, typename O>
__global__ void first_token_kernel(const D* dout, long long tok_stride, long long worker_stride, const I* ids, uint64_t T, uint64_t vocab,
                                   uint32_t dim, float scale, O* grads, long long stride, int accumulate, uint32_t* bad) {
  const uint64_t t = blockIdx.x, m = blockIdx.z;
  const I* id_row = ids + m * T;
  const long long id = (long long)id_row[t];
  if (id < 0) return;
  if ((uint64_t)id >= vocab) {
    if (bad != nullptr && threadIdx.x == 0 && blockIdx.y == 0) atomicAdd(bad, 1u);
    return;
  }
  int earlier = 0;
  for (uint64_t s = threadIdx.x; s < t; s += kThreads) earlier |= (long long)id_row[s] == id;
  if (__syncthreads_or(earlier)) return;
  for (uint32_t j0 = blockIdx.y * kThreads; j0 < dim; j0 += gridDim.y * kThreads) {
    const uint32_t j = j0 + threadIdx.x;
    if (j >= dim) continue;
    float sum = 0.f;
    for (uint64_t s = t; s < T; ++s)
      if ((long long)id_row[s] == id) sum += to_f32(dout[m * worker_stride + s * tok_stride + j]);
    O* to = grads + m * stride + (uint64_t)id * dim + j;
    *to = from_f32<O>((accumulate ? to_f32(*to) : 0.f) + scale * sum);
  }
}

bool is_real(int dt) { return dt == S3GD_F32 || dt == S3GD_BF16; }
bool is_index(int dt) { return dt == S3GD_I32 || dt == S3GD_I64; }

template <typename W, typename I, typename O>
cudaError_t lookup(const void* table, int64_t ts, uint64_t vocab, uint64_t dim, const void* ids, uint64_t n, float scale, void* out,
                   int64_t os, uint32_t* bad, cudaStream_t st) {
  count_launch();
  lookup_kernel<W, I, O><<<(unsigned)(n < 65536 ? n : 65536), kThreads, 0, st>>>(static_cast<const W*>(table), ts, vocab, (uint32_t)dim,
      static_cast<const I*>(ids), n, scale, static_cast<O*>(out), os, bad);
  return cudaGetLastError();
}

struct GradArgs {
  const void* dout; int64_t tok_stride, worker_stride;
  const void* ids; int M; uint64_t T, vocab, dim;
  float scale; void* grads; int64_t stride; int accumulate; uint32_t* bad;
};

template <typename D, typename I, typename O>
cudaError_t grad(const GradArgs& a, cudaStream_t st) {
  if (!a.accumulate) {
    const uint64_t n = a.vocab * a.dim, want = (n + 4095) / 4096;
    count_launch();
    zero_rows_kernel<O><<<dim3((unsigned)(want < 4096 ? want : 4096), a.M), kThreads, 0, st>>>(static_cast<O*>(a.grads), a.stride, n);
  }
  if (a.T > 0) {
    count_launch();
    const uint64_t by = (a.dim + kThreads - 1) / kThreads;
    first_token_kernel<D, I, O><<<dim3((unsigned)a.T, (unsigned)(by < 65535 ? by : 65535), a.M), kThreads, 0, st>>>(
        static_cast<const D*>(a.dout), a.tok_stride, a.worker_stride, static_cast<const I*>(a.ids), a.T, a.vocab, (uint32_t)a.dim, a.scale,
        static_cast<O*>(a.grads), a.stride, a.accumulate, a.bad);
  }
  return cudaGetLastError();
}

// calls f with a value of the types that the two element types and the index type name
template <typename F>
cudaError_t by_types(int in, int idx, int out, F f) {
  auto with_out = [&](auto a, auto b) { return out == S3GD_F32 ? f(a, b, float()) : f(a, b, __nv_bfloat16()); };
  auto with_idx = [&](auto a) { return idx == S3GD_I32 ? with_out(a, int32_t()) : with_out(a, int64_t()); };
  return in == S3GD_F32 ? with_idx(float()) : with_idx(__nv_bfloat16());
}

size_t grad_workspace(int M, uint64_t T, uint64_t vocab, uint64_t dim) {
  if (M < 1 || M > 65535 || vocab == 0 || dim == 0 || vocab >= (1ull << 31) || dim >= (1ull << 31) || T >= (1ull << 31) ||
      (uint64_t)M * T >= (1ull << 31))
    return 0;
  return align_up(kHdrWords * sizeof(uint32_t), 256);
}

}  // namespace
}  // namespace s3gd

using namespace s3gd;

extern "C" s3gd_status s3gd_embed(const void* table, int table_dtype, int64_t table_stride, uint64_t vocab, uint64_t dim, const void* ids,
                                  int ids_dtype, uint64_t n, float scale, void* out, int out_dtype, int64_t out_stride,
                                  uint32_t* opt_bad_count, void* stream) {
  if (!is_real(table_dtype) || !is_index(ids_dtype) || !is_real(out_dtype)) return S3GD_ERR_INVALID_ARG;
  if (vocab == 0 || dim == 0 || vocab >= (1ull << 31) || dim >= (1ull << 31) || n >= (1ull << 40)) return S3GD_ERR_INVALID_ARG;
  if (table == nullptr || table_stride < (int64_t)dim || out_stride < (int64_t)dim) return S3GD_ERR_INVALID_ARG;
  if (n > 0 && (ids == nullptr || out == nullptr)) return S3GD_ERR_INVALID_ARG;
  if (!is_aligned(table, dtype_bytes(table_dtype)) || !is_aligned(ids, dtype_bytes(ids_dtype)) || !is_aligned(out, dtype_bytes(out_dtype)) ||
      !is_aligned(opt_bad_count, 4))
    return S3GD_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (opt_bad_count != nullptr && cudaMemsetAsync(opt_bad_count, 0, 4, st) != cudaSuccess) return S3GD_ERR_CUDA;
  if (n == 0) return S3GD_OK;
  const cudaError_t e = by_types(table_dtype, ids_dtype, out_dtype, [&](auto w, auto i, auto o) {
    return lookup<decltype(w), decltype(i), decltype(o)>(table, table_stride, vocab, dim, ids, n, scale, out, out_stride, opt_bad_count, st);
  });
  return e == cudaSuccess ? S3GD_OK : S3GD_ERR_CUDA;
}

extern "C" size_t s3gd_embed_grad_workspace_bytes(int M, uint64_t T, uint64_t vocab, uint64_t dim) { return grad_workspace(M, T, vocab, dim); }

extern "C" s3gd_status s3gd_embed_grad(const void* dout, int dout_dtype, int64_t dout_stride, int64_t dout_worker_stride, const void* ids,
                                       int ids_dtype, int M, uint64_t T, uint64_t vocab, uint64_t dim, float scale, void* grads,
                                       int grads_dtype, int64_t grads_stride, int accumulate, uint32_t* opt_bad_count, void* ws,
                                       size_t ws_bytes, void* stream) {
  const size_t need = grad_workspace(M, T, vocab, dim);
  if (need == 0 || !is_real(dout_dtype) || !is_index(ids_dtype) || !is_real(grads_dtype)) return S3GD_ERR_INVALID_ARG;
  if (grads == nullptr || (M > 1 && grads_stride < (int64_t)(vocab * dim))) return S3GD_ERR_INVALID_ARG;
  if (T > 0 && (dout == nullptr || ids == nullptr || dout_stride < 0 || dout_worker_stride < 0)) return S3GD_ERR_INVALID_ARG;
  if (!is_aligned(dout, dtype_bytes(dout_dtype)) || !is_aligned(ids, dtype_bytes(ids_dtype)) || !is_aligned(grads, dtype_bytes(grads_dtype)) ||
      !is_aligned(opt_bad_count, 4))
    return S3GD_ERR_INVALID_ARG;
  if (ws == nullptr || ws_bytes < need || !is_aligned(ws, 256)) return S3GD_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (cudaMemsetAsync(ws, 0, kHdrWords * sizeof(uint32_t), st) != cudaSuccess) return S3GD_ERR_CUDA;
  if (opt_bad_count != nullptr && cudaMemsetAsync(opt_bad_count, 0, 4, st) != cudaSuccess) return S3GD_ERR_CUDA;
  const GradArgs a = {dout, dout_stride, dout_worker_stride, ids, M, T, vocab, dim, scale, grads, grads_stride, accumulate, opt_bad_count};
  const cudaError_t e = by_types(dout_dtype, ids_dtype, grads_dtype,
                                 [&](auto d, auto i, auto o) { return grad<decltype(d), decltype(i), decltype(o)>(a, st); });
  return e == cudaSuccess ? S3GD_OK : S3GD_ERR_CUDA;
}
