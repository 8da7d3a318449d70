// Whole orthogonalised updates of small matrices: one CTA per matrix, one launch for momentum, norm, all products and the
// update.  X (up to 128 x 256) and S stay in shared memory, as two fp16 pieces each, in the layout that the tensor cores read
// both ways: rows of 64 entries in 128 swizzled bytes serve as K-major operand for X X^T and S S^T and as MN-major operand for
// B X.  A step is three products, each followed by all eight warps taking the sums out of tensor memory and writing the next
// operand in place; the chain of these (about 3 us a step for 64 x 128), not bytes or operations, is what the time is made of.
#include "s3gd_ortho.cuh"
#include "s3gd_tcgen05.cuh"

namespace s3gd {
namespace {

constexpr int kSmallThreads = 256;
constexpr int kPanel = 128 * 128;                  // bytes of 128 rows x 64 entries

struct SmallArgs {
  Mat g, v;
  Store store;
  uint32_t* hdr;
  float mu, eps, a, b, c;
  int nesterov, has_v, steps, split, carried;
  int rows, cols, m, n;
  int panels_x, panels_s, tmem_cols;
};

struct SmallShared {
  uint64_t done;
  uint32_t tmem;
  double warp_sums[kSmallThreads / 32];
};

__device__ __forceinline__ int entry_offset(int i, int j) {       // bytes, of entry (i, j) in its piece
  return (j >> 6) * kPanel + i * 128 + ((((j >> 3) & 7) ^ (i & 7)) << 4) + (j & 7) * 2;
}

// eight neighbouring entries of row i as floats, from one or two pieces
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
__device__ __forceinline__ void write8(char* hi, char* lo, int off, const float* x) {
  __half2 h[4], l[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    h[e] = __floats2half2_rn(x[2 * e], x[2 * e + 1]);
    const float2 f = __half22float2(h[e]);
    l[e] = __floats2half2_rn(x[2 * e] - f.x, x[2 * e + 1] - f.y);
  }
  *reinterpret_cast<uint4*>(hi + off) = *reinterpret_cast<uint4*>(h);
  *reinterpret_cast<uint4*>(lo + off) = *reinterpret_cast<uint4*>(l);
}

template <typename T>
__device__ __forceinline__ void put8(const Store& s, int mat, int i, int j0, int m, int n, const float* x) {
  if (i >= m) return;
  T* base = reinterpret_cast<T*>(s.to.p) + (size_t)mat * s.to.batch;
  const size_t step = s.transpose ? s.to.row : 1;
  base += s.transpose ? (size_t)j0 * s.to.row + i : (size_t)i * s.to.row + j0;
  T old[8] = {};
  if (s.update)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (j0 + e < n) old[e] = base[e * step];
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (j0 + e < n) base[e * step] = from_f32<T>(s.update ? __fmaf_rn(-s.rate, x[e], __fmul_rn(s.keep, to_f32(old[e]))) : x[e]);
}

template <typename G>
__global__ void __launch_bounds__(kSmallThreads) small_kernel(const SmallArgs P) {
  extern __shared__ char smem_raw[];
  const uint32_t raw = smem_addr(smem_raw), base = (raw + 1023) & ~1023u;
  char* x_hi = smem_raw + (base - raw);
  char* x_lo = x_hi + P.panels_x * kPanel;
  char* s_hi = x_lo + P.panels_x * kPanel;
  char* s_lo = s_hi + P.panels_s * kPanel;
  SmallShared* sh = reinterpret_cast<SmallShared*>(s_lo + P.panels_s * kPanel);
  const uint32_t xa[2] = {smem_addr(x_hi), smem_addr(x_lo)}, sa[2] = {smem_addr(s_hi), smem_addr(s_lo)};
  const int warp = threadIdx.x >> 5, lane = lane_id(), mat = blockIdx.x;
  if (warp == 0) {
    if (lane == 0) {
      mbar_init(smem_addr(&sh->done), 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    tmem_alloc<1>(smem_addr(&sh->tmem), P.tmem_cols);
    tcgen05_fence_before();
  }
  for (int o = threadIdx.x * 16; o < 2 * (P.panels_x + P.panels_s) * kPanel; o += kSmallThreads * 16)
    *reinterpret_cast<uint4*>(x_hi + o) = make_uint4(0, 0, 0, 0);            // what lies beside m and n counts as zero
  grid_dependency_wait();
  // ---- momentum and norm (sum of squares in 64 bits), then X_0; the matrix is read twice, the second time from cache
  const G* g = reinterpret_cast<const G*>(P.g.p) + (size_t)mat * P.g.batch;
  float* v = reinterpret_cast<float*>(P.v.p) + (P.has_v ? (size_t)mat * P.v.batch : 0);
  const int count = P.rows * P.cols;
  constexpr int kAhead = 8;
  double sum = 0.0;
  for (int e0 = threadIdx.x; e0 < count; e0 += kAhead * kSmallThreads) {
    float u[kAhead], old[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int e = e0 + k * kSmallThreads, r = e / P.cols, c = e - r * P.cols;
      u[k] = e < count ? to_f32(g[(size_t)r * P.g.row + c]) : 0.f;
      old[k] = e < count && P.has_v ? v[(size_t)r * P.v.row + c] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int e = e0 + k * kSmallThreads, r = e / P.cols, c = e - r * P.cols;
      if (e < count && P.has_v) {
        const float nv = __fadd_rn(__fmul_rn(P.mu, old[k]), u[k]);
        v[(size_t)r * P.v.row + c] = nv;
        u[k] = P.nesterov ? __fadd_rn(u[k], __fmul_rn(P.mu, nv)) : nv;
      }
      sum += (double)u[k] * (double)u[k];
    }
  }
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) sh->warp_sums[warp] = sum;
  __syncthreads();
  sum = 0.0;
  for (int k = 0; k < kSmallThreads / 32; ++k) sum += sh->warp_sums[k];
  const float inv = (float)((double)kScaleX / (sqrt(sum) + (double)P.eps));
  const bool tall = P.rows > P.cols;
  for (int e0 = threadIdx.x; e0 < count; e0 += kAhead * kSmallThreads) {
    float u[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int e = e0 + k * kSmallThreads, r = e / P.cols, c = e - r * P.cols;
      u[k] = 0.f;
      if (e < count) {
        if (!P.has_v) u[k] = to_f32(g[(size_t)r * P.g.row + c]);
        else if (!P.nesterov) u[k] = v[(size_t)r * P.v.row + c];
        else u[k] = __fadd_rn(to_f32(g[(size_t)r * P.g.row + c]), __fmul_rn(P.mu, v[(size_t)r * P.v.row + c]));
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int e = e0 + k * kSmallThreads, r = e / P.cols, c = e - r * P.cols;
      if (e >= count) continue;
      const int off = tall ? entry_offset(c, r) : entry_offset(r, c);
      __half hi, lo;
      split_half(u[k] * inv, &hi, &lo);
      *reinterpret_cast<__half*>(x_hi + off) = hi;
      *reinterpret_cast<__half*>(x_lo + off) = lo;
    }
  }
  // ---- the products
  const int quad = warp & 3, half = warp >> 2, i = quad * 32 + lane;
  const int m16 = (P.m + 15) / 16, n16 = (P.n + 15) / 16, m32 = (P.m + 31) / 32, n32 = (P.n + 31) / 32;

  uint32_t phase = 0, tmem = 0;
  bool ok = true;
  // one product on the tensor cores: K in steps of 16; then every thread may take its row of the sums
  auto product = [&](const uint32_t* a, const uint32_t* b, bool b_mn, int n, int k16, bool split) {
    fence_async_smem();
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    tmem = sh->tmem;
    if (threadIdx.x == 0) {
      const uint32_t idesc = product_desc(128, n, b_mn);
      bool add = false;
      for (int p = split ? 0 : 2; p < 3; ++p)                                // hi lo + lo hi first, hi hi last: see the larger products
        for (int k = 0; k < k16; ++k) {
          const uint32_t at_a = a[p == 1] + (k >> 2) * kPanel + (k & 3) * 32;
          const uint32_t at_b = b[p == 0] + (b_mn ? k * 2048 : (k >> 2) * kPanel + (k & 3) * 32);
          mma_f16<1>(tmem, operand_desc(at_a), b_mn ? operand_desc(at_b, kPanel) : operand_desc(at_b), idesc, add);
          add = true;
        }
      mma_commit<1>(smem_addr(&sh->done));
    }
    __syncwarp();
    ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&sh->done), phase)) && ok;
    phase ^= 1;
    tcgen05_fence_after();
  };
  for (int step = 0; step < P.steps && ok; ++step) {
    const bool split = step < P.split;
    const uint32_t row = (uint32_t)(quad * 32) << 16;
    float acc[32];
    product(xa, xa, false, m16 * 16, n16, split);
#pragma unroll 1
    for (int c = half; c < m32; c += 2) {
      tmem_load32(tmem + row + c * 32, acc);
      tmem_load_wait();
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[q * 8 + e] *= kScaleS / (kScaleX * kScaleX);
        if (i < P.m) write8(s_hi, s_lo, entry_offset(i, c * 32 + q * 8), acc + q * 8);
      }
    }
    product(sa, sa, false, m16 * 16, m16, split);
#pragma unroll 1
    for (int c = half; c < m32; c += 2) {
      tmem_load32(tmem + row + c * 32, acc);
      tmem_load_wait();
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int off = entry_offset(i, c * 32 + q * 8);
        float s[8];
        read8(s_hi, s_lo, off, split, s);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          s[e] = __fmaf_rn(P.b * (kScaleB / kScaleS), s[e], __fmul_rn(P.c * (kScaleB / (kScaleS * kScaleS)), acc[q * 8 + e]));
        if (i < P.m) write8(s_hi, s_lo, off, s);
      }
    }
    product(sa, xa, true, n16 * 16, m16, split);
    const bool last = step + 1 == P.steps;
#pragma unroll 1
    for (int c = half; c < n32; c += 2) {
      tmem_load32(tmem + row + c * 32, acc);
      tmem_load_wait();
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int j = c * 32 + q * 8, off = entry_offset(i, j);
        float x[8];
        read8(x_hi, x_lo, off, step < P.carried, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __fmaf_rn(P.a, x[e], __fmul_rn(1.f / kScaleB, acc[q * 8 + e]));
        if (!last) {
          if (i < P.m) write8(x_hi, x_lo, off, x);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= 1.f / kScaleX;
          if (P.store.dtype == S3GD_F32) put8<float>(P.store, mat, i, j, P.m, P.n, x);
          else put8<__nv_bfloat16>(P.store, mat, i, j, P.m, P.n, x);
        }
      }
    }
  }
  if (!ok) atomicOr(&P.hdr[kHdrStatus], (uint32_t)kFlagInternal);            // a wait gave up; products are not in flight for that long
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  if (warp == 0) tmem_free<1>(sh->tmem, P.tmem_cols);
}

template <typename G>
cudaError_t launch(const SmallArgs& A, int batch, int bytes, cudaStream_t st) {
  static int done[kMaxDevices];
  cudaError_t e = opt_in_dynamic_smem(reinterpret_cast<const void*>(small_kernel<G>), bytes, done);
  if (e != cudaSuccess) return e;
  count_launch();
  return launch_after(small_kernel<G>, dim3(batch), dim3(kSmallThreads), bytes, st, A);
}

}  // namespace

bool is_small(const OrthoPlan& P) { return P.m <= 128 && P.n <= 256; }

cudaError_t launch_small(const OrthoPlan& P, const OrthoRequest& R, char* ws, cudaStream_t st) {
  SmallArgs A = {};
  A.g = R.g; A.v = R.v; A.store = R.out;
  A.hdr = reinterpret_cast<uint32_t*>(ws + P.off_hdr);
  A.mu = R.mu; A.eps = R.eps; A.a = R.a; A.b = R.b; A.c = R.c;
  A.nesterov = R.nesterov; A.has_v = R.has_v; A.steps = R.steps; A.split = R.split; A.carried = carried_steps(R.steps, R.split);
  A.rows = (int)P.rows; A.cols = (int)P.cols; A.m = P.m; A.n = P.n;
  A.panels_x = (P.n + 63) / 64;
  A.panels_s = (P.m + 63) / 64;
  A.tmem_cols = 32;                                  // 32-column loads must stay inside
  while (A.tmem_cols < (P.n + 31) / 32 * 32) A.tmem_cols *= 2;
  const int bytes = 1024 + 2 * (A.panels_x + A.panels_s) * kPanel + (int)sizeof(SmallShared);
  if (R.g_dtype == S3GD_F32) return launch<float>(A, P.batch, bytes, st);
  return R.g_dtype == S3GD_BF16 ? launch<__nv_bfloat16>(A, P.batch, bytes, st) : launch<int8_t>(A, P.batch, bytes, st);
}

}  // namespace s3gd
