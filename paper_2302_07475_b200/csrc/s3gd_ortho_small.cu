// Whole orthogonalised updates of small matrices: one CTA per matrix, one launch for momentum, norm, all products and the
// update.  X (up to 128 x 256) and S stay in shared memory, as two fp16 pieces each, in the layout that the tensor cores read
// both ways: rows of 64 entries in 128 swizzled bytes serve as K-major operand for X X^T and S S^T and as MN-major operand for
// B X.  A step is three products, each followed by all sixteen warps taking the sums out of tensor memory and writing the next
// operand in place.  The chain of these, not bytes or operations, is what the time is made of: 32 matrices of 64 x 128 fp32 take
// 31 us (2 MB, 0.9 GFLOP), about 5 us a step of three products; 16 x 16 still 19 us, from a CUDA graph too (the host's part of a
// call, 15 us, runs beside it).
#include "s3gd_ortho.cuh"
#include "s3gd_tcgen05.cuh"

namespace s3gd {
namespace {

constexpr int kGroups = 16;                        // of four entries per thread: 512 threads hold 128 x 256
constexpr int kPanel = 128 * 128;                  // bytes of 128 rows x 64 entries

struct SmallArgs {
  Mat g, v;
  Store store;
  uint32_t* hdr;
  float mu, eps, a, b, c;
  int nesterov, has_v, steps, split, carried;
  int rows, cols, m, n;
  int panels_x, panels_s, tmem_cols;
  int g_wide, v_wide;                              // rows and base allow four entries in one access
  int per_row;                                     // groups of four entries in a row, and what divides by it: exact below 2^16
  uint64_t reciprocal;
};

struct SmallShared {
  uint64_t done;
  uint32_t tmem;
  double warp_sums[16];
};

__device__ __forceinline__ int entry_offset(int i, int j) {       // bytes, of entry (i, j) in its piece
  return (j >> 6) * kPanel + i * 128 + ((((j >> 3) & 7) ^ (i & 7)) << 4) + (j & 7) * 2;
}

__device__ __forceinline__ void write8(char* hi, char* lo, int off, const float* x) {
  uint32_t h[4], l[4];
  split8(x, true, h, l);
  *reinterpret_cast<uint4*>(hi + off) = make_uint4(h[0], h[1], h[2], h[3]);
  *reinterpret_cast<uint4*>(lo + off) = make_uint4(l[0], l[1], l[2], l[3]);
}

template <typename G, int kSmallThreads>
__global__ void __launch_bounds__(kSmallThreads, 512 / kSmallThreads) small_kernel(const SmallArgs P) {
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
  if (mat == 0 && threadIdx.x < kHdrWords) P.hdr[threadIdx.x] = 0;           // a record, if any, comes seconds later
  // ---- momentum, norm (sum of squares in 64 bits) and X_0; u stays in registers in between
  const G* g = reinterpret_cast<const G*>(P.g.p) + (size_t)mat * P.g.batch;
  float* v = reinterpret_cast<float*>(P.v.p) + (P.has_v ? (size_t)mat * P.v.batch : 0);
  const int groups = P.rows * P.per_row;
  auto row_of = [&](int e) { return (int)(((uint64_t)(uint32_t)e * P.reciprocal) >> 32); };
  float u[kGroups][4];
  double sum = 0.0;
#pragma unroll
  for (int k = 0; k < kGroups; ++k) {
    u[k][0] = u[k][1] = u[k][2] = u[k][3] = 0.f;
    if (k * kSmallThreads >= groups) continue;               // the same for all threads: nothing is computed
    const int e = k * kSmallThreads + threadIdx.x, r = row_of(e), c = (e - r * P.per_row) * 4;
    if (e < groups) get4(g + (size_t)r * P.g.row + c, P.g_wide, P.cols - c, u[k]);
  }
  if (P.has_v) {
#pragma unroll
    for (int k0 = 0; k0 < kGroups; k0 += 4) {
      if (k0 * kSmallThreads >= groups) break;
      float old[4][4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int e = (k0 + k) * kSmallThreads + threadIdx.x, r = row_of(e), c = (e - r * P.per_row) * 4;
        if (e < groups) get4(v + (size_t)r * P.v.row + c, P.v_wide, P.cols - c, old[k]);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int e = (k0 + k) * kSmallThreads + threadIdx.x, r = row_of(e), c = (e - r * P.per_row) * 4;
        if (e >= groups) continue;
        float* p = v + (size_t)r * P.v.row + c;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float nv = __fadd_rn(__fmul_rn(P.mu, old[k][x]), u[k0 + k][x]);
          old[k][x] = nv;
          if (c + x < P.cols) u[k0 + k][x] = P.nesterov ? __fadd_rn(u[k0 + k][x], __fmul_rn(P.mu, nv)) : nv;
        }
        put4(p, P.v_wide, P.cols - c, old[k]);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kGroups; ++k) {
    if (k * kSmallThreads >= groups) break;
#pragma unroll
    for (int x = 0; x < 4; ++x) sum += (double)u[k][x] * (double)u[k][x];
  }
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) sh->warp_sums[warp] = sum;
  __syncthreads();
  sum = 0.0;
  for (int k = 0; k < kSmallThreads / 32; ++k) sum += sh->warp_sums[k];
  const Normaliser normalised(sqrt(sum), P.eps);
  const bool tall = P.rows > P.cols;
#pragma unroll
  for (int k = 0; k < kGroups; ++k) {
    if (k * kSmallThreads >= groups) break;
    const int e = k * kSmallThreads + threadIdx.x, r = row_of(e), c = (e - r * P.per_row) * 4;
    if (e >= groups) continue;
    __align__(8) __half hi[4], lo[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) split_half(normalised(u[k][x]), &hi[x], &lo[x]);
    if (!tall) {
      const int off = entry_offset(r, c);                    // four entries from a multiple of four: eight bytes
      *reinterpret_cast<uint2*>(x_hi + off) = *reinterpret_cast<uint2*>(hi);
      *reinterpret_cast<uint2*>(x_lo + off) = *reinterpret_cast<uint2*>(lo);
    } else {
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (c + x < P.cols) {
          const int off = entry_offset(c + x, r);
          *reinterpret_cast<__half*>(x_hi + off) = hi[x];
          *reinterpret_cast<__half*>(x_lo + off) = lo[x];
        }
    }
  }
  // ---- the products
  const int quad = warp & 3, part = warp >> 2, i = quad * 32 + lane;          // rows of a warp, and its part of the columns
  const int m16 = (P.m + 15) / 16, n16 = (P.n + 15) / 16, rows_here = quad * 32 < P.m;
  uint32_t phase = 0, tmem = 0;
  bool ok = true;
  // one product on the tensor cores: K in steps of 16; then every thread may take its row of the sums
  auto product = [&](const uint32_t* a, const uint32_t* b, bool b_mn, int n, int k16, bool split) {
    fence_async_smem();
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    tmem = sh->tmem;
    if (warp == 0) {                                         // the whole warp counts along, one lane issues
      const uint32_t idesc = product_desc(128, n, b_mn);
      auto pass = [&](uint32_t d, uint32_t at_a, uint32_t at_b, int from, int to, bool add) {
        const uint64_t da = operand_desc(at_a), db = operand_desc(at_b, b_mn ? kPanel : 16);
        for (int k = from; k < to; ++k) {
          const uint32_t step = (uint32_t)(k >> 2) * (kPanel / 16) + (uint32_t)(k & 3) * 2;
          mma_f16_elect(d, da + step, db + (b_mn ? (uint32_t)k * 128 : step), idesc, add);
          add = true;
        }
      };
      // two pieces: hi lo + lo hi before hi hi, as in the larger products, and the second half of hi hi into a sum of its own
      if (split) {
        pass(tmem, a[0], b[1], 0, k16, false);
        pass(tmem, a[1], b[0], 0, k16, true);
        pass(tmem, a[0], b[0], 0, k16 - k16 / 2, true);
        pass(tmem + P.tmem_cols / 2, a[0], b[0], k16 - k16 / 2, k16, false);
      } else {
        pass(tmem, a[0], b[0], 0, k16, false);
      }
      mma_commit_elect(smem_addr(&sh->done));
    }
    __syncwarp();
    if (ok) ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&sh->done), phase));   // a warp that gave up keeps to the barriers
    phase ^= 1;
    tcgen05_fence_after();
  };
  // 16 columns of this thread's row.  The tensor cores cut off what falls below the running sum; two shorter sums lose half of it.
  auto take16 = [&](int column, bool two, float* acc) {
    const uint32_t at = tmem + ((uint32_t)(quad * 32) << 16) + column;
    tmem_load16(at, acc);
    if (two) {
      float more[16];
      tmem_load16(at + P.tmem_cols / 2, more);
      tmem_load_wait();
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[e] += more[e];
    } else {
      tmem_load_wait();
    }
  };
  for (int step = 0; step < P.steps; ++step) {
    const bool split = step < P.split;
    float acc[16];
    product(xa, xa, false, m16 * 16, n16, split);
#pragma unroll 1
    for (int c = part; rows_here && c < m16; c += kSmallThreads / 128) {
      take16(c * 16, split && n16 > 1, acc);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[q * 8 + e] *= kScaleS / (kScaleX * kScaleX);
        if (i < P.m) write8(s_hi, s_lo, entry_offset(i, c * 16 + q * 8), acc + q * 8);
      }
    }
    product(sa, sa, false, m16 * 16, m16, split);
#pragma unroll 1
    for (int c = part; rows_here && c < m16; c += kSmallThreads / 128) {
      take16(c * 16, split && m16 > 1, acc);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int off = entry_offset(i, c * 16 + q * 8);
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
    for (int c = part; rows_here && c < n16; c += kSmallThreads / 128) {
      take16(c * 16, split && m16 > 1, acc);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int j = c * 16 + q * 8, off = entry_offset(i, j);
        float x[8];
        read8(x_hi, x_lo, off, step < P.carried, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __fmaf_rn(P.a, x[e], __fmul_rn(1.f / kScaleB, acc[q * 8 + e]));
        if (!last) {
          if (i < P.m) write8(x_hi, x_lo, off, x);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= 1.f / kScaleX;
          if (!ok) continue;
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

template <typename G, int kSmallThreads>
cudaError_t launch(const SmallArgs& A, int batch, int bytes, cudaStream_t st) {
  static int done[kMaxDevices];
  auto kernel = small_kernel<G, kSmallThreads>;
  cudaError_t e = opt_in_dynamic_smem(reinterpret_cast<const void*>(kernel), bytes, done);
  if (e != cudaSuccess) return e;
  count_launch();
  return launch_after(kernel, dim3(batch), dim3(kSmallThreads), bytes, st, A);
}

// Two CTAs of 256 threads share an SM where there are more matrices than SMs and each fits in half of one: 296 of 64 x 64
// fp32 take 37 us that way and 57 us with 512 threads.
template <typename G>
cudaError_t launch_by(const SmallArgs& A, int batch, int bytes, cudaStream_t st) {
  const bool half = batch > sm_count() && bytes <= 112 * 1024 && A.tmem_cols <= 256 && A.rows * A.per_row <= 256 * kGroups;
  return half ? launch<G, 256>(A, batch, bytes, st) : launch<G, 512>(A, batch, bytes, st);
}

}  // namespace

// What one CTA's shared memory holds.  One 64 x 128 fp32: 31 us, by the kernels for large matrices 90 us; 128 x 256: 60 and 97 us;
// 400 of them: 186 and 816 us.
bool is_small(const OrthoPlan& P) { return P.m <= 128 && P.n <= 256; }

cudaError_t launch_small(const OrthoPlan& P, const OrthoRequest& R, char* ws, cudaStream_t st) {
  SmallArgs A = {};
  A.g = R.g; A.v = R.v; A.store = R.out;
  A.hdr = reinterpret_cast<uint32_t*>(ws + P.off_hdr);
  A.mu = R.mu; A.eps = R.eps; A.a = R.a; A.b = R.b; A.c = R.c;
  A.nesterov = R.nesterov; A.has_v = R.has_v; A.steps = R.steps; A.split = R.split; A.carried = carried_steps(R.steps, R.split);
  A.rows = (int)P.rows; A.cols = (int)P.cols; A.m = P.m; A.n = P.n;
  A.per_row = (A.cols + 3) / 4;
  A.reciprocal = ((1ull << 32) + A.per_row - 1) / A.per_row;
  A.panels_x = (P.n + 63) / 64;
  A.panels_s = (P.m + 63) / 64;
  A.tmem_cols = 32;                                  // two sums
  while (A.tmem_cols < (P.n + 15) / 16 * 32) A.tmem_cols *= 2;
  const size_t g_four = 4 * dtype_bytes(R.g_dtype);
  A.g_wide = is_aligned(R.g.p, g_four) && R.g.row % 4 == 0 && (P.batch == 1 || R.g.batch % 4 == 0);
  A.v_wide = R.has_v && is_aligned(R.v.p, 16) && R.v.row % 4 == 0 && (P.batch == 1 || R.v.batch % 4 == 0);
  const int bytes = 1024 + 2 * (A.panels_x + A.panels_s) * kPanel + (int)sizeof(SmallShared);
  if (R.g_dtype == S3GD_F32) return launch_by<float>(A, P.batch, bytes, st);
  return R.g_dtype == S3GD_BF16 ? launch_by<__nv_bfloat16>(A, P.batch, bytes, st) : launch_by<int8_t>(A, P.batch, bytes, st);
}

}  // namespace s3gd
