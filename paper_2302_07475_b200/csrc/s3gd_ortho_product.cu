// The products of the Newton-Schulz steps on the tensor cores.
//
//   S = X X^T          symmetric: only tiles on and below the diagonal are computed, the others are their mirror image
//   B = b S + c S S    symmetric too (S S^T, both operands rows of S)
//   Y = a X + B X      B is its own transpose; X is read along its rows as the second operand (MN-major)
//
// One persistent kernel per product.  Operands are fp16 tiles brought by TMA into a ring of slots; one thread issues
// tcgen05.mma with fp32 sums in tensor memory, two sums in turn so that the epilogue of one tile runs under the products of
// the next.  kCta = 2: two CTAs of a cluster share a 256 x 256 tile and each holds half of either operand.
//
// Precision.  One fp16 piece per entry (11 bits), or two (kSplit, 22 bits): then hi hi + hi lo + lo hi, three products.
// The tensor cores add to the running fp32 sum without rounding to nearest, which biases a long sum of squares (the diagonal
// of S); with two pieces the sum is therefore taken out of tensor memory every kChunk slots of k and added in registers.
#include <atomic>

#include "s3gd_ortho.cuh"
#include "s3gd_tcgen05.cuh"

namespace s3gd {
namespace {

constexpr int kBlockK = 64;                       // entries of k per slot: one 128-byte row
constexpr int kSlotBytes = 32 * 1024;             // 128 rows of each operand
constexpr int kSlots = 5;
constexpr int kChunk = 2;                         // slots of k (128 entries) between two additions in registers, two pieces
constexpr int kEpiWarps = 8;
constexpr int kEpiBytes = 8 * 1024;               // per epilogue warp: 32 x 64 entries of either piece
constexpr int kThreads = 64 + 32 * kEpiWarps;     // one warp loads, one issues the products
constexpr int kSmemBytes = 1024 + kSlots * kSlotBytes + kEpiWarps * kEpiBytes + 256;
constexpr int kBand = 8;                          // tile rows that are worked on side by side, for reuse in L2

enum Kind : int { kGram = 0, kPoly = 1, kUpdate = 2, kFinal = 3 };

struct ProductArgs {
  CUtensorMap a, b, add, out, mirror;
  Store store;
  uint32_t* hdr;
  int m, n, k, batch;
  int tiles_m, tiles_n;
  int kind;
  int add_pieces, out_pieces;                     // 16-bit pieces of the matrix that is added, and of the result
  float c_add, c_acc;                             // result = c_add * add + c_acc * sum
};

struct Shared {                                   // behind the slots and the epilogue's buffers
  uint64_t full[kSlots], empty[kSlots], sum_full[2], sum_empty[2], add_full[kEpiWarps];
  uint32_t tmem;
};

__device__ __forceinline__ void tile_at(const ProductArgs& P, int t, bool symmetric, int* b, int* tm, int* tn) {
  if (symmetric) {
    const int per = P.tiles_m * (P.tiles_m + 1) / 2;
    *b = t / per;
    const int r = t - *b * per;
    int i = (int)((sqrtf(8.f * (float)r + 1.f) - 1.f) * 0.5f);
    while (i * (i + 1) / 2 > r) --i;
    while ((i + 1) * (i + 2) / 2 <= r) ++i;
    *tm = i;
    *tn = r - i * (i + 1) / 2;
  } else {
    const int per = P.tiles_m * P.tiles_n;
    *b = t / per;
    const int r = t - *b * per, band = r / (kBand * P.tiles_n), in = r - band * kBand * P.tiles_n;
    const int high = min(kBand, P.tiles_m - band * kBand);
    *tm = band * kBand + in % high;
    *tn = in / high;
  }
}

template <typename T>
__device__ __forceinline__ T stored(const Store& s, T old, float v) {
  return from_f32<T>(s.update ? __fmaf_rn(-s.rate, v, __fmul_rn(s.keep, to_f32(old))) : v);
}

// 32 rows x 64 columns of the caller's matrix from the warp's buffer (row r: 256 bytes, 16-byte pieces exchanged by r & 7)
template <typename T>
__device__ __forceinline__ void store_rows(const Store& s, const float* buf, int b, int i0, int j0, int m, int n) {
  T* base = reinterpret_cast<T*>(s.to.p) + (size_t)b * s.to.batch;
  const int lane = lane_id();
  if (s.wide) {
#pragma unroll 4
    for (int it = 0; it < 16; ++it) {
      const int r = it * 2 + lane / 16, q = lane % 16, j = j0 + q * 4;
      if (i0 + r >= m || j >= n) continue;
      const float4 v = *reinterpret_cast<const float4*>(buf + r * 64 + ((q ^ (r & 7)) << 2));
      T* p = base + (size_t)(i0 + r) * s.to.row + j;
      struct alignas(4 * sizeof(T)) Four { T v[4]; };
      if (j + 4 <= n) {
        Four o = {};
        if (s.update) o = *reinterpret_cast<const Four*>(p);
        o = {stored(s, o.v[0], v.x), stored(s, o.v[1], v.y), stored(s, o.v[2], v.z), stored(s, o.v[3], v.w)};
        *reinterpret_cast<Four*>(p) = o;
      } else {
        const float w[4] = {v.x, v.y, v.z, v.w};
        for (int e = 0; j + e < n; ++e) p[e] = stored(s, s.update ? p[e] : T(), w[e]);
      }
    }
  } else {
    for (int r = 0; r < 32 && i0 + r < m; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = h * 32 + lane;
        if (j0 + c >= n) continue;
        T* p = base + (size_t)(i0 + r) * s.to.row + j0 + c;
        *p = stored(s, s.update ? *p : T(), buf[r * 64 + (((c >> 2) ^ (r & 7)) << 2) + (c & 3)]);
      }
  }
}

template <typename T, int kN>
__device__ __forceinline__ void store_columns(const Store& s, const float* v, int b, int i, int j0, int m, int n) {
  T* base = reinterpret_cast<T*>(s.to.p) + (size_t)b * s.to.batch + i;
  if (i >= m) return;
#pragma unroll
  for (int e = 0; e < kN; ++e)
    if (j0 + e < n) {
      T* p = base + (size_t)(j0 + e) * s.to.row;
      *p = stored(s, s.update ? *p : T(), v[e]);
    }
}

template <int kCta, bool kSplit, bool kMn>
__global__ void __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ ProductArgs P) {
  extern __shared__ char smem_raw[];
  constexpr int kTile = 128 * kCta;               // rows and columns of a tile
  constexpr int kCols = kTile / 2;                // columns of one epilogue warp
  constexpr int kTmemCols = 2 * kTile;
  constexpr int kPieces = kSplit ? 2 : 1;
  const uint32_t raw = smem_addr(smem_raw);
  const uint32_t base = (raw + 1023) & ~1023u;
  char* base_ptr = smem_raw + (base - raw);
  Shared* sh = reinterpret_cast<Shared*>(base_ptr + kSlots * kSlotBytes + kEpiWarps * kEpiBytes);
  const int warp = threadIdx.x >> 5;
  const uint32_t rank = kCta == 2 ? cluster_rank() : 0;
  const bool symmetric = P.kind <= kPoly;
  const int tiles = P.batch * (symmetric ? P.tiles_m * (P.tiles_m + 1) / 2 : P.tiles_m * P.tiles_n);
  const int first = blockIdx.x / kCta, stride = gridDim.x / kCta;
  const int blocks_k = (P.k + kBlockK - 1) / kBlockK;

  if (warp == 0) {
    if (lane_id() == 0) {
      for (int s = 0; s < kSlots; ++s) {
        mbar_init(smem_addr(&sh->full[s]), 1);
        mbar_init(smem_addr(&sh->empty[s]), 1);
      }
      for (int s = 0; s < 2; ++s) {
        mbar_init(smem_addr(&sh->sum_full[s]), 1);
        mbar_init(smem_addr(&sh->sum_empty[s]), kCta * kEpiWarps);
      }
      for (int w = 0; w < kEpiWarps; ++w) mbar_init(smem_addr(&sh->add_full[w]), 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    tmem_alloc<kCta>(smem_addr(&sh->tmem), kTmemCols);
    tcgen05_fence_before();
  }
  __syncthreads();
  if (kCta == 2) cluster_sync();
  tcgen05_fence_after();
  const uint32_t tmem = sh->tmem;
  grid_dependency_wait();
  launch_dependents();

  bool ok = true;
  if (warp == 0) {
    if (lane_id() == 0) {                                   // ---- loads
      int slot = 0;
      uint32_t phase = 0;
      for (int t = first; t < tiles && ok; t += stride) {
        int b, tm, tn;
        tile_at(P, t, symmetric, &b, &tm, &tn);
        const int row_a = tm * kTile + (int)rank * 128, row_b = tn * kTile + (int)rank * 128;
        for (int kb = 0; kb < blocks_k && ok; ++kb)
          for (int piece = 0; piece < kPieces; ++piece) {
            if (!mbar_wait(smem_addr(&sh->empty[slot]), phase ^ 1)) { ok = false; break; }
            uint32_t bar = smem_addr(&sh->full[slot]);
            if (rank == 0) mbar_expect_tx(bar, kCta * kSlotBytes);
            if (kCta == 2) bar = cluster_addr(bar, 0);
            const uint32_t dst = base + slot * kSlotBytes;
            const int k0 = kb * kBlockK, z = 2 * b + piece;
            for (int h = 0; h < 2; ++h) tma_load<kCta>(dst + h * 8192, &P.a, k0, row_a + h * 64, z, bar);
            for (int h = 0; h < 2; ++h)
              if (kMn) tma_load<kCta>(dst + 16384 + h * 8192, &P.b, row_b + h * 64, k0, z, bar);
              else tma_load<kCta>(dst + 16384 + h * 8192, &P.b, k0, row_b + h * 64, z, bar);
            if (++slot == kSlots) { slot = 0; phase ^= 1; }
          }
      }
    }
  } else if (warp == 1) {
    if (lane_id() == 0 && rank == 0) {                      // ---- products
      constexpr uint32_t idesc = product_desc(kTile, kTile, kMn);
      int slot = 0;
      uint32_t phase = 0, sum = 0, sum_phase = 0;
      auto step = [&](uint32_t d, int sa, int sb, bool add) {
        const uint32_t a = base + sa * kSlotBytes, bb = base + sb * kSlotBytes + 16384;
        for (int k = 0; k < kBlockK / 16; ++k)
          mma_f16<kCta>(d, operand_desc(a + k * 32), kMn ? operand_desc(bb + k * 2048, 8192) : operand_desc(bb + k * 32), idesc, add || k > 0);
      };
      for (int t = first; t < tiles && ok; t += stride) {
        for (int kb = 0; kb < blocks_k && ok; ++kb) {
          const bool fresh = kSplit ? kb % kChunk == 0 : kb == 0;
          const bool last = kb + 1 == blocks_k || (kSplit && (kb + 1) % kChunk == 0);
          if (fresh && !mbar_wait(smem_addr(&sh->sum_empty[sum]), sum_phase ^ 1)) { ok = false; break; }
          const uint32_t d = tmem + sum * kTile;
          const int s0 = slot;
          const uint32_t p0 = phase;
          if (!mbar_wait(smem_addr(&sh->full[s0]), p0)) { ok = false; break; }
          tcgen05_fence_after();
          step(d, s0, s0, !fresh);
          if (++slot == kSlots) { slot = 0; phase ^= 1; }
          if (kSplit) {
            const int s1 = slot;
            if (!mbar_wait(smem_addr(&sh->full[s1]), phase)) { ok = false; break; }
            tcgen05_fence_after();
            step(d, s0, s1, true);
            step(d, s1, s0, true);
            mma_commit<kCta>(smem_addr(&sh->empty[s0]));
            mma_commit<kCta>(smem_addr(&sh->empty[s1]));
            if (++slot == kSlots) { slot = 0; phase ^= 1; }
          } else {
            mma_commit<kCta>(smem_addr(&sh->empty[s0]));
          }
          if (last) {
            mma_commit<kCta>(smem_addr(&sh->sum_full[sum]));
            sum ^= 1;
            if (sum == 0) sum_phase ^= 1;
          }
        }
      }
    }
  } else {                                                  // ---- epilogue
    const int w = warp - 2, quad = warp & 3, half = w >> 2, lane = lane_id();
    char* buf = base_ptr + kSlots * kSlotBytes + w * kEpiBytes;
    const uint32_t buf_addr = smem_addr(buf), add_bar = smem_addr(&sh->add_full[w]);
    const uint32_t empty_bar[2] = {cluster_addr(smem_addr(&sh->sum_empty[0]), 0), cluster_addr(smem_addr(&sh->sum_empty[1]), 0)};
    const bool has_add = P.kind != kGram;
    uint32_t sum = 0, sum_phase = 0, add_phase = 0;
    const int chunks = kSplit ? (blocks_k + kChunk - 1) / kChunk : 1;
    auto load_add = [&](int b, int i0, int j0) {            // one lane, once the buffer is free
      tma_store_wait_read();
      mbar_expect_tx(add_bar, P.add_pieces * 4096);
      for (int piece = 0; piece < P.add_pieces; ++piece) tma_load<1>(buf_addr + piece * 4096, &P.add, j0, i0, 2 * b + piece, add_bar);
    };
    for (int t = first; t < tiles && ok; t += stride) {
      int b, tm, tn;
      tile_at(P, t, symmetric, &b, &tm, &tn);
      const int i0 = tm * kTile + (int)rank * 128 + quad * 32, jt = tn * kTile + half * kCols;
      const bool here = i0 < P.m && jt < P.n;
      if (has_add && here && lane == 0) load_add(b, i0, jt);
      float acc[kCols];
      for (int c = 0; c < chunks; ++c) {
        if (!__all_sync(0xffffffffu, mbar_wait(smem_addr(&sh->sum_full[sum]), sum_phase))) { ok = false; break; }
        tcgen05_fence_after();
        const uint32_t at = tmem + ((uint32_t)(quad * 32) << 16) + sum * kTile + half * kCols;
        if (c == 0) {
#pragma unroll
          for (int x = 0; x < kCols; x += 32) tmem_load32(at + x, acc + x);
          tmem_load_wait();
        } else {
#pragma unroll
          for (int x = 0; x < kCols; x += 32) {
            float part[32];
            tmem_load32(at + x, part);
            tmem_load_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) acc[x + e] += part[e];
          }
        }
        tcgen05_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(empty_bar[sum]);
        sum ^= 1;
        if (sum == 0) sum_phase ^= 1;
      }
      if (!ok) break;
      if (!here) continue;
#pragma unroll
      for (int c = 0; c < kCols / 64; ++c) {
        const int j0 = jt + c * 64;
        if (j0 >= P.n) break;
        float* v = acc + c * 64;
        if (has_add) {
          if (c > 0 && lane == 0) load_add(b, i0, j0);
          if (!__all_sync(0xffffffffu, mbar_wait(add_bar, add_phase))) { ok = false; break; }
          add_phase ^= 1;
        } else {
          if (lane == 0) tma_store_wait_read();
          __syncwarp();
        }
        // row `lane` of the buffer: 16-byte pieces exchanged by lane & 7, as TMA lays them
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int off = lane * 128 + ((q ^ (lane & 7)) << 4);
          float add[8] = {};
          if (has_add) {
            const uint4 h4 = *reinterpret_cast<const uint4*>(buf + off);
            const __half2* h = reinterpret_cast<const __half2*>(&h4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = __half22float2(h[e]);
              add[2 * e] = f.x; add[2 * e + 1] = f.y;
            }
            if (P.add_pieces == 2) {
              const uint4 l4 = *reinterpret_cast<const uint4*>(buf + 4096 + off);
              const __half2* l = reinterpret_cast<const __half2*>(&l4);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 f = __half22float2(l[e]);
                add[2 * e] += f.x; add[2 * e + 1] += f.y;
              }
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) v[q * 8 + e] = __fmaf_rn(P.c_add, add[e], __fmul_rn(P.c_acc, v[q * 8 + e]));
          if (P.kind != kFinal) {
            __align__(16) __half hi[8], lo[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) split_half(v[q * 8 + e], &hi[e], &lo[e]);
            *reinterpret_cast<uint4*>(buf + off) = *reinterpret_cast<uint4*>(hi);
            if (P.out_pieces == 2) *reinterpret_cast<uint4*>(buf + 4096 + off) = *reinterpret_cast<uint4*>(lo);
          }
        }
        if (P.kind != kFinal) {
          fence_async_smem();
          __syncwarp();
          if (lane == 0) {
            tma_store(&P.out, j0, i0, 2 * b, buf_addr);
            if (P.out_pieces == 2) tma_store(&P.out, j0, i0, 2 * b + 1, buf_addr + 4096);
            tma_store_commit();
          }
          if (symmetric && tm != tn) {                      // the mirror image: row j0 + e, columns i0 ..
            if (lane == 0) tma_store_wait_read();
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 64; ++e) {
              __half hi, lo;
              split_half(v[e], &hi, &lo);
              *reinterpret_cast<__half*>(buf + e * 64 + lane * 2) = hi;
              if (P.out_pieces == 2) *reinterpret_cast<__half*>(buf + 4096 + e * 64 + lane * 2) = lo;
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
              tma_store(&P.mirror, i0, j0, 2 * b, buf_addr);
              if (P.out_pieces == 2) tma_store(&P.mirror, i0, j0, 2 * b + 1, buf_addr + 4096);
              tma_store_commit();
            }
          }
        } else if (P.store.transpose) {
          if (P.store.dtype == S3GD_F32) store_columns<float, 64>(P.store, v, b, i0 + lane, j0, P.m, P.n);
          else store_columns<__nv_bfloat16, 64>(P.store, v, b, i0 + lane, j0, P.m, P.n);
          fence_async_smem();
          __syncwarp();
        } else {
          __syncwarp();
          float* f = reinterpret_cast<float*>(buf);
#pragma unroll
          for (int q = 0; q < 16; ++q)
            *reinterpret_cast<float4*>(f + lane * 64 + ((q ^ (lane & 7)) << 2)) = make_float4(v[q * 4], v[q * 4 + 1], v[q * 4 + 2], v[q * 4 + 3]);
          __syncwarp();
          if (P.store.dtype == S3GD_F32) store_rows<float>(P.store, f, b, i0, j0, P.m, P.n);
          else store_rows<__nv_bfloat16>(P.store, f, b, i0, j0, P.m, P.n);
          fence_async_smem();
          __syncwarp();
        }
      }
    }
    if (lane == 0) tma_store_wait();
  }
  if (!ok) {                                                // a wait gave up: say so, let copies in flight land
    atomicOr(&P.hdr[kHdrStatus], (uint32_t)kFlagInternal);
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
  }
  __syncwarp();
  tcgen05_fence_before();
  __syncthreads();
  if (kCta == 2) cluster_sync();
  tcgen05_fence_after();
  if (warp == 0) tmem_free<kCta>(tmem, kTmemCols);
}

// ------------------------------------------------------------------ host
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
  static std::atomic<EncodeFn> cached{nullptr};
  EncodeFn f = cached.load(std::memory_order_acquire);
  if (f == nullptr) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
      return nullptr;
    f = reinterpret_cast<EncodeFn>(p);
    cached.store(f, std::memory_order_release);
  }
  return f;
}

// A 16-bit matrix of the workspace: box_x columns by box_y rows; swizzled where the columns fill 128 bytes.
bool make_map(CUtensorMap* map, void* p, int rows, int cols, int ld, int planes, int box_x, int box_y) {
  EncodeFn f = encode_fn();
  if (f == nullptr) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)rows * ld * 2};
  const cuuint32_t box[3] = {(cuuint32_t)box_x, (cuuint32_t)box_y, 1}, ones[3] = {1, 1, 1};
  return f(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, p, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
           box_x == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kCta, bool kSplit, bool kMn>
cudaError_t launch_product(ProductArgs& A, cudaStream_t st) {
  static int done[kMaxDevices];
  auto kernel = product_kernel<kCta, kSplit, kMn>;
  cudaError_t e = opt_in_dynamic_smem(reinterpret_cast<const void*>(kernel), kSmemBytes, done);
  if (e != cudaSuccess) return e;
  const int tile = 128 * kCta;
  A.tiles_m = (A.m + tile - 1) / tile;
  A.tiles_n = (A.n + tile - 1) / tile;
  const int64_t tiles = (int64_t)A.batch * (A.kind <= kPoly ? (int64_t)A.tiles_m * (A.tiles_m + 1) / 2 : (int64_t)A.tiles_m * A.tiles_n);
  const int64_t groups = sm_count() / kCta;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((tiles < groups ? tiles : groups) * kCta));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kCta; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = kCta == 2 ? 2 : 1;
  count_launch();
  return cudaLaunchKernelEx(&cfg, kernel, A);
}

template <bool kMn>
cudaError_t launch_by(ProductArgs& A, bool pair, bool split, cudaStream_t st) {
  if (pair) return split ? launch_product<2, true, kMn>(A, st) : launch_product<2, false, kMn>(A, st);
  return split ? launch_product<1, true, kMn>(A, st) : launch_product<1, false, kMn>(A, st);
}

}  // namespace

cudaError_t launch_products(const OrthoPlan& P, const OrthoRequest& R, char* ws, cudaStream_t st) {
  const int m = P.m, n = P.n, planes = 2 * P.batch;
  char* xs[2] = {ws + P.off_x, ws + P.off_y};
  CUtensorMap x_load[2], x_epi[2], s_load, s_epi, s_mirror, b_load, b_epi, b_mirror;
  bool ok = true;
  for (int i = 0; i < 2; ++i)
    ok = ok && make_map(&x_load[i], xs[i], m, n, P.ldx, planes, 64, 64) && make_map(&x_epi[i], xs[i], m, n, P.ldx, planes, 64, 32);
  ok = ok && make_map(&s_load, ws + P.off_s, m, m, P.lds, planes, 64, 64) && make_map(&s_epi, ws + P.off_s, m, m, P.lds, planes, 64, 32) &&
       make_map(&s_mirror, ws + P.off_s, m, m, P.lds, planes, 32, 64) && make_map(&b_load, ws + P.off_b, m, m, P.lds, planes, 64, 64) &&
       make_map(&b_epi, ws + P.off_b, m, m, P.lds, planes, 64, 32) && make_map(&b_mirror, ws + P.off_b, m, m, P.lds, planes, 32, 64);
  if (!ok) return cudaErrorInvalidValue;
  const bool pair = (int64_t)P.batch * ((m + 255) / 256) * ((n + 255) / 256) >= sm_count() / 2;
  const int carried = carried_steps(R.steps, R.split);
  for (int k = 0; k < R.steps; ++k) {
    const bool split = k < R.split;
    const int from = k & 1;
    ProductArgs A;
    A.hdr = reinterpret_cast<uint32_t*>(ws + P.off_hdr);
    A.batch = P.batch;
    A.store = R.out;
    A.add_pieces = A.out_pieces = split ? 2 : 1;
    A.kind = kGram; A.m = m; A.n = m; A.k = n;
    A.a = A.b = x_load[from]; A.add = s_epi; A.out = s_epi; A.mirror = s_mirror;
    A.c_add = 0.f; A.c_acc = kScaleS / (kScaleX * kScaleX);
    cudaError_t e = launch_by<false>(A, pair, split, st);
    if (e != cudaSuccess) return e;
    A.kind = kPoly; A.k = m;
    A.a = A.b = s_load; A.add = s_epi; A.out = b_epi; A.mirror = b_mirror;
    A.c_add = R.b * (kScaleB / kScaleS); A.c_acc = R.c * (kScaleB / (kScaleS * kScaleS));
    e = launch_by<false>(A, pair, split, st);
    if (e != cudaSuccess) return e;
    const bool last = k + 1 == R.steps;
    const float unit = last ? 1.f / kScaleX : 1.f;
    A.kind = last ? kFinal : kUpdate; A.n = n; A.k = m;
    A.a = b_load; A.b = x_load[from]; A.add = x_epi[from]; A.out = x_epi[from ^ 1];
    A.add_pieces = k < carried ? 2 : 1;
    A.out_pieces = k + 1 < carried ? 2 : 1;
    A.c_add = R.a * unit; A.c_acc = unit / kScaleB;
    e = launch_by<true>(A, pair, split, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace s3gd
