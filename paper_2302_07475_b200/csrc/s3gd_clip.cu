// The norm of each worker's gradients over many tensors, and clipping by it (see include/s3gd.h).
//
//     norm[m] = sqrt(sum over tensors i and entries j of g_i[m][j]^2),   c[m] = min(1, max_norm / (norm[m] + eps)),
//     out_i[m][j] = c[m] g_i[m][j].
//
// The tensors' addresses and sizes travel as the kernels' arguments (no copy to the device, nothing that a captured graph would
// have to keep alive), in groups where there are very many.  Each worker's tensors are cut into tiles of 8192 entries that begin on
// 16-byte boundaries; a CTA sums a run of tiles and writes one partial sum.  Whoever needs the norm adds the worker's partial sums in
// a fixed order: no atomics, and the result depends on sizes and alignment alone.
//
// Bound by memory: squares are read at 5.5 (bf16) to 6.5 TB/s, scaled at 6.2 to 6.6 TB/s of reads and writes together.  Clipping reads
// everything twice; the second time a part comes from the L2, where workers and tiles are taken last first.
//     norm of 53 bf16 tensors, 95.6e6 entries     35 us (floor 29), 41 from Python: the host's look at the list
//     the same clipped into an fp32 row          129 us (floor 87; 116 with the second read)
//     62 fp32 tensors of 100 workers, 1.12e9     2.06 ms (floor 1.36; 2.04 with the second read)
//     13 fp32 tensors, 28,000 entries              8 us, 21.5 from Python
// Both passes over many workers in one kernel, by tickets, were tried: a worker's entries then come from the L2 the second time, but
// its CTAs keep less on its way (registers of both passes) and take as long.
#include "s3gd_ops.cuh"
#include "s3gd_tcgen05.cuh"

namespace s3gd {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr uint32_t kTile = 8192;                   // entries of a tile
constexpr int kFewParts = 64, kMostParts = 640;    // tensors of one launch: kernel arguments of up to 32 KB
// Partial sums over all workers, and of each worker, at least; 512 where that makes no more than 2^21 of them.  (More of them let the last
// CTAs end together: 100 x ResNet-18 2.17 ms with 128 a worker, 2.09 with 256, 2.04 with 512.)
constexpr uint32_t kRunsAll = 2368, kRunsEach = 32, kRunsMost = 512, kRunsTotal = 1u << 21;

struct Part {
  const void* src;
  void* dst;
  uint64_t n;
  long long src_worker, dst_worker;
  uint32_t first_tile;
  uint32_t in_place;
};
struct ClipArgs {
  double* partial;     // [M x runs]
  float* norm;
  uint32_t* hdr;
  uint32_t count, tiles, per, runs, add;
  float max_norm, eps;
};
template <int kMax> struct Parts { Part p[kMax]; };

template <int kMax>
__device__ __forceinline__ uint32_t part_of(const Parts<kMax>& parts, uint32_t count, uint32_t tile) {
  uint32_t lo = 0, hi = count;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (parts.p[mid].first_tile <= tile) lo = mid; else hi = mid;
  }
  return lo;
}

// entries of a 16-byte access, and how many entries the address lies behind such a boundary
template <typename T> constexpr int kWide = 16 / (int)sizeof(T);

// What is scaled is read for the last time: wide loads tell the L2 so (67 MB into another buffer and a sum over that: 55 us, without
// the hint 59; the outputs stay).
__device__ __forceinline__ uint64_t drop_policy() {
  uint64_t p;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
template <typename P>
__device__ __forceinline__ P load_last(const void* from, uint64_t policy) {
  P v;
  uint32_t* w = reinterpret_cast<uint32_t*>(&v);
  if constexpr (sizeof(P) == 16)
    asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0,%1,%2,%3}, [%4], %5;" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(from), "l"(policy) : "memory");
  else if constexpr (sizeof(P) == 8)
    asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v2.u32 {%0,%1}, [%2], %3;" : "=r"(w[0]), "=r"(w[1]) : "l"(from), "l"(policy) : "memory");
  else
    v = *static_cast<const P*>(from);
  return v;
}
template <typename T>
__device__ __forceinline__ uint32_t behind(const T* p, int v) { return (uint32_t)(reinterpret_cast<uintptr_t>(p) / sizeof(T)) % v; }

// Squares of up to eight neighbours are added in 32 bits (off by 8 half steps of their sum at most), everything else in 64: one
// conversion for eight entries (where the conversions would otherwise take as long as the reads).  Sums that may have lost small
// squares, or overflowed, are taken again in 64 bits.
constexpr float kLeast = 8.2718061e-25f, kMost = 8.5070592e37f;                  // 2^-80, 2^126
template <int kN>
__device__ __forceinline__ double squares(const float* v) {
  float s = v[0] * v[0];
#pragma unroll
  for (int e = 1; e < kN; ++e) s = fmaf(v[e], v[e], s);
  if (s >= kLeast && s <= kMost) return s;
  double sum = 0;
#pragma unroll
  for (int e = 0; e < kN; ++e) sum += (double)v[e] * v[e];
  return sum;
}
// Entries of a tile that wide accesses miss, at the ends of a tensor: fewer than kVec before the first one and behind the last.
// f is called with the thread's entry, if it has one.
template <int kVec, typename F>
__device__ __forceinline__ void ragged_entries(long long begin, uint64_t n, F f) {
  const int t = (int)threadIdx.x;
  if (t >= 2 * kVec) return;
  if (t < kVec) {
    const long long at = begin + t;                // the first access begins before the tensor
    if (begin < 0 && at >= 0 && (uint64_t)at < n) f(at);
  } else {
    const long long last = (long long)n - (((long long)n - begin) & (kVec - 1)), at = last + t - kVec;
    if (last >= 0 && last >= begin && last < begin + (long long)kTile && (uint64_t)at < n) f(at);
  }
}
template <typename T>
__device__ __forceinline__ double tile_squares(const T* g, uint64_t n, uint32_t tile) {
  constexpr int kVec = kWide<T>, kLoads = kTile / (kThreads * kVec), kPacks = 8 / kVec;
  const long long begin = (long long)tile * kTile - behind(g, kVec), at = begin + threadIdx.x * kVec;
  const bool whole = begin >= 0 && (uint64_t)begin + kTile <= n;
  Pack<T, kVec> raw[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const long long c = at + i * kThreads * kVec;
    raw[i] = {};
    if (whole || (c >= 0 && (uint64_t)c + kVec <= n)) raw[i] = *reinterpret_cast<const Pack<T, kVec>*>(g + c);
  }
  double sum = 0;
#pragma unroll
  for (int i = 0; i < kLoads / kPacks; ++i) {
    float v[8];
#pragma unroll
    for (int e = 0; e < kPacks; ++e) load_floats<T, kVec>(raw[i * kPacks + e].v, v + e * kVec);
    sum += squares<8>(v);
  }
  if (!whole) ragged_entries<kVec>(begin, n, [&](long long c) { const double d = to_f32(g[c]); sum += d * d; });
  return sum;
}

// the CTA's sum, in every thread
__device__ __forceinline__ double cta_sum(double v) {
  __shared__ double room[kWarps];
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if (lane_id() == 0) room[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < kWarps; ++w) v += room[w];
  return v;
}
__device__ __forceinline__ double norm_of(const ClipArgs& a, uint32_t m) {
  double sum = 0;
  for (uint32_t i = threadIdx.x; i < a.runs; i += kThreads) sum += a.partial[(size_t)m * a.runs + i];
  return sqrt(cta_sum(sum));
}

// The factor, rounded to 32 bits.  One below their normal range (entries near fp32's end) would lose digits there, although what it makes
// of such entries may not: it is held times 2^126, and its products are taken back by that, exactly where they are normal.
struct Factor { float c; bool small; };
__device__ __forceinline__ Factor factor_of(const ClipArgs& a, double norm) {
  const double held = norm + (double)a.eps;
  if (held <= (double)a.max_norm) return {1.f, false};
  const double c = (double)a.max_norm / held;                                     // NaN stays NaN
  return c > 0 && c < 0x1p-126 ? Factor{(float)(c * 0x1p126), true} : Factor{(float)c, false};
}
// the CTA's sum of squares over a run of tiles of worker m, in every thread
template <typename S, int kMax>
__device__ __forceinline__ double run_squares(const Parts<kMax>& parts, const ClipArgs& a, uint32_t m, uint32_t run) {
  const uint32_t begin = run * a.per, end = min(begin + a.per, a.tiles);
  double sum = 0;
  uint32_t k = begin < end ? part_of(parts, a.count, begin) : 0;
  for (uint32_t tile = begin; tile < end; ++tile) {
    while (k + 1 < a.count && parts.p[k + 1].first_tile <= tile) ++k;
    const Part& p = parts.p[k];
    const uint32_t in = tile - p.first_tile;
    sum += tile_squares(static_cast<const S*>(p.src) + m * p.src_worker, p.n, in);
  }
  return cta_sum(sum);
}

// blockIdx.x: run of tiles, blockIdx.y: worker
template <typename S, int kMax>
__global__ void __launch_bounds__(kThreads) squares_kernel(const __grid_constant__ Parts<kMax> parts, const ClipArgs a) {
  grid_dependency_wait();
  const double sum = run_squares<S>(parts, a, blockIdx.y, blockIdx.x);
  double* to = a.partial + (size_t)blockIdx.y * a.runs + blockIdx.x;
  if (threadIdx.x == 0) *to = a.add ? *to + sum : sum;
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const ClipArgs a) {
  grid_dependency_wait();
  const double norm = norm_of(a, blockIdx.x);
  if (threadIdx.x == 0) a.norm[blockIdx.x] = (float)norm;
  if (blockIdx.x == 0 && threadIdx.x < 8) a.hdr[threadIdx.x] = 0;
}

// kBatch accesses of a tile, one behind the other; kWhole: all of them lie in the tensor
template <typename S, typename D, int kVec, int kBatch, bool kWhole>
__device__ __forceinline__ void scaled(const S* g, D* out, long long at, long long n, float c, uint64_t policy) {
  Pack<S, kVec> raw[kBatch];
#pragma unroll
  for (int i = 0; i < kBatch; ++i) {
    const long long j = at + i * kThreads * kVec;
    if (kWhole || (j >= 0 && j + kVec <= n)) raw[i] = load_last<Pack<S, kVec>>(g + j, policy);
  }
#pragma unroll
  for (int i = 0; i < kBatch; ++i) {
    const long long j = at + i * kThreads * kVec;
    if (!kWhole && (j < 0 || j + kVec > n)) continue;
    float v[kVec];
    load_floats<S, kVec>(raw[i].v, v);
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = __fmul_rn(v[e], c);
    Pack<D, kVec> o;
    store_floats<D, kVec>(o.v, v);
    *reinterpret_cast<Pack<D, kVec>*>(out + j) = o;
  }
}
template <typename S, typename D, int kVec>
__device__ __forceinline__ void tile_scaled(const S* g, D* out, uint64_t n, uint32_t tile, float c) {
  constexpr int kLoads = kTile / (kThreads * kVec), kSpan = kThreads * kVec;
  const long long begin = (long long)tile * kTile - behind(g, kVec), at = begin + threadIdx.x * kVec, end = (long long)n;
  const uint64_t policy = drop_policy();
  if (begin >= 0 && begin + (long long)kTile <= end) {
#pragma unroll 1
    for (int b = 0; b < kLoads; b += 8) scaled<S, D, kVec, 8, true>(g, out, at + b * kSpan, end, c, policy);
    return;
  }
#pragma unroll 1
  for (int b = 0; b < kLoads && begin + b * kSpan < end; b += 4) scaled<S, D, kVec, 4, false>(g, out, at + b * kSpan, end, c, policy);
  ragged_entries<kVec>(begin, n, [&](long long j) { out[j] = from_f32<D>(__fmul_rn(to_f32(g[j]), c)); });
}
// by a small factor: rare, an entry at a time
template <typename S, typename D>
__device__ __forceinline__ void tile_scaled_small(const S* g, D* out, uint64_t n, uint32_t tile, float c) {
  const uint64_t begin = (uint64_t)tile * kTile, end = begin + kTile < n ? begin + kTile : n;
#pragma unroll 1
  for (uint64_t j = begin + threadIdx.x; j < end; j += kThreads) out[j] = from_f32<D>(__fmul_rn(__fmul_rn(to_f32(g[j]), c), 0x1p-126f));
}
template <typename S, typename D>
__device__ __forceinline__ void tile_clipped(const Part& p, uint32_t m, uint32_t tile, Factor f) {
  const S* g = static_cast<const S*>(p.src) + m * p.src_worker;
  D* out = static_cast<D*>(p.dst) + m * p.dst_worker;
  const float c = f.c;
  if (f.small) { tile_scaled_small<S, D>(g, out, p.n, tile, c); return; }
  // four entries at a time where both sides lie alike, two or one where they do not
  if (behind(g, 4) == behind(out, 4)) tile_scaled<S, D, 4>(g, out, p.n, tile, c);
  else if (behind(g, 2) == behind(out, 2)) tile_scaled<S, D, 2>(g, out, p.n, tile, c);
  else tile_scaled<S, D, 1>(g, out, p.n, tile, c);
}

template <typename S, typename D, int kMax>
__device__ __forceinline__ void run_scaled(const Parts<kMax>& parts, const ClipArgs& a, uint32_t m, uint32_t run, Factor f) {
  const uint32_t begin = run * a.per, end = min(begin + a.per, a.tiles);
  uint32_t k = begin < end ? part_of(parts, a.count, begin) : 0;
  for (uint32_t tile = begin; tile < end; ++tile) {
    while (k + 1 < a.count && parts.p[k + 1].first_tile <= tile) ++k;
    const Part& p = parts.p[k];
    if (f.c == 1.f && !f.small && p.in_place) continue;
    const uint32_t in = tile - p.first_tile;
    tile_clipped<S, D>(p, m, in, f);
  }
}

template <typename S, typename D, int kMax>
__global__ void __launch_bounds__(kThreads, 4) scale_kernel(const __grid_constant__ Parts<kMax> parts, const ClipArgs a, uint32_t runs) {
  grid_dependency_wait();
  const uint32_t m = gridDim.y - 1 - blockIdx.y, run = runs - 1 - blockIdx.x;      // what was read last is in the L2
  const double norm = norm_of(a, m);
  if (run == 0 && threadIdx.x == 0) a.norm[m] = (float)norm;
  if (run == 0 && m == 0 && threadIdx.x < 8) a.hdr[threadIdx.x] = 0;
  run_scaled<S, D>(parts, a, m, run, factor_of(a, norm));
}

// Few tiles: a cluster of eight CTAs takes a worker's tiles, adds their squares and scales them, all in one launch.  What it saves is
// the host's second launch: 13 tensors of 14 tiles 22.5 us a call instead of 25.1, although the kernel takes 8.2 us and two of them,
// one behind the other in a captured graph, 6.4 (one tile a CTA: 2.9 and 3.3 us; 24 tiles: 6.5 and 4.7).
constexpr int kCluster = 8;
constexpr int kClusterWorkers = 8;
constexpr uint64_t kClusterTiles = 16;
template <typename S, typename D, int kMax>
__global__ void __launch_bounds__(kThreads) small_kernel(const __grid_constant__ Parts<kMax> parts, const ClipArgs a, bool scales) {
  grid_dependency_wait();
  const uint32_t m = blockIdx.y, rank = blockIdx.x;
  double* sums = a.partial + m * kCluster;
  const double sum = run_squares<S>(parts, a, m, rank);
  if (threadIdx.x == 0) sums[rank] = sum;
  cluster_sync();                                                    // the sums of all CTAs are there
  double total = 0;
#pragma unroll
  for (int k = 0; k < kCluster; ++k) total += __ldcg(sums + k);
  const double norm = sqrt(total);
  if (rank == 0 && threadIdx.x == 0) a.norm[m] = (float)norm;
  if (rank == 0 && m == 0 && threadIdx.x < 8) a.hdr[threadIdx.x] = 0;
  if (scales) run_scaled<S, D>(parts, a, m, rank, factor_of(a, norm));
}

// ------------------------------------------------------------------ host
uint32_t runs_each(int M) {
  const uint32_t even = (kRunsAll + M - 1) / M, share = kRunsTotal / M, some = share > kRunsMost ? kRunsMost : share < kRunsEach ? kRunsEach : share;
  return even > some ? even : some;
}
// M * runs_each(M) at most, and never less for more workers
size_t workspace_bytes(int M) {
  const uint64_t m = (uint64_t)M, some = kRunsMost * m < kRunsTotal ? kRunsMost * m : kRunsTotal;
  return 256 + align_up((kRunsAll + some + (kRunsEach + 1) * m) * sizeof(double), 256);
}

// tiles that n entries take wherever the first one lies
uint64_t tiles_of(uint64_t n) { return n == 0 ? 0 : (n + 8 - 1 + kTile - 1) / kTile; }

bool valid(const s3gd_part* parts, int count, int M, bool clip) {
  if (count < 0 || (count > 0 && parts == nullptr) || M < 1 || M > 65535) return false;
  for (int i = 0; i < count; ++i) {
    const s3gd_part& p = parts[i];
    if (!is_real(p.dtype) || (clip && !is_real(p.out_dtype)) || p.n >= (1ull << 40)) return false;
    if (p.n == 0) continue;
    if (p.data == nullptr || !is_aligned(p.data, dtype_bytes(p.dtype)) || (M > 1 && p.stride < 0)) return false;
    if (!clip) continue;
    if (p.out == nullptr || !is_aligned(p.out, dtype_bytes(p.out_dtype)) || (M > 1 && (p.out_stride < 0 || (uint64_t)p.out_stride < p.n))) return false;
    // in place: the same entries, not others of the same memory
    if (p.out == p.data && (p.dtype != p.out_dtype || (M > 1 && p.stride != p.out_stride))) return false;
  }
  return true;
}

cudaError_t launch_norm(const ClipArgs& base, uint32_t runs, int M, cudaStream_t st) {
  ClipArgs a = base;
  a.runs = runs;
  count_launch();
  return launch_after(norm_kernel, dim3(M), dim3(kThreads), 0, st, a);
}

// Runs of a worker's tiles: one for a tile where there are few.  (Several groups of tensors share the partial sums.)
uint64_t tiles_in(const s3gd_part* parts, int count) {
  uint64_t tiles = 0;
  for (int i = 0; i < count; ++i) tiles += tiles_of(parts[i].n);
  return tiles;
}
uint32_t runs_of(uint64_t tiles, uint32_t most) { return tiles < 1 ? 1 : tiles < most ? (uint32_t)tiles : most; }

// Calls f(Parts, ClipArgs of the group) for groups of at most kMax of the tensors that `takes` picks; `first`: partial sums are
// written, not added to.
template <int kMax, typename P, typename F>
cudaError_t by_group(const s3gd_part* parts, int count, int M, uint32_t runs, bool* first, ClipArgs a, P takes, F f) {
  a.runs = runs;
  for (int i = 0; i < count;) {
    Parts<kMax> group;
    a.count = 0;
    uint64_t tiles = 0;
    for (; i < count && a.count < kMax; ++i) {
      const s3gd_part& p = parts[i];
      const uint64_t more = tiles_of(p.n);
      if (more == 0 || !takes(p)) continue;
      if (tiles + more >= (1ull << 31)) break;
      Part& q = group.p[a.count++];
      q.src = p.data; q.dst = p.out; q.n = p.n; q.src_worker = M > 1 ? p.stride : 0; q.dst_worker = M > 1 ? p.out_stride : 0;
      q.first_tile = (uint32_t)tiles; q.in_place = p.out == p.data;
      tiles += more;
    }
    if (a.count == 0) break;
    a.tiles = (uint32_t)tiles;
    a.per = (uint32_t)((tiles + a.runs - 1) / a.runs);
    a.add = !*first;
    *first = false;
    const cudaError_t e = f(group, a);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

// Every tensor's type has launches of its own: a kernel for all of them together would need 254 registers.
template <int kMax>
cudaError_t enqueue_squares(const s3gd_part* parts, int count, int M, uint32_t runs, const ClipArgs& base, cudaStream_t st) {
  bool first = true;
  for (int dt : {(int)S3GD_F32, (int)S3GD_BF16}) {
    const cudaError_t e = by_real(dt, [&](auto s) {
      return by_group<kMax>(parts, count, M, runs, &first, base, [&](const s3gd_part& p) { return p.dtype == dt; }, [&](const Parts<kMax>& group, const ClipArgs& a) {
        count_launch();
        return launch_after(squares_kernel<decltype(s), kMax>, dim3(a.runs, M), dim3(kThreads), 0, st, group, a);
      });
    });
    if (e != cudaSuccess) return e;
  }
  return first ? cudaMemsetAsync(base.partial, 0, (size_t)M * runs * sizeof(double), st) : cudaSuccess;      // no entries at all
}

// Does one launch do?  (Tensors of one type each way.)
bool is_small(const s3gd_part* parts, int count, int M, bool clip) {
  if (M > kClusterWorkers || count < 1 || count > kFewParts || tiles_in(parts, count) > kClusterTiles || tiles_in(parts, count) == 0) return false;
  for (int i = 1; i < count; ++i)
    if (parts[i].dtype != parts[0].dtype || (clip && parts[i].out_dtype != parts[0].out_dtype)) return false;
  return true;
}
cudaError_t enqueue_small(const s3gd_part* parts, int count, int M, bool clip, const ClipArgs& base, cudaStream_t st) {
  bool first = true;
  return by_real(parts[0].dtype, [&](auto s) { return by_real(clip ? parts[0].out_dtype : (int)S3GD_F32, [&](auto d) {
    return by_group<kFewParts>(parts, count, M, kCluster, &first, base, [](const s3gd_part&) { return true; }, [&](const Parts<kFewParts>& group, const ClipArgs& a) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(kCluster, M); cfg.blockDim = dim3(kThreads); cfg.stream = st;
      cudaLaunchAttribute attr[2];
      attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
      attr[0].val.programmaticStreamSerializationAllowed = 1;
      attr[1].id = cudaLaunchAttributeClusterDimension;
      attr[1].val.clusterDim.x = kCluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
      cfg.attrs = attr; cfg.numAttrs = 2;
      count_launch();
      return cudaLaunchKernelEx(&cfg, small_kernel<decltype(s), decltype(d), kFewParts>, group, a, clip);
    });
  }); });
}
template <int kMax>
cudaError_t enqueue_clip(const s3gd_part* parts, int count, int M, const ClipArgs& base, cudaStream_t st) {
  if (is_small(parts, count, M, true)) return enqueue_small(parts, count, M, true, base, st);
  const uint32_t runs = runs_of(tiles_in(parts, count), runs_each(M));
  const cudaError_t e = enqueue_squares<kMax>(parts, count, M, runs, base, st);
  if (e != cudaSuccess) return e;
  bool first = true;
  for (int from : {(int)S3GD_F32, (int)S3GD_BF16})
    for (int to : {(int)S3GD_F32, (int)S3GD_BF16}) {
      const cudaError_t e = by_real(from, [&](auto s) { return by_real(to, [&](auto d) {
        return by_group<kMax>(parts, count, M, runs, &first, base, [&](const s3gd_part& p) { return p.dtype == from && p.out_dtype == to; },
                              [&](const Parts<kMax>& group, const ClipArgs& a) {
          const uint32_t busy = (a.tiles + a.per - 1) / a.per;
          count_launch();
          return launch_after(scale_kernel<decltype(s), decltype(d), kMax>, dim3(busy, M), dim3(kThreads), 0, st, group, a, busy);
        });
      }); });
      if (e != cudaSuccess) return e;
    }
  return first ? launch_norm(base, runs, M, st) : cudaSuccess;       // no entries at all: the norms are to be written all the same
}

ClipArgs clip_args(void* ws, float* norm) {
  ClipArgs a = {};
  a.hdr = static_cast<uint32_t*>(ws);
  a.partial = reinterpret_cast<double*>(static_cast<char*>(ws) + 256);
  a.norm = norm;
  return a;
}

}  // namespace
}  // namespace s3gd

using namespace s3gd;

extern "C" size_t s3gd_clip_workspace_bytes(int M) { return M < 1 || M > 65535 ? 0 : workspace_bytes(M); }

extern "C" s3gd_status s3gd_grad_norm(const s3gd_part* parts, int count, int M, float* out_norm, void* ws, size_t ws_bytes, void* stream) {
  if (!valid(parts, count, M, false) || out_norm == nullptr || !is_aligned(out_norm, 4)) return S3GD_ERR_INVALID_ARG;
  if (ws == nullptr || ws_bytes < workspace_bytes(M) || !is_aligned(ws, 256)) return S3GD_ERR_WORKSPACE;
  const ClipArgs a = clip_args(ws, out_norm);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (is_small(parts, count, M, false)) return enqueue_small(parts, count, M, false, a, st) == cudaSuccess ? S3GD_OK : S3GD_ERR_CUDA;
  const uint32_t runs = runs_of(tiles_in(parts, count), runs_each(M));
  cudaError_t e = count <= kFewParts ? enqueue_squares<kFewParts>(parts, count, M, runs, a, st) : enqueue_squares<kMostParts>(parts, count, M, runs, a, st);
  if (e == cudaSuccess) e = launch_norm(a, runs, M, st);
  return e == cudaSuccess ? S3GD_OK : S3GD_ERR_CUDA;
}

extern "C" s3gd_status s3gd_clip(const s3gd_part* parts, int count, int M, float max_norm, float eps, float* out_norm, void* ws,
                                 size_t ws_bytes, void* stream) {
  if (!valid(parts, count, M, true) || out_norm == nullptr || !is_aligned(out_norm, 4)) return S3GD_ERR_INVALID_ARG;
  if (!(max_norm >= 0.f && max_norm < INFINITY) || !(eps >= 0.f && eps < INFINITY)) return S3GD_ERR_INVALID_ARG;
  if (ws == nullptr || ws_bytes < workspace_bytes(M) || !is_aligned(ws, 256)) return S3GD_ERR_WORKSPACE;
  ClipArgs a = clip_args(ws, out_norm);
  a.max_norm = max_norm;
  a.eps = eps;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = count <= kFewParts ? enqueue_clip<kFewParts>(parts, count, M, a, st) : enqueue_clip<kMostParts>(parts, count, M, a, st);
  return e == cudaSuccess ? S3GD_OK : S3GD_ERR_CUDA;
}
