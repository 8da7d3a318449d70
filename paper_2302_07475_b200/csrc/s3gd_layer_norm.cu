// Layer norm over rows of a batch of workers, and its gradient with the workers' weight gradients (see include/s3gd.h).
//
// Forward: y = (x - mean) rstd w + b.  Backward, with xhat = (x - mean) rstd and g = dy w:
//     dx = rstd (g - mean(g) - xhat mean(g xhat)),   dw = sum over a worker's rows of dy xhat,   db = sum of dy.
// Mean and rstd are computed again from x, which the backward pass reads anyway: nothing is saved between the passes.
//
// Sums over a row.  The mean is taken first, then the sums of d = x - mean and d^2 (and of g and g d): the sum of d, which
// would be zero but for the mean's rounding, corrects both mean and variance, so that rows far from zero keep their digits.
//
// Weight gradients.  The rows of all workers, one worker after the other, are dealt to CTAs in runs of `per` rows, which may end with a
// worker's rows or go on with the next one's.  A CTA writes a partial sum for each worker that its run touches; where runs go on, run k
// and worker m meet in slot k + m (from one slot to the next in that order either k or m grows).  A last kernel adds a worker's slots in 64 bits, in ascending order: no atomics, and the
// result depends on sizes and alignment alone.
//
// Bound by memory in 32 bits, by the latency of dependent instructions in 16: 16 warps an SM hold their columns' weights and sums in
// up to 128 registers, and issue in 45 (forward) to 60 % of the cycles.  One call after the other, in a captured graph where the host
// would be slower (floor: every row read and written once at 6.57 TB/s):
//     forward   8 x 4096 x 512 fp32 -> bf16, 5 % empty    22.6 us (15)      backward  8 x 4096 x 512 fp32, 5 % empty       38 us (30)
//               65536 x 2048 bf16, residual                187 us (163)               65536 x 2048 bf16, residual         216 us (163)
//               32768 x 2048 bf16 / fp32                  63 / 105 us (41 / 82)       32768 x 2048 bf16 / fp32       102 / 147 us (61 / 123)
//               67041 x 1001 bf16 / fp32                  79 / 101 us (41 / 82)       67041 x 1001 bf16 / fp32       145 / 165 us (61 / 123)
//               1 x 1024 bf16                             4 us, 8.2 from Python       200 x 768 fp32, added to      8.2 us, 17 from Python
// Rows of more than 8192 entries (4096 x 16384 bf16: 122 us forward, 216 us backward; floors 41 and 61) are read two or three times, after
// the first from L1 or L2; what takes longer is that every entry is added in 64 bits, and one access a thread at a time.
// Where M is above 296 runs go on from worker to worker, and a CTA adds its groups' sums once for each worker it touches: 65535 workers of
// one row of 512 fp32 take 6.9 ms (floor 0.1), 20000 of three 2.1 ms, 2000 of 33 256 us (floor 63), 290 of 226 87 us (62).
#include "s3gd_ops.cuh"
#include "s3gd_tcgen05.cuh"

namespace s3gd {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr uint64_t kMaxDim = 65535ull * kThreads;   // a grid dimension of tiles with one entry a thread: 2^24 - 256
constexpr int kRuns = kDefaultSMs;                 // runs of rows at least, where there are as many rows
constexpr uint64_t kMaxRun = 4096;                 // rows of a run at most: 32-bit sums stay short

struct Rows {                                      // [M x T] rows of `dim` entries; p NULL: not given
  const void* p;
  long long tok, worker;
  long long last;                                  // entries from the first to behind the last
};
struct NormArgs {
  Rows x, add, total, y;
  const void *weight, *bias;
  bool param_bf16, ids64;
  const void* ids;
  uint32_t T, N, dim, per;
  float eps;
};
struct NormGradArgs {
  Rows dy, x, dtotal, dx;
  const void *weight, *ids;
  bool weight_bf16, ids64, grads_bf16, accumulate;
  uint32_t M, T, N, dim, pad, per, runs;
  uint32_t shares;                                 // runs of a worker, where they end with its rows; 0: they may go on with the next worker's
  bool cluster;                                    // a worker's runs are a cluster's CTAs, which join their sums themselves
  float eps;
  void *dweight, *dbias;
  long long grads_stride;
  uint32_t* hdr;
  float4* stats;
  float* partial;
};

template <typename T>
__device__ __forceinline__ T* row_of(const Rows& r, uint32_t m, uint32_t t) {
  return static_cast<T*>(const_cast<void*>(r.p)) + m * r.worker + t * r.tok;
}
__device__ __forceinline__ bool is_empty(const void* ids, bool ids64, uint32_t r) {
  if (ids == nullptr) return false;
  return ids64 ? static_cast<const long long*>(ids)[r] < 0 : static_cast<const int*>(ids)[r] < 0;
}
__device__ __forceinline__ float param_at(const void* p, bool bf16, uint32_t c, float otherwise) {
  if (p == nullptr) return otherwise;
  return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[c]) : static_cast<const float*>(p)[c];
}
// the CTA's sums of kCount values, in every thread
template <int kCount>
__device__ __forceinline__ void cta_sums(double (&v)[kCount], double (&room)[kCount][kWarps]) {
#pragma unroll
  for (int i = 0; i < kCount; ++i)
    for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  __syncthreads();
  if (lane_id() == 0)
    for (int i = 0; i < kCount; ++i) room[i][threadIdx.x >> 5] = v[i];
  __syncthreads();
  for (int i = 0; i < kCount; ++i) {
    v[i] = 0;
    for (int w = 0; w < kWarps; ++w) v[i] += room[i][w];
  }
}

// ------------------------------------------------------------------ weight gradients from the partial sums
// [dw | db] of worker m, column `col` of 2 pad
__device__ __forceinline__ void put_weight_gradient(const NormGradArgs& a, uint32_t m, uint32_t col, double sum) {
  const uint32_t c = col < a.pad ? col : col - a.pad;
  void* base = col < a.pad ? a.dweight : a.dbias;
  if (base == nullptr || c >= a.dim) return;
  if (a.grads_bf16) {
    __nv_bfloat16* to = static_cast<__nv_bfloat16*>(base) + m * a.grads_stride + c;
    *to = __double2bfloat16(a.accumulate ? sum + (double)__bfloat162float(*to) : sum);      // to nearest, in one rounding
  } else {
    float* to = static_cast<float*>(base) + m * a.grads_stride + c;
    *to = (float)(a.accumulate ? sum + (double)*to : sum);
  }
}
// blockIdx.x: 32 columns of [dw | db] (pad entries each), blockIdx.y: worker.  The warps take neighbouring slots in turn.
constexpr int kJoinWarps = 16;
__global__ void __launch_bounds__(kJoinWarps * 32) norm_join_kernel(NormGradArgs a) {
  __shared__ double room[kJoinWarps][32];
  const uint32_t w = threadIdx.x >> 5, lane = lane_id(), m = blockIdx.y, col = blockIdx.x * 32 + lane;
  grid_dependency_wait();
  if (blockIdx.x == 0 && m == 0 && threadIdx.x < 8) a.hdr[threadIdx.x] = 0;
  if (a.dweight == nullptr && a.dbias == nullptr) return;
  double sum = 0;
  if (a.T > 0 && col < 2 * a.pad) {
    const uint32_t first = a.shares ? m * (a.shares - 1) : (uint32_t)((uint64_t)m * a.T / a.per);      // slot k + m
    const uint32_t last = a.shares ? first + a.shares - 1 : (uint32_t)(((uint64_t)(m + 1) * a.T - 1) / a.per);
    const float* from = a.partial + (size_t)m * 2 * a.pad + col;
#pragma unroll 8
    for (uint32_t k = first + w; k <= last; k += kJoinWarps) sum += from[(size_t)k * 2 * a.pad];
  }
  room[w][lane] = sum;
  __syncthreads();
  if (w != 0 || col >= 2 * a.pad) return;
  for (int k = 1; k < kJoinWarps; ++k) sum += room[k][lane];
  put_weight_gradient(a, m, col, sum);
}

// ------------------------------------------------------------------ rows that threads hold in registers
// A group of `tpr` threads (part of a warp, a power of two, or whole warps) takes a row, kEach entries a thread: chunks of
// neighbouring kVec entries.  Rows to come are on their way into a ring in shared memory meanwhile (cp.async; empty places are
// not read).
constexpr int kRowThreads = 512, kRowWarps = kRowThreads / 32;
// Few rows: a cluster of eight CTAs takes a worker's rows and joins their sums itself, which saves the second launch.  One row a group
// at most (16 rows of 768: 7.0 us, with a second launch 7.1; 200 rows 12.1 and 8.8; what it saves besides is the host's second launch)
// and eight workers (8 x 16 rows of 768: 7.0 and 7.7 us; 16 workers: 14 and 8 us, more clusters than there is room for at once).
constexpr int kCluster = 8;
constexpr int kClusterWorkers = 8;
constexpr int kEach = 16, kPairs = kEach / 2;
constexpr uint64_t kMaxRowDim = (uint64_t)kRowThreads * kEach;

template <int kBytes>
__device__ __forceinline__ void copy_async(uint32_t at, const void* from) {   // at: shared memory
  if (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(kBytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// Two entries at a time (one instruction for both).
__device__ __forceinline__ unsigned long long bits(float2 a) { return *reinterpret_cast<unsigned long long*>(&a); }
__device__ __forceinline__ float2 pair(unsigned long long a) { return *reinterpret_cast<float2*>(&a); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
  return pair(d);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits(a)), "l"(bits(b)));
  return pair(d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  unsigned long long d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits(a)), "l"(bits(b)));
  return pair(d);
}
template <typename T>
__device__ __forceinline__ float2 rounded(float2 a) {
  if constexpr (sizeof(T) == 4) return a;
  const __nv_bfloat162 o = __floats2bfloat162_rn(a.x, a.y);
  const uint32_t w = *reinterpret_cast<const uint32_t*>(&o);
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }
__device__ __forceinline__ void clear(float2* v) {
#pragma unroll
  for (int i = 0; i < kPairs; ++i) v[i] = both(0.f);
}
__device__ __forceinline__ float total_of(const float2* v) {
  float2 q = v[0];
#pragma unroll
  for (int i = 1; i < kPairs; ++i) q = add2(q, v[i]);
  return q.x + q.y;
}

// The columns of a thread: kEach / kVec chunks, `step` apart.  Rows of more than 256 entries (kTiles) are dealt out evenly to the warps
// of the group, up to 512 to a warp, with a step that is known beforehand; shorter ones take a part of a warp, the smallest that holds
// them.  Either way the lower half of the chunks is there in every thread, but for a few entries by themselves (kTiny).
enum Form : int { kTiny = 0, kShort = 1, kTiles = 2, kFullTiles = 3 };      // kFullTiles: 512 columns to every warp
template <int kVec, int kForm>
struct Columns {
  static constexpr int kChunks = kEach / kVec;
  uint32_t c, any_step, limit;                     // first column; step; column behind the last one of the warp (of the row)
  __device__ __forceinline__ uint32_t step() const { return kForm >= kTiles ? 32 * kVec : any_step; }
  __device__ __forceinline__ bool has(int k) const { return kForm == kFullTiles || (kForm != kTiny && k < kChunks / 2) || c + k * step() < limit; }
};
// columns of a warp: the row's, dealt out evenly
template <int kVec>
__device__ __forceinline__ uint32_t tile_columns(uint32_t tpr, uint32_t dim) {
  const uint32_t warps = tpr / 32;
  return (dim + warps * kVec - 1) / (warps * kVec) * kVec;
}
template <int kVec, int kForm>
__device__ __forceinline__ Columns<kVec, kForm> columns(uint32_t tpr, uint32_t dim) {
  const uint32_t l = threadIdx.x % tpr;
  if (kForm < kTiles) return {l * kVec, tpr * kVec, dim};
  const uint32_t tile = tile_columns<kVec>(tpr, dim), first = l / 32 * tile;
  return {first + l % 32 * kVec, 32 * kVec, min(first + tile, dim)};
}

__device__ __forceinline__ void group_sync(uint32_t tpr) {
  if (tpr <= 32) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(1 + threadIdx.x / tpr), "r"(tpr) : "memory");     // at most eight groups
}

// A tensor's part of a ring stage.  Rows that wide accesses fit (kVec > 1): every thread copies the entries that it will read itself,
// and nobody waits for anybody.  Other rows (kVec 1): the group copies the row's 16-byte granules, whatever lies in them beside the
// row, and reads entries after a barrier.
template <typename T, int kVec>
struct Ring {
  static constexpr bool kShared = kVec == 1;
  static constexpr int kBytes = kVec * (int)sizeof(T), kChunks = kEach / kVec;
  static constexpr int kStage = kEach * (int)sizeof(T) * kRowThreads + (kShared ? kRowThreads / 4 * 16 : 0);
  const T* next;                                   // the group's row that is copied next, from the thread's first column (kShared: from the first)
  long long turn;                                  // entries from a row to the group's next
  uintptr_t begin, end;                            // what the tensor's entries lie between
  uint32_t own, low, bytes;                        // where the thread's (group's) entries begin in a stage; address of the row that is read next; of a row

  __device__ __forceinline__ void start(const Rows& r, uint32_t m, uint32_t t, uint32_t groups, uint32_t tpr, uint32_t c, uint32_t dim) {
    bytes = dim * (uint32_t)sizeof(T);
    next = row_of<T>(r, m, t);
    turn = groups * r.tok;
    begin = reinterpret_cast<uintptr_t>(r.p);
    end = reinterpret_cast<uintptr_t>(static_cast<const T*>(r.p) + r.last);
    low = (uint32_t)reinterpret_cast<uintptr_t>(next);
    if (kShared) own = threadIdx.x / tpr * (tpr * kEach * (uint32_t)sizeof(T) + 16);
    else { own = threadIdx.x * kBytes; next += c; }
  }
  // stage: offset of the tensor's part in the ring
  template <typename Cols>
  __device__ __forceinline__ void copy(char* ring, uint32_t stage, const Cols& at, uint32_t tpr) const {
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(ring) + stage + own;
    if (kShared) {
      const uintptr_t from = reinterpret_cast<uintptr_t>(next), past = from + bytes, first = from & ~(uintptr_t)15;
      for (uint32_t i = threadIdx.x % tpr * 16; first + i < past; i += tpr * 16) {
        if (first + i >= begin && first + i + 16 <= end) copy_async<16>(to + i, reinterpret_cast<const void*>(first + i));
        else                                       // at the ends of the tensor: only its own entries
          for (uint32_t e = 0; e < 16; e += sizeof(T))
            if (first + i + e >= from && first + i + e < past)
              *reinterpret_cast<T*>(ring + stage + own + i + e) = *reinterpret_cast<const T*>(first + i + e);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kChunks; ++k)
        if (at.has(k)) copy_async<kShared ? 16 : kBytes>(to + k * kRowThreads * kBytes, next + k * at.step());
    }
  }
  __device__ __forceinline__ void advance() { next += turn; }
  __device__ __forceinline__ void done() { if (kShared) low += (uint32_t)turn * (uint32_t)sizeof(T); }
  // ahead: 1 for the row after the one that is read next
  template <typename Cols>
  __device__ __forceinline__ void read(const char* ring, uint32_t stage, const Cols& at, float2* v, int ahead = 0) const {
    float* f = reinterpret_cast<float*>(v);
    uint32_t from = stage + own;
    if (kShared) from += ((low + (ahead ? (uint32_t)turn * (uint32_t)sizeof(T) : 0u)) & 15) + at.c * (uint32_t)sizeof(T);
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      const T* chunk = reinterpret_cast<const T*>(ring + from + (kShared ? k * at.step() * (uint32_t)sizeof(T) : k * kRowThreads * kBytes));
      if (at.has(k)) load_floats<T, kVec>(chunk, f + k * kVec);
      else
#pragma unroll
        for (int e = 0; e < kVec; ++e) f[k * kVec + e] = 0.f;
    }
  }
};
__host__ __device__ constexpr int stages_of(int bytes, int room) { return room / bytes > 5 ? 5 : room / bytes; }

template <typename T, int kVec, int kForm>
__device__ __forceinline__ void store_row(T* row, const Columns<kVec, kForm>& at, const float2* v) {
#pragma unroll
  for (int k = 0; k < kEach / kVec; ++k)
    if (at.has(k)) store_floats<T, kVec>(row + k * at.step(), reinterpret_cast<const float*>(v) + k * kVec);
}
template <int kVec, int kForm>
__device__ __forceinline__ void load_param(const void* p, bool bf16, const Columns<kVec, kForm>& at, float otherwise, float2* v) {
#pragma unroll
  for (int k = 0; k < kEach / kVec; ++k)
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      reinterpret_cast<float*>(v)[k * kVec + e] = at.has(k) ? param_at(p, bf16, at.c + k * at.step() + e, otherwise) : 0.f;
}
// v - mean, zero in columns that the thread does not have
template <int kVec, int kForm>
__device__ __forceinline__ void centre(float2* v, float mean, const Columns<kVec, kForm>& at) {
#pragma unroll
  for (int i = 0; i < kPairs; ++i) v[i] = add2(v[i], both(-mean));
#pragma unroll
  for (int e = 0; e < kEach; ++e)
    if (!at.has(e / kVec)) reinterpret_cast<float*>(v)[e] = 0.f;
}

// Sums over the group, in every thread of it: kCount values and, with kNext, one more.  Over a warp two or four sums share the
// exchanges: each step leaves a lane with half as many sums of twice as many lanes.  Calls in turn take another room each.
struct Room { float4 sums[kRowWarps]; float next[kRowWarps]; };
template <int kCount, bool kNext>
__device__ __forceinline__ void group_sums(float (&v)[kCount == 0 ? 1 : kCount], float& next, Room& room, uint32_t tpr) {
  constexpr uint32_t kAll = 0xffffffffu;
  if (tpr < 32) {
#pragma unroll
    for (uint32_t o = 1; o < 32; o *= 2) {
      if (o >= tpr) break;
#pragma unroll
      for (int i = 0; i < kCount; ++i) v[i] += __shfl_xor_sync(kAll, v[i], o);
      if (kNext) next += __shfl_xor_sync(kAll, next, o);
    }
    return;
  }
  const uint32_t lane = lane_id();
  float one = 0.f;                                 // lane l: sum number l % kCount
  if constexpr (kCount == 2) {
    const bool odd = lane & 1;
    one = (odd ? v[1] : v[0]) + __shfl_xor_sync(kAll, odd ? v[0] : v[1], 1);
  } else if constexpr (kCount == 4) {
    const bool odd = lane & 1, high = lane & 2;
    const float a = (odd ? v[1] : v[0]) + __shfl_xor_sync(kAll, odd ? v[0] : v[1], 1);
    const float b = (odd ? v[3] : v[2]) + __shfl_xor_sync(kAll, odd ? v[2] : v[3], 1);
    one = (high ? b : a) + __shfl_xor_sync(kAll, high ? a : b, 2);
  }
#pragma unroll
  for (uint32_t o = 1; o < 32; o *= 2) {
    if (kCount > 0 && o >= kCount) one += __shfl_xor_sync(kAll, one, o);
    if (kNext) next += __shfl_xor_sync(kAll, next, o);
  }
  if (tpr == 32) {
#pragma unroll
    for (int i = 0; i < kCount; ++i) v[i] = __shfl_sync(kAll, one, i);
    return;
  }
  const uint32_t w = threadIdx.x / 32, warps = tpr / 32, first = threadIdx.x / tpr * warps;
  if (kCount > 0 && lane < kCount) reinterpret_cast<float*>(room.sums + w)[lane] = one;
  if (kNext && lane == 0) room.next[w] = next;
  group_sync(tpr);
  float4 all = make_float4(0.f, 0.f, 0.f, 0.f);
  next = 0.f;
  for (uint32_t k = 0; k < warps; ++k) {
    if constexpr (kCount == 4) {
      const float4 more = room.sums[first + k];
      all.x += more.x; all.y += more.y; all.z += more.z; all.w += more.w;
    } else if constexpr (kCount == 2) {
      const float2 more = *reinterpret_cast<const float2*>(room.sums + first + k);
      all.x += more.x; all.y += more.y;
    }
    if (kNext) next += room.next[first + k];
  }
  if constexpr (kCount > 0) { v[0] = all.x; v[1] = all.y; }
  if constexpr (kCount > 2) { v[2] = all.z; v[3] = all.w; }
}

// The variance from the mean of (v - mean)^2 and `shift`, the mean of v - mean.  Where all entries are equal, v - mean is one number d in
// every column: zero, or what the mean's rounding left.  The sums have at most 31 roundings, with 1 / dim's, so the mean square is at most
// (1 + 31 u) d^2 and shift^2 at least (1 - 60 u) d^2, u = 2^-24: taking 128 u more than shift^2 leaves nothing, as the formula has it.  In other
// rows that is no more than the mean square's own rounding where shift is as large as the deviation, and vanishes with shift^2.
// 512 threads' sums below the normal range are off by 2^-150 each: what lies below 2^-116 has lost digits and counts as nothing, too.
__device__ __forceinline__ float variance(float square, float shift) {
  const float rest = fmaf(-shift * (1.f + 0x1p-17f), shift, square);
  return !(square < INFINITY) ? NAN : rest < 0x1p-116f ? 0.f : rest;           // NaN: squares beyond fp32's range, too
}

// One worker's rows begin .. end of a run, of which the group takes every groups-th.
struct Segment {
  uint32_t m, t, turns, row, groups;
  int left;                                        // rows from the group's next one on
  const void* ids;
  bool ids64;
  __device__ __forceinline__ bool there(uint32_t k) const {          // is there a token k turns from the first?
    return k * groups < (uint32_t)left && !is_empty(ids, ids64, row + k * groups);
  }
};
__device__ __forceinline__ Segment segment(uint32_t begin, uint32_t end, uint32_t m, uint32_t T, uint32_t groups, uint32_t group, const void* ids, bool ids64) {
  return {m, begin - m * T + group, (end - begin + groups - 1) / groups, begin + group, groups, end - begin > group ? (int)(end - begin - group) : 0, ids, ids64};
}

// The two kernels have the same course.  Turn k: wait until its row has arrived, send for row k + kStages - 1 (into the stage that
// turn k - 1 read), take the row's sums.  The sum of row k + 1 is taken in turn k and travels with the others, which leaves one exchange
// a row (65536 x 2048 bf16, gradient with residual: 289 -> 223 us; 32768 x 2048 fp32 gradient: 156 -> 147).  That needs three stages: in
// fp32 the gradient with dtotal has two, where waiting for row k + 1 would leave nothing on its way.  Backward, rows entry by entry:
// 128 registers do not hold the next row as well.
constexpr int kNormRoom = 204 * 1024;              // shared memory of the ring
template <typename X, int kVec, bool kAdd>
constexpr int kNormStage = Ring<X, kVec>::kStage * (kAdd ? 2 : 1);

// Rows begin .. end of worker m.
template <typename X, typename Y, int kVec, bool kAdd, typename Cols>
__device__ __forceinline__ void norm_rows(const NormArgs& a, uint32_t begin, uint32_t end, uint32_t m, uint32_t tpr, const Cols& at, char* ring,
                                          Room* rooms, const float2* w, const float2* b) {
  using RingX = Ring<X, kVec>;
  constexpr int kStage = kNormStage<X, kVec, kAdd>, kStages = stages_of(kStage, kNormRoom);
  static_assert(kStages >= 3, "the next row is read a turn ahead");
  const uint32_t groups = kRowThreads / tpr;
  const float over = 1.f / a.dim;
  Segment s = segment(begin, end, m, a.T, groups, threadIdx.x / tpr, a.ids, a.ids64);
  RingX x, add;
  x.start(a.x, m, s.t, groups, tpr, at.c, a.dim);
  if (kAdd) add.start(a.add, m, s.t, groups, tpr, at.c, a.dim);
  Y* row_y = row_of<Y>(a.y, m, s.t) + at.c;
  X* row_t = kAdd ? row_of<X>(a.total, m, s.t) + at.c : nullptr;
  uint32_t to = 0, from = 0;
  auto after = [](uint32_t stage) { return stage == (kStages - 1) * kStage ? 0u : stage + kStage; };
  auto issue = [&](bool real) {
    if (real) {
      x.copy(ring, to, at, tpr);
      if (kAdd) add.copy(ring, to + RingX::kStage, at, tpr);
    }
    copy_commit();
    x.advance();
    if (kAdd) add.advance();
    to = after(to);
  };
  auto read = [&](uint32_t stage, float2* v, int ahead) {
    x.read(ring, stage, at, v, ahead);
    if (!kAdd) return;
    float2 u[kPairs];
    add.read(ring, stage + RingX::kStage, at, u, ahead);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) v[i] = rounded<X>(add2(v[i], u[i]));
  };
  group_sync(tpr);                                                   // the segment before is read: ring and rooms are free
  uint32_t flags = 0;                                                // bit k: the row k turns ahead is there
#pragma unroll
  for (int k = 0; k + 1 < kStages; ++k) {
    const bool real = s.there(k);
    issue(real);
    flags |= (uint32_t)real << k;
  }
  bool coming = s.there(kStages - 1);
  float2 v[kPairs], u[kPairs];                                       // this row, the next one
  float sum = 0.f, none[1];
  copy_wait<kStages - 2>();
  if (RingX::kShared) group_sync(tpr);
  if (flags & 1) read(from, u, 0);
  else clear(u);
  sum = total_of(u);
  group_sums<0, true>(none, sum, rooms[1], tpr);
  for (uint32_t k = 0; k < s.turns; ++k) {
    copy_wait<kStages - 3>();
    if (RingX::kShared) group_sync(tpr);
    issue(coming);
    flags |= (uint32_t)coming << (kStages - 1);
    coming = s.there(k + kStages);
    const bool real = flags & 1, more = flags & 2, in = (int)(k * groups) < s.left;
    flags >>= 1;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) v[i] = u[i];
    if (more) read(after(from), u, 1);
    else clear(u);
    if (kAdd && in) store_row(row_t, at, v);
    centre(v, sum * over, at);
    float2 s0 = v[0], s1 = mul2(v[0], v[0]);
#pragma unroll
    for (int i = 1; i < kPairs; ++i) {
      s0 = add2(s0, v[i]);
      s1 = fma2(v[i], v[i], s1);
    }
    float sums[2] = {(s0.x + s0.y) * over, (s1.x + s1.y) * over};     // the row's mean, so that sums of large squares fit
    sum = total_of(u);
    group_sums<2, true>(sums, sum, rooms[k & 1], tpr);
    const float shift = sums[0], rstd = rsqrtf(variance(sums[1], shift) + a.eps);
    if (in) {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) v[i] = fma2(fma2(v[i], both(rstd), both(-shift * rstd)), w[i], b[i]);
      if (!real) clear(v);
      store_row(row_y, at, v);
    }
    row_y += groups * a.y.tok;
    if (kAdd) row_t += groups * a.total.tok;
    x.done();
    if (kAdd) add.done();
    from = after(from);
  }
}

template <typename X, typename Y, int kVec, int kForm, bool kAdd>
__global__ void __launch_bounds__(kRowThreads, 1) norm_row_kernel(NormArgs a, uint32_t tpr) {
  extern __shared__ __align__(16) char ring[];
  __shared__ Room rooms[2];
  if (threadIdx.x / tpr >= kRowThreads / tpr) return;                // warps that make no group
  const Columns<kVec, kForm> at = columns<kVec, kForm>(tpr, a.dim);
  const uint32_t r0 = blockIdx.x * a.per, r1 = min(r0 + a.per, a.N);
  float2 w[kPairs], b[kPairs];
  load_param(a.weight, a.param_bf16, at, 1.f, w);
  load_param(a.bias, a.param_bf16, at, 0.f, b);
  for (uint32_t begin = r0; begin < r1;) {                           // one worker's rows at a time
    const uint32_t m = begin / a.T, end = (uint32_t)min((uint64_t)r1, (uint64_t)(m + 1) * a.T);
    norm_rows<X, Y, kVec, kAdd>(a, begin, end, m, tpr, at, ring, rooms, w, b);
    begin = end;
  }
}

constexpr int kGradRoom = 204 * 1024;
template <typename D, typename X, int kVec, bool kMore>
constexpr int kGradStage = Ring<D, kVec>::kStage + Ring<X, kVec>::kStage * (kMore ? 2 : 1);

// Rows begin .. end of worker m; the group's sums of the weight gradients.
template <typename D, typename X, int kVec, bool kMore, typename Cols>
__device__ __forceinline__ void grad_rows(const NormGradArgs& a, uint32_t begin, uint32_t end, uint32_t m, uint32_t tpr, const Cols& at, char* ring,
                                          Room* rooms, const float2* w, float2* dw, float2* db) {
  using RingD = Ring<D, kVec>; using RingX = Ring<X, kVec>;
  constexpr int kStage = kGradStage<D, X, kVec, kMore>, kStages = stages_of(kStage, kGradRoom);
  constexpr bool kAhead = kStages >= 3 && kVec > 1;
  const uint32_t groups = kRowThreads / tpr;
  const float over = 1.f / a.dim;
  Segment s = segment(begin, end, m, a.T, groups, threadIdx.x / tpr, a.ids, a.ids64);
  RingD dy;
  RingX x, dt;
  dy.start(a.dy, m, s.t, groups, tpr, at.c, a.dim);
  x.start(a.x, m, s.t, groups, tpr, at.c, a.dim);
  if (kMore) dt.start(a.dtotal, m, s.t, groups, tpr, at.c, a.dim);
  X* row_o = row_of<X>(a.dx, m, s.t) + at.c;
  uint32_t to = 0, from = 0;
  auto after = [](uint32_t stage) { return stage == (kStages - 1) * kStage ? 0u : stage + kStage; };
  auto issue = [&](bool real) {
    if (real) {
      x.copy(ring, to, at, tpr);
      dy.copy(ring, to + RingX::kStage, at, tpr);
      if (kMore) dt.copy(ring, to + RingX::kStage + RingD::kStage, at, tpr);
    }
    copy_commit();
    dy.advance();
    x.advance();
    if (kMore) dt.advance();
    to = after(to);
  };
  group_sync(tpr);                                                   // the segment before is read: ring and rooms are free
  uint32_t flags = 0;                                                // bit k: the row k turns ahead is there
#pragma unroll
  for (int k = 0; k + 1 < kStages; ++k) {
    const bool real = s.there(k);
    issue(real);
    flags |= (uint32_t)real << k;
  }
  bool coming = s.there(kStages - 1);
  float2 v[kPairs], g[kPairs];
  float sum = 0.f, none[1];
  if (kAhead) {
    copy_wait<kStages - 2>();
    if (flags & 1) {
      x.read(ring, from, at, v);
      sum = total_of(v);
    }
    group_sums<0, true>(none, sum, rooms[1], tpr);
  }
  for (uint32_t k = 0; k < s.turns; ++k) {
    copy_wait<kAhead ? kStages - 3 : kStages - 2>();
    if (RingX::kShared) group_sync(tpr);
    issue(coming);
    flags |= (uint32_t)coming << (kStages - 1);
    coming = s.there(k + kStages);
    const bool real = flags & 1, more = flags & 2, in = (int)(k * groups) < s.left;
    flags >>= 1;
    if (real) {
      x.read(ring, from, at, v);
      dy.read(ring, from + RingX::kStage, at, g);
    } else {
      clear(v);
      clear(g);
    }
    if (!kAhead) {
      sum = total_of(v);
      group_sums<0, true>(none, sum, rooms[1], tpr);
    }
    centre(v, sum * over, at);
    float2 s0 = both(0.f), s1 = s0, s2 = s0, s3 = s0;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const float2 gw = mul2(g[i], w[i]);
      s0 = add2(s0, v[i]);
      s1 = fma2(v[i], v[i], s1);
      s2 = add2(s2, gw);
      s3 = fma2(gw, v[i], s3);
    }
    float sums[4] = {(s0.x + s0.y) * over, (s1.x + s1.y) * over, (s2.x + s2.y) * over, (s3.x + s3.y) * over};
    sum = 0.f;
    if (kAhead && more) {
      float2 u[kPairs];
      x.read(ring, after(from), at, u, 1);
      sum = total_of(u);
    }
    group_sums<4, kAhead>(sums, sum, rooms[kAhead ? k & 1 : 0], tpr);
    const float shift = sums[0], rstd = rsqrtf(variance(sums[1], shift) + a.eps);
    const float mg = sums[2], mgx = fmaf(-shift, mg, sums[3]) * rstd;
    if (real) {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float2 xhat = fma2(v[i], both(rstd), both(-shift * rstd));
        dw[i] = fma2(g[i], xhat, dw[i]);
        db[i] = add2(db[i], g[i]);
        v[i] = mul2(fma2(xhat, both(-mgx), fma2(g[i], w[i], both(-mg))), both(rstd));
      }
      if (kMore) {
        float2 o[kPairs];
        dt.read(ring, from + RingX::kStage + RingD::kStage, at, o);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) v[i] = add2(v[i], o[i]);
      }
    }
    if (a.dx.p != nullptr && in) {
      if (!real) clear(v);
      store_row(row_o, at, v);
    }
    row_o += groups * a.dx.tok;
    dy.done();
    x.done();
    if (kMore) dt.done();
    from = after(from);
  }
}

template <typename D, typename X, int kVec, int kForm, bool kMore>
__global__ void __launch_bounds__(kRowThreads, 1) grad_row_kernel(NormGradArgs a, uint32_t tpr) {
  constexpr int kStage = kGradStage<D, X, kVec, kMore>, kStages = stages_of(kStage, kGradRoom);
  extern __shared__ __align__(16) char ring[];
  float* flush = reinterpret_cast<float*>(ring);                     // between two segments, when no row is on its way
  static_assert(kStages * kStage >= kRowThreads * 2 * kEach * (int)sizeof(float));
  __shared__ Room rooms[2];
  const uint32_t groups = kRowThreads / tpr;
  const bool busy = threadIdx.x / tpr < groups;                      // not a warp that makes no group
  const Columns<kVec, kForm> at = columns<kVec, kForm>(tpr, a.dim);
  grid_dependency_wait();
  uint32_t r0 = blockIdx.x * a.per, r1 = min(r0 + a.per, a.N);
  if (a.shares) {
    r0 = min(blockIdx.x * a.per, a.T) + blockIdx.y * a.T;
    r1 = min((blockIdx.x + 1) * a.per, a.T) + blockIdx.y * a.T;
  }
  float2 w[kPairs], dw[kPairs], db[kPairs];
  load_param(a.weight, a.weight_bf16, at, 1.f, w);
  for (uint32_t begin = r0; begin < r1;) {                           // one worker's rows at a time
    const uint32_t m = begin / a.T, end = (uint32_t)min((uint64_t)r1, (uint64_t)(m + 1) * a.T);
    clear(dw);
    clear(db);
    if (busy) grad_rows<D, X, kVec, kMore>(a, begin, end, m, tpr, at, ring, rooms, w, dw, db);
    if (a.partial != nullptr) {                                      // the groups' sums
      float* out = a.partial + (size_t)(blockIdx.x + m * (a.shares ? a.shares : 1u)) * 2 * a.pad;
#pragma unroll
      for (int i = 0; i < kPairs; ++i)                               // groups of one warp
        for (uint32_t o = tpr; o < 32; o *= 2) {
          dw[i] = add2(dw[i], pair(__shfl_xor_sync(0xffffffffu, bits(dw[i]), o)));
          db[i] = add2(db[i], pair(__shfl_xor_sync(0xffffffffu, bits(db[i]), o)));
        }
      const uint32_t tile = kForm >= kTiles ? tile_columns<kVec>(tpr, a.dim) : a.dim;
      const uint32_t apart = tpr < 32 ? 32 : tpr, past = tpr < 32 ? kRowThreads : groups * tpr;   // threads from one sum of a column to the next
      __syncthreads();
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        flush[e * kRowThreads + threadIdx.x] = reinterpret_cast<float*>(dw)[e];
        flush[(kEach + e) * kRowThreads + threadIdx.x] = reinterpret_cast<float*>(db)[e];
      }
      __syncthreads();
      for (uint32_t i = threadIdx.x; i < 2 * kEach * tpr; i += kRowThreads) {
        const uint32_t row = i / tpr, l = i % tpr, e = row % kEach;
        const uint32_t in = (kForm >= kTiles ? l % 32 : l) * kVec + e / kVec * at.step() + e % kVec, col = kForm >= kTiles ? l / 32 * tile + in : in;
        float sum = 0.f;
        for (uint32_t j = l; j < past; j += apart) sum += flush[row * kRowThreads + j];
        if (in < tile && col < a.dim) out[(row < kEach ? 0 : a.pad) + col] = sum;
      }
      if (end < r1) __syncthreads();
    }
    begin = end;
  }
  if (!a.cluster) return;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 8) a.hdr[threadIdx.x] = 0;
  if (a.partial == nullptr) return;
  cluster_sync();                                                    // the partial sums of all CTAs are there
  const float* from = a.partial + (size_t)blockIdx.y * a.shares * 2 * a.pad;
  for (uint32_t col = blockIdx.x * kRowThreads + threadIdx.x; col < 2 * a.pad; col += kCluster * kRowThreads) {
    double sum = 0;
    for (uint32_t k = 0; k < a.shares; ++k) sum += __ldcg(from + (size_t)k * 2 * a.pad + col);
    put_weight_gradient(a, blockIdx.y, col, sum);
  }
}

// ------------------------------------------------------------------ rows of any length, read once for each sum
template <typename X, typename Y, int kVec>
__global__ void __launch_bounds__(kThreads) norm_long_kernel(NormArgs a) {
  __shared__ double room1[1][kWarps], room2[2][kWarps];
  for (uint32_t r = blockIdx.x; r < a.N; r += gridDim.x) {
    const uint32_t m = r / a.T, t = r % a.T;
    const X* x = row_of<X>(a.x, m, t);
    X* total = a.total.p == nullptr ? nullptr : row_of<X>(a.total, m, t);
    Y* y = row_of<Y>(a.y, m, t);
    if (is_empty(a.ids, a.ids64, r)) {
      const float zero[kVec] = {};
      for (uint32_t c = threadIdx.x * kVec; c < a.dim; c += kThreads * kVec) {
        store_floats<Y, kVec>(y + c, zero);
        if (total != nullptr) store_floats<X, kVec>(total + c, zero);
      }
      continue;
    }
    double sum[1] = {};
    for (uint32_t c = threadIdx.x * kVec; c < a.dim; c += kThreads * kVec) {
      float v[kVec], u[kVec];
      load_floats<X, kVec>(x + c, v);
      if (a.add.p != nullptr) {
        load_floats<X, kVec>(row_of<X>(a.add, m, t) + c, u);
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = to_f32(from_f32<X>(v[e] + u[e]));
        store_floats<X, kVec>(total + c, v);
      }
#pragma unroll
      for (int e = 0; e < kVec; ++e) sum[0] += v[e];
    }
    cta_sums(sum, room1);
    if (total != nullptr) x = total;               // each thread reads back what it wrote itself
    const float mean = (float)(sum[0] / a.dim);
    double sums[2] = {};
    for (uint32_t c = threadIdx.x * kVec; c < a.dim; c += kThreads * kVec) {
      float v[kVec];
      load_floats<X, kVec>(x + c, v);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const double d = v[e] - mean;
        sums[0] += d;
        sums[1] += d * d;
      }
    }
    cta_sums(sums, room2);
    const double rest = sums[0] / a.dim;
    const float shift = (float)rest, rstd = (float)(1.0 / sqrt(fmax(sums[1] / a.dim - rest * rest, 0.0) + a.eps));
    for (uint32_t c = threadIdx.x * kVec; c < a.dim; c += kThreads * kVec) {
      float v[kVec];
      load_floats<X, kVec>(x + c, v);
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        v[e] = fmaf((v[e] - mean - shift) * rstd, param_at(a.weight, a.param_bf16, c + e, 1.f), param_at(a.bias, a.param_bf16, c + e, 0.f));
      store_floats<Y, kVec>(y + c, v);
    }
  }
}

// Two times four numbers for every row: the mean in two pieces, rstd; mean of g, mean of g xhat.
template <typename D, typename X, int kVec>
__global__ void __launch_bounds__(kThreads) stats_long_kernel(NormGradArgs a) {
  __shared__ double room1[1][kWarps], room4[4][kWarps];
  for (uint32_t r = blockIdx.x; r < a.N; r += gridDim.x) {
    if (is_empty(a.ids, a.ids64, r)) continue;
    const uint32_t m = r / a.T, t = r % a.T;
    const X* x = row_of<X>(a.x, m, t);
    const D* dy = row_of<D>(a.dy, m, t);
    double sum[1] = {};
    for (uint32_t c = threadIdx.x * kVec; c < a.dim; c += kThreads * kVec) {
      float v[kVec];
      load_floats<X, kVec>(x + c, v);
#pragma unroll
      for (int e = 0; e < kVec; ++e) sum[0] += v[e];
    }
    cta_sums(sum, room1);
    const float mean = (float)(sum[0] / a.dim);
    double s[4] = {};
    for (uint32_t c = threadIdx.x * kVec; c < a.dim; c += kThreads * kVec) {
      float v[kVec], g[kVec];
      load_floats<X, kVec>(x + c, v);
      load_floats<D, kVec>(dy + c, g);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const double d = v[e] - mean, w = g[e] * param_at(a.weight, a.weight_bf16, c + e, 1.f);
        s[0] += d;
        s[1] += d * d;
        s[2] += w;
        s[3] += w * d;
      }
    }
    cta_sums(s, room4);
    const double rest = s[0] / a.dim, rstd = 1.0 / sqrt(fmax(s[1] / a.dim - rest * rest, 0.0) + a.eps);
    if (threadIdx.x == 0) {
      a.stats[2 * (size_t)r] = make_float4(mean, (float)rest, (float)rstd, 0.f);
      a.stats[2 * (size_t)r + 1] = make_float4((float)(s[2] / a.dim), (float)((s[3] - rest * s[2]) * rstd / a.dim), 0.f, 0.f);
    }
  }
}

// blockIdx.x: run of rows, blockIdx.y: tile of columns.  dx of the tile, and its partial sums of the weight gradients.
template <typename D, typename X, int kVec>
__global__ void __launch_bounds__(kThreads) grad_long_kernel(NormGradArgs a) {
  grid_dependency_wait();
  const uint32_t r0 = blockIdx.x * a.per, r1 = min(r0 + a.per, a.N), c = (blockIdx.y * kThreads + threadIdx.x) * kVec;
  if (c >= a.dim) return;
  float w[kVec], dw[kVec] = {}, db[kVec] = {};
#pragma unroll
  for (int e = 0; e < kVec; ++e) w[e] = param_at(a.weight, a.weight_bf16, c + e, 1.f);
  for (uint32_t r = r0; r < r1; ++r) {
    const uint32_t m = r / a.T, t = r % a.T;
    float o[kVec] = {};
    if (!is_empty(a.ids, a.ids64, r)) {
      const float4 s = a.stats[2 * (size_t)r], q = a.stats[2 * (size_t)r + 1];
      float x[kVec], g[kVec];
      load_floats<X, kVec>(row_of<X>(a.x, m, t) + c, x);
      load_floats<D, kVec>(row_of<D>(a.dy, m, t) + c, g);
      if (a.dtotal.p != nullptr) load_floats<X, kVec>(row_of<X>(a.dtotal, m, t) + c, o);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float xhat = (x[e] - s.x - s.y) * s.z;
        dw[e] = fmaf(g[e], xhat, dw[e]);
        db[e] += g[e];
        o[e] = fmaf(s.z, fmaf(-xhat, q.y, fmaf(g[e], w[e], -q.x)), o[e]);
      }
    }
    if (a.dx.p != nullptr) store_floats<X, kVec>(row_of<X>(a.dx, m, t) + c, o);
    if (a.partial != nullptr && (r + 1 == r1 || t + 1 == a.T)) {
      float* to = a.partial + (size_t)(blockIdx.x + m) * 2 * a.pad + c;
      store_floats<float, kVec>(to, dw);
      store_floats<float, kVec>(to + a.pad, db);
#pragma unroll
      for (int e = 0; e < kVec; ++e) dw[e] = db[e] = 0.f;
    }
  }
}

// ------------------------------------------------------------------ host
struct NormGradLayout {
  uint32_t per, runs, pad;
  size_t off_stats, off_partial, total;
};
bool norm_grad_layout(int M, uint64_t T, uint64_t dim, NormGradLayout* L) {
  if (M < 1 || M > 65535 || dim == 0 || dim > kMaxDim || T >= (1ull << 31) || (uint64_t)M * T >= (1ull << 31)) return false;
  const uint64_t N = (uint64_t)M * T;
  uint64_t per = (N + kRuns - 1) / kRuns;
  per = per < 1 ? 1 : per > kMaxRun ? kMaxRun : per;
  L->per = (uint32_t)per;
  L->runs = (uint32_t)((N + per - 1) / per);
  L->pad = (uint32_t)((dim + 3) / 4 * 4);
  L->off_stats = align_up(kHdrWords * sizeof(uint32_t), 256);
  L->off_partial = align_up(L->off_stats + (dim > kMaxRowDim ? N * 2 * sizeof(float4) : 0), 256);
  // slots: runs + M, which never shrinks as N grows if runs is counted as follows
  const uint64_t most = (N < 2 * kRuns ? N : (uint64_t)2 * kRuns) + N / kMaxRun + M + 1;
  L->total = align_up(L->off_partial + most * 2 * L->pad * sizeof(float), 256);
  return true;
}

// widest access of rows: 8 (16-bit types only) or 4 entries where base and distances of every tensor allow it, else single ones
struct Given { Rows r; int dtype; };
int row_width(const Given* g, int n, uint64_t dim, int M, uint64_t T) {
  int v = dim % 8 == 0 ? 8 : dim % 4 == 0 && dim > kEach / 2 ? 4 : 1;
  for (int i = 0; i < n; ++i) {
    if (g[i].r.p == nullptr) continue;
    if (g[i].dtype != S3GD_BF16 && v == 8) v = 4;
    v = allowed(v, g[i].r.p, g[i].dtype, T > 1 ? g[i].r.tok : 0, M > 1 ? g[i].r.worker : 0);
  }
  return v >= 4 ? v : 1;
}
// entries from the first to behind the last
void measure(Rows* r, int M, uint64_t T, uint64_t dim) { r->last = (M - 1) * r->worker + (long long)(T - 1) * r->tok + (long long)dim; }
// inputs may repeat a row (distance 0); what is written must not overlap itself
bool readable(const Rows& r, int dtype) { return is_aligned(r.p, dtype_bytes(dtype)) && r.tok >= 0 && r.worker >= 0; }
bool writable(const Rows& r, int dtype, int M, uint64_t T, uint64_t dim) {
  if (!is_aligned(r.p, dtype_bytes(dtype)) || r.tok < 0 || r.worker < 0) return false;
  const uint64_t tok = (uint64_t)r.tok, worker = (uint64_t)r.worker;
  if (T > 1 && tok < dim) return false;
  if (M == 1) return true;
  // workers one behind the other, or interleaved (each token's row of all workers side by side)
  return worker >= (T > 1 ? (T - 1) * tok : 0) + dim || (worker >= dim && (T == 1 || tok >= (uint64_t)(M - 1) * worker + dim));
}
// an output that begins where an input does: in place, so it must lie the same
bool lies_alike(const Rows& out, int out_dtype, const Rows& in, int in_dtype, int M, uint64_t T) {
  return out.p == nullptr || out.p != in.p || (out_dtype == in_dtype && (T == 1 || out.tok == in.tok) && (M == 1 || out.worker == in.worker));
}
// do the workers' rows of two gradients have entries in common?  (stride >= dim where there are several)
bool rows_meet(const void* a, const void* b, size_t size, uint64_t dim, int M, int64_t stride) {
  if (a == nullptr || b == nullptr) return false;
  const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
  const uint64_t apart = (p < q ? q - p : p - q) / size;
  if (M == 1) return apart < dim;
  const uint64_t rows = apart / (uint64_t)stride, rest = apart % (uint64_t)stride;
  return (rows < (uint64_t)M && rest < dim) || (rows + 1 < (uint64_t)M && (uint64_t)stride - rest < dim);
}
// threads of a row: part of a warp (the fewest that hold it, but four where groups copy rows together), or a warp for every 512 entries
uint32_t threads_per_row(uint64_t dim, int vec) {
  if (dim > 16 * kEach) return (uint32_t)((dim + 32 * kEach - 1) / (32 * kEach)) * 32;
  uint32_t n = vec == 1 ? 4 : 1;
  while (n * kEach < dim) n *= 2;
  return n;
}
// f is called with the width of an access and the form of a row, as types.  16-bit rows alone may be read eight entries at a time.
template <bool kWide, typename F>
cudaError_t by_row_form(int vec, uint64_t dim, F f) {
  const bool tiles = dim > 16 * kEach;
  if (vec == 1) return tiles ? f(Width<1>(), Width<kTiles>()) : dim <= 2 * kEach ? f(Width<1>(), Width<kTiny>()) : f(Width<1>(), Width<kShort>());
  const bool whole = dim % (32 * kEach) == 0;
  if (kWide && vec == 8) {
    constexpr int kVec = kWide ? 8 : 4;
    return whole ? f(Width<kVec>(), Width<kFullTiles>()) : tiles ? f(Width<kVec>(), Width<kTiles>()) : f(Width<kVec>(), Width<kShort>());
  }
  return whole ? f(Width<4>(), Width<kFullTiles>()) : tiles ? f(Width<4>(), Width<kTiles>()) : f(Width<4>(), Width<kShort>());
}
template <typename X, typename Y, int kVec, int kForm, bool kAdd>
cudaError_t enqueue_norm_rows(NormArgs a, cudaStream_t st) {
  static int done[kMaxDevices];
  constexpr int kStage = kNormStage<X, kVec, kAdd>, kBytes = stages_of(kStage, kNormRoom) * kStage;
  auto kernel = norm_row_kernel<X, Y, kVec, kForm, kAdd>;
  const cudaError_t e = opt_in_dynamic_smem(reinterpret_cast<const void*>(kernel), kBytes, done);
  if (e != cudaSuccess) return e;
  const uint32_t runs = sm_count();
  a.per = (a.N + runs - 1) / runs;
  kernel<<<(a.N + a.per - 1) / a.per, kRowThreads, kBytes, st>>>(a, threads_per_row(a.dim, kVec));
  return cudaGetLastError();
}
template <typename D, typename X, int kVec, int kForm, bool kMore>
cudaError_t enqueue_grad_rows(const NormGradArgs& a, cudaStream_t st) {
  static int done[kMaxDevices];
  constexpr int kStage = kGradStage<D, X, kVec, kMore>, kBytes = stages_of(kStage, kGradRoom) * kStage;
  auto kernel = grad_row_kernel<D, X, kVec, kForm, kMore>;
  const cudaError_t e = opt_in_dynamic_smem(reinterpret_cast<const void*>(kernel), kBytes, done);
  if (e != cudaSuccess) return e;
  const uint32_t tpr = threads_per_row(a.dim, kVec);
  if (!a.cluster) return launch_after(kernel, a.shares ? dim3(a.shares, a.M) : dim3(a.runs), dim3(kRowThreads), kBytes, st, a, tpr);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kCluster, a.M); cfg.blockDim = dim3(kRowThreads); cfg.dynamicSmemBytes = kBytes; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kCluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, a, tpr);
}
// How rows are dealt to CTAs.  A turn of a CTA takes a row for each of its groups, and what a worker's rows cost a CTA besides
// (filling the ring, adding the groups' sums) is worth kSegmentTurns turns: runs either go on from one worker to the next, which
// keeps all CTAs equally busy, or end with the worker, one or two rounds of CTAs, whichever is over sooner (8 x 4096 x 512 fp32: 36.2 us,
// with runs that go on 39.6; 16 x 200 x 128: 6.8 and 14.2; 40 x 2000 x 1024, where they go on: 179).
constexpr uint32_t kLeastRun = 8;                  // rows of a run at least, where its CTA has as many groups: fewer sums to join
constexpr uint64_t kSegmentTurns = 4;
void plan_runs(NormGradArgs* a, uint32_t groups) {
  const uint64_t least = groups < kLeastRun ? groups : kLeastRun, M = a->M, T = a->T;
  auto turns = [&](uint64_t rows) { return (rows + groups - 1) / groups; };
  if (M <= kClusterWorkers && T <= (uint64_t)kCluster * groups) {
    a->cluster = true;
    a->per = (uint32_t)((T + kCluster - 1) / kCluster);
    a->shares = (uint32_t)((T + a->per - 1) / a->per);
    return;
  }
  if (a->per < least) a->per = (uint32_t)least;
  a->runs = (uint32_t)((a->N + a->per - 1) / a->per);
  const uint64_t segments = M == 1 ? 1 : (a->per + T - 1) / T + (T % a->per != 0);
  uint64_t best = (a->runs + kRuns - 1) / kRuns * (turns(a->per) + (segments - 1) + segments * kSegmentTurns);
  for (uint64_t rounds = 1; rounds <= 2 && M > 1; ++rounds) {
    uint64_t shares = rounds * kRuns / M;
    if (shares == 0) continue;
    uint64_t per = (T + shares - 1) / shares;
    per = per < least ? least : per;
    if (per > kMaxRun) continue;
    shares = (T + per - 1) / per;
    const uint64_t cost = (M * shares + kRuns - 1) / kRuns * (turns(per) + kSegmentTurns);
    if (cost >= best) continue;
    best = cost;
    a->per = (uint32_t)per;
    a->shares = (uint32_t)shares;
  }
}
template <typename F>
cudaError_t by_row_width(int v, F f) { return v >= 4 ? f(Width<4>()) : f(Width<1>()); }

}  // namespace
}  // namespace s3gd

using namespace s3gd;

extern "C" s3gd_status s3gd_layer_norm(const void* x, int x_dtype, int64_t x_stride, int64_t x_worker_stride, const void* opt_add,
                                       int64_t add_stride, int64_t add_worker_stride, void* opt_total, int64_t total_stride,
                                       int64_t total_worker_stride, const void* opt_weight, const void* opt_bias, int param_dtype,
                                       const void* opt_ids, int ids_dtype, int M, uint64_t T, uint64_t dim, float eps, void* y, int y_dtype,
                                       int64_t y_stride, int64_t y_worker_stride, void* stream) {
  if (!is_real(x_dtype) || !is_real(y_dtype) || !is_real(param_dtype) || !is_index(ids_dtype)) return S3GD_ERR_INVALID_ARG;
  if (M < 1 || M > 65535 || dim == 0 || dim > kMaxDim || T >= (1ull << 31) || (uint64_t)M * T >= (1ull << 31)) return S3GD_ERR_INVALID_ARG;
  if (!(eps >= 0.f && eps < INFINITY) || (opt_add == nullptr) != (opt_total == nullptr)) return S3GD_ERR_INVALID_ARG;
  NormArgs a = {};
  a.x = {x, x_stride, x_worker_stride};
  a.add = {opt_add, add_stride, add_worker_stride};
  a.total = {opt_total, total_stride, total_worker_stride};
  a.y = {y, y_stride, y_worker_stride};
  if (!is_aligned(opt_weight, dtype_bytes(param_dtype)) || !is_aligned(opt_bias, dtype_bytes(param_dtype)) ||
      !is_aligned(opt_ids, dtype_bytes(ids_dtype)))
    return S3GD_ERR_INVALID_ARG;
  if (T == 0) return S3GD_OK;
  if (x == nullptr || y == nullptr || !readable(a.x, x_dtype) || !writable(a.y, y_dtype, M, T, dim)) return S3GD_ERR_INVALID_ARG;
  if (opt_add != nullptr && (!readable(a.add, x_dtype) || !writable(a.total, x_dtype, M, T, dim) || y == opt_total)) return S3GD_ERR_INVALID_ARG;
  if (!lies_alike(a.y, y_dtype, a.x, x_dtype, M, T) || !lies_alike(a.total, x_dtype, a.x, x_dtype, M, T) ||
      !lies_alike(a.total, x_dtype, a.add, x_dtype, M, T))
    return S3GD_ERR_INVALID_ARG;
  a.weight = opt_weight; a.bias = opt_bias; a.param_bf16 = param_dtype == S3GD_BF16;
  a.ids = opt_ids; a.ids64 = ids_dtype == S3GD_I64;
  a.T = (uint32_t)T; a.N = (uint32_t)((uint64_t)M * T); a.dim = (uint32_t)dim; a.eps = eps;
  for (Rows* r : {&a.x, &a.add}) measure(r, M, T, dim);
  const Given all[] = {{a.x, x_dtype}, {a.add, x_dtype}, {a.total, x_dtype}, {a.y, y_dtype}};
  const int vec = row_width(all, 4, dim, M, T);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  count_launch();
  const cudaError_t e = by_real(x_dtype, [&](auto xt) { return by_real(y_dtype, [&](auto yt) {
    using X = decltype(xt); using Y = decltype(yt);
    if (dim <= kMaxRowDim)
      return by_row_form<sizeof(X) == 2 && sizeof(Y) == 2>(vec, dim, [&](auto v, auto f) {
        constexpr int kVec = decltype(v)::value, kForm = decltype(f)::value;
        return opt_add != nullptr ? enqueue_norm_rows<X, Y, kVec, kForm, true>(a, st) : enqueue_norm_rows<X, Y, kVec, kForm, false>(a, st);
      });
    return by_row_width(vec, [&](auto v) {
      const unsigned most = 8u * sm_count();
      norm_long_kernel<X, Y, decltype(v)::value><<<a.N < most ? a.N : most, kThreads, 0, st>>>(a);
      return cudaGetLastError();
    });
  }); });
  return e == cudaSuccess ? S3GD_OK : S3GD_ERR_CUDA;
}

extern "C" size_t s3gd_layer_norm_grad_workspace_bytes(int M, uint64_t T, uint64_t dim) {
  NormGradLayout L;
  return norm_grad_layout(M, T, dim, &L) ? L.total : 0;
}

extern "C" s3gd_status s3gd_layer_norm_grad(const void* dy, int dy_dtype, int64_t dy_stride, int64_t dy_worker_stride, const void* x,
                                            int x_dtype, int64_t x_stride, int64_t x_worker_stride, const void* opt_dtotal,
                                            int64_t dtotal_stride, int64_t dtotal_worker_stride, const void* opt_weight, int weight_dtype,
                                            const void* opt_ids, int ids_dtype, int M, uint64_t T, uint64_t dim, float eps, void* opt_dx,
                                            int64_t dx_stride, int64_t dx_worker_stride, void* opt_dweight, void* opt_dbias,
                                            int grads_dtype, int64_t grads_stride, int accumulate, void* ws, size_t ws_bytes,
                                            void* stream) {
  NormGradLayout L;
  if (!norm_grad_layout(M, T, dim, &L) || !is_real(dy_dtype) || !is_real(x_dtype) || !is_real(weight_dtype) || !is_index(ids_dtype) ||
      !is_real(grads_dtype) || !(eps >= 0.f && eps < INFINITY))
    return S3GD_ERR_INVALID_ARG;
  const bool weights = opt_dweight != nullptr || opt_dbias != nullptr;
  if ((opt_dx == nullptr && !weights) || (opt_dtotal != nullptr && opt_dx == nullptr)) return S3GD_ERR_INVALID_ARG;
  if (weights && M > 1 && (grads_stride < 0 || (uint64_t)grads_stride < dim)) return S3GD_ERR_INVALID_ARG;
  NormGradArgs a = {};
  a.dy = {dy, dy_stride, dy_worker_stride};
  a.x = {x, x_stride, x_worker_stride};
  a.dtotal = {opt_dtotal, dtotal_stride, dtotal_worker_stride};
  a.dx = {opt_dx, dx_stride, dx_worker_stride};
  if (!is_aligned(opt_weight, dtype_bytes(weight_dtype)) || !is_aligned(opt_ids, dtype_bytes(ids_dtype)) ||
      !is_aligned(opt_dweight, dtype_bytes(grads_dtype)) || !is_aligned(opt_dbias, dtype_bytes(grads_dtype)))
    return S3GD_ERR_INVALID_ARG;
  if (T > 0 && (dy == nullptr || x == nullptr || !readable(a.dy, dy_dtype) || !readable(a.x, x_dtype) ||
                (opt_dtotal != nullptr && !readable(a.dtotal, x_dtype)) || (opt_dx != nullptr && !writable(a.dx, x_dtype, M, T, dim))))
    return S3GD_ERR_INVALID_ARG;
  if (ws == nullptr || ws_bytes < L.total || !is_aligned(ws, 256)) return S3GD_ERR_WORKSPACE;
  if (rows_meet(opt_dweight, opt_dbias, dtype_bytes(grads_dtype), dim, M, grads_stride)) return S3GD_ERR_INVALID_ARG;
  if (T > 0 && (!lies_alike(a.dx, x_dtype, a.dy, dy_dtype, M, T) || !lies_alike(a.dx, x_dtype, a.x, x_dtype, M, T) ||
                !lies_alike(a.dx, x_dtype, a.dtotal, x_dtype, M, T)))
    return S3GD_ERR_INVALID_ARG;
  a.weight = opt_weight; a.weight_bf16 = weight_dtype == S3GD_BF16;
  a.ids = opt_ids; a.ids64 = ids_dtype == S3GD_I64;
  a.grads_bf16 = grads_dtype == S3GD_BF16; a.accumulate = accumulate != 0;
  a.M = M; a.T = (uint32_t)T; a.N = (uint32_t)((uint64_t)M * T); a.dim = (uint32_t)dim; a.pad = L.pad; a.per = L.per; a.runs = L.runs;
  a.eps = eps; a.dweight = opt_dweight; a.dbias = opt_dbias; a.grads_stride = M > 1 ? grads_stride : 0;
  char* base = static_cast<char*>(ws);
  a.hdr = reinterpret_cast<uint32_t*>(base);
  a.stats = reinterpret_cast<float4*>(base + L.off_stats);
  a.partial = weights ? reinterpret_cast<float*>(base + L.off_partial) : nullptr;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (a.N > 0) {
    for (Rows* r : {&a.dy, &a.x, &a.dtotal}) measure(r, M, T, dim);
    const Given all[] = {{a.dy, dy_dtype}, {a.x, x_dtype}, {a.dtotal, x_dtype}, {a.dx, x_dtype}};
    const int vec = row_width(all, 4, dim, M, T);
    const unsigned most = 8u * sm_count(), grid = a.N < most ? a.N : most;
    const unsigned wide = vec >= 4 ? 4 : 1, tiles = (unsigned)((dim + kThreads * wide - 1) / (kThreads * wide));
    if (tiles > 65535) return S3GD_ERR_INVALID_ARG;
    count_launch(dim > kMaxRowDim ? 2 : 1);
    if (dim <= kMaxRowDim) plan_runs(&a, kRowThreads / threads_per_row(dim, vec));
    e = by_real(dy_dtype, [&](auto dt) { return by_real(x_dtype, [&](auto xt) {
      using D = decltype(dt); using X = decltype(xt);
      if (dim <= kMaxRowDim)
        return by_row_form<sizeof(D) == 2 && sizeof(X) == 2>(vec, dim, [&](auto v, auto f) {
          constexpr int kVec = decltype(v)::value, kForm = decltype(f)::value;
          return opt_dtotal != nullptr ? enqueue_grad_rows<D, X, kVec, kForm, true>(a, st) : enqueue_grad_rows<D, X, kVec, kForm, false>(a, st);
        });
      return by_row_width(vec, [&](auto v) {
        constexpr int kVec = decltype(v)::value;
        stats_long_kernel<D, X, kVec><<<grid, kThreads, 0, st>>>(a);
        const cudaError_t first = cudaGetLastError();
        if (first != cudaSuccess) return first;
        return launch_after(grad_long_kernel<D, X, kVec>, dim3(a.runs, tiles), dim3(kThreads), 0, st, a);
      });
    }); });
  }
  if (e == cudaSuccess && !a.cluster) {
    count_launch();
    e = launch_after(norm_join_kernel, dim3(weights ? (2 * a.pad + 31) / 32 : 1, weights ? M : 1), dim3(kJoinWarps * 32), 0, st, a);
  }
  return e == cudaSuccess ? S3GD_OK : S3GD_ERR_CUDA;
}
