// Embedding table: scaled lookup, and the gradient of M workers written into their rows (see include/s3gd.h).
//
// Lookup.  A warp takes 512 columns of one token's row, all loads under way before the first store.  Bound by memory: 65536
// rows of 1000 from fp32 to bf16 take 39 us, 331 MB if every row were read once (51 us at 6.5 TB/s); common words are read
// from L2.
//
// Gradient.  Every entry of a worker's vocab x dim block is written once: a warp takes kRows neighbouring rows and 512
// columns, finds the tokens of its rows, sums their gradients in registers and stores sums or zeros.  Few tokens per worker
// (kDirectTokens, kDirectWork) the warp looks through itself, in one launch; more are first sorted by id (stable, so that
// each row's tokens come in ascending order) and the warp finds its rows by search.  A token that takes more than a chunk of
// places would leave one warp with all of them: its places are summed a chunk at a time by separate warps (aligned in the
// sorted order, so at most two such tokens meet a chunk) and joined by a last kernel in ascending order.  The list of these
// tokens is written in whatever order they are found; each is then worked on by itself.
// Bound by memory and, for few tokens to a row, by the chain search - place - gradient: 131072 tokens bf16 into 65536 x 2048
// fp32 take 252 us (1064 MB: 163 us at 6.5 TB/s; sort 37, rows 193, joining 20 by themselves), eight workers of 4096 tokens
// into 16000 x 512 each 86 us (326 MB: 50 us).
#include "s3gd_ops.cuh"

namespace s3gd {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kLane = 16;                          // columns per lane
constexpr int kTileCols = 32 * kLane;              // columns per warp
constexpr int kRows = 8;                           // rows of the table per warp
// Tokens per worker, and tokens times rows, that warps look through themselves: 512 tokens, 8000 rows of 768: 14.2 us, sorted
// 18.5 us; 64 tokens: 12.4 and 15.9 us; 1024 tokens: 18.5 us either way; 512 tokens, 100000 rows: 87 us, sorted 70 us.
constexpr int kDirectTokens = 512;
constexpr uint64_t kDirectWork = 1ull << 24;
constexpr int kHdrCommon = 16;                     // header word: common tokens found
constexpr int kMinChunk = 32, kMaxChunks = 8192;   // places per partial sum at least (64: 107 instead of 94 us for the eight
                                                   // workers above); partial sums per worker at most

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

// the widest access that base and distances allow, no wider than what keeps 32 lanes busy on `dim` columns
int widest(uint64_t dim) {
  int v = 8;
  while (v > 1 && (dim % v != 0 || dim < 32u * v)) v /= 2;
  return v;
}
int allowed(int v, const void* p, int dtype, int64_t stride_a, int64_t stride_b) {
  const size_t size = dtype_bytes(dtype);
  while (v > 1 && (!is_aligned(p, v * size < 16 ? v * size : 16) || stride_a % v != 0 || stride_b % v != 0)) v /= 2;
  return v;
}

// ------------------------------------------------------------------ lookup
template <typename W, typename I, typename O, int kVec>
__global__ void __launch_bounds__(kThreads) lookup_kernel(const W* table, long long table_stride, uint64_t vocab, uint32_t dim, const I* ids,
                                                          uint64_t n, float scale, O* out, long long out_stride, uint32_t* bad) {
  const uint32_t tiles = (dim + kTileCols - 1) / kTileCols;
  const uint64_t item = (uint64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const uint64_t t = item / tiles;
  const uint32_t tile = (uint32_t)(item % tiles), lane = lane_id();
  if (t >= n) return;
  const long long id = (long long)ids[t];
  const bool there = id >= 0 && (uint64_t)id < vocab;
  if (id >= 0 && !there && tile == 0 && bad != nullptr && lane == 0) atomicAdd(bad, 1u);
  const uint32_t c0 = tile * kTileCols + lane * kVec;
  const W* from = table + (there ? id : 0) * table_stride;
  O* to = out + (long long)t * out_stride;
  Pack<W, kVec> w[kLane / kVec];
#pragma unroll
  for (int a = 0; a < kLane / kVec; ++a)
    if (there && c0 + a * 32 * kVec < dim) w[a] = *reinterpret_cast<const Pack<W, kVec>*>(from + c0 + a * 32 * kVec);
#pragma unroll
  for (int a = 0; a < kLane / kVec; ++a) {
    if (c0 + a * 32 * kVec >= dim) continue;
    float v[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = there ? __fmul_rn(scale, to_f32(w[a].v[e])) : 0.f;
    store_pack<O, kVec>(to + c0 + a * 32 * kVec, v);
  }
}

// ------------------------------------------------------------------ sort of the tokens by id
// Least significant digit first, digits of at most 9 bits, tiles of 2048 or 4096 tokens of one worker.  Empty places and ids out of
// range take the key `vocab` and end up behind all others.
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
constexpr int kSortEach = 8, kSortTile = kSortThreads * kSortEach;   // of a long row, or the whole of a short one
constexpr int kFewEach = 4, kFewTiles = 64;       // rows of up to 64 tiles of 2048 are cut into these: more
                                                   // CTAs, shorter chains (131072 tokens: 246 instead of 273 us)
constexpr int kMaxDigit = 9, kBins = 1 << kMaxDigit;

struct SortPlan { int passes, bits; };
SortPlan sort_plan(uint64_t vocab) {
  int need = 1;
  while ((vocab >> need) != 0) ++need;             // keys 0 .. vocab
  SortPlan p;
  p.passes = (need + kMaxDigit - 1) / kMaxDigit;
  p.bits = (need + p.passes - 1) / p.passes;
  return p;
}

template <typename I>
__device__ __forceinline__ uint32_t key_of(I id, uint32_t vocab) {
  return id >= 0 && (unsigned long long)id < vocab ? (uint32_t)id : vocab;
}

struct TileSort {                                  // shared memory of one tile
  uint32_t count[kSortWarps][kBins];               // tokens of a digit per warp, then those in earlier warps
  uint32_t base[kBins];
  uint32_t warp_total[kSortWarps];
};

// Rank of every token among those of its digit in the tile.  Warp w holds places (w * kSortEach + r) * 32 + lane in key[r].
template <int kSortEach>
__device__ __forceinline__ void tile_ranks(TileSort& s, const uint32_t* key, uint32_t n, int shift, int bits, uint32_t* rank, uint32_t* total) {
  const uint32_t w = threadIdx.x >> 5, lane = lane_id(), mask = (1u << bits) - 1u;
  for (int i = threadIdx.x; i < kSortWarps * kBins; i += kSortThreads) s.count[i / kBins][i % kBins] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    const bool in = w * (kSortEach * 32) + r * 32 + lane < n;
    const uint32_t d = in ? (key[r] >> shift) & mask : kBins;      // places behind the end match only each other
    const uint32_t peers = __match_any_sync(0xffffffffu, d);
    uint32_t before = 0;
    if (in) before = s.count[w][d];
    __syncwarp();
    if (in && (peers & lanemask_lt()) == 0) s.count[w][d] = before + __popc(peers);
    __syncwarp();
    rank[r] = before + __popc(peers & lanemask_lt());
  }
  __syncthreads();
  uint32_t sum = 0;                                // thread d: digit d
  for (int v = 0; v < kSortWarps; ++v) {
    const uint32_t c = s.count[v][threadIdx.x];
    s.count[v][threadIdx.x] = sum;
    sum += c;
  }
  *total = sum;
  __syncthreads();
}

// s.base[d] = sum of `total` over the digits below d
__device__ __forceinline__ void digit_bases(TileSort& s, uint32_t total) {
  const uint32_t w = threadIdx.x >> 5, lane = lane_id();
  uint32_t v = total;
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= (uint32_t)o) v += u;
  }
  if (lane == 31) s.warp_total[w] = v;
  __syncthreads();
  uint32_t before = 0;
  for (uint32_t k = 0; k < w; ++k) before += s.warp_total[k];
  s.base[threadIdx.x] = before + v - total;
  __syncthreads();
}
static_assert(kBins == kSortThreads, "one thread per digit");

// All passes in shared memory: one CTA per worker, T <= kSortTile.
template <typename I>
__global__ void __launch_bounds__(kSortThreads) sort_small_kernel(const I* ids, uint32_t T, uint32_t vocab, SortPlan plan, uint32_t* keys,
                                                                  uint32_t* places, uint32_t* bad, uint32_t* hdr) {
  extern __shared__ char sort_smem[];
  TileSort& s = *reinterpret_cast<TileSort*>(sort_smem);
  uint32_t* buf_key = reinterpret_cast<uint32_t*>(sort_smem + sizeof(TileSort));
  uint32_t* buf_place = buf_key + kSortTile;
  const size_t row = (size_t)blockIdx.x * T;
  const uint32_t first = (threadIdx.x >> 5) * (kSortEach * 32) + lane_id();
  grid_dependency_wait();
  if (blockIdx.x == 0 && threadIdx.x < kHdrWords) hdr[threadIdx.x] = 0;
  uint32_t key[kSortEach], place[kSortEach], rank[kSortEach], out_of_range = 0;
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    place[r] = first + r * 32;
    key[r] = vocab;
    if (place[r] < T) {
      const I id = ids[row + place[r]];
      key[r] = key_of(id, vocab);
      out_of_range += id >= 0 && key[r] == vocab;
    }
  }
  if (bad != nullptr && out_of_range) atomicAdd(bad, out_of_range);
  for (int p = 0; p < plan.passes; ++p) {
    uint32_t total;
    const int shift = p * plan.bits;
    tile_ranks<kSortEach>(s, key, T, shift, plan.bits, rank, &total);
    digit_bases(s, total);
    const bool last = p + 1 == plan.passes;
#pragma unroll
    for (int r = 0; r < kSortEach; ++r)
      if (first + r * 32 < T) {
        const uint32_t d = (key[r] >> shift) & ((1u << plan.bits) - 1u);
        const uint32_t to = s.base[d] + s.count[threadIdx.x >> 5][d] + rank[r];
        if (last) { keys[row + to] = key[r]; places[row + to] = place[r]; }
        else { buf_key[to] = key[r]; buf_place[to] = place[r]; }
      }
    if (last) break;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortEach; ++r)
      if (first + r * 32 < T) { key[r] = buf_key[first + r * 32]; place[r] = buf_place[first + r * 32]; }
    __syncthreads();
  }
}

// One pass over longer rows, first half: how often each digit occurs in each tile, as count[worker][tile][digit].
template <typename I, bool kFirst, int kSortEach>
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const I* ids, const uint32_t* keys, uint32_t T, uint32_t vocab, uint32_t tiles,
                                                                  int shift, int bits, uint32_t* counts, uint32_t* bad, uint32_t* hdr) {
  __shared__ uint32_t count[kBins];
  const uint32_t tile = blockIdx.x;
  const size_t row = (size_t)blockIdx.y * T;
  count[threadIdx.x] = 0;
  __syncthreads();
  grid_dependency_wait();
  if (kFirst && tile + blockIdx.y == 0 && threadIdx.x < kHdrWords) hdr[threadIdx.x] = 0;
  uint32_t out_of_range = 0;
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    const uint32_t at = (tile * kSortEach + r) * kSortThreads + threadIdx.x;
    uint32_t d = kBins;
    if (at < T) {
      uint32_t key;
      if (kFirst) {
        const I id = ids[row + at];
        key = key_of(id, vocab);
        out_of_range += id >= 0 && key == vocab;
      } else {
        key = keys[row + at];
      }
      d = (key >> shift) & ((1u << bits) - 1u);
    }
    const uint32_t peers = __match_any_sync(0xffffffffu, d);       // a common word would serialise its additions
    if (d < kBins && (peers & lanemask_lt()) == 0) atomicAdd(&count[d], __popc(peers));
  }
  if (kFirst && bad != nullptr && out_of_range) atomicAdd(bad, out_of_range);
  __syncthreads();
  counts[((size_t)blockIdx.y * tiles + tile) * kBins + threadIdx.x] = count[threadIdx.x];
}

// second half: every token to its place
template <typename I, bool kFirst, int kSortEach>
__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(const I* ids, const uint32_t* keys, const uint32_t* places, uint32_t T,
                                                                    uint32_t vocab, uint32_t tiles, int shift, int bits, const uint32_t* counts,
                                                                    uint32_t* to_keys, uint32_t* to_places) {
  extern __shared__ char sort_smem[];
  TileSort& s = *reinterpret_cast<TileSort*>(sort_smem);
  const uint32_t tile = blockIdx.x, first = tile * (kSortThreads * kSortEach) + (threadIdx.x >> 5) * (kSortEach * 32) + lane_id();
  const size_t row = (size_t)blockIdx.y * T;
  grid_dependency_wait();
  uint32_t key[kSortEach], place[kSortEach], rank[kSortEach];
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    const uint32_t at = first + r * 32;
    key[r] = vocab; place[r] = at;
    if (at < T) {
      if (kFirst) key[r] = key_of(ids[row + at], vocab);
      else { key[r] = keys[row + at]; place[r] = places[row + at]; }
    }
  }
  uint32_t in_tile;
  tile_ranks<kSortEach>(s, key, min(T - tile * (kSortThreads * kSortEach), (uint32_t)(kSortThreads * kSortEach)), shift, bits, rank, &in_tile);
  const uint32_t* mine = counts + (size_t)blockIdx.y * tiles * kBins + threadIdx.x;
  uint32_t all = 0, before = 0;
#pragma unroll 16
  for (uint32_t k = 0; k < tiles; ++k) {
    const uint32_t c = mine[(size_t)k * kBins];
    all += c;
    before += k < tile ? c : 0u;
  }
  digit_bases(s, all);
  s.base[threadIdx.x] += before;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortEach; ++r)
    if (first + r * 32 < T) {
      const uint32_t d = (key[r] >> shift) & ((1u << bits) - 1u);
      const size_t to = row + s.base[d] + s.count[threadIdx.x >> 5][d] + rank[r];
      to_keys[to] = key[r];
      to_places[to] = place[r];
    }
}

// ------------------------------------------------------------------ sums
struct GradArgs {
  const void* dout;
  long long tok_stride, worker_stride;
  const void* ids;
  int M;
  uint32_t T, vocab, dim, tiles;                   // tiles: of kTileCols columns
  float scale;
  void* grads;
  long long stride;
  int accumulate;
  uint32_t *bad, *hdr;
  const uint32_t *keys, *places;                   // sorted
  uint4* common;                                   // {row, first place, behind the last, worker} of the common tokens, in no order
  uint32_t* common_count;
  float* partial;                                  // [M][chunks][2][pad]: the chunk's sum for the token that enters it / that leaves it
  uint32_t chunk, chunks, pad;
};

template <typename D, int kVec>
__device__ __forceinline__ void add_row(const D* src, uint32_t c0, uint32_t dim, float* acc) {
#pragma unroll
  for (int a = 0; a < kLane / kVec; ++a) {
    if (c0 + a * 32 * kVec >= dim) continue;
    const Pack<D, kVec> x = *reinterpret_cast<const Pack<D, kVec>*>(src + c0 + a * 32 * kVec);
#pragma unroll
    for (int e = 0; e < kVec; ++e) acc[a * kVec + e] += to_f32(x.v[e]);
  }
}

// acc += the rows at places[0 .. n), in that order, four loads under way
template <typename D, int kVec, typename F>
__device__ __forceinline__ void add_rows(const D* base, long long tok_stride, F place, uint32_t n, uint32_t c0, uint32_t dim, float* acc) {
  uint32_t i = 0;
  for (; i + 4 <= n; i += 4) {
    const D* src[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) src[u] = base + (long long)place(i + u) * tok_stride;
#pragma unroll
    for (int a = 0; a < kLane / kVec; ++a) {
      if (c0 + a * 32 * kVec >= dim) continue;
      Pack<D, kVec> x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = *reinterpret_cast<const Pack<D, kVec>*>(src[u] + c0 + a * 32 * kVec);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < kVec; ++e) acc[a * kVec + e] += to_f32(x[u].v[e]);
    }
  }
  for (; i < n; ++i) add_row<D, kVec>(base + (long long)place(i) * tok_stride, c0, dim, acc);
}

template <typename O, int kVec>
__device__ __forceinline__ void put_row(O* to, uint32_t c0, uint32_t dim, const float* acc, float scale, bool accumulate) {
#pragma unroll
  for (int a = 0; a < kLane / kVec; ++a) {
    if (c0 + a * 32 * kVec >= dim) continue;
    O* p = to + c0 + a * 32 * kVec;
    float v[kVec];
    if (accumulate) {
      const Pack<O, kVec> old = *reinterpret_cast<const Pack<O, kVec>*>(p);
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] = __fmaf_rn(scale, acc[a * kVec + e], to_f32(old.v[e]));
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] = __fmul_rn(scale, acc[a * kVec + e]);
    }
    store_pack<O, kVec>(p, v);
  }
}

__device__ __forceinline__ uint32_t lower_bound(const uint32_t* keys, uint32_t lo, uint32_t n, uint32_t key) {
  while (n > 0) {
    const uint32_t half = n / 2;
    if (__ldg(keys + lo + half) < key) { lo += half + 1; n -= half + 1; }
    else n = half;
  }
  return lo;
}

// The same by half a warp, each half for a key of its own: sixteen probes a round, so that 131072 keys take five rounds of
// dependent loads instead of seventeen.
__device__ __forceinline__ uint32_t lower_bound16(const uint32_t* keys, uint32_t n, uint32_t key) {
  const uint32_t lane = lane_id(), sub = lane & 15, shift = lane & 16;
  uint32_t lo = 0;
  while (__any_sync(0xffffffffu, n > 0)) {
    const uint32_t seg = (n + 17) / 17, at = (sub + 1) * seg - 1;              // probes seg apart; n == 0: none is inside
    const bool below = n > 0 && at < n && __ldg(keys + lo + at) < key;
    const uint32_t skip = __popc((__ballot_sync(0xffffffffu, below) >> shift) & 0xffffu) * seg;
    lo += skip;
    n = n > 0 ? min(seg - 1, n - skip) : 0u;
  }
  return lo;
}

// Lane r <= kRows gets the first place of row v0 + r.
__device__ __forceinline__ uint32_t row_bounds(const uint32_t* keys, uint32_t T, uint64_t v0, uint32_t vocab) {
  const uint32_t lane = lane_id();
  const uint32_t end_key = (uint32_t)min(v0 + kRows, (uint64_t)vocab);
  const uint32_t ends = lower_bound16(keys, T, lane < 16 ? (uint32_t)v0 : end_key);
  const uint32_t s = __shfl_sync(0xffffffffu, ends, 0), n = __shfl_sync(0xffffffffu, ends, 16) - s;
  const uint32_t key = (uint32_t)min(v0 + min(lane, (uint32_t)kRows), (uint64_t)vocab);
  if (n > 32) return lower_bound(keys, s, n, key);
  const uint32_t mine = lane < n ? __ldg(keys + s + lane) : vocab;
  uint32_t bound = s;
#pragma unroll
  for (int r = 1; r <= kRows; ++r) {
    const uint32_t below = __popc(__ballot_sync(0xffffffffu, lane < n && mine < (uint32_t)min(v0 + r, (uint64_t)vocab)));
    if (lane >= (uint32_t)r) bound = s + below;
  }
  return bound;
}

// Rows of the table, few tokens: each warp looks through the ids itself.
template <typename D, typename I, typename O, int kVec>
__global__ void __launch_bounds__(kThreads) rows_direct_kernel(GradArgs g) {
  __shared__ uint32_t found[kWarps][kDirectTokens];
  const uint32_t w = threadIdx.x >> 5, lane = lane_id(), m = blockIdx.z, tile = blockIdx.y;
  const uint32_t v0 = (blockIdx.x * kWarps + w) * kRows;
  if (blockIdx.x + tile + m == 0 && threadIdx.x < kHdrWords) g.hdr[threadIdx.x] = 0;
  const I* ids = static_cast<const I*>(g.ids) + (size_t)m * g.T;
  const D* dout = static_cast<const D*>(g.dout) + m * g.worker_stride;
  O* grads = static_cast<O*>(g.grads) + m * g.stride;
  if (v0 >= g.vocab) return;
  uint32_t n = 0, out_of_range = 0, keys[kDirectTokens / 32];
#pragma unroll
  for (int k = 0; k < kDirectTokens / 32; ++k) {                               // all ids under way at once
    const uint32_t t = k * 32 + lane;
    keys[k] = g.vocab;
    if (t >= g.T) continue;
    const I id = ids[t];
    keys[k] = key_of(id, g.vocab);
    out_of_range += id >= 0 && keys[k] == g.vocab;
  }
#pragma unroll
  for (int k = 0; k < kDirectTokens / 32; ++k) {
    if (k * 32 >= g.T) break;
    const bool mine = keys[k] < g.vocab && keys[k] >= v0 && keys[k] < v0 + kRows;
    const uint32_t votes = __ballot_sync(0xffffffffu, mine);
    if (mine) found[w][n + __popc(votes & lanemask_lt())] = (keys[k] - v0) << 16 | (k * 32 + lane);
    n += __popc(votes);
  }
  if (v0 != 0 || tile != 0) out_of_range = 0;                                  // counted once
  if (g.bad != nullptr && out_of_range) atomicAdd(g.bad, out_of_range);
  __syncwarp();
  const uint32_t c0 = tile * kTileCols + lane * kVec;
  for (uint32_t r = 0; r < kRows && v0 + r < g.vocab; ++r) {
    float acc[kLane] = {};
    bool any = false;
    for (uint32_t i = 0; i < n; ++i) {
      const uint32_t f = found[w][i];
      if (f >> 16 != r) continue;
      any = true;
      add_row<D, kVec>(dout + (long long)(f & 0xffffu) * g.tok_stride, c0, g.dim, acc);
    }
    if (any || !g.accumulate) put_row<O, kVec>(grads + (uint64_t)(v0 + r) * g.dim, c0, g.dim, acc, g.scale, g.accumulate);
  }
}

// From the sorted tokens.  blockIdx.x: first the warps that sum chunks of common tokens (the longest work), then the rows.
template <typename D, typename O, int kVec>
__global__ void __launch_bounds__(kThreads) rows_sorted_kernel(GradArgs g, uint32_t chunk_blocks) {
  const uint32_t w = threadIdx.x >> 5, lane = lane_id(), m = blockIdx.z, tile = blockIdx.y;
  const uint32_t* keys = g.keys + (size_t)m * g.T;
  const uint32_t* places = g.places + (size_t)m * g.T;
  const D* dout = static_cast<const D*>(g.dout) + m * g.worker_stride;
  const uint32_t c0 = tile * kTileCols + lane * kVec;
  grid_dependency_wait();
  if (blockIdx.x < chunk_blocks) {
    const uint32_t c = blockIdx.x * kWarps + w;
    if (c >= g.chunks) return;
    const uint32_t begin = c * g.chunk, end = min(begin + g.chunk, g.T);
    // side 0: the token at the chunk's first place; side 1: the one at its last, where that is another
    const uint32_t key0 = keys[begin], key1 = keys[end - 1];
    for (int side = 0; side < 2; ++side) {
      const uint32_t key = side == 0 ? key0 : key1;
      if (key == g.vocab || (side == 1 && key1 == key0)) continue;
      const uint32_t bound = lower_bound16(keys, g.T, key + (lane >> 4));            // first place, and behind the last
      const uint32_t s = __shfl_sync(0xffffffffu, bound, 0), e = __shfl_sync(0xffffffffu, bound, 16);
      if (e - s <= g.chunk) continue;
      const uint32_t from = max(s, begin), n = min(e, end) - from;
      float acc[kLane] = {};
      add_rows<D, kVec>(dout, g.tok_stride, [&](uint32_t i) { return __ldg(places + from + i); }, n, c0, g.dim, acc);
      float* to = g.partial + (((size_t)m * g.chunks + c) * 2 + (s <= begin ? 0 : 1)) * g.pad;
#pragma unroll
      for (int a = 0; a < kLane / kVec; ++a)
        if (c0 + a * 32 * kVec < g.dim) store_pack<float, kVec>(to + c0 + a * 32 * kVec, acc + a * kVec);
    }
    return;
  }
  const uint64_t v0 = ((uint64_t)(blockIdx.x - chunk_blocks) * kWarps + w) * kRows;
  if (v0 >= g.vocab) return;
  O* grads = static_cast<O*>(g.grads) + m * g.stride;
  const uint32_t bound = row_bounds(keys, g.T, v0, g.vocab);
  uint32_t window = __shfl_sync(0xffffffffu, bound, 0);      // 32 places from here on are in the lanes' `place`
  uint32_t place = window + lane < g.T ? __ldg(places + window + lane) : 0u;
  for (uint32_t r = 0; r < kRows && v0 + r < g.vocab; ++r) {
    const uint32_t s = __shfl_sync(0xffffffffu, bound, r), e = __shfl_sync(0xffffffffu, bound, r + 1);
    if (e - s > g.chunk) {
      if (tile == 0 && lane == 0) g.common[atomicAdd(g.common_count, 1u)] = make_uint4((uint32_t)(v0 + r), s, e, m);
      continue;
    }
    if (e == s && g.accumulate) continue;
    float acc[kLane] = {};
    for (uint32_t at = s; at < e; at += 32) {
      const uint32_t n = min(32u, e - at);
      if (at + n > window + 32) {
        window = at;
        place = window + lane < g.T ? __ldg(places + window + lane) : 0u;
      }
      add_rows<D, kVec>(dout, g.tok_stride, [&](uint32_t i) { return __shfl_sync(0xffffffffu, place, at - window + i); }, n, c0, g.dim, acc);
    }
    put_row<O, kVec>(grads + (v0 + r) * g.dim, c0, g.dim, acc, g.scale, g.accumulate);
  }
}

// Common tokens: a CTA for each and 512 columns adds its partial sums, eight runs of them side by side, in ascending order.
template <typename O, int kVec>
__global__ void __launch_bounds__(kThreads) join_kernel(GradArgs g) {
  __shared__ float part[kWarps][kTileCols];
  const uint32_t w = threadIdx.x >> 5, lane = lane_id();
  grid_dependency_wait();
  const uint32_t items = *g.common_count * g.tiles;
  for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint4 common = g.common[item / g.tiles];
    const uint32_t s = common.y, e = common.z, m = common.w;
    const uint32_t c0 = item % g.tiles * kTileCols + lane * kVec;
    const uint32_t from = s / g.chunk, count = (e - 1) / g.chunk - from + 1, each = (count + kWarps - 1) / kWarps;
    float acc[kLane] = {};
    const float* base = g.partial + (size_t)m * g.chunks * 2 * g.pad;
    add_rows<float, kVec>(base, 1, [&](uint32_t i) -> long long {
      const uint32_t k = from + w * each + i;
      return ((long long)k * 2 + (s <= k * g.chunk ? 0 : 1)) * g.pad;
    }, w * each < count ? min(each, count - w * each) : 0u, c0, g.dim, acc);
#pragma unroll
    for (int x = 0; x < kLane; ++x) part[w][x * 32 + lane] = acc[x];
    __syncthreads();
    if (w == 0) {
      for (int k = 1; k < kWarps; ++k)
#pragma unroll
        for (int x = 0; x < kLane; ++x) acc[x] += part[k][x * 32 + lane];
      put_row<O, kVec>(static_cast<O*>(g.grads) + m * g.stride + (uint64_t)common.x * g.dim, c0, g.dim, acc, g.scale, g.accumulate);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ host
bool is_real(int dt) { return dt == S3GD_F32 || dt == S3GD_BF16; }
bool is_index(int dt) { return dt == S3GD_I32 || dt == S3GD_I64; }

template <typename F>
cudaError_t by_real(int dt, F f) { return dt == S3GD_F32 ? f(float()) : f(__nv_bfloat16()); }
template <typename F>
cudaError_t by_index(int dt, F f) { return dt == S3GD_I32 ? f(int32_t()) : f(int64_t()); }
template <int kN> struct Width { static constexpr int value = kN; };
template <typename F>
cudaError_t by_width(int v, F f) { return v == 8 ? f(Width<8>()) : v == 4 ? f(Width<4>()) : v == 2 ? f(Width<2>()) : f(Width<1>()); }

struct GradLayout {
  uint32_t chunk, chunks, pad, sort_tiles;
  bool direct, few;
  size_t off_keys[2], off_places[2], off_counts, off_common, off_partial, total;
};
bool grad_layout(int M, uint64_t T, uint64_t vocab, uint64_t dim, GradLayout* L) {
  if (M < 1 || M > 65535 || vocab == 0 || dim == 0 || vocab >= (1ull << 31) || dim >= (1ull << 31) || T >= (1ull << 31) ||
      (uint64_t)M * T >= (1ull << 31))
    return false;
  L->direct = T <= kDirectTokens && T * vocab <= kDirectWork;
  uint64_t chunk = (T + kMaxChunks - 1) / kMaxChunks;
  L->chunk = (uint32_t)(chunk < kMinChunk ? kMinChunk : chunk);
  L->chunks = (uint32_t)((T + L->chunk - 1) / L->chunk);
  L->pad = (uint32_t)((dim + 7) / 8 * 8);
  L->few = T <= (uint64_t)kFewTiles * kSortThreads * kFewEach;
  const uint64_t tile = kSortThreads * (L->few ? kFewEach : kSortEach);
  L->sort_tiles = (uint32_t)((T + tile - 1) / tile);
  size_t off = align_up(kHdrWords * sizeof(uint32_t), 256);
  if (!L->direct) {
    const size_t list = (size_t)M * T * sizeof(uint32_t);
    for (int i = 0; i < 2; ++i) {
      L->off_keys[i] = off;    off = align_up(off + list, 256);
      L->off_places[i] = off;  off = align_up(off + list, 256);
    }
    // Room that does not shrink where T grows past the point at which tiles or chunks become longer, so that a workspace for
    // many tokens serves fewer.
    const size_t tiles = !L->few && L->sort_tiles < kFewTiles ? kFewTiles : L->sort_tiles;
    const size_t chunks = L->chunk > kMinChunk ? kMaxChunks : L->chunks;
    L->off_counts = off;   off = align_up(off + (size_t)M * kBins * tiles * sizeof(uint32_t), 256);
    L->off_common = off;   off = align_up(off + (size_t)M * chunks * sizeof(uint4), 256);   // each takes more than a chunk
    L->off_partial = off;  off = align_up(off + (size_t)M * chunks * 2 * L->pad * sizeof(float), 256);
  }
  L->total = off;
  return true;
}

template <typename I, int kEach>
cudaError_t sort_passes(const GradArgs& g, const GradLayout& L, const SortPlan& plan, uint32_t** keys, uint32_t** places, uint32_t* counts, int* where,
                        cudaStream_t st) {
  const I* ids = static_cast<const I*>(g.ids);
  const dim3 grid(L.sort_tiles, g.M), block(kSortThreads);
  for (int p = 0; p < plan.passes; ++p) {
    const int from = (p + 1) & 1, to = p & 1, shift = p * plan.bits;
    auto count = p == 0 ? sort_count_kernel<I, true, kEach> : sort_count_kernel<I, false, kEach>;
    auto scatter = p == 0 ? sort_scatter_kernel<I, true, kEach> : sort_scatter_kernel<I, false, kEach>;
    count_launch(2);
    cudaError_t e = launch_after(count, grid, block, 0, st, ids, keys[from], g.T, g.vocab, L.sort_tiles, shift, plan.bits, counts, g.bad, g.hdr);
    if (e != cudaSuccess) return e;
    e = launch_after(scatter, grid, block, sizeof(TileSort), st, ids, keys[from], places[from], g.T, g.vocab, L.sort_tiles, shift, plan.bits, counts,
                     keys[to], places[to]);
    if (e != cudaSuccess) return e;
    *where = to;
  }
  return cudaSuccess;
}

template <typename I>
cudaError_t sort_tokens(const GradArgs& g, const GradLayout& L, char* ws, int* where, cudaStream_t st) {
  const SortPlan plan = sort_plan(g.vocab);
  const I* ids = static_cast<const I*>(g.ids);
  uint32_t *keys[2], *places[2];
  for (int i = 0; i < 2; ++i) {
    keys[i] = reinterpret_cast<uint32_t*>(ws + L.off_keys[i]);
    places[i] = reinterpret_cast<uint32_t*>(ws + L.off_places[i]);
  }
  uint32_t* counts = reinterpret_cast<uint32_t*>(ws + L.off_counts);
  *where = 0;
  if (g.T <= kSortTile) {
    static int done[kMaxDevices];
    const int bytes = (int)sizeof(TileSort) + 2 * kSortTile * 4;
    cudaError_t e = opt_in_dynamic_smem(reinterpret_cast<const void*>(sort_small_kernel<I>), bytes, done);
    if (e != cudaSuccess) return e;
    count_launch();
    return launch_after(sort_small_kernel<I>, dim3(g.M), dim3(kSortThreads), bytes, st, ids, g.T, g.vocab, plan, keys[0], places[0], g.bad, g.hdr);
  }
  return L.few ? sort_passes<I, kFewEach>(g, L, plan, keys, places, counts, where, st) : sort_passes<I, kSortEach>(g, L, plan, keys, places, counts, where, st);
}

cudaError_t enqueue_grad(GradArgs g, const GradLayout& L, int dout_dtype, int ids_dtype, int grads_dtype, char* ws, cudaStream_t st) {
  int vec = widest(g.dim);
  vec = allowed(vec, g.dout, dout_dtype, g.tok_stride, g.M > 1 ? g.worker_stride : 0);
  vec = allowed(vec, g.grads, grads_dtype, g.dim, g.M > 1 ? g.stride : 0);
  const uint32_t row_blocks = (uint32_t)(((uint64_t)g.vocab + kWarps * kRows - 1) / (kWarps * kRows));
  if (L.direct) {
    count_launch();
    return by_real(dout_dtype, [&](auto d) { return by_index(ids_dtype, [&](auto i) { return by_real(grads_dtype, [&](auto o) {
      return by_width(vec, [&](auto v) {
        rows_direct_kernel<decltype(d), decltype(i), decltype(o), decltype(v)::value><<<dim3(row_blocks, g.tiles, g.M), kThreads, 0, st>>>(g);
        return cudaGetLastError();
      }); }); }); });
  }
  int where = 0;
  cudaError_t e = by_index(ids_dtype, [&](auto i) { return sort_tokens<decltype(i)>(g, L, ws, &where, st); });
  if (e != cudaSuccess) return e;
  g.keys = reinterpret_cast<uint32_t*>(ws + L.off_keys[where]);
  g.places = reinterpret_cast<uint32_t*>(ws + L.off_places[where]);
  g.partial = reinterpret_cast<float*>(ws + L.off_partial);
  g.common = reinterpret_cast<uint4*>(ws + L.off_common);
  g.common_count = g.hdr + kHdrCommon;
  const uint32_t chunk_blocks = (L.chunks + kWarps - 1) / kWarps;
  count_launch(2);
  e = by_real(dout_dtype, [&](auto d) { return by_real(grads_dtype, [&](auto o) { return by_width(vec, [&](auto v) {
    return launch_after(rows_sorted_kernel<decltype(d), decltype(o), decltype(v)::value>, dim3(chunk_blocks + row_blocks, g.tiles, g.M),
                        dim3(kThreads), 0, st, g, chunk_blocks);
  }); }); });
  if (e != cudaSuccess) return e;
  const uint64_t most = (uint64_t)g.M * L.chunks * g.tiles, some = 4 * sm_count();
  const uint32_t joins = (uint32_t)(most < some ? most : some);
  return by_real(grads_dtype, [&](auto o) { return by_width(vec, [&](auto v) {
    return launch_after(join_kernel<decltype(o), decltype(v)::value>, dim3(joins), dim3(kThreads), 0, st, g);
  }); });
}

}  // namespace
}  // namespace s3gd

using namespace s3gd;

extern "C" s3gd_status s3gd_embed(const void* table, int table_dtype, int64_t table_stride, uint64_t vocab, uint64_t dim, const void* ids,
                                  int ids_dtype, uint64_t n, float scale, void* out, int out_dtype, int64_t out_stride,
                                  uint32_t* opt_bad_count, void* stream) {
  if (!is_real(table_dtype) || !is_index(ids_dtype) || !is_real(out_dtype)) return S3GD_ERR_INVALID_ARG;
  if (vocab == 0 || dim == 0 || vocab >= (1ull << 31) || dim >= (1ull << 31) || n >= (1ull << 31)) return S3GD_ERR_INVALID_ARG;
  if (table == nullptr || table_stride < (int64_t)dim || out_stride < (int64_t)dim) return S3GD_ERR_INVALID_ARG;
  if (n > 0 && (ids == nullptr || out == nullptr)) return S3GD_ERR_INVALID_ARG;
  if (!is_aligned(table, dtype_bytes(table_dtype)) || !is_aligned(ids, dtype_bytes(ids_dtype)) || !is_aligned(out, dtype_bytes(out_dtype)) ||
      !is_aligned(opt_bad_count, 4))
    return S3GD_ERR_INVALID_ARG;
  const uint64_t blocks = (n * ((dim + kTileCols - 1) / kTileCols) + kWarps - 1) / kWarps;
  if (blocks >= (1ull << 31)) return S3GD_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (opt_bad_count != nullptr && cudaMemsetAsync(opt_bad_count, 0, 4, st) != cudaSuccess) return S3GD_ERR_CUDA;
  if (n == 0) return S3GD_OK;
  int vec = allowed(widest(dim), table, table_dtype, vocab > 1 ? table_stride : 0, 0);
  vec = allowed(vec, out, out_dtype, n > 1 ? out_stride : 0, 0);
  count_launch();
  const cudaError_t e = by_real(table_dtype, [&](auto w) { return by_index(ids_dtype, [&](auto i) { return by_real(out_dtype, [&](auto o) {
    return by_width(vec, [&](auto v) {
      using W = decltype(w); using I = decltype(i); using O = decltype(o);
      lookup_kernel<W, I, O, decltype(v)::value><<<(unsigned)blocks, kThreads, 0, st>>>(
          static_cast<const W*>(table), table_stride, vocab, (uint32_t)dim, static_cast<const I*>(ids), n, scale, static_cast<O*>(out), out_stride,
          opt_bad_count);
      return cudaGetLastError();
    }); }); }); });
  return e == cudaSuccess ? S3GD_OK : S3GD_ERR_CUDA;
}

extern "C" size_t s3gd_embed_grad_workspace_bytes(int M, uint64_t T, uint64_t vocab, uint64_t dim) {
  GradLayout L;
  return grad_layout(M, T, vocab, dim, &L) ? L.total : 0;
}

extern "C" s3gd_status s3gd_embed_grad(const void* dout, int dout_dtype, int64_t dout_stride, int64_t dout_worker_stride, const void* ids,
                                       int ids_dtype, int M, uint64_t T, uint64_t vocab, uint64_t dim, float scale, void* grads,
                                       int grads_dtype, int64_t grads_stride, int accumulate, uint32_t* opt_bad_count, void* ws,
                                       size_t ws_bytes, void* stream) {
  GradLayout L;
  if (!grad_layout(M, T, vocab, dim, &L) || !is_real(dout_dtype) || !is_index(ids_dtype) || !is_real(grads_dtype)) return S3GD_ERR_INVALID_ARG;
  const uint64_t tiles = (dim + kTileCols - 1) / kTileCols;
  if (tiles > 65535) return S3GD_ERR_INVALID_ARG;
  if (grads == nullptr || (M > 1 && (grads_stride < 0 || (uint64_t)grads_stride < vocab * dim))) return S3GD_ERR_INVALID_ARG;
  if (T > 0 && (dout == nullptr || ids == nullptr || dout_stride < 0 || dout_worker_stride < 0)) return S3GD_ERR_INVALID_ARG;
  if (!is_aligned(dout, dtype_bytes(dout_dtype)) || !is_aligned(ids, dtype_bytes(ids_dtype)) || !is_aligned(grads, dtype_bytes(grads_dtype)) ||
      !is_aligned(opt_bad_count, 4))
    return S3GD_ERR_INVALID_ARG;
  if (ws == nullptr || ws_bytes < L.total || !is_aligned(ws, 256)) return S3GD_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (opt_bad_count != nullptr && cudaMemsetAsync(opt_bad_count, 0, 4, st) != cudaSuccess) return S3GD_ERR_CUDA;
  GradArgs g = {};
  g.dout = dout; g.tok_stride = dout_stride; g.worker_stride = dout_worker_stride;
  g.ids = ids; g.M = M; g.T = (uint32_t)T; g.vocab = (uint32_t)vocab; g.dim = (uint32_t)dim; g.tiles = (uint32_t)tiles;
  g.scale = scale; g.grads = grads; g.stride = grads_stride; g.accumulate = accumulate; g.bad = opt_bad_count;
  g.chunk = L.chunk; g.chunks = L.chunks; g.pad = L.pad;
  g.hdr = static_cast<uint32_t*>(ws);
  return enqueue_grad(g, L, dout_dtype, ids_dtype, grads_dtype, static_cast<char*>(ws), st) == cudaSuccess ? S3GD_OK : S3GD_ERR_CUDA;
}
