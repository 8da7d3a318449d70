// The products of the Newton-Schulz steps on the tensor cores.
//
//   S = X X^T          symmetric: only tiles on and below the diagonal are computed, the others are their mirror image
//   B = b S + c S S    symmetric too (S S^T, both operands rows of S)
//   Y = a X + B X      B is its own transpose; X is read along its rows as the second operand (MN-major)
//
// One kernel per product.  Operands are fp16 tiles brought by TMA into slots; one thread issues tcgen05.mma with fp32 sums in
// tensor memory, two sums in turn, and eight warps take the sums out and finish the tile.  wide_kernel: two CTAs share a
// 256 x 256 tile (cta_group::2), each with half of either operand, and go from tile to tile, so that the epilogue of one runs
// under the products of the next.  narrow_kernel: 128 x 128 tiles, each by a cluster of up to eight CTAs that share out k and
// join their sums through distributed shared memory.  launch_product's model of their times chooses, in effect the second where
// its tiles are fewer than SMs.
//
// Precision.  Two fp16 pieces per entry (kSplit, 22 bits): hi hi + hi lo + lo hi, three products.  Or, in steps for which the
// caller asks for it, one (11 bits).
// The tensor cores cut off, rather than round, what falls below the running fp32 sum, which biases a long sum of squares (the
// diagonal of S); with two pieces the sum is therefore taken out of tensor memory every kChunk slots of k and added in
// registers, and the small products go first.
//
// Bounds.  Large: the tensor cores under the power cap; 8192 x 8192 runs five steps in 28.9 to 30.4 ms, 1.08 to 1.14 PFLOP/s of
// three products for each of the m^2 n + m^3 + 2 m^2 n operations a step (a plain bf16 product of the library sustains 1.37 here;
// the tensor pipes are active 64 to 67 % of the cycles at 4096 x 4096); with one piece 9.2 to 10.1 ms.  Tiles of a last round
// that fill half of it or less are cut in two (4 x 2048 x 2048 fp32: 2.09 -> 1.99 ms); a last round between half and full is
// lost time.  Middle: the chain of kernels; a product of 1024 x 1024 takes 12 to 13 us, of which 1.3 pass between two kernels, 1.5
// until the first operands arrive, 5 in the products (bound by L2: 64 KB per CTA and 64 entries of k, 12.6 TB/s over 128 CTAs)
// and 3 to 4 in the epilogue; with one piece 9 us.
#include <atomic>

#include "s3gd_ortho.cuh"
#include "s3gd_tcgen05.cuh"

namespace s3gd {
namespace {

constexpr int kBlockK = 64;                       // entries of k per slot: one 128-byte row
constexpr int kSlotBytes = 32 * 1024;             // 128 rows of each operand
constexpr int kSlots = 5;
constexpr int kChunk = 2;                         // slots of k between two additions in registers, two pieces (4: 5 % faster for
                                                  // large fp32 results, but 1.9e-6 off instead of 1.1e-6 at 1024 x 1024; 1: 20 % slower)
constexpr int kEpiWarps = 8;
constexpr int kEpiBytes = 8 * 1024;               // per epilogue warp: 32 x 64 entries of either piece
constexpr int kImageBytes = 4 * 1024;             // and, wide kernel with two pieces, the mirror image of half of them
constexpr int kThreads = 128 + 32 * kEpiWarps;    // warp 0 loads, warp 1 issues the products; the epilogue begins at warp 4
template <bool kSplit> constexpr int kWideSlots = kSplit ? kSlots - 1 : kSlots;   // the images take the place of one
constexpr int kSmemBytes = 1024 + kSlots * kSlotBytes + kEpiWarps * kEpiBytes + 256;
static_assert(kEpiWarps * kImageBytes <= kSlotBytes, "");
constexpr int kBand = 8;                          // tile rows that are worked on side by side, for reuse in L2

enum Kind : int { kGram = 0, kPoly = 1, kUpdate = 2, kFinal = 3 };

struct ProductArgs {
  CUtensorMap a, b, add, out, mirror;
  Store store;
  uint32_t* hdr;
  int m, n, k, batch;
  int tiles_m, tiles_n, ways;                     // ways: CTAs that share a tile of the narrow kernel
  int whole;                                      // wide kernel: tiles that are not cut in two
  int b_mn;                                       // b is read with k down its rows
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

// Eight entries of row `lane` of a 32-row part (two to a word), as column `lane` of its mirror image: row c of the image is 64
// bytes.  Neighbouring lanes exchange half of their entries so that words are written; odd lanes go through theirs in another
// order, which keeps the two off each other's banks.
__device__ __forceinline__ void mirror8(char* image, int c0, const uint32_t* h) {
  const int lane = lane_id(), odd = lane & 1;
  const uint32_t g0 = __shfl_xor_sync(0xffffffffu, odd ? h[0] : h[2], 1), g1 = __shfl_xor_sync(0xffffffffu, odd ? h[1] : h[3], 1);
  uint32_t* to = reinterpret_cast<uint32_t*>(image + c0 * 64) + (lane >> 1);
  if (!odd) {
    to[0] = __byte_perm(h[0], g0, 0x5410);
    to[16] = __byte_perm(h[0], g0, 0x7632);
    to[32] = __byte_perm(h[1], g1, 0x5410);
    to[48] = __byte_perm(h[1], g1, 0x7632);
  } else {
    to[5 * 16] = __byte_perm(g0, h[2], 0x7632);
    to[4 * 16] = __byte_perm(g0, h[2], 0x5410);
    to[7 * 16] = __byte_perm(g1, h[3], 0x7632);
    to[6 * 16] = __byte_perm(g1, h[3], 0x5410);
  }
}

// ------------------------------------------------------------------ the three roles
// The slots of a CTA.  One piece: a ring of kSlots.  Two pieces: a ring of kHiSlots for the leading pieces of both operands and
// one of the rest for the trailing pieces.
constexpr int kHiSlots = 3;
struct Ring {
  int first, count, slot;
  uint32_t phase;
  __device__ __forceinline__ Ring(int f, int c) : first(f), count(c), slot(f), phase(0) {}
  __device__ __forceinline__ void next() {
    if (++slot == first + count) { slot = first; phase ^= 1; }
  }
};

// Loads slots k of [from, to): 128 rows of the first operand from row_a, and 64 * boxes_b of the second from row_b.
template <int kCta, bool kSplit>
__device__ __forceinline__ bool load_slots(const ProductArgs& P, Shared* sh, uint32_t base, uint32_t rank, int b, int row_a, int row_b, int boxes_b,
                                           int from, int to, Ring* ring) {
  for (int kb = from; kb < to; ++kb)
    for (int piece = 0; piece < (kSplit ? 2 : 1); ++piece) {
      Ring& r = ring[piece];
      if (!mbar_wait(smem_addr(&sh->empty[r.slot]), r.phase ^ 1)) return false;
      uint32_t bar = smem_addr(&sh->full[r.slot]);
      if (rank == 0) mbar_expect_tx(bar, kCta * (16384 + boxes_b * 8192));
      if (kCta == 2) bar = cluster_addr(bar, 0);
      const uint32_t dst = base + r.slot * kSlotBytes;
      const int k0 = kb * kBlockK, z = 2 * b + piece;
      for (int h = 0; h < 2; ++h) tma_load<kCta>(dst + h * 8192, &P.a, k0, row_a + h * 64, z, bar);
      const int xb = P.b_mn ? row_b : k0, yb = P.b_mn ? k0 : row_b;
      tma_load<kCta>(dst + 16384, &P.b, xb, yb, z, bar);    // written out: a loop of a length not known costs 4 % of the large products
      if (boxes_b == 2) tma_load<kCta>(dst + 16384 + 8192, &P.b, P.b_mn ? xb + 64 : xb, P.b_mn ? yb : yb + 64, z, bar);
      r.next();
    }
  return true;
}

// The two sums in tensor memory that take turns.
struct Turn {
  uint32_t sum = 0, phase = 0;
  __device__ __forceinline__ void next() {
    sum ^= 1;
    if (sum == 0) phase ^= 1;
  }
};

// Products of `blocks` slots of k into `columns` columns.  Two pieces: hi lo + lo hi before hi hi, so that fewer additions are cut off at the size of
// the full sum.
template <int kCta, bool kSplit>
__device__ __forceinline__ bool issue_products(Shared* sh, uint32_t base, uint32_t tmem, int blocks, int columns, bool b_mn, Ring* ring,
                                               Turn* turn) {
  constexpr int kTile = 128 * kCta;
  const uint32_t idesc = product_desc(kTile, columns, b_mn), b_next = b_mn ? 8192 : 16, b_step = (b_mn ? 2048 : 32) / 16;
  auto product = [&](uint32_t d, int sa, int sb, bool add) {
    const uint64_t a = operand_desc(base + sa * kSlotBytes), b = operand_desc(base + sb * kSlotBytes + 16384, b_next);
#pragma unroll
    for (int k = 0; k < kBlockK / 16; ++k) mma_f16<kCta>(d, a + 2 * k, b + b_step * k, idesc, add || k > 0);
  };
  for (int kb = 0; kb < blocks;) {
    if (!mbar_wait(smem_addr(&sh->sum_empty[turn->sum]), turn->phase ^ 1)) return false;
    tcgen05_fence_after();
    const uint32_t d = tmem + turn->sum * kTile;
    if (kSplit) {
      const int n = min(kChunk, blocks - kb);
      for (int c = 0; c < n; ++c) {
        const int hi = ring[0].slot, lo = ring[1].slot;
        if (!mbar_wait(smem_addr(&sh->full[hi]), ring[0].phase)) return false;
        if (!mbar_wait(smem_addr(&sh->full[lo]), ring[1].phase)) return false;
        tcgen05_fence_after();
        product(d, hi, lo, c > 0);
        product(d, lo, hi, true);
        mma_commit<kCta>(smem_addr(&sh->empty[lo]));
        product(d, hi, hi, true);
        mma_commit<kCta>(smem_addr(&sh->empty[hi]));
        ring[0].next();
        ring[1].next();
      }
      kb += n;
    } else {
      for (int k = 0; k < blocks; ++k) {
        if (!mbar_wait(smem_addr(&sh->full[ring[0].slot]), ring[0].phase)) return false;
        tcgen05_fence_after();
        product(d, ring[0].slot, ring[0].slot, k > 0);
        mma_commit<kCta>(smem_addr(&sh->empty[ring[0].slot]));
        ring[0].next();
      }
      kb = blocks;
    }
    mma_commit<kCta>(smem_addr(&sh->sum_full[turn->sum]));
    turn->next();
  }
  return true;
}
__host__ __device__ constexpr int sums_of(bool split, int blocks) { return split ? (blocks + kChunk - 1) / kChunk : 1; }

// One epilogue warp's part of `sums` consecutive sums, added up: 32 rows (lanes), kCols columns from `column`.
template <int kTile, int kCols>
__device__ __forceinline__ bool take_sums(Shared* sh, uint32_t tmem, int quad, int column, int sums, const uint32_t* empty_bar, Turn* turn,
                                          float* acc) {
  for (int c = 0; c < sums; ++c) {
    if (!__all_sync(0xffffffffu, mbar_wait(smem_addr(&sh->sum_full[turn->sum]), turn->phase))) return false;
    tcgen05_fence_after();
    const uint32_t at = tmem + ((uint32_t)(quad * 32) << 16) + turn->sum * kTile + column;
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
    if (lane_id() == 0) mbar_arrive_cluster(empty_bar[turn->sum]);
    turn->next();
  }
  return true;
}

// Brings the 32 x 64 entries at (i0, j0) of the matrix that is added into the warp's buffer (one lane).
__device__ __forceinline__ void load_add(const ProductArgs& P, uint32_t buf_addr, uint32_t bar, int b, int i0, int j0) {
  tma_store_wait_read();
  mbar_expect_tx(bar, P.add_pieces * 4096);
  for (int piece = 0; piece < P.add_pieces; ++piece) tma_load<1>(buf_addr + piece * 4096, &P.add, j0, i0, 2 * b + piece, bar);
}

// Eight entries of row i from their sums in x: c_add * what is added (in the buffer at `off`) + c_acc * x, to the caller's matrix
// or, in the place of what was added, as they are stored; and as column c0.. of the mirror image.
__device__ __forceinline__ void finish8(const ProductArgs& P, char* buf, int off, char* image, int image_lo, int c0, bool mirror, int b, int i, int j,
                                        float* x) {
  if (P.kind == kGram) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= P.c_acc;
  } else {
    float add[8];
    read8(buf, buf + 4096, off, P.add_pieces == 2, add);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __fmaf_rn(P.c_add, add[e], __fmul_rn(P.c_acc, x[e]));
  }
  if (P.kind == kFinal) {
    if (P.store.dtype == S3GD_F32) put8<float>(P.store, b, i, j, P.m, P.n, x);
    else put8<__nv_bfloat16>(P.store, b, i, j, P.m, P.n, x);
    return;
  }
  const bool two = P.out_pieces == 2;
  uint32_t hi[4], lo[4];
  split8(x, two, hi, lo);
  *reinterpret_cast<uint4*>(buf + off) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
  if (two) *reinterpret_cast<uint4*>(buf + 4096 + off) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  if (!mirror) return;
  mirror8(image, c0, hi);
  if (two) mirror8(image + image_lo, c0, lo);
}

// Barriers, tensor memory, the wait for the kernel before: the same for both kernels.  Returns the tensor memory's address.
template <int kCta>
__device__ __forceinline__ uint32_t set_up(const ProductArgs& P, Shared* sh, int columns) {
  const int warp = threadIdx.x >> 5;
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
    tmem_alloc<kCta>(smem_addr(&sh->tmem), columns);
    tcgen05_fence_before();
  } else if (warp == 1 && lane_id() == 0) {
    tma_prefetch(&P.a); tma_prefetch(&P.b); tma_prefetch(&P.add); tma_prefetch(&P.out); tma_prefetch(&P.mirror);
  }
  __syncthreads();
  if (kCta == 2) cluster_sync();
  tcgen05_fence_after();
  grid_dependency_wait();
  launch_dependents();
  return sh->tmem;
}
template <int kCta>
__device__ __forceinline__ void tear_down(const ProductArgs& P, bool ok, uint32_t tmem, int columns, bool cluster) {
  if (!ok) {                                                // a wait gave up: say so, let copies in flight land
    atomicOr(&P.hdr[kHdrStatus], (uint32_t)kFlagInternal);
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
  }
  __syncwarp();
  tcgen05_fence_before();
  __syncthreads();
  if (cluster) cluster_sync();
  tcgen05_fence_after();
  if (threadIdx.x < 32) tmem_free<kCta>(tmem, columns);
}

// Many tiles: persistent, two CTAs to a 256 x 256 tile.
template <bool kSplit>
__global__ void __launch_bounds__(kThreads, 1) wide_kernel(const __grid_constant__ ProductArgs P) {
  extern __shared__ char smem_raw[];
  constexpr int kTile = 256, kCols = 128;
  const uint32_t raw = smem_addr(smem_raw);
  const uint32_t base = (raw + 1023) & ~1023u;
  constexpr int kOwnSlots = kWideSlots<kSplit>, kOwnEpi = kEpiBytes + (kSplit ? kImageBytes : 0);
  char* epi = smem_raw + (base - raw) + kOwnSlots * kSlotBytes;
  Shared* sh = reinterpret_cast<Shared*>(epi + kEpiWarps * kOwnEpi);
  const int warp = threadIdx.x >> 5;
  const uint32_t rank = cluster_rank();
  const bool symmetric = P.kind <= kPoly;
  const int tiles = P.batch * (symmetric ? P.tiles_m * (P.tiles_m + 1) / 2 : P.tiles_m * P.tiles_n);
  const int first = blockIdx.x / 2, stride = gridDim.x / 2;
  const int blocks = (P.k + kBlockK - 1) / kBlockK;
  // Tiles beyond P.whole are worked on as two halves of 128 columns each.
  const int items = P.whole + 2 * (tiles - P.whole);
  auto item_at = [&](int t, int* b, int* tm, int* tn, int* column) {
    const int over = t - P.whole;
    tile_at(P, over < 0 ? t : P.whole + over / 2, symmetric, b, tm, tn);
    *column = *tn * kTile + (over < 0 ? 0 : (over & 1) * 128);
    return over < 0 ? kTile : kTile / 2;
  };
  const uint32_t tmem = set_up<2>(P, sh, 512);
  Ring ring[2] = {Ring(0, kSplit ? kOwnSlots / 2 : kOwnSlots), Ring(kOwnSlots / 2, kOwnSlots / 2)};
  Turn turn;
  bool ok = true;
  if (warp == 0) {
    if (lane_id() == 0)
      for (int t = first; t < items && ok; t += stride) {
        int b, tm, tn, column;
        const int columns = item_at(t, &b, &tm, &tn, &column);
        ok = load_slots<2, kSplit>(P, sh, base, rank, b, tm * kTile + (int)rank * 128, column + (int)rank * columns / 2, columns / 128, 0, blocks, ring);
      }
  } else if (warp == 1) {
    if (lane_id() == 0 && rank == 0)
      for (int t = first; t < items && ok; t += stride)
        ok = issue_products<2, kSplit>(sh, base, tmem, blocks, t < P.whole ? kTile : kTile / 2, P.b_mn, ring, &turn);
  } else if (warp >= 4) {
    const int w = warp - 4, quad = warp & 3, half = w >> 2, lane = lane_id();
    char* buf = epi + w * kOwnEpi;
    const uint32_t buf_addr = smem_addr(buf), add_bar = smem_addr(&sh->add_full[w]);
    const uint32_t empty_bar[2] = {cluster_addr(smem_addr(&sh->sum_empty[0]), 0), cluster_addr(smem_addr(&sh->sum_empty[1]), 0)};
    const bool has_add = P.kind != kGram;
    uint32_t add_phase = 0;
    for (int t = first; t < items && ok; t += stride) {
      int b, tm, tn, column;
      const int own = item_at(t, &b, &tm, &tn, &column) / 2;   // columns of this warp
      const int i0 = tm * kTile + (int)rank * 128 + quad * 32, jt = column + half * own;
      const bool here = i0 < P.m && jt < P.n;
      if (has_add && here && lane == 0) load_add(P, buf_addr, add_bar, b, i0, jt);
      const bool mirror = symmetric && tm != tn;
      float acc[kSplit ? kCols : 1];
      if (kSplit) {
        ok = take_sums<kTile, kCols>(sh, tmem, quad, half * own, sums_of(true, blocks), empty_bar, &turn, acc);
      } else {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&sh->sum_full[turn.sum]), turn.phase));
        tcgen05_fence_after();
      }
      if (!ok) break;
      // 32 columns at a time, one copy of the code: the kernels are short and instructions come late
#pragma unroll 1
      for (int s = 0; s < own / 32; ++s) {
        const int j0 = jt + s / 2 * 64, odd = s & 1;
        float v[32];
        if (kSplit) {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = s < 2 ? (odd ? acc[32 + e] : acc[e]) : (odd ? acc[96 + e] : acc[64 + e]);
        } else {
          tmem_load32(tmem + ((uint32_t)(quad * 32) << 16) + turn.sum * kTile + half * own + s * 32, v);
          tmem_load_wait();
          if (s + 1 == own / 32) {
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(empty_bar[turn.sum]);
          }
        }
        if (!here || j0 >= P.n || !ok) continue;
        if (!odd) {                                          // a new 32 x 64 part of the buffer
          if (has_add) {
            if (s > 0 && lane == 0) load_add(P, buf_addr, add_bar, b, i0, j0);
            ok = __all_sync(0xffffffffu, mbar_wait(add_bar, add_phase));
            if (!ok) continue;
            add_phase ^= 1;
          } else {
            if (lane == 0) tma_store_wait_read();
            __syncwarp();
          }
        } else if (kSplit && mirror) {                       // the image's buffer may still be read
          if (lane == 0) tma_store_wait_read();
          __syncwarp();
        }
        // two pieces: both pieces' images of 32 columns behind the buffer; one: they fit in its second half, in turn
        char* image = kSplit ? buf + kEpiBytes : buf + 4096 + odd * 2048;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const int q = odd * 4 + p;
          finish8(P, buf, lane * 128 + ((q ^ (lane & 7)) << 4), image, 2048, p * 8, mirror, b, i0 + lane, j0 + q * 8, v + p * 8);
        }
        if (P.kind == kFinal) {                              // what is added next lands where this was read
          if (odd) {
            fence_async_smem();
            __syncwarp();
          }
          continue;
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (odd)
            for (int piece = 0; piece < P.out_pieces; ++piece) tma_store(&P.out, j0, i0, 2 * b + piece, buf_addr + piece * 4096);
          if (mirror && j0 + odd * 32 < P.n)
            for (int piece = 0; piece < P.out_pieces; ++piece) tma_store(&P.mirror, i0, j0 + odd * 32, 2 * b + piece, smem_addr(image) + piece * 2048);
          tma_store_commit();
        }
      }
      if (!kSplit) turn.next();
    }
    if (lane == 0) tma_store_wait_read();
  }
  tear_down<2>(P, ok, tmem, 512, true);
}

// Few tiles: a cluster of P.ways CTAs takes one 128 x 128 tile, each a part of k.  The eight 32 x 64 parts of the tile are dealt
// over the CTAs.  Every CTA lays its sums into its own shared memory (the slots are free by then) and reads those of its parts
// from all of them, in the order of the parts of k; all eight warps of a CTA finish its parts, eight columns at a time.
// One kernel for all kinds of product and ways, with its epilogue in one short loop: the products of a step follow one another
// within microseconds, and code that is not in the instruction cache costs each of them up to three.
template <bool kSplit>
__global__ void __launch_bounds__(kThreads, 1) narrow_kernel(const __grid_constant__ ProductArgs P) {
  extern __shared__ char smem_raw[];
  constexpr int kTile = 128, kCols = 64;
  const uint32_t raw = smem_addr(smem_raw);
  const uint32_t base = (raw + 1023) & ~1023u;
  char* base_ptr = smem_raw + (base - raw);
  char* epi = base_ptr + kSlots * kSlotBytes;
  Shared* sh = reinterpret_cast<Shared*>(epi + kEpiWarps * kEpiBytes);
  const int warp = threadIdx.x >> 5, ways = P.ways, mine = 8 / ways;     // mine: parts per CTA, and 8-column pieces per warp
  const uint32_t rank = ways > 1 ? cluster_rank() : 0;
  const bool symmetric = P.kind <= kPoly, has_add = P.kind != kGram;
  const int blocks = (P.k + kBlockK - 1) / kBlockK;
  const int from = (int)rank * blocks / ways, to = ((int)rank + 1) * blocks / ways;
  int b, tm, tn;
  tile_at(P, blockIdx.x / ways, symmetric, &b, &tm, &tn);
  const uint32_t tmem = set_up<1>(P, sh, 256);
  const int w = (warp - 4) & 7, quad = warp & 3, lane = lane_id();
  // what this warp finishes: pieces q0 .. q0 + mine of part `part` (ways 1: the part whose sums it holds)
  const int pl = ways == 1 ? quad * 2 + (w >> 2) : w * mine / 8, part = (int)rank * mine + pl, q0 = w * mine % 8;
  const int i0 = tm * kTile + (part >> 1) * 32, j0 = tn * kTile + (part & 1) * kCols;
  const bool here = warp >= 4 && i0 < P.m && j0 < P.n, leads = q0 == 0 && lane == 0;
  char* buf = epi + pl * kEpiBytes;                           // what is added, then the result
  char* side = base_ptr + 8 * 8192 + pl * 8192;               // its mirror image
  const uint32_t buf_addr = smem_addr(buf), add_bar = smem_addr(&sh->add_full[pl]);
  Ring ring[2] = {Ring(0, kSplit ? kHiSlots : kSlots), Ring(kHiSlots, kSlots - kHiSlots)};
  Turn turn;
  bool ok = true;
  if (warp == 0) {
    if (lane == 0) ok = load_slots<1, kSplit>(P, sh, base, 0, b, tm * kTile, tn * kTile, 2, from, to, ring);
  } else if (warp == 1) {
    if (lane == 0) ok = issue_products<1, kSplit>(sh, base, tmem, to - from, kTile, P.b_mn, ring, &turn);
  } else if (warp >= 4) {
    if (has_add && here && leads) load_add(P, buf_addr, add_bar, b, i0, j0);
    const uint32_t empty_bar[2] = {cluster_addr(smem_addr(&sh->sum_empty[0]), rank), cluster_addr(smem_addr(&sh->sum_empty[1]), rank)};
    float acc[kCols];
    ok = take_sums<kTile, kCols>(sh, tmem, quad, (w >> 2) * kCols, sums_of(kSplit, to - from), empty_bar, &turn, acc);
    char* sums = base_ptr + (quad * 2 + (w >> 2)) * 8192 + lane * 16;
#pragma unroll
    for (int q = 0; q < 16; ++q) *reinterpret_cast<float4*>(sums + q * 512) = make_float4(acc[q * 4], acc[q * 4 + 1], acc[q * 4 + 2], acc[q * 4 + 3]);
  }
  if (ways > 1) {
    __syncwarp();
    cluster_sync();
  }
  const bool mirror = symmetric && tm != tn;
  if (here) {
    if (has_add) ok = __all_sync(0xffffffffu, mbar_wait(add_bar, 0)) && ok;
#pragma unroll 1
    for (int q = q0; q < q0 + mine; ++q) {
      float4 got[8][2];
      const uint32_t at = base + (uint32_t)part * 8192u + (uint32_t)q * 1024u + lane * 16;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        if (r >= ways) break;
        const uint32_t from_r = ways > 1 ? cluster_addr(at, r) : at;
#pragma unroll
        for (int l = 0; l < 2; ++l)
          asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                       : "=f"(got[r][l].x), "=f"(got[r][l].y), "=f"(got[r][l].z), "=f"(got[r][l].w) : "r"(from_r + l * 512)
                       : "memory");                           // ways 1: after this lane's own stores above
      }
      float x[8] = {got[0][0].x, got[0][0].y, got[0][0].z, got[0][0].w, got[0][1].x, got[0][1].y, got[0][1].z, got[0][1].w};
#pragma unroll
      for (int r = 1; r < 8; ++r) {
        if (r >= ways) break;
        x[0] += got[r][0].x; x[1] += got[r][0].y; x[2] += got[r][0].z; x[3] += got[r][0].w;
        x[4] += got[r][1].x; x[5] += got[r][1].y; x[6] += got[r][1].z; x[7] += got[r][1].w;
      }
      finish8(P, buf, lane * 128 + ((q ^ (lane & 7)) << 4), side, 4096, q * 8, mirror, b, i0 + lane, j0 + q * 8, x);
    }
  }
  if (ways > 1) {
    __syncwarp();
    cluster_arrive();                                         // the others may go once this CTA has read their sums
  }
  if (here && P.kind != kFinal) {
    fence_async_smem();
    if (ways == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + pl), "r"(32 * ways) : "memory");   // the warps of a part
    if (leads && ok) {
      for (int piece = 0; piece < P.out_pieces; ++piece) {
        tma_store(&P.out, j0, i0, 2 * b + piece, buf_addr + piece * 4096);
        if (!mirror) continue;
        tma_store(&P.mirror, i0, j0, 2 * b + piece, smem_addr(side) + piece * 4096);
        if (j0 + 32 < P.n) tma_store(&P.mirror, i0, j0 + 32, 2 * b + piece, smem_addr(side) + piece * 4096 + 2048);
      }
      tma_store_commit();
      tma_store_wait_read();
    }
  }
  tear_down<1>(P, ok, tmem, 256, false);
  if (ways > 1) {
    __syncwarp();
    cluster_wait();
  }
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

cudaError_t launch_cluster(void (*kernel)(ProductArgs), const ProductArgs& A, unsigned grid, int cluster, int* done, cudaStream_t st) {
  cudaError_t e = opt_in_dynamic_smem(reinterpret_cast<const void*>(kernel), kSmemBytes, done);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
  count_launch();
  return cudaLaunchKernelEx(&cfg, kernel, A);
}

int64_t tiles_of(const ProductArgs& A, int tile) {
  const int64_t tm = (A.m + tile - 1) / tile, tn = (A.n + tile - 1) / tile;
  return A.batch * (A.kind <= kPoly ? tm * (tm + 1) / 2 : tm * tn);
}

// Clusters of `ways` CTAs of this kernel that run at a time (the SMs of a GPC are not always a multiple of it); asked once.
int clusters_at_a_time(void (*kernel)(ProductArgs), int ways, int* cached) {
  int dev = 0;
  const bool keep = cudaGetDevice(&dev) == cudaSuccess && dev >= 0 && dev < kMaxDevices;
  int n = keep ? __atomic_load_n(&cached[dev], __ATOMIC_RELAXED) : 0;
  if (n > 0) return n;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ways);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ways; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n <= 0) n = sm_count() / ways;
  if (keep) __atomic_store_n(&cached[dev], n, __ATOMIC_RELAXED);
  return n;
}

// Which kernel, and over how many CTAs a narrow tile's k is dealt: what takes least time, in units of 0.14 us, by a model of
// the measured times.  A slot of k takes two units for each product of pieces in either kernel (the wide one does four times the
// work in it, on two SMs).  On top come, for every wave of narrow tiles, its start, first loads and epilogue, the pieces that a
// warp finishes, and the joining of parts of k; for the wide kernel, whose epilogues run under products, the start and the last.
// Five steps in us with the choice left to the model | all products wide | narrow with 1, 2, 4, 8 CTAs to a tile, two pieces:
//   256 x 256      109 |  172 |  154  121  108  108        2731 x 1000      367 |  540 |  502  389  537  852
//   512 x 512      123 |  253 |  200  147  123  164        2048 x 2048      629 |  637 |  635  760 1089 1870
//   512 x 4608     184 |  516 |  421  309  333  515        3000 x 3000     1986 | 2085 | 2488 2614 3139 4936
//   1024 x 1024    196 |  351 |  286  197  281  472        12 x 600 x 900   613 |  613 |  705  805 1275 2499
// It takes several waves of narrow tiles for slower than they are where there are two: 1500 x 1500 runs in 469 (wide) and would
// in 382 (narrow, one CTA), 30 x 300 x 300 in 447 and 335.
constexpr int kSlotUnits = 2, kNarrowStart = 40, kWideStart = 76;
constexpr int kJoinUnits[4] = {0, 3, 5, 14};

template <bool kSplit>
cudaError_t launch_product(ProductArgs& A, cudaStream_t st) {
  static int done_wide[kMaxDevices], done_narrow[kMaxDevices], at_a_time[4][kMaxDevices];
  const int pairs = sm_count() / 2, pieces = kSplit ? 3 : 1;
  const int64_t wide = tiles_of(A, 256), narrow = tiles_of(A, 128), blocks = (A.k + kBlockK - 1) / kBlockK;
  // The last round of wide tiles is cut into halves where they fit into one: it takes half as long then.
  const int64_t over = wide % pairs, whole = over * 2 <= pairs ? wide - over : wide;
  int64_t best = (whole / pairs * 2 + (whole % pairs != 0 ? 2 : 0) + (whole < wide ? 1 : 0)) * blocks * pieces * kSlotUnits / 2 + kWideStart;
  A.ways = 0;
  auto kernel = narrow_kernel<kSplit>;
  cudaError_t e = opt_in_dynamic_smem(reinterpret_cast<const void*>(kernel), kSmemBytes, done_narrow);
  if (e != cudaSuccess) return e;
  for (int i = 0; i < 4; ++i) {
    const int ways = 1 << i;
    if (blocks < ways || narrow * ways >= (1ll << 31)) break;
    const int room = ways > 1 ? clusters_at_a_time(kernel, ways, at_a_time[i]) : sm_count();
    const int64_t cost = (narrow + room - 1) / room * (kNarrowStart + 8 / ways + (blocks + ways - 1) / ways * pieces * kSlotUnits + kJoinUnits[i]);
    if (cost < best) { best = cost; A.ways = ways; }
  }
  const int tile = A.ways == 0 ? 256 : 128;
  A.tiles_m = (A.m + tile - 1) / tile;
  A.tiles_n = (A.n + tile - 1) / tile;
  if (A.ways == 0) {
    A.whole = (int)whole;
    const int64_t items = whole + 2 * (wide - whole);
    return launch_cluster(wide_kernel<kSplit>, A, (unsigned)(items < pairs ? items : pairs) * 2, 2, done_wide, st);
  }
  return launch_cluster(kernel, A, (unsigned)(narrow * A.ways), A.ways, done_narrow, st);
}

cudaError_t launch_by(ProductArgs& A, bool split, cudaStream_t st) { return split ? launch_product<true>(A, st) : launch_product<false>(A, st); }

}  // namespace

cudaError_t launch_products(const OrthoPlan& P, const OrthoRequest& R, char* ws, cudaStream_t st) {
  const int m = P.m, n = P.n, planes = 2 * P.batch;
  char* xs[2] = {ws + P.off_x, ws + P.off_y};
  CUtensorMap x_load[2], x_epi[2], s_load, s_epi, s_mirror, b_load, b_epi, b_mirror;
  bool ok = true;
  for (int i = 0; i < 2; ++i)
    ok = ok && make_map(&x_load[i], xs[i], m, n, P.ldx, planes, 64, 64) && make_map(&x_epi[i], xs[i], m, n, P.ldx, planes, 64, 32);
  ok = ok && make_map(&s_load, ws + P.off_s, m, m, P.lds, planes, 64, 64) && make_map(&s_epi, ws + P.off_s, m, m, P.lds, planes, 64, 32) &&
       make_map(&s_mirror, ws + P.off_s, m, m, P.lds, planes, 32, 32) && make_map(&b_load, ws + P.off_b, m, m, P.lds, planes, 64, 64) &&
       make_map(&b_epi, ws + P.off_b, m, m, P.lds, planes, 64, 32) && make_map(&b_mirror, ws + P.off_b, m, m, P.lds, planes, 32, 32);
  if (!ok) return cudaErrorInvalidValue;
  const int carried = carried_steps(R.steps, R.split);
  for (int k = 0; k < R.steps; ++k) {
    const bool split = k < R.split;
    const int from = k & 1;
    ProductArgs A;
    A.hdr = reinterpret_cast<uint32_t*>(ws + P.off_hdr);
    A.batch = P.batch;
    A.store = R.out;
    A.add_pieces = A.out_pieces = split ? 2 : 1;
    A.kind = kGram; A.m = m; A.n = m; A.k = n; A.b_mn = 0;
    A.a = A.b = x_load[from]; A.add = s_epi; A.out = s_epi; A.mirror = s_mirror;
    A.c_add = 0.f; A.c_acc = kScaleS / (kScaleX * kScaleX);
    cudaError_t e = launch_by(A, split, st);
    if (e != cudaSuccess) return e;
    A.kind = kPoly; A.k = m;
    A.a = A.b = s_load; A.add = s_epi; A.out = b_epi; A.mirror = b_mirror;
    A.c_add = R.b * (kScaleB / kScaleS); A.c_acc = R.c * (kScaleB / (kScaleS * kScaleS));
    e = launch_by(A, split, st);
    if (e != cudaSuccess) return e;
    const bool last = k + 1 == R.steps;
    const float unit = last ? 1.f / kScaleX : 1.f;
    A.kind = last ? kFinal : kUpdate; A.n = n; A.k = m; A.b_mn = 1;
    A.a = b_load; A.b = x_load[from]; A.add = x_epi[from]; A.out = x_epi[from ^ 1];
    A.add_pieces = k < carried ? 2 : 1;
    A.out_pieces = k + 1 < carried ? 2 : 1;
    A.c_add = R.a * unit; A.c_acc = unit / kScaleB;
    e = launch_by(A, split, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace s3gd
