// The kernel of the matrix products: tcgen05 with both operands brought to
// shared memory by TMA and the sums in tensor memory.
//
// One block an SM walks over tiles of 128 x 64 results, or a pair of blocks (a
// cluster; their SMs' tensor cores work as one) over tiles of 256 x 256, of which
// each block loads half of either operand and keeps the sums of 128 rows.  Two
// threads load blocks of 64 of the contracted index into a ring of stages, a third
// (in a pair the first block's) multiplies them, and eight or sixteen warps take the sums out
// of tensor memory, two accumulators in turn, so that an epilogue runs beside the
// next tile's products.
//
// Of bf16 products of 8192^3: 578 us, 1900 TFLOP/s (a library product: 541); 503
// without the loads, 665 with four stages: what is left is the loads' latency, for which six stages of 32 KB
// are what fits.  Four blocks that share an operand by TMA multicast: 608, as
// clusters of four leave 8 of 152 SMs idle.
//
// The tensor cores' own sums are rounded towards zero, by up to one unit in the
// last place each 16 products: over thousands of them the error grows past that
// of fp32 sums.  So an accumulator takes `chunk` blocks only; the warps
// add it to sums in registers (128 or 64 a thread), rounded to nearest, while the
// other accumulator fills.  Some 16 blocks (1024 products) where the result has 32 bits
// (12, two for each pair of parts, where the operands have), 32 in f16, 128 in bf16: taking sums out costs the products up
// to a tenth at 8.  An accumulator's pairs of parts come one after another, the smallest first: what is added to a small
// sum loses little, and only the largest pair's steps are rounded at the size of the result (pair by pair at each block, the weight gradient of
// 2048 rows in three parts was off by 1.2e-6 of its norm, so by 3.9e-7; of 777 rows in fp32 by 5.5e-7, so by 1.1e-7).
#pragma once

#include "device_common.cuh"
#include "products.cuh"

namespace dq {

constexpr int kTileRows = 128;
constexpr int kBlockDepth = 64;       // 128 bytes: a row of the 128-byte swizzle

// kWarps: those that take the sums, of a tile of 256 columns.  Sixteen hide more of an epilogue's latencies (8 x 2048 rows of
// 1024 x 4096 with GELU: 114 us, 131 with eight), eight spill less and store from two buffers (without: 95 and 100).
template <int BN, int kWarps = 8>
struct ProductShape {
  static constexpr int kPair = BN == 256 ? 2 : 1;     // blocks that work on a tile
  static constexpr int kRows = kPair * kTileRows;  // of a tile
  static constexpr int kBColumns = BN / kPair;     // of the second operand that a block loads
  static constexpr int kABytes = kTileRows * kBlockDepth * 2;
  static constexpr int kBBytes = kBColumns * kBlockDepth * 2;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kStages = BN == 256 ? 6 : 8;
  // four warps that load and multiply, and those that take the sums: a quarter of the rows and kWidth columns each
  static constexpr int kSumWarps = BN == 256 ? kWarps : 8;
  static constexpr int kThreads = 128 + 32 * kSumWarps;
  static constexpr int kWidth = BN / (kSumWarps / 4);
  static constexpr int kBuffers = 16 / kSumWarps;  // of TurnStore
  // registers of either kind; together at most those that the block is launched with, 96 * 640 or 168 * 384
  static constexpr int kFewRegisters = kSumWarps == 16 ? 56 : 64, kManyRegisters = kSumWarps == 16 ? 104 : 216;
  static_assert(128 * kFewRegisters + 32 * kSumWarps * kManyRegisters <= (65536 / kThreads / 8 * 8) * kThreads, "registers");
  static constexpr int kTurnBytes = 16 * 2048;
  // stages, transposing buffers, barriers; and what it takes to start on a boundary of 1024 bytes
  static constexpr int kSmem = kStages * kStageBytes + kTurnBytes + 256 + 1024;
};

template <int BN, typename Epilogue>
using ShapeOf = ProductShape<BN, Epilogue::kWarps>;

// ---- tcgen05 ----
template <int kPair>
__device__ __forceinline__ void tensor_memory_allocate(uint32_t* to, uint32_t columns) {
  if constexpr (kPair == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(to)), "r"(columns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(to)), "r"(columns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
}
template <int kPair>
__device__ __forceinline__ void tensor_memory_free(uint32_t at, uint32_t columns) {
  if constexpr (kPair == 2)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
  else
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Arrives at `bar` (in a pair, of both blocks) when the products so far are done.
template <int kPair>
__device__ __forceinline__ void tensor_commit(uint64_t* bar) {
  if constexpr (kPair == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                     smem_addr(bar)),
                 "h"((uint16_t)3)
                 : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar))
                 : "memory");
}
template <int kPair>
__device__ __forceinline__ void tensor_multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t kind, bool add) {
  if constexpr (kPair == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(kind), "r"((uint32_t)add)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(kind), "r"((uint32_t)add)
        : "memory");
}
// 32 columns of this warp's 32 lanes: lane l gets row l.  The warp executes it as one.
__device__ __forceinline__ void tensor_load32(uint32_t at, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
        "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
        "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(at));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// The address of the pair's first block's object at the place of this block's.
__device__ __forceinline__ uint32_t first_block(const void* p) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(smem_addr(p)));
  return at;
}
__device__ __forceinline__ uint32_t block_in_pair() {
  uint32_t rank;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  return rank;
}
__device__ __forceinline__ void pair_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A box into this block's shared memory, counted by the barrier at `bar` (shared::cluster: a pair's is the first block's).
template <int kPair>
__device__ __forceinline__ void tma_load_4d(uint32_t to, const void* tmap, int32_t x, int32_t y, int32_t z, int32_t w,
                                            uint32_t bar) {
  if constexpr (kPair == 2)
    asm volatile(
        "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
            to),
        "l"(tmap), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
            to),
        "l"(tmap), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
        : "memory");
}

// Shared-memory descriptor of an operand's 16 (contracted) x 64... slice with the 128-byte swizzle.  Rows along the
// contracted index: 8 rows are 1024 bytes apart from the next 8.  Rows across it: 8 of the contracted index are 1024
// bytes apart from the next 8, and 64 of the other index 64 * 128 bytes from the next 64.
__device__ __forceinline__ uint64_t operand_descriptor(uint32_t at, bool across) {
  const uint64_t lead = across ? (kBlockDepth * 128) >> 4 : 1;
  return (uint64_t)((at & 0x3ffff) >> 4) | lead << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// What a warp has ready of its 32 rows, 64 bytes of a row at a time, goes through shared memory and from there by TMA.
// Lane l holds row l; its packs of 16 bytes stand in the order of the 64-byte swizzle, in which eight lanes' packs meet in
// no bank.  Rows outside the matrix are not written, and columns by 16 bytes.
template <int kBuffers>
struct TurnStore {
  uint8_t* buffer;  // kBuffers x 2048 bytes, used in turn
  int lane;
  uint32_t n = 0;

  __device__ __forceinline__ void put(const uint4 (&packs)[4], const CUtensorMap* map, int column, int row, int worker, int part) {
    uint8_t* const to = buffer + (n % kBuffers) * 2048;
    ++n;
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kBuffers - 1) : "memory");
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c) *reinterpret_cast<uint4*>(to + lane * 64 + ((c ^ (lane / 2 & 3)) * 16)) = packs[c];
    fence_proxy_async_shared();
    __syncwarp();
    if (lane == 0) {
      asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%1, %2, %3, %4}], [%5];" ::"l"(map), "r"(column),
                   "r"(row), "r"(worker), "r"(part), "r"(smem_addr(to))
                   : "memory");
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }

  // 32 columns as T
  template <typename T>
  __device__ __forceinline__ void put32(const float (&x)[32], const CUtensorMap* map, int column, int row, int worker) {
    constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < 32; i += 4 * E) {
      uint4 packs[4];
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int e = 0; e < E; e += 2) set_pair<T>(packs[c], e, make_float2(x[i + c * E + e], x[i + c * E + e + 1]));
      put(packs, map, column + i, row, worker, 0);
    }
  }

  // Single values, for matrices that TMA cannot write (of two buffers): 32 columns that lane r holds of row r; then column l
  // of any row.  No two of the packs that a warp writes or the values that it reads at once meet in a bank.
  __device__ __forceinline__ void turn(const float* x) {
    static_assert(kBuffers == 2, "32 x 32 values");
    float* const to = reinterpret_cast<float*>(buffer);
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 8; ++c)
      *reinterpret_cast<float4*>(to + lane * 32 + (c ^ (lane & 7)) * 4) = make_float4(x[4 * c], x[4 * c + 1], x[4 * c + 2], x[4 * c + 3]);
    __syncwarp();
  }
  __device__ __forceinline__ float turned(int r) const {
    return reinterpret_cast<const float*>(buffer)[r * 32 + ((lane / 4) ^ (r & 7)) * 4 + (lane & 3)];
  }
};

struct ProductTile {
  int worker;
  int64_t row, column;  // of the tile's first result
  int begin, end;       // blocks of the contracted index
  int64_t piece;        // of a split tile: its place among all pieces; else -1
};

// Item t of the walk: the whole tiles, then the pieces of the split ones.
template <int BN>
__device__ __forceinline__ ProductTile product_tile(const ProductArgs& p, int64_t t) {
  ProductTile tile;
  int piece = 0, pieces = 1;
  tile.piece = -1;
  if (t >= p.whole) {
    tile.piece = t - p.whole;
    pieces = p.pieces;
    piece = (int)(tile.piece % pieces);
    t = p.whole + tile.piece / pieces;
  }
  const int per_worker = p.tiles_m * p.tiles_n;
  tile.worker = (int)(t / per_worker);
  const int in = (int)(t - (int64_t)tile.worker * per_worker);
  // eight rows of tiles at a time: what runs at once shares operands in L2
  constexpr int kGroup = 8;
  const int group = in / (kGroup * p.tiles_n), left = in - group * kGroup * p.tiles_n;
  const int high = p.tiles_m - group * kGroup < kGroup ? p.tiles_m - group * kGroup : kGroup;
  tile.row = (int64_t)(group * kGroup + left % high) * ProductShape<BN>::kRows;
  tile.column = (int64_t)(left / high) * BN;
  tile.begin = (int)((int64_t)p.kblocks * piece / pieces);
  tile.end = (int)((int64_t)p.kblocks * (piece + 1) / pieces);
  return tile;
}

// Items of a product: whole tiles, and pieces.
__host__ __device__ inline int64_t product_items(const ProductArgs& p) {
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n * p.workers;
  return p.whole + (tiles - p.whole) * p.pieces;
}

// Where a warp keeps its sums of a piece: four columns of 32 rows after another.
template <typename S>
__device__ __forceinline__ float4* piece_sums(const ProductArgs& p, int64_t piece, int rank, int warp, int lane) {
  return reinterpret_cast<float4*>(p.partial) + ((piece * S::kPair + rank) * S::kSumWarps + warp) * (8 * S::kWidth) + lane;
}

template <int BN, typename Epilogue>
__global__ void __launch_bounds__(ShapeOf<BN, Epilogue>::kThreads, 1) product_kernel(const __grid_constant__ ProductArgs p) {
  dq_pdl_enter();
  using S = ShapeOf<BN, Epilogue>;
  constexpr int kPair = S::kPair;
  extern __shared__ __align__(1024) uint8_t raw[];
  uint8_t* const smem = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
  uint8_t* const turn = smem + S::kStages * S::kStageBytes;
  uint64_t* const full = reinterpret_cast<uint64_t*>(smem + S::kStages * S::kStageBytes + S::kTurnBytes);
  uint64_t* const empty = full + S::kStages;
  uint64_t* const sum_full = empty + S::kStages;
  uint64_t* const sum_empty = sum_full + 2;
  uint32_t* const at_shared = reinterpret_cast<uint32_t*>(sum_empty + 2);
  static_assert((2 * S::kStages + 4) * 8 + 4 <= 256, "barriers");
  constexpr uint32_t kColumns = 2 * BN;

  const int warp = (int)threadIdx.x / 32, lane = (int)threadIdx.x & 31;
  const int rank = kPair == 2 ? (int)block_in_pair() : 0;
  if (threadIdx.x == 0) {
    // full and sum_empty of a pair's first block count for both; empty and sum_full are each block's own
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(sum_full + s, 1);
      mbar_init(sum_empty + s, S::kSumWarps * kPair);
    }
    mbar_fence_init();
  }
  __syncwarp();
  if (warp == 2) tensor_memory_allocate<kPair>(at_shared, kColumns);
  tensor_fence_before();
  __syncthreads();
  if constexpr (kPair == 2) pair_barrier();
  tensor_fence_after();
  const uint32_t sums = *at_shared;

  const int64_t tiles = product_items(p);
  const int64_t first = blockIdx.x / S::kPair, step = gridDim.x / S::kPair;
  const int terms = p.terms.count;
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kFewRegisters));
    if ((warp == 0 || warp == 3) && lane == 0) {
      // One thread loads A, another B: a stage is 512 clocks of the tensor cores, and one thread that issues all of its
      // loads takes longer (8192^3: 655 us).
      const bool is_a = warp == 0;
      const CUtensorMap* const map = is_a ? &p.a : &p.b;
      const bool across = is_a ? p.a_across : p.b_across, one_matrix = is_a ? p.a_shared : p.b_shared;
      const bool counts = is_a && rank == 0;  // announces the stage's bytes
      const int offset = rank * (is_a ? kTileRows : S::kBColumns);
      const bool two = across && (is_a ? kTileRows : S::kBColumns) > 64;  // boxes of 64 x 64
      const uint32_t bars = kPair == 2 ? first_block(full) : smem_addr(full);
      const uint32_t base = smem_addr(smem) + (is_a ? 0 : S::kABytes);
      uint32_t s = 0, phase = 1, n = 0;  // stage, what to wait for, stages filled so far
      bool ok = true;
      for (int64_t t = first; ok && t < tiles; t += step) {
        const ProductTile tile = product_tile<BN>(p, t);
        const int worker = one_matrix ? 0 : tile.worker;
        const int at = (int)(is_a ? tile.row : tile.column) + offset;
        for (int begin = tile.begin; ok && begin < tile.end; begin += p.group) {
          const int end = (begin + p.group < tile.end ? begin + p.group : tile.end) * kBlockDepth;
          for (int term = 0; ok && term < terms; ++term) {
            const int part = is_a ? p.terms.a[term] : p.terms.b[term];
            for (int k = begin * kBlockDepth; k < end; k += kBlockDepth) {
              if (!(ok = mbar_wait_bounded(empty + s, phase, p.err))) break;
              if (counts) mbar_arrive_expect_tx(full + s, kPair * S::kStageBytes);
              const uint32_t to = base + s * S::kStageBytes, bar = bars + s * 8;
              const int x = across ? at : k, y = across ? k : at;
              tma_load_4d<kPair>(to, map, x, y, worker, part, bar);
              if (two) tma_load_4d<kPair>(to + 8192, map, x + 64, y, worker, part, bar);
              ++n;
              if (++s == S::kStages) s = 0, phase ^= 1;
            }
          }
        }
      }
      // what is still on its way into shared memory (of a pair, both blocks') arrives before the block ends
      if (counts)
        for (uint32_t i = n > S::kStages ? n - S::kStages : 0; i < n; ++i)
          mbar_wait_bounded(full + i % S::kStages, i / S::kStages & 1, p.err);
    } else if (warp == 1 && lane == 0 && rank == 0) {
      // D in fp32 | type and direction of A and B | N / 8 | M / 16
      const uint32_t kind = 1u << 4 | (p.half ? 0u : 1u << 7 | 1u << 10) | (uint32_t)p.a_across << 15 |
                            (uint32_t)p.b_across << 16 | (uint32_t)(BN / 8) << 17 | (uint32_t)(S::kRows / 16) << 24;
      const uint64_t da = operand_descriptor(smem_addr(smem), p.a_across);
      const uint64_t db = operand_descriptor(smem_addr(smem + S::kABytes), p.b_across);
      const uint32_t step_a = p.a_across ? 2048 >> 4 : 32 >> 4, step_b = p.b_across ? 2048 >> 4 : 32 >> 4;
      uint32_t s = 0, phase = 0, n = 0, c = 0;  // stage, what to wait for, stages used, accumulators filled
      const int chunk = p.chunk;
      bool ok = true;
      for (int64_t t = first; ok && t < tiles; t += step) {
        const ProductTile tile = product_tile<BN>(p, t);
        for (int left = (tile.end - tile.begin) * terms; ok && left > 0; left -= chunk, ++c) {
          const uint32_t d = sums + (c & 1) * BN;
          if (!(ok = mbar_wait_bounded(sum_empty + (c & 1), (c / 2 & 1) ^ 1, p.err))) break;
          tensor_fence_after();
          const int count = left < chunk ? left : chunk;
          for (int i = 0; i < count; ++i, ++n) {
            if (!(ok = mbar_wait_bounded(full + s, phase, p.err))) break;
            tensor_fence_after();
            const uint64_t at = (uint64_t)(s * (S::kStageBytes >> 4));
#pragma unroll
            for (int k = 0; k < kBlockDepth / 16; ++k)
              tensor_multiply<kPair>(d, da + at + k * step_a, db + at + k * step_b, kind, i > 0 || k > 0);
            tensor_commit<kPair>(empty + s);
            if (++s == S::kStages) s = 0, phase ^= 1;
          }
          if (ok) tensor_commit<kPair>(sum_full + (c & 1));
        }
      }
      // the products end before the block does
      for (uint32_t i = n > S::kStages ? n - S::kStages : 0; i < n; ++i)
        mbar_wait_bounded(empty + i % S::kStages, i / S::kStages & 1, p.err);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kManyRegisters));
    const int sub = warp & 3, slice = (warp - 4) / 4;
    TurnStore<S::kBuffers> store{turn + (warp - 4) * (S::kTurnBytes / S::kSumWarps), lane};
    uint32_t c = 0;
    bool ok = true;
    for (int64_t t = first; ok && t < tiles; t += step) {
      const ProductTile tile = product_tile<BN>(p, t);
      const int total = (tile.end - tile.begin) * terms;
      float v[S::kWidth];
#pragma unroll
      for (int i = 0; i < S::kWidth; ++i) v[i] = 0.f;
      for (int done = 0; done < total; done += p.chunk, ++c) {
        // each lane polls for itself, and all go on or none: what follows is executed by whole warps
        if (!(ok = __all_sync(kFullMask, mbar_wait_bounded(sum_full + (c & 1), c / 2 & 1, p.err)))) break;
        __syncwarp();
        tensor_fence_after();
        const uint32_t from = sums + ((uint32_t)(32 * sub) << 16) + (c & 1) * BN + slice * S::kWidth;
#pragma unroll
        for (int i = 0; i < S::kWidth; i += 32) {
          uint32_t x[32];
          tensor_load32(from + i, x);
#pragma unroll
          for (int j = 0; j < 32; ++j) v[i + j] = __fadd_rn(v[i + j], __uint_as_float(x[j]));
        }
        tensor_fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (kPair == 2)
            asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(
                             first_block(sum_empty + (c & 1)))
                         : "memory");
          else
            mbar_arrive(sum_empty + (c & 1));
        }
      }
      if (!ok) break;
      if (tile.piece >= 0) {
        float4* const to = piece_sums<S>(p, tile.piece, rank, warp - 4, lane);
#pragma unroll
        for (int j = 0; j < S::kWidth / 4; ++j) to[32 * j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
      } else {
        Epilogue::template run<BN>(p, tile, tile.row + rank * kTileRows + 32 * sub, tile.column + slice * S::kWidth, v, store);
      }
      __syncwarp();  // lanes whose rows are outside the matrix may come first
    }
    bulk_wait_all();
  }
  __syncwarp();  // the single threads' lanes
  tensor_fence_before();
  __syncthreads();
  if constexpr (kPair == 2) pair_barrier();
  tensor_fence_after();
  if (warp == 2) tensor_memory_free<kPair>(sums, kColumns);
}

// The pieces' sums of the split tiles in order, and what is done with them.  A warp for each of the
// tile's, two to a block.
template <int BN, typename Epilogue>
__global__ void __launch_bounds__(64) join_kernel(const __grid_constant__ ProductArgs p) {
  dq_pdl_enter();
  using S = ShapeOf<BN, Epilogue>;
  constexpr int kBlocks = S::kPair * S::kSumWarps / 2;  // of a tile
  __shared__ __align__(1024) uint8_t turn[2 * 2048 * S::kBuffers];
  const int in = (int)(blockIdx.x % kBlocks) * 2 + (int)threadIdx.x / 32, lane = (int)threadIdx.x & 31;
  const int rank = in / S::kSumWarps, warp = in % S::kSumWarps;
  const int64_t first = (int64_t)(blockIdx.x / kBlocks) * p.pieces;
  const ProductTile tile = product_tile<BN>(p, p.whole + first);
  float v[S::kWidth];
#pragma unroll
  for (int i = 0; i < S::kWidth; ++i) v[i] = 0.f;
  for (int piece = 0; piece < p.pieces; ++piece) {
    const float4* const from = piece_sums<S>(p, first + piece, rank, warp, lane);
#pragma unroll
    for (int j = 0; j < S::kWidth / 4; ++j) {
      const float4 x = from[32 * j];
      v[4 * j] = __fadd_rn(v[4 * j], x.x);
      v[4 * j + 1] = __fadd_rn(v[4 * j + 1], x.y);
      v[4 * j + 2] = __fadd_rn(v[4 * j + 2], x.z);
      v[4 * j + 3] = __fadd_rn(v[4 * j + 3], x.w);
    }
  }
  TurnStore<S::kBuffers> store{turn + threadIdx.x / 32 * (2048 * S::kBuffers), lane};
  Epilogue::template run<BN>(p, tile, tile.row + rank * kTileRows + 32 * (warp & 3), tile.column + warp / 4 * S::kWidth, v, store);
  bulk_wait_all();
}

// Host: the tensor map of an operand.  Boxes of 64 of the contracted index and a block's `tile` rows, or of 64 x 64.
inline bool encode_operand(const ProductOperand& o, int64_t rows, int64_t depth, int32_t workers, int tile, CUtensorMap* out) {
  const TensorMapEncoder encode = tensor_map_encoder();
  if (!encode) return false;
  const int batches = o.shared ? 1 : workers;
  const auto stride = [&](int64_t s, int count) { return (cuuint64_t)(count > 1 ? s : o.ld) * 2; };
  const cuuint64_t dims[4] = {(cuuint64_t)(o.across ? rows : depth), (cuuint64_t)(o.across ? depth : rows),
                              (cuuint64_t)batches, (cuuint64_t)o.parts};
  const cuuint64_t strides[3] = {(cuuint64_t)o.ld * 2, stride(o.batch, batches), stride(o.part, o.parts)};
  const cuuint32_t boxes[4] = {64u, (cuuint32_t)(o.across ? 64 : tile), 1u, 1u};
  const cuuint32_t steps[4] = {1u, 1u, 1u, 1u};
  return encode(out, o.half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
                const_cast<void*>(o.data), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Results that TMA cannot write (product_rows.cu).
template <int BN>
cudaError_t launch_product_rows(const ProductArgs& args, cudaStream_t stream, uint64_t* launches);

// Host: the tensor map of a matrix that is stored, [parts][workers][rows][columns], in boxes of 64 bytes of 32 rows.
inline bool encode_result(void* data, int32_t dtype, int64_t columns, int64_t rows, int32_t workers, int32_t parts, int64_t ld,
                          int64_t batch, int64_t part, CUtensorMap* out) {
  const TensorMapEncoder encode = tensor_map_encoder();
  if (!encode) return false;
  const int64_t size = dtype == DQGAN_F32 ? 4 : 2;
  const auto stride = [&](int64_t s, int count) { return (cuuint64_t)((count > 1 ? s : ld) * size); };
  const cuuint64_t dims[4] = {(cuuint64_t)columns, (cuuint64_t)rows, (cuuint64_t)workers, (cuuint64_t)parts};
  const cuuint64_t strides[3] = {(cuuint64_t)(ld * size), stride(batch, workers), stride(part, parts)};
  const cuuint32_t boxes[4] = {(cuuint32_t)(64 / size), 32u, 1u, 1u};
  const cuuint32_t steps[4] = {1u, 1u, 1u, 1u};
  const CUtensorMapDataType type = dtype == DQGAN_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == DQGAN_F16  ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                         : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  return encode(out, type, 4, data, dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
                CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Fills what the kernel needs of a product; false where its sizes are beyond the kernel's.
template <int BN>
inline bool product_args(const Product& p, int chunk, uint32_t* err, ProductArgs* out) {
  out->rows = p.rows;
  out->columns = p.columns;
  out->workers = p.workers;
  out->kblocks = (int32_t)ceil_div(p.depth, kBlockDepth);
  out->group = chunk / p.terms.count;
  out->chunk = out->group * p.terms.count;
  out->tiles_m = (int32_t)ceil_div(p.rows, ProductShape<BN>::kRows);
  out->tiles_n = (int32_t)ceil_div(p.columns, BN);
  out->terms = p.terms;
  out->a_across = p.a.across;
  out->b_across = p.b.across;
  out->a_shared = p.a.shared;
  out->b_shared = p.b.shared;
  out->half = p.a.half;
  out->err = err;
  out->whole = (int64_t)out->tiles_m * out->tiles_n * p.workers;
  out->pieces = 1;
  return p.rows <= INT32_MAX && p.columns <= INT32_MAX && p.depth <= INT32_MAX &&
         (int64_t)out->tiles_m * out->tiles_n <= INT32_MAX &&
         encode_operand(p.a, p.rows, p.depth, p.workers, kTileRows, &out->a) &&
         encode_operand(p.b, p.columns, p.depth, p.workers, ProductShape<BN>::kBColumns, &out->b);
}

// Tiles that the device works on at once.
template <int BN, typename Epilogue>
inline cudaError_t product_slots(int* slots) {
  static std::atomic<int> kept[kKeptDevices];
  using S = ShapeOf<BN, Epilogue>;
  if (S::kPair == 1) return resident_ctas(product_kernel<BN, Epilogue>, S::kThreads, S::kSmem, S::kSmem, kept, slots);
  int dev = 0;
  cudaError_t st = cudaGetDevice(&dev);
  if (st != cudaSuccess) return st;
  if (dev < 0 || dev >= kKeptDevices) return cudaErrorInvalidDevice;
  *slots = kept[dev].load(std::memory_order_acquire);
  if (*slots != 0) return cudaSuccess;
  if ((st = cudaFuncSetAttribute(product_kernel<BN, Epilogue>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem)) !=
      cudaSuccess)
    return st;
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = S::kPair;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  lc.gridDim = dim3(S::kPair * 1024);
  lc.blockDim = dim3(S::kThreads);
  lc.dynamicSmemBytes = S::kSmem;
  lc.attrs = attr;
  lc.numAttrs = 1;
  int clusters = 0;
  if ((st = cudaOccupancyMaxActiveClusters(&clusters, product_kernel<BN, Epilogue>, &lc)) != cudaSuccess) return st;
  if (clusters < 1) return cudaErrorInvalidConfiguration;
  *slots = clusters;
  kept[dev].store(clusters, std::memory_order_release);
  return cudaSuccess;
}

template <int BN, typename Epilogue>
inline cudaError_t launch_product(const ProductArgs& p, cudaStream_t stream, uint64_t* launches) {
  using S = ShapeOf<BN, Epilogue>;
  int slots = 0;
  cudaError_t st = product_slots<BN, Epilogue>(&slots);
  if (st != cudaSuccess) return st;
  const int64_t items = product_items(p);
  const int grid = (int)(items < slots ? items : slots) * S::kPair;
  ++*launches;
  st = launch_pdl_cluster(product_kernel<BN, Epilogue>, S::kPair, dim3(grid), dim3(S::kThreads), S::kSmem, stream, p);
  const int64_t split = (int64_t)p.tiles_m * p.tiles_n * p.workers - p.whole;
  if (st != cudaSuccess || split == 0) return st;
  ++*launches;
  return launch_pdl(join_kernel<BN, Epilogue>, dim3((unsigned)(split * S::kPair * S::kSumWarps / 2)), dim3(64), 0, stream, p);
}

}  // namespace dq
