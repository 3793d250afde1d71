// Embedding lookup with scaling, and its gradient over the tokens sorted by id.
//
//   y_i = scale table[id_i];   dtable[v] = scale sum over i with id_i = v of dy_i
//
// Both are bound by memory: a row of the table (or of dy) read and one written
// per token, one operation a value; the gradient also writes every row of
// the table's gradient that no token fell on, which is most of its traffic
// where the vocabulary is larger than the batch.
#include "device_common.cuh"
#include "operators.cuh"

namespace dq {
namespace {

// The place's id, or the vocabulary where it holds no token.
__device__ __forceinline__ int32_t token_at(const EmbeddingArgs& a, int64_t i) {
  if (a.token_bits == 32) {
    const int32_t id = static_cast<const int32_t*>(a.ids)[i];
    return (uint32_t)id < (uint32_t)a.vocab ? id : (int32_t)a.vocab;
  }
  const int64_t id = static_cast<const int64_t*>(a.ids)[i];
  return (uint64_t)id < (uint64_t)a.vocab ? (int32_t)id : (int32_t)a.vocab;
}

// ---------------------------------------------------------------------------
// Forward: `lanes` threads take a row, each kAtOnce pieces of it at once: 16 bytes
// of y (kVec: rows of table and y are aligned for that) or one value; the next row's
// id is on its way meanwhile.  8 x 4096 rows of 1024 fp32 values to bf16: 23 us, 87 %
// of 6694.5 GB/s; of 1023 (single values) 49 us, from a bf16 table 61 us (41 %, 25 %).
// ---------------------------------------------------------------------------
constexpr int kForwardThreads = 256;
// 8 x 4096 rows of 1023 values: 49 us with 8 single fp32 values at once, 57 with 4; bf16 ones 76 and 61
constexpr int at_once(bool vec, int size) { return vec || size == 2 ? 4 : 8; }

template <typename E, typename T, bool kVec>
__global__ void __launch_bounds__(kForwardThreads) embedding_forward_kernel(EmbeddingArgs a, int lanes) {
  dq_pdl_enter();
  constexpr int N = kVec ? 16 / (int)sizeof(T) : 1, kAtOnce = at_once(kVec, (int)sizeof(E));  // values of a piece, pieces
  constexpr int kWords = (N * (int)sizeof(E) + 7) / 8;                       // of the table, in 8 bytes
  const int lane = threadIdx.x % lanes, groups = kForwardThreads / lanes;
  const int64_t all = a.tokens * a.workers, stride = (int64_t)gridDim.x * groups;
  const auto id_at = [&](int64_t i) { return i < all ? token_at(a, i) : (int32_t)a.vocab; };
  int64_t i = (int64_t)blockIdx.x * groups + threadIdx.x / lanes;
  int32_t next_id = id_at(i);
  for (; i < all; i += stride) {
    const int32_t id = next_id;
    const bool live = id < a.vocab;
    next_id = id_at(i + stride);  // on its way while this row is
    const E* row = static_cast<const E*>(a.table) +
                   (live ? (int64_t)((uint32_t)i / (uint32_t)a.tokens) * a.p_stride + (int64_t)id * a.width : 0);
    T* y = static_cast<T*>(a.y) + i * a.ld;
    for (int c0 = lane * N; c0 < a.width; c0 += lanes * N * kAtOnce) {
      uint2 p[kAtOnce][kWords];
      float single[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int c = c0 + k * lanes * N;
        if (!live || c >= a.width) continue;
        if constexpr (!kVec) {
          single[k] = to_float(row[c]);
        } else if constexpr (kWords == 1) {
          p[k][0] = *reinterpret_cast<const uint2*>(row + c);
        } else {
#pragma unroll
          for (int w = 0; w < kWords; w += 2) {
            const uint4 q = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(row + c) + 8 * w);
            p[k][w] = make_uint2(q.x, q.y);
            p[k][w + 1] = make_uint2(q.z, q.w);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int c = c0 + k * lanes * N;
        if (c >= a.width) continue;
        if constexpr (!kVec) {
          y[c] = from_float<T>(live ? single[k] * a.scale : 0.f);
        } else {
          uint4 q;
#pragma unroll
          for (int e = 0; e < N; ++e)
            reinterpret_cast<T*>(&q)[e] = from_float<T>(live ? to_float(reinterpret_cast<const E*>(p[k])[e]) * a.scale : 0.f);
          __stcs(reinterpret_cast<uint4*>(y + c), q);
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Backward, in three kernels:
//   1. a cluster of blocks per worker sorts its places by id, the places of an id in
//      order, while the other blocks write zeros to the rows that no token fell on.
//      The sort takes 13 us for 4096 places, 25 for 32,768 and 84 for 131,072 on at most
//      eight SMs a worker, and hides behind the zeros of a large table;
//   2. the sorted places are cut into chunks; a chunk's rows of dy are read
//      once and summed id by id.  A run of one id that lies in the chunk is the result;
//      what a run that crosses into other chunks has there goes to the scratch space;
//   3. such runs' parts are added up in order.
// Nothing is added atomically, so the same call gives the same bits.  Measured: 8 x 4096
// tokens of 32,000 x 1024 171 us (97 % of 6694.5 GB/s, 136 of them zeros), 131,072 tokens
// of 128,000 x 4096 602 us (79 %: zeros 300 us at 5.0 TB/s, sums 276 us at 5.9 TB/s, joins
// about 20 us); small ones are bound by the three kernels' latencies: 2 x 333 tokens 16 us.
// Where no zeros hide it the sort stands in the way: added to the same 8 tables 66 us (45 %),
// 131,072 tokens added to 128,000 x 1024 214 us (38 %), 8 x 31,395 f16 tokens of 3541 x 109
// 79 us (13 %).
// ---------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kSortMost = 20480;  // places of one block: two buffers of them in shared memory
constexpr int kCarryMost = kSortMost / 2;  // up to here with their ids, which else are read again
constexpr int kSection = 8 * kSortMost;  // places that are sorted at once; more are taken in turn, and added
constexpr int kMostBins = 512;
constexpr int kSortShared = 8 * kSortMost + 2 * kSortWarps * kMostBins;  // at most
constexpr int kFillRows = 1 << 16;  // rows of one filling block, a bit each

// Scratch: per worker the sorted ids and places of a section; then the chunks' parts.
struct Sorted {
  int32_t* ids;
  int32_t* places;
};
__host__ __device__ inline int64_t section_of(int64_t tokens) { return tokens < kSection ? tokens : kSection; }
__host__ __device__ inline Sorted sorted_of(const EmbeddingArgs& a, int64_t m) {
  const int64_t n = section_of(a.tokens);
  int32_t* base = static_cast<int32_t*>(a.scratch) + m * 2 * n;
  return {base, base + n};
}

__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_block(const void* p, int rank) {  // the same place in another block of the cluster
  uint32_t there;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(smem_addr(p)), "r"(rank));
  return there;
}

// The lanes whose digit of `width` bits is this lane's (-1: none), a bit at a time: a
// warp's match instruction takes several times as long.
__device__ __forceinline__ unsigned lanes_with(int digit, int width) {
  unsigned same = __ballot_sync(kFullMask, digit >= 0);
#pragma unroll
  for (int b = 0; b < 9; ++b)
    if (b < width) {
      const unsigned set = __ballot_sync(kFullMask, digit >> b & 1);
      same &= digit >> b & 1 ? set : ~set;
    }
  return digit >= 0 ? same : 0u;
}

// Sorts the n places from `begin` on of worker m by id, `share` of them to each
// of the cluster's blocks: passes of up to 9 bits from the lowest, each of which keeps
// the order within a digit.  A warp counts the digits of its part of the block's
// places, the counts are added up over warps, blocks and digits, and every place goes
// to where its digit's earlier ones end, in the shared memory of the block that holds
// that position.  kCarry: its id goes with it.  One SM's issue slots bound it (about
// 100 instructions for 32 places and pass), hence the cluster.
template <bool kCarry>
__device__ void sort_section(const EmbeddingArgs& a, int64_t m, int64_t begin, int n, int share, int rank, int ranks,
                             unsigned char* dynamic) {
  // places, counted from `begin`, and above kPlaceBits a place's rank among its warp's with the digit; then (kCarry) ids
  constexpr int kPlaceBits = 18;
  static_assert(kSection <= 1 << kPlaceBits && kSortMost / kSortWarps + 32 < 1 << (32 - kPlaceBits), "packed places");
  constexpr uint32_t kPlace = (1u << kPlaceBits) - 1u;
  uint32_t* from = reinterpret_cast<uint32_t*>(dynamic);
  uint32_t* to = from + (kCarry ? 2 : 1) * share;
  uint16_t* counts = reinterpret_cast<uint16_t*>(to + (kCarry ? 2 : 1) * share);  // [warp][bin]
  __shared__ uint32_t totals[kMostBins], bases[kMostBins], warp_sums[kSortWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const int mine = max(0, min(share, n - rank * share));
  const int part = (mine + kSortThreads - 1) / kSortThreads * 32;  // places of a warp
  const int lo = min(warp * part, mine), hi = min(lo + part, mine);
  const int bits = 32 - __clz((int)a.vocab), passes = (bits + 8) / 9, width = (bits + passes - 1) / passes;
  const int bins = 1 << width;
  const int64_t at = m * a.tokens + begin;
  const Sorted out = sorted_of(a, m);
  constexpr int kBatch = 4;  // ids on their way at once
#pragma unroll 4
  for (int i = threadIdx.x; i < mine; i += kSortThreads) {
    const uint32_t place = (uint32_t)(rank * share + i);
    from[i] = place;
    if (kCarry) from[share + i] = (uint32_t)token_at(a, at + place);
  }
  const auto id_of = [&](int i) { return kCarry ? (int32_t)from[share + i] : token_at(a, at + (from[i] & kPlace)); };
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * width;
    for (int i = threadIdx.x; i < kSortWarps * bins / 2; i += kSortThreads) reinterpret_cast<uint32_t*>(counts)[i] = 0;
    __syncthreads();
    uint16_t* const mine_counts = counts + warp * bins;
    for (int i0 = lo; i0 < hi; i0 += 32 * kBatch) {
      int32_t id[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) id[k] = i0 + 32 * k + lane < hi ? id_of(i0 + 32 * k + lane) : -1;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (i0 + 32 * k >= hi) break;
        const int digit = id[k] >= 0 ? id[k] >> shift & (bins - 1) : -1;
        const unsigned same = lanes_with(digit, width);
        uint32_t earlier = 0;
        if (digit >= 0) earlier = mine_counts[digit];
        __syncwarp();
        if (digit >= 0) {
          if (__ffs(same) - 1 == lane) mine_counts[digit] = (uint16_t)(earlier + __popc(same));
          from[i0 + 32 * k + lane] |= (earlier + __popc(same & ((1u << lane) - 1u))) << kPlaceBits;
        }
        __syncwarp();
      }
    }
    __syncthreads();
    // counts: the block's places of the digit in earlier warps; totals: in the block
    if (threadIdx.x < bins) {
      uint32_t sum = 0;
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = counts[w * bins + threadIdx.x];
        counts[w * bins + threadIdx.x] = (uint16_t)sum;
        sum += c;
      }
      totals[threadIdx.x] = sum;
    }
    if (ranks > 1) cluster_wait();
    else __syncthreads();
    uint32_t all = 0, earlier = 0;
    if (threadIdx.x < bins) {
      uint32_t c[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) {  // all on their way at once
        c[r] = 0;
        if (r < ranks) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c[r]) : "r"(in_block(totals + threadIdx.x, r)));
      }
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        all += c[r];
        if (r < rank) earlier += c[r];
      }
    }
    // bases: the section's places of lower digits, and of this one in earlier blocks
    uint32_t scan = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_up_sync(kFullMask, scan, o);
      if (lane >= o) scan += up;
    }
    if (lane == 31) warp_sums[warp] = scan;
    __syncthreads();
    if (threadIdx.x < bins) {
      for (int w = 0; w < warp; ++w) scan += warp_sums[w];
      bases[threadIdx.x] = scan - all + earlier;
    }
    __syncthreads();
    const bool last = pass == passes - 1;
#pragma unroll 4
    for (int i = lo + lane; i < hi; i += 32) {
      const uint32_t place = from[i] & kPlace;
      const int32_t id = id_of(i);
      const int digit = id >> shift & (bins - 1);
      const uint32_t where = bases[digit] + mine_counts[digit] + (from[i] >> kPlaceBits);
      if (last) {
        out.places[where] = (int32_t)(begin + place);
        out.ids[where] = id;
      } else {
        const int r = ranks == 1 ? 0 : (int)(where / (uint32_t)share);
        const uint32_t there = in_block(to + (where - r * (uint32_t)share), r);
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(there), "r"(place) : "memory");
        if (kCarry) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(there + 4 * (uint32_t)share), "r"(id) : "memory");
      }
    }
    // the other blocks' places have come, and nobody needs these totals any more
    if (ranks > 1) cluster_wait();
    else __syncthreads();
    uint32_t* const t = from;
    from = to;
    to = t;
  }
}

// Zeros to rows [v0, v1) of worker m's gradient that none of its n places from `begin` on holds
// (skip: look for those; else to all).
__device__ void fill_rows(const EmbeddingArgs& a, int64_t m, int64_t begin, int n, int64_t v0, int64_t v1, bool skip,
                          unsigned char* dynamic) {
  uint32_t* held = reinterpret_cast<uint32_t*>(dynamic);  // a bit a row
  const int rows = (int)(v1 - v0), lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  if (skip) {
    for (int i = threadIdx.x; i < (rows + 31) / 32; i += kSortThreads) held[i] = 0;
    __syncthreads();
    constexpr int kBatch = 8;
    const int64_t at = m * a.tokens + begin;
    for (int i0 = threadIdx.x; i0 < n; i0 += kSortThreads * kBatch) {
      int32_t id[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) id[k] = i0 + k * kSortThreads < n ? token_at(a, at + i0 + k * kSortThreads) : -1;
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (id[k] >= v0 && id[k] < v1) atomicOr(held + (int)(id[k] - v0) / 32, 1u << (int)(id[k] - v0) % 32);
    }
    __syncthreads();
  }
  float* const table = a.dtable + m * a.g_stride;
  for (int r = warp; r < rows; r += kSortWarps) {
    if (skip && (held[r / 32] >> r % 32 & 1u)) continue;
    float* row = table + (v0 + r) * a.width;
    // up to 3 values before the first 16-byte boundary, then 16 bytes at a time
    const int head = min((int)((16 - (uintptr_t)row % 16) % 16 / 4), (int)a.width), packs = ((int)a.width - head) / 4;
    const int tail = head + 4 * packs;
    if (lane < head) row[lane] = 0.f;
    if (tail + lane < a.width) row[tail + lane] = 0.f;
    float4* to = reinterpret_cast<float4*>(row + head);
    for (int i = lane; i < packs; i += 32) __stcs(to + i, make_float4(0.f, 0.f, 0.f, 0.f));
  }
}

// Blocks [0, workers * ranks) sort, the others fill `rows` rows each, `fills` blocks to a worker.
__global__ void __launch_bounds__(kSortThreads, 2)
    embedding_sort_kernel(EmbeddingArgs a, int64_t begin, int n, int share, int ranks, int rows, int fills, int skip) {
  dq_pdl_enter();
  dq_pdl_release();  // the sums' blocks may take up places as this grid's last ones come free
  extern __shared__ __align__(16) unsigned char dynamic[];
  const int sorters = n > 0 ? a.workers * ranks : 0;
  if ((int)blockIdx.x < sorters) {
    if (share <= kCarryMost) sort_section<true>(a, blockIdx.x / ranks, begin, n, share, blockIdx.x % ranks, ranks, dynamic);
    else sort_section<false>(a, blockIdx.x / ranks, begin, n, share, blockIdx.x % ranks, ranks, dynamic);
    return;
  }
  const int64_t fill = blockIdx.x - sorters;
  if (fill >= (int64_t)fills * a.workers) return;  // the cluster's spare blocks
  const int64_t v0 = fill % fills * rows;
  fill_rows(a, fill / fills, begin, n, v0, min64(v0 + rows, a.vocab), skip != 0, dynamic);
}

// A thread of the second kernel takes 8 columns: one 16-byte pack of dy, two in 32
// bits; where rows of dy are not aligned, shifted out of the aligned packs that hold them.
constexpr int kSumThreads = 128, kCols = 8, kSlice = kSumThreads * kCols;

struct Chunks {
  int32_t size;   // places of a chunk
  int32_t count;  // chunks of a worker
  int32_t lanes;  // threads that take a chunk's columns, at most kSumThreads
  int32_t near;   // rows_near of dy
};

// A worker's chunk's two parts, each a row of `width` sums: 0: of the run that comes
// from the chunk before; 1: of one that begins here and goes on.
__device__ __forceinline__ float* part_of(const EmbeddingArgs& a, const Chunks& ch, int64_t m, int64_t chunk, int which) {
  float* parts = reinterpret_cast<float*>(static_cast<int32_t*>(a.scratch) +
                                          (2 * section_of(a.tokens) * a.workers + 3) / 4 * 4);
  return parts + ((m * ch.count + chunk) * 2 + which) * ((a.width + 3) / 4 * 4);
}

// Blocks on an SM: three to five as registers come out; one instance would miss its fourth by 10 registers.
constexpr int sum_blocks(bool in, bool out, int size) { return in && !out && size == 2 ? 4 : 0; }

// kIn: rows of dy start on 16-byte boundaries; kOut: the table's gradient's do.
template <typename T, bool kIn, bool kOut>
__global__ void __launch_bounds__(kSumThreads, sum_blocks(kIn, kOut, sizeof(T))) embedding_sum_kernel(EmbeddingArgs a, int n, Chunks ch) {
  dq_pdl_enter();
  dq_pdl_release();
  constexpr int E = 16 / (int)sizeof(T), P = kCols / E, Q = kIn ? P : P + 1;  // packs of a row: its own, read
  constexpr int kAhead = Q * (kIn ? 2 : 1) <= 2 ? 8 : 4;                      // rows of dy on their way at once
  __shared__ __align__(16) float turned[kOut ? 1 : kSumThreads * kCols];
  const int lane = threadIdx.x % ch.lanes, groups = kSumThreads / ch.lanes;
  const int64_t which = (int64_t)blockIdx.x * groups + threadIdx.x / ch.lanes;
  if (which >= (int64_t)a.workers * ch.count) return;
  const int64_t m = which / ch.count, chunk = which % ch.count;
  const Sorted s = sorted_of(a, m);
  const int lo = (int)chunk * ch.size, hi = min(lo + ch.size, n), width = (int)a.width;
  const int c0 = (int)blockIdx.y * kSlice + lane * kCols;
  const T* dy = static_cast<const T*>(a.dy) + m * a.tokens * a.ld;
  float* const table = a.dtable + m * a.g_stride;

  float sum[kCols];
#pragma unroll
  for (int k = 0; k < kCols; ++k) sum[k] = 0.f;
  bool came = lo > 0 && s.ids[lo - 1] == s.ids[lo];  // the run at hand began in an earlier chunk
  const auto flush = [&](int32_t id, bool goes) {
    if (came || goes) {
      float* out = part_of(a, ch, m, chunk, came ? 0 : 1);
#pragma unroll
      for (int k = 0; k < kCols; k += 4)
        if (c0 + k < width)  // up to whole packs
          *reinterpret_cast<float4*>(out + c0 + k) = make_float4(sum[k], sum[k + 1], sum[k + 2], sum[k + 3]);
    } else if (kOut) {
      float* out = table + (int64_t)id * width + c0;
#pragma unroll
      for (int k = 0; k < kCols; k += 4) {
        if (c0 + k >= width) continue;
        float4* q = reinterpret_cast<float4*>(out + k);
        float4 v = make_float4(sum[k] * a.scale, sum[k + 1] * a.scale, sum[k + 2] * a.scale, sum[k + 3] * a.scale);
        if (a.accumulate) {
          const float4 old = *q;
          v = make_float4(old.x + v.x, old.y + v.y, old.z + v.z, old.w + v.w);
        }
        __stcs(q, v);
      }
    } else {
      // the lanes' columns turned, so that neighbouring lanes write neighbouring columns
      const int seg = min(ch.lanes, 32), l = lane % seg;
      float* mine = turned + (threadIdx.x - l) * kCols;  // of this warp, or group
      const unsigned mask = seg == 32 ? kFullMask : ((1u << seg) - 1u) << (threadIdx.x % 32 - l);
#pragma unroll
      for (int k = 0; k < kCols; k += 4)
        *reinterpret_cast<float4*>(mine + l * kCols + k) = make_float4(sum[k], sum[k + 1], sum[k + 2], sum[k + 3]);
      __syncwarp(mask);
      const int first = c0 - l * kCols;
      float* out = table + (int64_t)id * width + first;
#pragma unroll
      for (int k = 0; k < kCols; ++k) {
        const int c = l + k * seg;
        if (first + c >= width) continue;
        const float v = mine[c] * a.scale;
        out[c] = a.accumulate ? out[c] + v : v;
      }
      __syncwarp(mask);
    }
#pragma unroll
    for (int k = 0; k < kCols; ++k) sum[k] = 0.f;
    came = false;
  };

  const int32_t after = hi < n ? s.ids[hi] : (int32_t)a.vocab;  // of the next chunk's first place
  // Batches with a row whose packs might reach beyond dy are read by single values.
  constexpr bool kWhole = kIn && kOut && E == 4;  // rows end with a pack
  const Rows inside = rows_inside((int)a.tokens, a.workers, (int)m, ch.near, !kIn && c0 == 0,
                                  c0 + 2 * kCols > width && !(kIn && width % E == 0));
  int32_t next_id[kAhead + 1], next_place[kAhead];
  const auto places_at = [&](int j0) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      next_id[j] = j0 + j < hi ? s.ids[j0 + j] : (int32_t)a.vocab;
      next_place[j] = j0 + j < hi ? s.places[j0 + j] : inside.begin;
    }
    next_id[kAhead] = j0 + kAhead < hi ? s.ids[j0 + kAhead] : after;
  };
  places_at(lo);
  for (int j0 = lo; j0 < hi; j0 += kAhead) {
    int32_t id[kAhead + 1];
    uint4 x[kAhead][Q];
    int shift[kIn ? 1 : kAhead];
    int first = next_place[0], last = next_place[0];
#pragma unroll
    for (int j = 1; j < kAhead; ++j) {
      first = min(first, next_place[j]);
      last = max(last, next_place[j]);
    }
    if (!kWhole && (first < inside.begin || last >= inside.end)) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        id[j] = next_id[j];
        const T* row = dy + (int64_t)next_place[j] * a.ld + c0;
        if (!kIn) shift[j] = 0;
#pragma unroll
        for (int c = 0; c < kCols; ++c)
          reinterpret_cast<T*>(&x[j][c / E])[c % E] = id[j] < a.vocab && c0 + c < width ? row[c] : from_float<T>(0.f);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        id[j] = next_id[j];
        const T* row = dy + (int64_t)next_place[j] * a.ld + c0;
        const int s16 = kIn ? 0 : (int)((uintptr_t)row & 15u);
        if (!kIn) shift[j] = s16;
        const uint4* from = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(row) - s16);
        const int bytes = (width - c0) * (int)sizeof(T) + s16;  // before the row's end
        if (id[j] < a.vocab) {
#pragma unroll
          for (int p = 0; p < Q; ++p)
            if (16 * p < bytes) x[j][p] = kIn ? __ldcs(from + p) : from[p];
        }
      }
    }
    id[kAhead] = next_id[kAhead];
    places_at(j0 + kAhead);  // on their way while these rows are
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (j0 + j >= hi || id[j] >= a.vocab) break;  // the places without a token come last
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const uint4 y = kIn ? x[j][p] : funnel16(x[j][p], x[j][kIn ? p : p + 1], shift[kIn ? 0 : j]);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 v = pair_of<T>(y, e);
          sum[p * E + e] += v.x;
          sum[p * E + e + 1] += v.y;
        }
      }
      const bool ends_chunk = j0 + j + 1 == hi;
      const int32_t next = ends_chunk ? after : id[j + 1];
      if (next != id[j]) flush(id[j], false);
      else if (ends_chunk) flush(id[j], true);
    }
  }
}

// The parts of the run that begins in a chunk and goes on, if one does: `lanes`
// threads (32, 64 or 128) take 4 columns each; with 128 the block's two halves take
// half of the parts each.
constexpr int kJoinThreads = 256, kJoinSlice = 512;

__global__ void __launch_bounds__(kJoinThreads) embedding_join_kernel(EmbeddingArgs a, int n, Chunks ch, int lanes) {
  dq_pdl_enter();
  __shared__ float4 shared[kJoinThreads / 2];
  const bool halves = lanes == kJoinThreads / 2;
  const int group = threadIdx.x / lanes, t = threadIdx.x % lanes;
  const int64_t which = halves ? blockIdx.x : (int64_t)blockIdx.x * (kJoinThreads / lanes) + group;
  if (which >= (int64_t)a.workers * ch.count) return;
  const int64_t m = which / ch.count, chunk = which % ch.count;
  const Sorted s = sorted_of(a, m);
  const int lo = (int)chunk * ch.size, hi = lo + ch.size;
  if (hi >= n) return;  // nothing after it
  const int lane = threadIdx.x & 31;
  const int64_t after = hi + (int64_t)(lane + 1) * ch.size;  // the first place of the chunk after chunk + 1 + lane
  const int32_t id = s.ids[hi], id_last = s.ids[hi - 1], id_first = s.ids[lo], id_before = lo > 0 ? s.ids[lo - 1] : -1;
  const int32_t id_after = after < n ? s.ids[after] : -1;
  if (id >= a.vocab || id_last != id) return;
  if (id_first == id && id_before == id) return;  // it began earlier
  // the run's last chunk: the first whose next one starts with another id
  int64_t last = chunk + 1;
  unsigned ends = __ballot_sync(kFullMask, id_after != id);
  while (ends == 0) {
    last += 32;
    const int64_t next = (last + lane + 1) * ch.size;
    ends = __ballot_sync(kFullMask, next >= n || s.ids[next] != id);
  }
  last += __ffs(ends) - 1;
  const int64_t count = last - chunk + 1, mid = halves ? (count + 1) / 2 : count;
  const int64_t first = group == 0 || !halves ? 0 : mid, end = group == 0 || !halves ? mid : count;
  const int c = (int)blockIdx.y * kJoinSlice + 4 * t;  // the parts' rows are padded to whole packs
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < a.width)
#pragma unroll 8
    for (int64_t i = first; i < end; ++i) {
      const float4 v = *reinterpret_cast<const float4*>(part_of(a, ch, m, chunk + i, i == 0 ? 1 : 0) + c);
      sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
    }
  if (halves) {
    if (group == 1) shared[t] = sum;
    __syncthreads();
    if (group == 1) return;
    const float4 v = shared[t];
    sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
  }
  if (c >= a.width) return;
  const float total[4] = {sum.x * a.scale, sum.y * a.scale, sum.z * a.scale, sum.w * a.scale};
  float* out = a.dtable + m * a.g_stride + (int64_t)id * a.width + c;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (c + k < a.width) out[k] = a.accumulate ? out[k] + total[k] : total[k];
}

int lanes_for(int64_t width, int per_thread, int most) {
  int lanes = 1;
  while (lanes < most && (int64_t)lanes * per_thread < width) lanes *= 2;
  return lanes;
}

// Chunks small enough for 16 blocks of the second kernel on every SM (four at once: 131,072 tokens of 128,000 x
// 4096 602 us, with 32 blocks and as many more parts to join 611), of at least 16 places; at most 1024 to a worker,
// so that a run through many of them is soon joined.
constexpr int64_t kSumBlocks = 152 * 16;

Chunks chunks_of(int64_t n, int64_t width, int64_t workers) {
  Chunks ch{};
  ch.lanes = lanes_for(width, kCols, kSumThreads);
  const int64_t slices = ceil_div(width, kSlice), groups = kSumThreads / ch.lanes;
  ch.size = (int32_t)max64(max64(16, ceil_div(n, 1024)), ceil_div(n * workers * slices, kSumBlocks * groups));
  ch.count = (int32_t)max64(1, ceil_div(n, ch.size));
  return ch;
}

}  // namespace

size_t embedding_scratch_bytes(int64_t, int64_t width, int64_t max_tokens, int32_t workers) {
  const int64_t n = section_of(max_tokens);
  // the most chunks that any smaller number of tokens makes: n workers slices / size <= blocks groups
  const Chunks ch = chunks_of(n, width, workers);
  const int64_t slices = ceil_div(width, kSlice), groups = kSumThreads / ch.lanes;
  const int64_t chunks = min64(workers * ceil_div(n, 16), kSumBlocks * groups / slices + workers);
  return 4 * (size_t)((2 * n * workers + 3) / 4 * 4) + 8 * (size_t)chunks * (size_t)((width + 3) / 4 * 4);
}

cudaError_t launch_embedding_forward(const EmbeddingArgs& a, cudaStream_t stream, uint64_t* launches) {
  const int64_t n = a.tokens * a.workers;
  if (n == 0) return cudaSuccess;
  ++*launches;
  return with_dtype(a.table_dtype, [&](auto e) {
    return with_dtype(a.dtype, [&](auto t) {
      using E = decltype(e);
      using T = decltype(t);
      constexpr int N = 16 / (int)sizeof(T), kBytes = N * (int)sizeof(E), kAlign = kBytes < 16 ? kBytes : 16;
      const bool vec = a.width % N == 0 && (uintptr_t)a.y % 16 == 0 && a.ld % N == 0 &&
                       (uintptr_t)a.table % kAlign == 0 && a.width * (int64_t)sizeof(E) % kAlign == 0 &&
                       a.p_stride * (int64_t)sizeof(E) % kAlign == 0;
      const int lanes = lanes_for(a.width, (vec ? N : 1) * at_once(vec, (int)sizeof(E)), kForwardThreads);
      const auto kern = vec ? embedding_forward_kernel<E, T, true> : embedding_forward_kernel<E, T, false>;
      static std::atomic<int> kept[2][kKeptDevices];
      int resident = 0;
      const cudaError_t st = resident_ctas(kern, kForwardThreads, 0, 0, kept[vec ? 1 : 0], &resident);
      if (st != cudaSuccess) return st;
      const int64_t blocks = min64(ceil_div(n, kForwardThreads / lanes), resident);
      return launch_pdl(kern, dim3((unsigned)blocks), dim3(kForwardThreads), 0, stream, a, lanes);
    });
  });
}

cudaError_t launch_embedding_backward(const EmbeddingArgs& args, cudaStream_t stream, uint64_t* launches) {
  EmbeddingArgs a = args;
  int64_t begin = 0;
  do {
    const int n = (int)min64(a.tokens - begin, kSection);
    // 1. sort and fill
    int ranks = 1;
    while (ranks < 8 && ceil_div(n, ranks) > 1024) ranks *= 2;  // 32,768 places: 27 us in one block, 20 in eight
    const int share = (int)max64(ceil_div(n, ranks), 1);
    const int64_t sorters = n > 0 ? (int64_t)a.workers * ranks : 0;
    int64_t rows = 1, fills = 0;
    bool skip = false;
    int shared = n > 0 ? (share <= kCarryMost ? 16 : 8) * share + 2 * kSortWarps * kMostBins : 0;
    if (!a.accumulate) {
      // filling blocks for whole waves of the GPU, of at least a 16th MB each, and of four times the bytes
      // of the ids that a block looks through to find the rows to leave alone
      const int64_t all = 4 * a.width * a.vocab, ids = (int64_t)n * a.token_bits / 8;
      skip = n > 0 && all >= max64(64 << 10, 4 * ids);
      if (skip) shared = (int)max64(shared, kFillRows / 8);
      const int64_t at_once = max64(1, device_sms()) * (shared <= (100 << 10) ? 2 : 1);
      const int64_t waves = max64(1, min64(8, a.workers * all / (at_once * max64(64 << 10, skip ? 4 * ids : 0))));
      fills = max64(1, (waves * at_once - sorters) / a.workers);
      rows = min64(max64(ceil_div(a.vocab, fills), ceil_div(64 << 10, 4 * a.width)), kFillRows);
      fills = ceil_div(a.vocab, rows);
    }
    const int64_t blocks = ceil_div(sorters + fills * a.workers, ranks) * ranks;
    static std::atomic<int> kept[kKeptDevices];
    int resident = 0;
    cudaError_t st = resident_ctas(embedding_sort_kernel, kSortThreads, kSortShared, kSortShared, kept, &resident);
    if (st != cudaSuccess) return st;
    if (blocks > 0) {
      ++*launches;
      st = launch_pdl_cluster(embedding_sort_kernel, ranks, dim3((unsigned)blocks), dim3(kSortThreads), (size_t)shared,
                              stream, a, begin, n, share, ranks, (int)rows, (int)fills, skip ? 1 : 0);
      if (st != cudaSuccess) return st;
    }
    if (n == 0) return cudaSuccess;
    // 2. and 3. sum
    const int size = a.dtype == DQGAN_F32 ? 4 : 2;
    const bool in = (uintptr_t)a.dy % 16 == 0 && a.ld * size % 16 == 0;
    const bool out = a.width % 4 == 0 && (uintptr_t)a.dtable % 16 == 0 && a.g_stride % 4 == 0;
    Chunks ch = chunks_of(n, a.width, a.workers);
    ch.near = rows_near(a.ld * size);
    const dim3 grid((unsigned)ceil_div((int64_t)a.workers * ch.count, kSumThreads / ch.lanes),
                    (unsigned)ceil_div(a.width, kSlice));
    ++*launches;
    st = with_dtype(a.dtype, [&](auto t) {
      using T = decltype(t);
      const auto kern = in ? (out ? embedding_sum_kernel<T, true, true> : embedding_sum_kernel<T, true, false>)
                           : (out ? embedding_sum_kernel<T, false, true> : embedding_sum_kernel<T, false, false>);
      return launch_pdl(kern, grid, dim3(kSumThreads), 0, stream, a, n, ch);
    });
    if (st != cudaSuccess) return st;
    if (ch.count > 1) {
      const int lanes = (int)max64(32, lanes_for(a.width, 4, kJoinThreads / 2));
      const int chunks_a_block = lanes == kJoinThreads / 2 ? 1 : kJoinThreads / lanes;
      ++*launches;
      st = launch_pdl(embedding_join_kernel,
                      dim3((unsigned)ceil_div((int64_t)a.workers * ch.count, chunks_a_block),
                           (unsigned)ceil_div(a.width, kJoinSlice)),
                      dim3(kJoinThreads), 0, stream, a, n, ch, lanes);
      if (st != cudaSuccess) return st;
    }
    begin += n;
    a.accumulate = 1;
  } while (begin < a.tokens);
  return cudaSuccess;
}

}  // namespace dq
