// Embedding lookup with scaling, and its gradient over the tokens sorted by id.
#include "device_common.cuh"
#include "operators.cuh"

namespace dq {
namespace {

constexpr int kThreads = 256;

// The place's id, or -1 where it holds no token.
__device__ __forceinline__ int32_t token_at(const EmbeddingArgs& a, int64_t i) {
  const int64_t id = a.token_bits == 32 ? static_cast<const int32_t*>(a.ids)[i] : static_cast<const int64_t*>(a.ids)[i];
  return id >= 0 && id < a.vocab ? (int32_t)id : -1;
}

// One block per place.
template <typename E, typename T>
__global__ void __launch_bounds__(kThreads) embedding_forward_kernel(EmbeddingArgs a) {
  dq_pdl_enter();
  const int64_t i = blockIdx.x;
  const int32_t id = token_at(a, i);
  T* y = static_cast<T*>(a.y) + i * a.ld;
  const E* row = static_cast<const E*>(a.table) + i / a.tokens * a.p_stride + (int64_t)max(id, 0) * a.width;
  for (int64_t c = threadIdx.x; c < a.width; c += kThreads)
    y[c] = from_float<T>(id < 0 ? 0.f : to_float(row[c]) * a.scale);
}

// Scratch, per worker: vocab + 1 starts of the ids' runs, then the places
// sorted by id (and by place within an id).
struct Sorted {
  int32_t* starts;
  int32_t* places;
};
__host__ __device__ inline Sorted sorted_of(const EmbeddingArgs& a, int64_t m) {
  int32_t* base = static_cast<int32_t*>(a.scratch) + m * (a.vocab + 1 + a.tokens);
  return {base, base + a.vocab + 1};
}

__global__ void __launch_bounds__(kThreads) embedding_clear_kernel(EmbeddingArgs a) {
  dq_pdl_enter();
  const int64_t v = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (v <= a.vocab) sorted_of(a, blockIdx.y).starts[v] = 0;
}

__global__ void __launch_bounds__(kThreads) embedding_count_kernel(EmbeddingArgs a) {
  dq_pdl_enter();
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.tokens) return;
  const int32_t id = token_at(a, blockIdx.y * a.tokens + i);
  if (id >= 0) atomicAdd(sorted_of(a, blockIdx.y).starts + id, 1);
}

// Counts to starts: one warp per worker.
__global__ void __launch_bounds__(32) embedding_scan_kernel(EmbeddingArgs a) {
  dq_pdl_enter();
  int32_t* starts = sorted_of(a, blockIdx.x).starts;
  const int lane = threadIdx.x;
  int32_t before = 0;
  for (int64_t v0 = 0; v0 <= a.vocab; v0 += 32) {
    const int64_t v = v0 + lane;
    const int32_t n = v <= a.vocab ? starts[v] : 0;
    int32_t s = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int32_t up = __shfl_up_sync(kFullMask, s, o);
      if (lane >= o) s += up;
    }
    if (v <= a.vocab) starts[v] = before + s - n;
    before += __shfl_sync(kFullMask, s, 31);
  }
}

// A place's rank within its id's run: the earlier places with the same id.
__global__ void __launch_bounds__(kThreads) embedding_place_kernel(EmbeddingArgs a) {
  dq_pdl_enter();
  __shared__ int32_t tile[kThreads];
  const int64_t first = blockIdx.y * a.tokens, i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int32_t id = i < a.tokens ? token_at(a, first + i) : -1;
  int32_t rank = 0;
  for (int64_t j0 = 0; j0 <= (int64_t)blockIdx.x * kThreads; j0 += kThreads) {
    __syncthreads();
    tile[threadIdx.x] = j0 + threadIdx.x < a.tokens ? token_at(a, first + j0 + threadIdx.x) : -1;
    __syncthreads();
    for (int j = 0; j < kThreads; ++j) rank += tile[j] == id && j0 + j < i ? 1 : 0;
  }
  const Sorted s = sorted_of(a, blockIdx.y);
  if (id >= 0) s.places[s.starts[id] + rank] = (int32_t)i;
}

// One block per row of a worker's table.
template <typename T>
__global__ void __launch_bounds__(kThreads) embedding_gradient_kernel(EmbeddingArgs a) {
  dq_pdl_enter();
  const int64_t v = blockIdx.x, m = blockIdx.y;
  const Sorted s = sorted_of(a, m);
  const int32_t begin = s.starts[v], end = s.starts[v + 1];
  if (begin == end && a.accumulate) return;
  float* out = a.dtable + m * a.g_stride + v * a.width;
  for (int64_t c = threadIdx.x; c < a.width; c += kThreads) {
    float sum = 0.f;
    for (int32_t j = begin; j < end; ++j)
      sum += to_float(static_cast<const T*>(a.dy)[(m * a.tokens + s.places[j]) * a.ld + c]);
    sum *= a.scale;
    out[c] = a.accumulate ? out[c] + sum : sum;
  }
}

}  // namespace

size_t embedding_scratch_bytes(int64_t vocab, int64_t, int64_t max_tokens, int32_t workers) {
  return 4 * (size_t)workers * (size_t)(vocab + 1 + max_tokens);
}

cudaError_t launch_embedding_forward(const EmbeddingArgs& a, cudaStream_t stream, uint64_t* launches) {
  const int64_t n = a.tokens * a.workers;
  if (n == 0) return cudaSuccess;
  ++*launches;
  return with_dtype(a.table_dtype, [&](auto e) {
    return with_dtype(a.dtype, [&](auto t) {
      return launch_pdl(embedding_forward_kernel<decltype(e), decltype(t)>, dim3((unsigned)n), dim3(kThreads), 0,
                        stream, a);
    });
  });
}

cudaError_t launch_embedding_backward(const EmbeddingArgs& a, cudaStream_t stream, uint64_t* launches) {
  const dim3 block(kThreads), by_token((unsigned)ceil_div(a.tokens, kThreads), a.workers);
  cudaError_t st = launch_pdl(embedding_clear_kernel, dim3((unsigned)ceil_div(a.vocab + 1, kThreads), a.workers), block,
                              0, stream, a);
  ++*launches;
  if (st == cudaSuccess && a.tokens > 0) {
    *launches += 3;
    if ((st = launch_pdl(embedding_count_kernel, by_token, block, 0, stream, a)) == cudaSuccess &&
        (st = launch_pdl(embedding_scan_kernel, dim3(a.workers), dim3(32), 0, stream, a)) == cudaSuccess)
      st = launch_pdl(embedding_place_kernel, by_token, block, 0, stream, a);
  }
  if (st != cudaSuccess) return st;
  ++*launches;
  return with_dtype(a.dtype, [&](auto t) {
    return launch_pdl(embedding_gradient_kernel<decltype(t)>, dim3((unsigned)a.vocab, a.workers), block, 0, stream, a);
  });
}

}  // namespace dq
