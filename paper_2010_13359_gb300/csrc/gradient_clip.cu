// The global norm of every worker's gradient over many tensors, and its clipping on the way into the row that the
// worker step compresses:
//
//   n = sqrt(sum over all tensors of g^2);  out = min(1, max_norm / (n + eps)) g
//
// Two passes, bound by memory: the norm reads every value, the clipping reads it
// again and writes it.  Both cut the tensors into units of up to 16,384 values and
// give each block a run of them; the second pass walks them backwards, so that it
// finds in L2 what the first one read last.
//
// Up to 2^18 values a worker take one launch of a cluster each.
//
// A block's thread sums the squares of at most 64 values of a unit in fp32, then in
// fp64, and the blocks' sums are joined in a fixed order.  Where a thread's fp32 sum
// leaves [2^-80, 2^120], its squares are taken again in fp64.
#include "device_common.cuh"
#include "operators.cuh"

namespace dq {

namespace {

constexpr int kClipThreads = 256, kMostUnit = 16384, kLeastUnit = 2048;
constexpr int kTableTensors = 640;  // of one launch: kernel parameters are limited to 32,764 bytes
constexpr int kMaxTables = 8;
constexpr int kClipBlocks = 152 * 4;

struct ClipTensor {
  const void* from;
  void* to;
  int64_t size, from_stride, to_stride;
  int64_t unit;  // the tensor's first unit in its table
};

struct ClipLaunch {
  double* sums;     // of block b and worker m at [b + m], this table's
  int64_t units;    // of one worker
  int32_t blocks;
};

struct ClipArgs {
  ClipLaunch tables[kMaxTables];
  int32_t count_tables, table;
  int32_t norm_table;  // the first that has units: its second pass writes the norms
  int32_t workers;
  int32_t count;  // tensors of this table
  int32_t unit;   // values
  double max_norm, eps;
  float* norms;
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

template <int kTensors>
struct ClipTable {
  ClipTensor t[kTensors];
};

__device__ __forceinline__ int64_t first_unit(const ClipArgs& a, const ClipLaunch& l, int64_t block) {
  return clip_first_unit(l.units, a.workers, block, l.blocks);
}

__device__ __forceinline__ double block_sum_double(double x, double* shared) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(kFullMask, x, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x / 32] = x;
  __syncthreads();
  double s = shared[0];
  for (int i = 1; i < kClipThreads / 32; ++i) s += shared[i];
  return s;
}

template <int kTensors>
__device__ __forceinline__ int tensor_of(const ClipTable<kTensors>& table, int count, int64_t unit) {
  int low = 0, high = count - 1;  // the last tensor that begins at or before the unit
  while (low < high) {
    const int mid = (low + high + 1) / 2;
    if (table.t[mid].unit <= unit)
      low = mid;
    else
      high = mid - 1;
  }
  return low;
}

// Values before the first pack of 16 bytes.
template <typename T>
__device__ __forceinline__ int head_of(const T* p, int64_t n) {
  return (int)min64(n, (int64_t)((16 - ((uintptr_t)p & 15)) & 15) / (int64_t)sizeof(T));
}

// Sum of the squares of this thread's values of a unit.
template <typename T>
__device__ __forceinline__ double unit_squares(const T* p, int n) {
  constexpr int E = 16 / (int)sizeof(T);
  const int head = head_of(p, n), packs = (n - head) / E, tail = head + packs * E;
  const uint4* const body = reinterpret_cast<const uint4*>(p + head);
  float s[4] = {};
  uint32_t any = 0;
  const auto one = [&](const T& value) {
    const float x = to_float(value);
    s[0] = fmaf(x, x, s[0]);
    any |= __float_as_uint(x);
  };
  if ((int)threadIdx.x < head) one(p[threadIdx.x]);
  if ((int)threadIdx.x < n - tail) one(p[tail + threadIdx.x]);
  for (int i = (int)threadIdx.x; i < packs; i += 8 * kClipThreads) {
    uint4 pack[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) pack[k] = i + k * kClipThreads < packs ? body[i + k * kClipThreads] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      any |= (pack[k].x | pack[k].y) | (pack[k].z | pack[k].w);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 v = pair_of<T>(pack[k], e);
        s[e & 2] = fmaf(v.x, v.x, s[e & 2]);
        s[(e & 2) + 1] = fmaf(v.y, v.y, s[(e & 2) + 1]);
      }
    }
  }
  const float sum = (s[0] + s[1]) + (s[2] + s[3]);
  if ((sum >= 0x1p-80f && sum <= 0x1p120f) || any == 0) return sum;
  double d = 0.;
  const auto again = [&](const T& value) { d += (double)to_float(value) * (double)to_float(value); };
  if ((int)threadIdx.x < head) again(p[threadIdx.x]);
  if ((int)threadIdx.x < n - tail) again(p[tail + threadIdx.x]);
  for (int i = head + (int)threadIdx.x * E; i < tail; i += kClipThreads * E)
    for (int e = 0; e < E; ++e) again(p[i + e]);
  return d;
}

template <typename T, int kTensors>
__global__ void __launch_bounds__(kClipThreads, 4) norm_kernel(const __grid_constant__ ClipArgs a,
                                                             const __grid_constant__ ClipTable<kTensors> table) {
  dq_pdl_enter();
  __shared__ double shared[kClipThreads / 32];
  const ClipLaunch& l = a.tables[a.table];
  const int64_t begin = first_unit(a, l, blockIdx.x), end = first_unit(a, l, (int64_t)blockIdx.x + 1);
  double sum = 0.;
  for (int64_t u = begin; u < end; ++u) {
    const int64_t worker = u / l.units, unit = u - worker * l.units;
    const ClipTensor& t = table.t[tensor_of(table, a.count, unit)];
    const int64_t at = (unit - t.unit) * a.unit;
    sum += unit_squares(static_cast<const T*>(t.from) + worker * t.from_stride + at, (int)min64(a.unit, t.size - at));
    if (u + 1 == end || unit + 1 == l.units) {
      const double total = block_sum_double(sum, shared);
      if (threadIdx.x == 0) l.sums[blockIdx.x + worker] = total;
      sum = 0.;
    }
  }
}

// The norm of a worker's gradient from the blocks' sums of all tables.
__device__ __forceinline__ double worker_norm(const ClipArgs& a, int64_t worker, double* shared) {
  double sum = 0.;
  for (int i = 0; i < a.count_tables; ++i) {
    const ClipLaunch& l = a.tables[i];
    if (l.units == 0) continue;
    // the blocks that hold the worker's first and last unit
    const int64_t first = clip_block_of(l.units, a.workers, worker * l.units, l.blocks);
    const int64_t last = clip_block_of(l.units, a.workers, (worker + 1) * l.units - 1, l.blocks);
    for (int64_t b = first + threadIdx.x; b <= last; b += kClipThreads) sum += l.sums[b + worker];
  }
  return sqrt(block_sum_double(sum, shared));
}

__global__ void __launch_bounds__(kClipThreads) norms_kernel(const __grid_constant__ ClipArgs a) {
  dq_pdl_enter();
  __shared__ double shared[kClipThreads / 32];
  const double norm = worker_norm(a, blockIdx.x, shared);
  if (threadIdx.x == 0) a.norms[blockIdx.x] = (float)norm;
}

// The factor of a worker's values, in two steps: one below fp32's range, which large values bring back into it, by a power
// of two first, which is exact.
struct ClipFactor {
  float shift, factor;
};
__device__ __forceinline__ ClipFactor clip_factor(const ClipArgs& a, double norm) {
  const double scale = isfinite(norm) ? fmin(1., a.max_norm / (norm + a.eps)) : 1.;
  const float shift = scale < 0x1p-150 ? 0x1p-126f : scale < 0x1p-64 ? 0x1p-64f : 1.f;
  return {shift, (float)(scale / shift)};
}

template <typename T, typename O>
__device__ __forceinline__ void scale_unit(const T* from, O* to, int n, float shift, float factor, const T* begin, const T* end) {
  constexpr int E = 16 / (int)sizeof(T);
  const int head = head_of(from, n);
  const auto one = [&](int i) { to[i] = from_float<O>(to_float(from[i]) * shift * factor); };
  if ((((uintptr_t)(to + head)) & 15) != 0) {  // the two sides' packs do not meet: the places' ones, shifted out of the tensor's
    constexpr int F = 16 / (int)sizeof(O);
    const int first = head_of(to, n), eights = (n - first) / 8, rest = first + eights * 8;
    if ((int)threadIdx.x < first) one(threadIdx.x);
    if ((int)threadIdx.x < n - rest) one(rest + threadIdx.x);
    for (int i = (int)threadIdx.x; i < eights; i += 2 * kClipThreads) {
      float x[2][8];
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (i + k * kClipThreads < eights) read8_near(from + first + 8 * (i + k * kClipThreads), 8, begin, end, x[k]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (i + k * kClipThreads >= eights) break;
        uint4* const at = reinterpret_cast<uint4*>(to + first + 8 * (i + k * kClipThreads));
#pragma unroll
        for (int q = 0; q < 8 / F; ++q) {
          uint4 pack;
#pragma unroll
          for (int e = 0; e < F; e += 2)
            set_pair<O>(pack, e, make_float2(x[k][q * F + e] * shift * factor, x[k][q * F + e + 1] * shift * factor));
          __stcs(at + q, pack);
        }
      }
    }
    return;
  }
  const int packs = (n - head) / E, tail = head + packs * E;
  if ((int)threadIdx.x < head) one(threadIdx.x);
  if ((int)threadIdx.x < n - tail) one(tail + threadIdx.x);
  const uint4* const body = reinterpret_cast<const uint4*>(from + head);
  const bool wide = ((uintptr_t)(to + head) & 31) == 0;
  for (int i = (int)threadIdx.x; i < packs; i += 4 * kClipThreads) {
    uint4 pack[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * kClipThreads < packs) pack[k] = __ldcs(body + i + k * kClipThreads);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (i + k * kClipThreads >= packs) break;
      uint4 out[sizeof(O) * E / 16];
      constexpr int F = 16 / (int)sizeof(O);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 v = pair_of<T>(pack[k], e);
        set_pair<O>(out[e / F], e % F, make_float2(v.x * shift * factor, v.y * shift * factor));
      }
      uint4* const at = reinterpret_cast<uint4*>(to + head) + (int64_t)(i + k * kClipThreads) * (sizeof(out) / 16);
      if constexpr (sizeof(out) == 32) {
        if (wide)
          asm volatile("st.global.cs.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(out[0].x), "r"(out[0].y),
                       "r"(out[0].z), "r"(out[0].w), "r"(out[1].x), "r"(out[1].y), "r"(out[1].z), "r"(out[1].w)
                       : "memory");
        else
          __stcs(at, out[0]), __stcs(at + 1, out[1]);
      } else {
        __stcs(at, out[0]);
      }
    }
  }
}

template <typename T, typename O, int kTensors>
__global__ void __launch_bounds__(kClipThreads, 4) scale_kernel(const __grid_constant__ ClipArgs a,
                                                              const __grid_constant__ ClipTable<kTensors> table) {
  dq_pdl_enter();
  __shared__ double shared[kClipThreads / 32];
  const ClipLaunch& l = a.tables[a.table];
  const int64_t begin = first_unit(a, l, blockIdx.x), end = first_unit(a, l, (int64_t)blockIdx.x + 1);
  int64_t known = -1;
  ClipFactor f{1.f, 1.f};
  for (int64_t u = end - 1; u >= begin; --u) {
    const int64_t worker = u / l.units, unit = u - worker * l.units;
    if (worker != known) {
      const double norm = worker_norm(a, worker, shared);
      f = clip_factor(a, norm);
      known = worker;
      // one block has the worker's first unit of the last table that is walked
      if (a.norms && threadIdx.x == 0 && a.table == a.norm_table && worker * l.units >= begin) a.norms[worker] = (float)norm;
    }
    const ClipTensor& t = table.t[tensor_of(table, a.count, unit)];
    const int64_t at = (unit - t.unit) * a.unit;
    scale_unit(static_cast<const T*>(t.from) + worker * t.from_stride + at,
               static_cast<O*>(t.to) + worker * t.to_stride + at, (int)min64(a.unit, t.size - at), f.shift, f.factor,
               static_cast<const T*>(t.from) + worker * t.from_stride, static_cast<const T*>(t.from) + worker * t.from_stride + t.size);
  }
}

// Few values: a cluster of eight blocks a worker does both passes in one launch, its sums exchanged through shared memory.
constexpr int kFewBlocks = 8;
constexpr int64_t kFewValues = 1 << 18;
template <typename T, typename O, int kTensors>
__global__ void __launch_bounds__(kClipThreads) few_values_kernel(const __grid_constant__ ClipArgs a,
                                                                   const __grid_constant__ ClipTable<kTensors> table, bool scale) {
  dq_pdl_enter();
  __shared__ double shared[kClipThreads / 32], sums[kFewBlocks];
  cluster_arrive();  // every block of the cluster runs before another touches its shared memory
  const ClipLaunch& l = a.tables[0];
  const int64_t worker = blockIdx.x / kFewBlocks;
  const int rank = (int)(blockIdx.x % kFewBlocks);
  double sum = 0.;
  const auto each = [&](int64_t unit, auto&& f) {
    const ClipTensor& t = table.t[tensor_of(table, a.count, unit)];
    const int64_t at = (unit - t.unit) * a.unit;
    f(t, static_cast<const T*>(t.from) + worker * t.from_stride + at, at, (int)min64(a.unit, t.size - at));
  };
  int64_t unit = rank;
  for (; unit < l.units; unit += kFewBlocks)
    each(unit, [&](const ClipTensor&, const T* from, int64_t, int n) { sum += unit_squares(from, n); });
  sum = block_sum_double(sum, shared);
  cluster_wait();
  if (threadIdx.x < kFewBlocks) {
    uint32_t to;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_addr(sums + rank)), "r"((uint32_t)threadIdx.x));
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to), "d"(sum) : "memory");
  }
  cluster_arrive();
  cluster_wait();
  double total = 0.;
  for (int i = 0; i < kFewBlocks; ++i) total += sums[i];
  const double norm = sqrt(total);
  if (a.norms && rank == 0 && threadIdx.x == 0) a.norms[worker] = (float)norm;
  if (!scale) return;
  const ClipFactor f = clip_factor(a, norm);
  for (unit -= kFewBlocks; unit >= 0; unit -= kFewBlocks)
    each(unit, [&](const ClipTensor& t, const T* from, int64_t at, int n) {
      scale_unit(from, static_cast<O*>(t.to) + worker * t.to_stride + at, n, f.shift, f.factor, from - at, from - at + t.size);
    });
}

template <typename T, typename O, int kTensors>
cudaError_t launch_clip(const ClipShape& s, int64_t count, const dqgan_tensor* from, const dqgan_tensor* to,
                        float max_norm, float* norms, void* scratch, cudaStream_t stream, uint64_t* launches) {
  ClipArgs a{};
  a.workers = s.workers;
  a.max_norm = max_norm;
  a.eps = s.eps;
  a.norms = norms;
  a.count_tables = (int32_t)ceil_div(count, kTensors);
  int64_t values = 0;
  for (int64_t k = 0; k < count; ++k) values += from[k].size;
  a.unit = kMostUnit;  // smaller where the GPU has blocks to spare
  while (a.unit > kLeastUnit && values / a.unit * s.workers < kClipBlocks) a.unit /= 2;
  ClipTable<kTensors> table{};
  const auto fill = [&](int i) {
    a.table = i;
    a.count = 0;
    int64_t units = 0;
    for (int64_t k = (int64_t)i * kTensors; k < count && k < (int64_t)(i + 1) * kTensors; ++k) {
      if (from[k].size == 0) continue;
      table.t[a.count++] = {from[k].data, to ? to[k].data : nullptr, from[k].size, from[k].stride, to ? to[k].stride : 0, units};
      units += ceil_div(from[k].size, a.unit);
    }
    ClipLaunch& l = a.tables[i];
    l.units = units;
    l.blocks = (int32_t)min64(units * s.workers, kClipBlocks);
    l.sums = static_cast<double*>(scratch) + (int64_t)i * (kClipBlocks + s.workers);
  };
  cudaError_t st = cudaSuccess;
  if (a.count_tables == 1 && values > 0 && values <= kFewValues) {
    a.unit = kLeastUnit;
    fill(0);
    ++*launches;
    return launch_pdl_cluster(few_values_kernel<T, O, kTensors>, kFewBlocks, dim3((unsigned)s.workers * kFewBlocks), dim3(kClipThreads),
                              0, stream, a, table, to != nullptr);
  }
  for (int i = 0; i < a.count_tables && st == cudaSuccess; ++i) {
    fill(i);
    if (a.tables[i].units == 0) continue;
    ++*launches;
    st = launch_pdl(norm_kernel<T, kTensors>, dim3((unsigned)a.tables[i].blocks), dim3(kClipThreads), 0, stream, a, table);
  }
  if (st != cudaSuccess) return st;
  while (a.norm_table < a.count_tables - 1 && a.tables[a.norm_table].units == 0) ++a.norm_table;
  if (norms && (!to || values == 0)) {
    ++*launches;
    st = launch_pdl(norms_kernel, dim3((unsigned)s.workers), dim3(kClipThreads), 0, stream, a);
  }
  for (int i = a.count_tables - 1; to && i >= 0 && st == cudaSuccess; --i) {
    fill(i);
    if (a.tables[i].units == 0) continue;
    ++*launches;
    st = launch_pdl(scale_kernel<T, O, kTensors>, dim3((unsigned)a.tables[i].blocks), dim3(kClipThreads), 0, stream, a, table);
  }
  return st;
}

}  // namespace

size_t clip_scratch_bytes(const ClipShape& s) { return (size_t)kMaxTables * (kClipBlocks + s.workers) * sizeof(double); }

cudaError_t launch_gradient_clip(const ClipShape& s, int64_t count, const dqgan_tensor* from, const dqgan_tensor* to,
                                 float max_norm, float* norms, void* scratch, cudaStream_t stream, uint64_t* launches) {
  static_assert(sizeof(ClipArgs) + sizeof(ClipTable<kTableTensors>) <= 32764, "kernel parameters");
  return with_dtype(s.dtype, [&](auto t) {
    using T = decltype(t);
    const auto run = [&](auto o) {
      using O = decltype(o);
      return count <= 32 ? launch_clip<T, O, 32>(s, count, from, to, max_norm, norms, scratch, stream, launches)
                         : launch_clip<T, O, kTableTensors>(s, count, from, to, max_norm, norms, scratch, stream, launches);
    };
    return s.out_dtype == DQGAN_F32 ? run(float{}) : run(t);
  });
}

}  // namespace dq
