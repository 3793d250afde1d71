// Layer norm over the rows of W workers, and its gradient.
//
//   mu = mean(x), s^2 = mean((x - mu)^2), r = 1 / sqrt(s^2 + eps), h = (x - mu) r
//   y = h weight + bias
//   a = dy weight, dx = r (a - mean(a) - h mean(a h)), dweight = sum dy h, dbias = sum dy
//
// Both directions are bound by memory (forward: 2, backward: 3 values moved per
// element at 8 and 14 operations), so each row is read once and kept on chip: a
// group of kLanes threads holds it, 16 values to a thread.  The variance is taken
// from the deviations, in a second sum over the same registers, so that a large
// mean costs no digits.  Rows longer than 16,384 values are read again from the
// caches instead, and so are those of the backward pass in fp32 above 8192: a row of
// x and one of dy take up to 128 KB there, which leaves no room for rows ahead.
#include "device_common.cuh"
#include "operators.cuh"

namespace dq {
namespace {

constexpr int kPerThread = 16;  // values of a row in one thread
constexpr int kMaxOnChip = 1024 * kPerThread;

// A thread's share of a row: N packs of E values.  kVec: pack i of lane t holds
// values (i * kLanes + t) * E and the E - 1 after it; else (rows that do not
// start on 16-byte boundaries) value e of pack i is (i * E + e) * kLanes + t, so
// that single-element accesses of a warp are adjacent.  Such rows come into shared
// memory as the aligned packs that hold them, copied by all of a row's threads.
template <typename T, int kLanes, bool kVec>
struct Slice {
  static constexpr int E = 16 / (int)sizeof(T);
  static constexpr int N = kPerThread / E;

  __device__ __forceinline__ static int at(int i, int e, int lane) {
    return kVec ? (i * kLanes + lane) * E + e : (i * E + e) * kLanes + lane;
  }

  // The row's packs, 0 past its end.
  __device__ __forceinline__ static void load(const T* row, int width, int lane, uint4 (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (kVec && at(i, E - 1, lane) < width) {
        x[i] = *reinterpret_cast<const uint4*>(row + at(i, 0, lane));
      } else {
        T* v = reinterpret_cast<T*>(&x[i]);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = at(i, e, lane) < width ? row[at(i, e, lane)] : from_float<T>(0.f);
      }
    }
  }

  // Packs of a row vector in the ring, and where this thread's row begins in them.
  __host__ __device__ static constexpr int ring_packs(int threads) { return threads * N + (kVec ? 0 : threads / kLanes); }
  __device__ __forceinline__ static int ring_at() { return kVec ? (int)threadIdx.x : (int)threadIdx.x / kLanes * (kLanes * N + 1); }

  // The row into a ring stage, 0 past its end.  all: where the tensor begins, if the row may be so near to that that
  // its first pack begins before; nothing there is read.  (Only a group's first row may: rows of less than 16 bytes, of
  // which several are, have a group of 8 threads each.)
  __device__ __forceinline__ static void fetch(const T* row, int width, int lane, uint4* to, int threads,
                                               const T* all = nullptr) {
    const int shift = kVec ? 0 : (int)((uintptr_t)row & 15u);
    const char* from = reinterpret_cast<const char*>(row) - shift;
    to += ring_at();
#pragma unroll
    for (int i = 0; i < (kVec ? N : N + 1); ++i) {
      if (i == N && lane > 0) break;  // one pack more than the threads' N
      const int pack = i * kLanes + lane, left = shift + width * (int)sizeof(T) - 16 * pack;
      const int bytes = left >= 16 ? 16 : left > 0 ? left : 0;
      if (!kVec && i == 0 && lane == 0 && all && (uintptr_t)from < (uintptr_t)all) {
#pragma unroll 1
        for (int e = 0; e < (16 - shift) / (int)sizeof(T); ++e)
          reinterpret_cast<T*>(to)[shift / (int)sizeof(T) + e] = e < width ? row[e] : from_float<T>(0.f);
        continue;
      }
      copy16_async(kVec ? to + i * threads : to + pack, from + (bytes > 0 ? 16 * pack : 0), bytes);
    }
  }

  // What fetch brought.
  __device__ __forceinline__ static void take(const uint4* from, const T* row, int lane, int threads, uint4 (&x)[N]) {
    from += ring_at();
    if (kVec) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = from[i * threads];
      return;
    }
    const T* values = reinterpret_cast<const T*>(reinterpret_cast<const char*>(from) + ((uintptr_t)row & 15u));
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) reinterpret_cast<T*>(&x[i])[e] = values[at(i, e, lane)];
  }

  __device__ __forceinline__ static void store(T* row, int width, int lane, const uint4 (&y)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (kVec && at(i, E - 1, lane) < width) {
        __stcs(reinterpret_cast<uint4*>(row + at(i, 0, lane)), y[i]);
      } else {
        const T* v = reinterpret_cast<const T*>(&y[i]);
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (at(i, e, lane) < width) row[at(i, e, lane)] = v[e];
      }
    }
  }

  // f(i, e, column) for every value of the row that this lane holds.
  template <typename F>
  __device__ __forceinline__ static void each(int width, int lane, F&& f) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (at(i, e, lane) < width) f(i, e, at(i, e, lane));
  }

  // A worker's parameters at this lane's columns (`missing` where there are none
  // or past the end).  They come from the caches; 16 bytes at a time where they
  // are aligned, which a parameter vector's segments need not be.
  __device__ __forceinline__ static void params(const float* p, float missing, int width, int lane,
                                                float2 (&w)[N][E / 2]) {
    const bool aligned = ((uintptr_t)p & 15u) == 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (kVec && p && aligned && at(i, E - 1, lane) < width) {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
          const float4 v = *reinterpret_cast<const float4*>(p + at(i, e, lane));
          w[i][e / 2] = make_float2(v.x, v.y);
          w[i][e / 2 + 1] = make_float2(v.z, v.w);
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const int c0 = at(i, e, lane), c1 = at(i, e + 1, lane);
          w[i][e / 2] = make_float2(p && c0 < width ? p[c0] : missing, p && c1 < width ? p[c1] : missing);
        }
      }
    }
  }
};

// The first half of a sum of K values over the kLanes threads of a row: above a
// warp, each warp's sum goes to its slots of `shared`.
template <int kLanes, int K>
__device__ __forceinline__ void row_sum_publish(float (&v)[K], float* shared) {
  constexpr int kWide = kLanes < 32 ? kLanes : 32;
#pragma unroll
  for (int o = kWide / 2; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(kFullMask, v[k], o);
  if constexpr (kLanes > 32)
    if ((threadIdx.x & 31) == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) shared[threadIdx.x / 32 * K + k] = v[k];
}

// Waits for the other threads of this thread's row.
template <int kLanes>
__device__ __forceinline__ void row_wait() {
  if constexpr (kLanes <= 32) __syncwarp();
  else
    asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / kLanes), "n"(kLanes) : "memory");
}

// The second half, after row_wait: the warps' sums in a fixed tree; every thread
// gets the total.
template <int kLanes, int K>
__device__ __forceinline__ void row_sum_collect(float (&v)[K], const float* shared) {
  if constexpr (kLanes > 32) {
    constexpr int kWarps = kLanes / 32;
    const float* mine = shared + (int)threadIdx.x / kLanes * kWarps * K;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float s[kWarps];
#pragma unroll
      for (int i = 0; i < kWarps; ++i) s[i] = mine[i * K + k];
#pragma unroll
      for (int w = 1; w < kWarps; w *= 2)
#pragma unroll
        for (int i = 0; i + w < kWarps; i += 2 * w) s[i] += s[i + w];
      v[k] = s[0];
    }
  }
}

// A block's threads: one row for each kLanes of them.  Register use decides
// (forward: three blocks of 256 on an SM; backward: one of 512).
template <int kLanes>
constexpr int forward_threads() {
  return kLanes > 256 ? kLanes : 256 / kLanes * kLanes;
}
template <int kLanes>
constexpr int backward_threads() {
  return kLanes > 512 ? kLanes : 512 / kLanes * kLanes;
}

// Rows on their way or at work in shared memory, as far as they fit.
template <typename T, int kLanes, bool kVec>
constexpr int forward_stages() {
  constexpr int kFit = ((kLanes > 256 ? 132 : 68) << 10) / (16 * Slice<T, kLanes, kVec>::ring_packs(forward_threads<kLanes>()));
  return kFit > 4 ? 4 : kFit;
}
template <typename T, int kLanes, bool kVec>
constexpr int backward_stages() {
  constexpr int kFit = (208 << 10) / (32 * Slice<T, kLanes, kVec>::ring_packs(backward_threads<kLanes>()));
  return kFit > 6 ? 6 : kFit;
}

// Forward.  Blocks walk over a worker's rows, with its weight and bias in
// registers.  The next rows are on their way while one is worked on: every
// thread copies its own packs to its own places in shared memory, so no barrier
// guards them (rows that are not aligned are copied and taken by all of a row's
// threads, between the barriers of its two sums).  kWhole: the width is a multiple
// of a pack, so no pack needs looking into.
//
// Measured (of 6694.5 GB/s): 16,384 rows of 1024 bf16 values 12.7 us (79 %), of 4096
// 46 us (87 %), of 5120 63 us (80 %), of 4095 65 us (62 %: single-element reads and
// writes), of 4096 fp32 ones 95 us (85 %); four rows of 512 on each of four workers 2.5 us.
// Groups of 512 and 1024 threads have 64 registers a thread and spill 8 to 92 bytes.
template <typename T, int kLanes, bool kVec, bool kWhole>
__global__ void __launch_bounds__(forward_threads<kLanes>(), kLanes > 512 ? 1 : kLanes > 256 ? 2 : 3)
    layer_norm_forward_kernel(LayerNormArgs a) {
  dq_pdl_enter();
  using S = Slice<T, kLanes, kVec>;
  constexpr int kThreads = forward_threads<kLanes>(), kGroups = kThreads / kLanes;
  constexpr int kStages = forward_stages<T, kLanes, kVec>(), kPacks = S::ring_packs(kThreads);
  constexpr bool ragged = !kWhole;
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ float shared[2][kThreads / 32];
  uint4* ring = reinterpret_cast<uint4*>(dynamic);  // [stage][packs]
  const int width = (int)a.width, lane = threadIdx.x % kLanes;
  const int64_t m = blockIdx.y, step = (int64_t)gridDim.x * kGroups;
  const int64_t first = (int64_t)blockIdx.x * kGroups;
  const T* xs = static_cast<const T*>(a.x) + m * a.rows * a.x_ld;
  T* ys = static_cast<T*>(a.out) + m * a.rows * a.out_ld;
  const auto fetch = [&](int64_t r, int stage, const T* all = nullptr) {
    if (r < a.rows) S::fetch(xs + r * a.x_ld, width, lane, ring + stage * kPacks, kThreads, all);
    copies_begun();
  };
  const int64_t mine = first + threadIdx.x / kLanes;
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) fetch(mine + s * step, s, s == 0 ? static_cast<const T*>(a.x) : nullptr);
  float2 w[S::N][S::E / 2], b[S::N][S::E / 2];
  S::params(a.weight ? a.weight + m * a.p_stride : nullptr, 1.f, width, lane, w);
  S::params(a.bias ? a.bias + m * a.p_stride : nullptr, 0.f, width, lane, b);
  const float inv_width = 1.f / (float)width;
  int stage = 0;
  if (!kVec) {
    wait_copies<kStages - 2>();
    row_wait<kLanes>();
  }
  for (int64_t r0 = first; r0 < a.rows; r0 += step) {
    const int64_t r = r0 + threadIdx.x / kLanes;
    const bool live = r < a.rows;
    uint4 p[S::N];
    if (kVec) {
      fetch(r + (kStages - 1) * step, stage == 0 ? kStages - 1 : stage - 1);
      wait_copies<kStages - 1>();
    }
    S::take(ring + stage * kPacks, xs + r * a.x_ld, lane, kThreads, p);
    stage = stage + 1 == kStages ? 0 : stage + 1;
    float2 x[S::N][S::E / 2], t = both(0.f);
#pragma unroll
    for (int i = 0; i < S::N; ++i)
#pragma unroll
      for (int e = 0; e < S::E; e += 2) {
        x[i][e / 2] = pair_of<T>(p[i], e);
        t = add2(t, x[i][e / 2]);
      }
    float s[1] = {t.x + t.y};
    row_sum_publish<kLanes, 1>(s, shared[0]);
    row_wait<kLanes>();
    if (!kVec) {  // the row before was taken by all; the next one has come when they meet again
      fetch(r + (kStages - 1) * step, stage >= 2 ? stage - 2 : stage + kStages - 2);
      wait_copies<kStages - 2>();
    }
    row_sum_collect<kLanes, 1>(s, shared[0]);
    const float mean = s[0] * inv_width;
    t = both(0.f);
#pragma unroll
    for (int i = 0; i < S::N; ++i) {  // nothing past the row's end counts
      float2 u = both(0.f);
#pragma unroll
      for (int e = 0; e < S::E; e += 2) {
        float2 d = add2(x[i][e / 2], both(-mean));
        x[i][e / 2] = d;
        if (ragged) {
          if (S::at(i, e, lane) >= width) d.x = 0.f;
          if (S::at(i, e + 1, lane) >= width) d.y = 0.f;
        }
        u = fma2(d, d, u);
      }
      if (ragged || S::at(i, 0, lane) < width) t = add2(t, u);
    }
    s[0] = t.x + t.y;
    row_sum_publish<kLanes, 1>(s, shared[1]);
    row_wait<kLanes>();
    row_sum_collect<kLanes, 1>(s, shared[1]);
    const float rstd = rsqrtf(fmaf(s[0], inv_width, a.eps));  // 2 units at most, at a sixth of the division's instructions
#pragma unroll
    for (int i = 0; i < S::N; ++i)
#pragma unroll
      for (int e = 0; e < S::E; e += 2)
        set_pair<T>(p[i], e, fma2(mul2(x[i][e / 2], both(rstd)), w[i][e / 2], b[i][e / 2]));
    if (live) {
      S::store(ys + r * a.out_ld, width, lane, p);
      if (lane == 0 && a.mean) {
        a.mean[m * a.rows + r] = mean;
        a.rstd[m * a.rows + r] = rstd;
      }
    }
  }
}

// A row of the scratch space, in floats: whole 16-byte packs.
__host__ __device__ constexpr int64_t part_stride(int64_t width) { return (width + 3) / 4 * 4; }

// Backward.  A block walks over rows of one worker, its rows ahead on their way
// as above, and keeps each column's sums for dweight and dbias in registers; what
// it has at the end goes to its row of the scratch space, and a second kernel
// adds the blocks' rows up in order (with one block per worker it is the
// result).  A row's sums are published while the row before is finished from its
// packs in shared memory, which hides the exchange between the row's warps:
// one barrier a row.
//
// Measured: 16,384 rows of 4096 bf16 values 74 us with the join (82 % of 6694.5 GB/s),
// in fp32 133 us (91 %); of 8192 (512 a worker) 52 us (58 %) and of 1024 27 us (56 %):
// one block's 16 warps leave the row's chain exposed there.  Rows that are not
// aligned: of 4095 bf16 values 107 us (56 %).  Groups of 768 (fp32) and 1024 threads spill,
// up to 312 bytes of stores a thread in fp32: 4096 rows of 12,288 fp32 values 131 us
// (69 %), of 16,384 218 us (55 %), in bf16 81 us and 116 us (55 %, 52 %).  Tried: 32
// values a thread with the weights in shared memory, 79 us and 58 us.
template <typename T, int kLanes, bool kVec>
__global__ void __launch_bounds__(backward_threads<kLanes>(), 1) layer_norm_backward_kernel(LayerNormArgs a) {
  dq_pdl_enter();
  using S = Slice<T, kLanes, kVec>;
  constexpr int kThreads = backward_threads<kLanes>(), kGroups = kThreads / kLanes;
  constexpr int kStages = backward_stages<T, kLanes, kVec>(), kPacks = S::ring_packs(kThreads);
  constexpr bool kRing = kStages >= 3;  // else a row is read again from the caches
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ float shared[2][kThreads / 32 * 2];
  uint4* ring = reinterpret_cast<uint4*>(dynamic);  // [stage][x, dy][packs]
  const int width = (int)a.width, lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int64_t m = blockIdx.y, parts = gridDim.x, step = parts * kGroups;
  const int64_t first = (int64_t)blockIdx.x * kGroups;
  const T* xs = static_cast<const T*>(a.x) + m * a.rows * a.x_ld;
  const T* dys = static_cast<const T*>(a.dy) + m * a.rows * a.dy_ld;

  const auto fetch = [&](int64_t r, int stage, bool begins = false) {
    if (!kRing) return;
    if (r < a.rows) {
      uint4* to = ring + stage * 2 * kPacks;
      S::fetch(xs + r * a.x_ld, width, lane, to, kThreads, begins ? static_cast<const T*>(a.x) : nullptr);
      S::fetch(dys + r * a.dy_ld, width, lane, to + kPacks, kThreads, begins ? static_cast<const T*>(a.dy) : nullptr);
    }
    copies_begun();
  };
  const auto take = [&](int64_t r, int stage, uint4 (&x)[S::N], uint4 (&g)[S::N]) {
    if (kRing) {
      S::take(ring + stage * 2 * kPacks, xs + r * a.x_ld, lane, kThreads, x);
      S::take(ring + stage * 2 * kPacks + kPacks, dys + r * a.dy_ld, lane, kThreads, g);
    } else {
      S::load(xs + r * a.x_ld, width, lane, x);
      S::load(dys + r * a.dy_ld, width, lane, g);
    }
  };
#pragma unroll
  for (int s = 0; s < kStages - 2; ++s) fetch(first + group + s * step, s, s == 0);

  float2 w[S::N][S::E / 2], sw[S::N][S::E / 2], sb[S::N][S::E / 2];
  S::params(a.weight ? a.weight + m * a.p_stride : nullptr, 1.f, width, lane, w);
#pragma unroll
  for (int i = 0; i < S::N; ++i)
#pragma unroll
    for (int e = 0; e < S::E / 2; ++e) sw[i][e] = sb[i][e] = both(0.f);
  const float inv_width = 1.f / (float)width;

  float s[2] = {0.f, 0.f}, mean = 0.f, rstd = 0.f;  // of the row before
  float next_mean = 0.f, next_rstd = 0.f;           // of the row at hand
  if (first + group < a.rows) {
    next_mean = a.mean[m * a.rows + first + group];
    next_rstd = a.rstd[m * a.rows + first + group];
  }
  int stage = 0, before = 0, parity = 0;
  if (!kVec && kRing) {
    wait_copies<kStages >= 3 ? kStages - 3 : 0>();
    row_wait<kLanes>();
  }
  int64_t last = -1;  // the row before
  for (int64_t r0 = first; r0 < a.rows + step; r0 += step) {
    const int64_t r = r0 + group;
    float sum[2] = {0.f, 0.f};
    const float new_mean = next_mean, new_rstd = next_rstd;
    if (kRing) {  // the stage of the row before last is free
      fetch(r + (kStages - 2) * step, stage + kStages - 2 >= kStages ? stage - 2 : stage + kStages - 2);
      // rows that all of their threads copy: the one after this has come when they meet at the turn's end
      wait_copies<kVec ? (kStages >= 2 ? kStages - 2 : 0) : (kStages >= 3 ? kStages - 3 : 0)>();
    }
    if (r < a.rows) {
      if (r + step < a.rows) {
        next_mean = a.mean[m * a.rows + r + step];
        next_rstd = a.rstd[m * a.rows + r + step];
      }
      uint4 x[S::N], g[S::N];
      take(r, stage, x, g);
      float2 s0 = both(0.f), s1 = both(0.f);
#pragma unroll
      for (int i = 0; i < S::N; ++i)
#pragma unroll
        for (int e = 0; e < S::E; e += 2) {  // past the row's end dy is 0
          const float2 h = mul2(add2(pair_of<T>(x[i], e), both(-new_mean)), both(new_rstd));
          const float2 d = pair_of<T>(g[i], e);
          sw[i][e / 2] = fma2(d, h, sw[i][e / 2]);
          sb[i][e / 2] = add2(sb[i][e / 2], d);
          const float2 wd = mul2(d, w[i][e / 2]);
          s0 = add2(s0, wd);
          s1 = fma2(wd, h, s1);
        }
      sum[0] = s0.x + s0.y;
      sum[1] = s1.x + s1.y;
    }
    row_sum_publish<kLanes, 2>(sum, shared[parity]);
    if (last >= 0 && a.out) {
      uint4 x[S::N], g[S::N];
      take(last, before, x, g);
      row_sum_collect<kLanes, 2>(s, shared[parity ^ 1]);
      // dx = rstd (dy w - c1 - h c2)
      const float c1 = s[0] * inv_width, c2 = s[1] * inv_width;
#pragma unroll
      for (int i = 0; i < S::N; ++i)
#pragma unroll
        for (int e = 0; e < S::E; e += 2) {
          const float2 h = mul2(add2(pair_of<T>(x[i], e), both(-mean)), both(rstd));
          const float2 wd = fma2(pair_of<T>(g[i], e), w[i][e / 2], both(-c1));
          set_pair<T>(g[i], e, mul2(fma2(h, both(-c2), wd), both(rstd)));
        }
      S::store(static_cast<T*>(a.out) + (m * a.rows + last) * a.out_ld, width, lane, g);
    }
    row_wait<kLanes>();
    s[0] = sum[0];
    s[1] = sum[1];
    mean = new_mean;
    rstd = new_rstd;
    last = r < a.rows ? r : -1;
    before = stage;
    stage = stage + 1 == kStages ? 0 : stage + 1;
    parity ^= 1;
  }
  dq_pdl_release();  // the join's blocks, if any, may take up places as this grid's come free
  if (!a.dweight && !a.dbias) return;
  // the groups' sums in order, through shared memory in the ring's place
  float* sums = reinterpret_cast<float*>(dynamic);
  if (kRing) asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const auto value = [&](int i, int e) {
      const float2 v = which == 0 ? sw[i][e / 2] : sb[i][e / 2];
      return e % 2 == 0 ? v.x : v.y;
    };
    if (kGroups > 1) {
      __syncthreads();
      S::each(width, lane, [&](int i, int e, int c) { sums[group * width + c] = value(i, e); });
      __syncthreads();
    }
    float* out = which == 0 ? a.dweight : a.dbias;
    if (!out) continue;
    out += m * a.g_stride;
    const bool whole = parts == 1;
    float* part = a.scratch + ((m * parts + blockIdx.x) * 2 + which) * part_stride(a.width);
    const auto put = [&](int c, float v) {
      if (whole) out[c] = a.accumulate ? out[c] + v : v;
      else part[c] = v;
    };
    if (kGroups > 1) {
      for (int c = threadIdx.x; c < width; c += kThreads) {
        float v = sums[c];
        for (int k = 1; k < kGroups; ++k) v += sums[k * width + c];
        put(c, v);
      }
    } else {
      S::each(width, lane, [&](int i, int e, int c) { put(c, value(i, e)); });
    }
  }
}

// The blocks' rows of the scratch space, added up in order: a block takes 128
// columns of one worker's dweight or dbias, its warps every kJoinWarps-th row.
constexpr int kJoinWarps = 8;

__global__ void __launch_bounds__(kJoinWarps * 32) layer_norm_join_kernel(LayerNormArgs a, int parts) {
  dq_pdl_enter();
  __shared__ float4 shared[kJoinWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, which = blockIdx.z;
  const int64_t m = blockIdx.y, c = ((int64_t)blockIdx.x * 32 + lane) * 4;
  float* out = which == 0 ? a.dweight : a.dbias;
  if (!out) return;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < a.width)
#pragma unroll 4
    for (int p = warp; p < parts; p += kJoinWarps) {
      const float4 w = *reinterpret_cast<const float4*>(a.scratch + ((m * parts + p) * 2 + which) * part_stride(a.width) + c);
      v = make_float4(v.x + w.x, v.y + w.y, v.z + w.z, v.w + w.w);
    }
  shared[warp][lane] = v;
  __syncthreads();
  if (warp != 0) return;
#pragma unroll
  for (int i = 1; i < kJoinWarps; ++i) {
    const float4 w = shared[i][lane];
    v = make_float4(v.x + w.x, v.y + w.y, v.z + w.z, v.w + w.w);
  }
  out += m * a.g_stride + c;
  const float sums[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (c + k < a.width) out[k] = a.accumulate ? out[k] + sums[k] : sums[k];
}

// Rows of more than kMaxOnChip values, one block each: further passes over the
// row come out of the caches, a value at a time.  4000 rows of 20,000 bf16 values
// forward 131 us (36 % of 6694.5 GB/s), backward, where the parameters' sums read x and dy
// once more, 377 us (19 %).
constexpr int kLongThreads = 512;

template <typename T>
__global__ void __launch_bounds__(kLongThreads) layer_norm_forward_long_kernel(LayerNormArgs a) {
  dq_pdl_enter();
  __shared__ float shared[32];
  const int64_t row = blockIdx.x;
  const int64_t m = row / a.rows;
  const T* x = static_cast<const T*>(a.x) + row * a.x_ld;
  T* y = static_cast<T*>(a.out) + row * a.out_ld;
  const float* weight = a.weight ? a.weight + m * a.p_stride : nullptr;
  const float* bias = a.bias ? a.bias + m * a.p_stride : nullptr;
  float s = 0.f;
  for (int64_t c = threadIdx.x; c < a.width; c += kLongThreads) s += to_float(x[c]);
  const float mean = block_sum(s, shared) / (float)a.width;
  s = 0.f;
  for (int64_t c = threadIdx.x; c < a.width; c += kLongThreads) {
    const float d = to_float(x[c]) - mean;
    s = fmaf(d, d, s);
  }
  const float rstd = 1.f / sqrtf(block_sum(s, shared) / (float)a.width + a.eps);
  for (int64_t c = threadIdx.x; c < a.width; c += kLongThreads) {
    const float h = (to_float(x[c]) - mean) * rstd;
    y[c] = from_float<T>(fmaf(h, weight ? weight[c] : 1.f, bias ? bias[c] : 0.f));
  }
  if (threadIdx.x == 0 && a.mean) {
    a.mean[row] = mean;
    a.rstd[row] = rstd;
  }
}

template <typename T>
__global__ void __launch_bounds__(kLongThreads) layer_norm_dx_long_kernel(LayerNormArgs a) {
  dq_pdl_enter();
  __shared__ float shared[32];
  const int64_t row = blockIdx.x;
  const int64_t m = row / a.rows;
  const T* x = static_cast<const T*>(a.x) + row * a.x_ld;
  const T* dy = static_cast<const T*>(a.dy) + row * a.dy_ld;
  T* dx = static_cast<T*>(a.out) + row * a.out_ld;
  const float* weight = a.weight ? a.weight + m * a.p_stride : nullptr;
  const float mean = a.mean[row], rstd = a.rstd[row];
  float s1 = 0.f, s2 = 0.f;
  for (int64_t c = threadIdx.x; c < a.width; c += kLongThreads) {
    const float g = to_float(dy[c]) * (weight ? weight[c] : 1.f);
    s1 += g;
    s2 = fmaf(g, (to_float(x[c]) - mean) * rstd, s2);
  }
  const float c1 = block_sum(s1, shared) / (float)a.width;
  const float c2 = block_sum(s2, shared) / (float)a.width;
  for (int64_t c = threadIdx.x; c < a.width; c += kLongThreads) {
    const float g = to_float(dy[c]) * (weight ? weight[c] : 1.f);
    const float h = (to_float(x[c]) - mean) * rstd;
    dx[c] = from_float<T>(rstd * (g - fmaf(h, c2, c1)));
  }
}

// dweight and dbias: a block takes 32 columns of one worker; its 8 warps take
// every eighth row and their sums are added in order.
template <typename T>
__global__ void __launch_bounds__(256) layer_norm_dparams_long_kernel(LayerNormArgs a) {
  dq_pdl_enter();
  __shared__ float sw[8][32], sb[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const int64_t m = blockIdx.y, c = (int64_t)blockIdx.x * 32 + lane;
  float w = 0.f, b = 0.f;
  if (c < a.width)
    for (int64_t r = warp; r < a.rows; r += 8) {
      const int64_t row = m * a.rows + r;
      const float g = to_float(static_cast<const T*>(a.dy)[row * a.dy_ld + c]);
      const float h = (to_float(static_cast<const T*>(a.x)[row * a.x_ld + c]) - a.mean[row]) * a.rstd[row];
      w = fmaf(g, h, w);
      b += g;
    }
  sw[warp][lane] = w;
  sb[warp][lane] = b;
  __syncthreads();
  if (warp != 0 || c >= a.width) return;
  for (int i = 1; i < 8; ++i) {
    w += sw[i][lane];
    b += sb[i][lane];
  }
  if (a.dweight) {
    float* out = a.dweight + m * a.g_stride + c;
    *out = a.accumulate ? *out + w : w;
  }
  if (a.dbias) {
    float* out = a.dbias + m * a.g_stride + c;
    *out = a.accumulate ? *out + b : b;
  }
}

// Blocks of the backward pass over all workers.
int64_t backward_blocks(int64_t workers) { return max64(workers, device_sms()); }

template <int kLanes>
struct Lanes {
  static constexpr int value = kLanes;
};

// Calls f with the number of threads that hold a row of `width` values.
template <typename F>
cudaError_t with_lanes(int64_t width, F&& f) {
  if (width <= 8 * kPerThread) return f(Lanes<8>{});
  if (width <= 16 * kPerThread) return f(Lanes<16>{});
  if (width <= 32 * kPerThread) return f(Lanes<32>{});
  if (width <= 64 * kPerThread) return f(Lanes<64>{});
  if (width <= 96 * kPerThread) return f(Lanes<96>{});
  if (width <= 128 * kPerThread) return f(Lanes<128>{});
  if (width <= 192 * kPerThread) return f(Lanes<192>{});
  if (width <= 256 * kPerThread) return f(Lanes<256>{});
  if (width <= 384 * kPerThread) return f(Lanes<384>{});
  if (width <= 512 * kPerThread) return f(Lanes<512>{});
  if (width <= 768 * kPerThread) return f(Lanes<768>{});
  return f(Lanes<1024>{});
}

bool rows_aligned(const void* p, int64_t ld, size_t size) {
  return ((uintptr_t)p & 15u) == 0 && ld * (int64_t)size % 16 == 0;
}

template <typename T, int kLanes, bool kVec, bool kWhole>
cudaError_t forward(const LayerNormArgs& a, cudaStream_t stream) {
  constexpr int kThreads = forward_threads<kLanes>(), kGroups = kThreads / kLanes;
  constexpr int kShared = forward_stages<T, kLanes, kVec>() * 16 * Slice<T, kLanes, kVec>::ring_packs(kThreads);
  static std::atomic<int> kept[kKeptDevices];
  int resident = 0;
  const cudaError_t st =
      resident_ctas(layer_norm_forward_kernel<T, kLanes, kVec, kWhole>, kThreads, kShared, kShared, kept, &resident);
  if (st != cudaSuccess) return st;
  const int64_t blocks = min64(max64(resident / a.workers, 1), ceil_div(a.rows, kGroups));
  return launch_pdl(layer_norm_forward_kernel<T, kLanes, kVec, kWhole>, dim3((unsigned)blocks, (unsigned)a.workers),
                    dim3(kThreads), kShared, stream, a);
}

template <typename T, int kLanes, bool kVec>
cudaError_t backward(const LayerNormArgs& a, cudaStream_t stream, uint64_t* launches) {
  constexpr int kThreads = backward_threads<kLanes>(), kGroups = kThreads / kLanes;
  constexpr int kStages = backward_stages<T, kLanes, kVec>();
  constexpr int kRing = kStages >= 3 ? kStages * 32 * Slice<T, kLanes, kVec>::ring_packs(kThreads) : 0;
  constexpr int kSums = kGroups > 1 ? kThreads * kPerThread * 4 : 0;
  constexpr int kShared = kRing > kSums ? kRing : kSums;
  static std::atomic<int> kept[kKeptDevices];
  int resident = 0;
  cudaError_t st = resident_ctas(layer_norm_backward_kernel<T, kLanes, kVec>, kThreads, kShared, kShared, kept, &resident);
  if (st != cudaSuccess) return st;
  const bool sums = a.dweight || a.dbias;
  const int64_t most = sums ? backward_blocks(a.workers) : max64(a.workers, resident);
  const int64_t parts = max64(1, min64(most / a.workers, ceil_div(a.rows, kGroups)));
  ++*launches;
  st = launch_pdl(layer_norm_backward_kernel<T, kLanes, kVec>, dim3((unsigned)parts, (unsigned)a.workers), dim3(kThreads),
                  kShared, stream, a);
  if (st != cudaSuccess || !sums || parts == 1) return st;
  ++*launches;
  return launch_pdl(layer_norm_join_kernel, dim3((unsigned)ceil_div(a.width, 128), (unsigned)a.workers, 2),
                    dim3(kJoinWarps * 32), 0, stream, a, (int)parts);
}

}  // namespace

size_t layer_norm_scratch_bytes(int64_t width, int32_t workers) {
  return width <= kMaxOnChip ? 8 * (size_t)part_stride(width) * (size_t)backward_blocks(workers) : 0;
}

cudaError_t launch_layer_norm_forward(const LayerNormArgs& a, cudaStream_t stream, uint64_t* launches) {
  const int64_t rows = a.rows * a.workers;
  if (rows == 0) return cudaSuccess;
  ++*launches;
  return with_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    if (a.width > kMaxOnChip)
      return launch_pdl(layer_norm_forward_long_kernel<T>, dim3((unsigned)rows), dim3(kLongThreads), 0, stream, a);
    const bool vec = rows_aligned(a.x, a.x_ld, sizeof(T)) && rows_aligned(a.out, a.out_ld, sizeof(T));
    return with_lanes(a.width, [&](auto lanes) {
      constexpr int kLanes = decltype(lanes)::value;
      if (!vec) return forward<T, kLanes, false, false>(a, stream);
      return a.width % (16 / (int64_t)sizeof(T)) == 0 ? forward<T, kLanes, true, true>(a, stream)
                                                       : forward<T, kLanes, true, false>(a, stream);
    });
  });
}

cudaError_t launch_layer_norm_backward(const LayerNormArgs& a, cudaStream_t stream, uint64_t* launches) {
  const int64_t rows = a.rows * a.workers;
  return with_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    if (a.width <= kMaxOnChip) {
      const bool vec = rows_aligned(a.x, a.x_ld, sizeof(T)) && rows_aligned(a.dy, a.dy_ld, sizeof(T)) &&
                       (!a.out || rows_aligned(a.out, a.out_ld, sizeof(T)));
      return with_lanes(a.width, [&](auto lanes) {
        constexpr int kLanes = decltype(lanes)::value;
        return vec ? backward<T, kLanes, true>(a, stream, launches) : backward<T, kLanes, false>(a, stream, launches);
      });
    }
    // the parameters' gradients first: dx may be dy
    if (a.dweight || a.dbias) {
      ++*launches;
      const cudaError_t st = launch_pdl(layer_norm_dparams_long_kernel<T>,
                                        dim3((unsigned)ceil_div(a.width, 32), a.workers), dim3(256), 0, stream, a);
      if (st != cudaSuccess) return st;
    }
    if (!a.out || rows == 0) return cudaSuccess;
    ++*launches;
    return launch_pdl(layer_norm_dx_long_kernel<T>, dim3((unsigned)rows), dim3(kLongThreads), 0, stream, a);
  });
}

}  // namespace dq
