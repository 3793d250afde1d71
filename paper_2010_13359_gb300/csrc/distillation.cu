// Distillation from a teacher's top logits: the loss of each row, and its
// gradient with respect to the student's logits.
//
//   p_k = exp(t_k / T - L), q = softmax(z / T), P = sum p_k
//   loss = c T^2 sum p_k (log p_k - log q_id_k), dz = scale c T (P q - p at the ids)
//
// Bound by memory: the logits in, the gradient out, and about five operations and
// one exponential a value for each of the two passes over a row (its softmax's
// maximum and sum, then the gradient).  So a row is read once and held in
// shared memory between them.
#include <cmath>
#include <type_traits>

#include "device_common.cuh"
#include "operators.cuh"

namespace dq {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxEntries = 1024;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float teacher_value(const DistillationArgs& a, int64_t row, int k) {
  const int64_t i = row * a.teacher_ld + k;
  if (a.teacher_dtype == DQGAN_F32) return static_cast<const float*>(a.values)[i];
  if (a.teacher_dtype == DQGAN_BF16) return to_float(static_cast<const __nv_bfloat16*>(a.values)[i]);
  return to_float(static_cast<const __half*>(a.values)[i]);
}

// 2^x, subnormal results flushed to 0.
__device__ __forceinline__ float exp2_ftz(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float block_max(float x, float* shared) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(kFullMask, x, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x / 32] = x;
  __syncthreads();
  x = shared[0];
  for (int i = 1; i < kThreads / 32; ++i) x = fmaxf(x, shared[i]);
  return x;
}

// Rows that do not fit on chip: one block each, which reads its row once for the
// maximum, once for the sum and once for the gradient, the later times out of the
// L2 as far as that holds them, a value at a time: 256 rows of 1,000,003 bf16 values
// 3.97 ms, 4 % of 6694.5 GB/s.
template <typename T, DistillationWay kWay>
__global__ void __launch_bounds__(kThreads) distillation_long_kernel(DistillationArgs a) {
  dq_pdl_enter();
  __shared__ float shared[32];
  __shared__ int32_t id[kMaxEntries];
  __shared__ float p[kMaxEntries], fix[kMaxEntries];
  const int64_t row = blockIdx.x;
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  T* dz = kWay == DistillationWay::kForward ? nullptr : static_cast<T*>(a.dlogits) + row * a.dld;
  const float c = a.weights ? a.weights[row] : 1.f;
  const float inv_t = 1.f / a.temperature;

  // the teacher's entries: p holds t, then the probabilities.  log p = (t - most) / T - lse_t, the difference first,
  // so that the type's lowest values do not overflow (most: 0 where L is given)
  float most = -INFINITY;
  bool some = false;
  for (int k = threadIdx.x; k < a.k; k += kThreads) {
    const int32_t v = a.ids[row * a.teacher_ld + k];
    const float t = teacher_value(a, row, k);
    const bool there = v >= 0 && v < a.vocab && t != -INFINITY;
    id[k] = there ? v : -1;
    p[k] = there ? t : -INFINITY;
    if (there) most = fmaxf(most, t);
    some = some || there;
  }
  const bool any = __syncthreads_or(some ? 1 : 0);
  if (!any || c == 0.f) {
    if (threadIdx.x == 0 && kWay != DistillationWay::kBackward) {
      a.loss[row] = 0.f;
      if (a.lse) a.lse[row] = 0.f;
    }
    if (kWay != DistillationWay::kForward)
      for (int64_t v = threadIdx.x; v < a.vocab; v += kThreads) dz[v] = from_float<T>(0.f);
    return;
  }
  float lse_t;
  if (a.teacher_lse) {
    most = 0.f;
    lse_t = a.teacher_lse[row];
  } else {
    most = block_max(most, shared);
    float s = 0.f;
    for (int k = threadIdx.x; k < a.k; k += kThreads)
      if (id[k] >= 0) s += expf((p[k] - most) * inv_t);
    lse_t = logf(block_sum(s, shared));
  }

  // q_v = exp((z_v - top) / T) / sum; in the gradient alone exp(z_v / T - lse)
  float top = 0.f, sum = 1.f, log_sum = 0.f;
  if (kWay == DistillationWay::kBackward) {
    log_sum = a.lse[row];
  } else {
    top = -INFINITY;
    for (int64_t v = threadIdx.x; v < a.vocab; v += kThreads) top = fmaxf(top, to_float(z[v]));
    top = block_max(top, shared);
    float s = 0.f;
    for (int64_t v = threadIdx.x; v < a.vocab; v += kThreads) s += expf((to_float(z[v]) - top) * inv_t);
    sum = block_sum(s, shared);
    log_sum = logf(sum);
  }
  const auto q_of = [&](T x) {
    return kWay == DistillationWay::kBackward ? expf(to_float(x) * inv_t - log_sum)
                                              : expf((to_float(x) - top) * inv_t) / sum;
  };

  float loss = 0.f, mass = 0.f;
  for (int k = threadIdx.x; k < a.k; k += kThreads)
    if (id[k] >= 0) {
      const float logp = (p[k] - most) * inv_t - lse_t;
      const float pk = expf(logp);
      if (pk != 0.f) loss += pk * (logp - ((to_float(z[id[k]]) - top) * inv_t - log_sum));
      mass += pk;
      p[k] = pk;
    }
  mass = block_sum(mass, shared);
  if (kWay != DistillationWay::kBackward) {
    loss = block_sum(loss, shared);
    if (threadIdx.x == 0) {
      a.loss[row] = c * a.temperature * a.temperature * loss;
      if (a.lse) a.lse[row] = top * inv_t + log_sum;
    }
  }
  if (kWay == DistillationWay::kForward) return;
  const float factor = a.scale * c * a.temperature;
  __syncthreads();
  // the gradient at an id, by its first entry; all logits of entries are read before dz is written
  for (int k = threadIdx.x; k < a.k; k += kThreads) {
    if (id[k] < 0) continue;
    bool first = true;
    float sum = 0.f;
    for (int j = 0; j < a.k; ++j)
      if (id[j] == id[k]) {
        if (j < k) first = false;
        sum += p[j];
      }
    if (first) fix[k] = factor * (q_of(z[id[k]]) * mass - sum);
  }
  __syncthreads();
  for (int64_t v = threadIdx.x; v < a.vocab; v += kThreads)
    dz[v] = from_float<T>(factor * (q_of(z[v]) * mass));
  __syncthreads();
  for (int k = threadIdx.x; k < a.k; k += kThreads) {
    if (id[k] < 0) continue;
    bool first = true;
    for (int j = 0; j < k; ++j) first = first && id[j] != id[k];
    if (first) dz[id[k]] = from_float<T>(fix[k]);
  }
}

// The kernel for rows that fit on chip: a row belongs to a cluster of `pieces`
// blocks (1 to 8), each of which holds its piece in shared memory, every worker
// thread the packs that it copied there itself.  A warp takes its own maximum and
// sum of exponentials and writes the pair to every block of the cluster; one
// cluster barrier later each block joins all pairs and turns its packs into the
// gradient.  Clusters stay on the GPU and take row after row: as a thread has used
// a pack for the last time it copies the next row's into its place.  Helper warps
// prepare the teacher's entries of the next row meanwhile, and write the entries'
// own gradients when the workers are through: as an extra task of a worker warp
// they took half of the block's time at the barrier.
//
// Measured (of 6694.5 GB/s): both passes over 8192 x 128,000 bf16 761 us (82 %),
// over 4096 x 32,000 89 us (86 %), in fp32 191 us (82 %), in place 206 us; the loss alone
// 438 us (72 %) and 54 us (69 %); the gradient alone of 1023 x 50,001 fp32 70 us (88 %).  Issue slots are 63 % used and the rest goes to the row's two exchanges
// (cluster barrier, join) and to the start of each row's loads.  Rows of a few
// thousand values are bound by the latency of a row's chain: 8000 x 2300 with 8
// entries 37 us, a quarter of the bandwidth.
//
// Rows need not start on 16-byte boundaries: packs are aligned ones that lie in the
// row, and the values before the first and after the last pack belong to the first
// helper warp, a lane each.
constexpr int kMostWorkers = 256;
constexpr int kMostShared = 220 << 10;

template <typename T>
struct Packs {
  static constexpr int E = 16 / (int)sizeof(T);

  static __device__ __forceinline__ float value(const uint4& p, int e) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(reinterpret_cast<const uint32_t*>(&p)[e]);
    else return to_float(reinterpret_cast<const T*>(&p)[e]);
  }

  static __device__ __forceinline__ float max_of(const uint4& p) {  // NaN where nothing else
    if constexpr (sizeof(T) == 4) {
      return fmaxf(fmaxf(value(p, 0), value(p, 1)), fmaxf(value(p, 2), value(p, 3)));
    } else if constexpr (std::is_same<T, __half>::value) {
      const __half2* v = reinterpret_cast<const __half2*>(&p);
      const __half2 m = __hmax2(__hmax2(v[0], v[1]), __hmax2(v[2], v[3]));
      return fmaxf(__low2float(m), __high2float(m));
    } else {
      const __nv_bfloat162* v = reinterpret_cast<const __nv_bfloat162*>(&p);
      const __nv_bfloat162 m = __hmax2(__hmax2(v[0], v[1]), __hmax2(v[2], v[3]));
      return fmaxf(__low2float(m), __high2float(m));
    }
  }
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(kFullMask, x, o);
  return x;
}
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(kFullMask, x, o));
  return x;
}

// What a block's helpers make of the teacher's entries, for the block's part [lo, hi) of
// the vocabulary.  Arrays of k: t ((value - the greatest) / T, the difference first, so
// that the type's lowest values do not overflow and large ones keep their digits, or
// value / T where L is given; -inf where there is no entry), z (the logits at the ids), at
// (the id where this entry stands for it and it is in the part, else below 0), sum (p
// summed over the id's entries, where `at` has it).
struct Teacher {
  float* t;
  float* z;
  int32_t* at;
  float* sum;
};
__host__ __device__ constexpr int32_t teacher_bytes(int32_t k) { return 16 * ((4 * k + 3) / 4); }

template <int kHelpers>
constexpr int helper_warps() {
  return kHelpers / 32;
}
// What the helpers leave for a row beside the arrays.
template <int kHelpers>
struct TeacherTotals {
  float lse;                                // log p = t - lse: log sum exp t, or L
  float mass[helper_warps<kHelpers>()];     // sums of p of each helper warp
  int32_t any[helper_warps<kHelpers>()];    // whether it had entries
  float most[helper_warps<kHelpers>()], exps[helper_warps<kHelpers>()];  // on the way to L
  int32_t twice;                            // whether an id of the part came more than once
};

template <int kHelpers>
__device__ __forceinline__ void helpers_wait() {
  __syncwarp();
  if constexpr (kHelpers > 32) asm volatile("bar.sync 2, %0;" ::"n"(kHelpers) : "memory");
}

// seen: a bit for every value of the part, which finds ids that come twice at one
// atomic an entry (a hash table cost up to 17 us a row where ids were a fixed step apart).
template <typename T, int kHelpers>
__device__ __forceinline__ void prepare_teacher(const DistillationArgs& a, int64_t row, const Teacher& t,
                                                TeacherTotals<kHelpers>& totals, uint4* seen, int me, int lo, int hi, bool want_all,
                                                const T* z) {
  const int lane = me & 31, warp = me / 32;
  const float inv_t = 1.f / a.temperature;
  constexpr int kBatch = 2;  // loads of each kind on their way at once
  float most = -INFINITY;
  bool any = false;
  for (int k0 = me; k0 < a.k; k0 += kBatch * kHelpers) {
    int32_t id[kBatch];
    float v[kBatch], x[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int k = k0 + kHelpers * i;
      id[i] = k < a.k ? a.ids[row * a.teacher_ld + k] : -1;
      v[i] = k < a.k ? teacher_value(a, row, k) : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (id[i] >= a.vocab || v[i] == -INFINITY) id[i] = -1;
      const bool mine = id[i] >= lo && id[i] < hi;
      x[i] = id[i] >= 0 && (mine || want_all) ? to_float(z[id[i]]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int k = k0 + kHelpers * i;
      if (id[i] < 0) v[i] = -INFINITY;
      else any = true;
      most = fmaxf(most, v[i]);
      if (k >= a.k) continue;
      t.t[k] = a.teacher_lse ? v[i] * inv_t : v[i];
      t.at[k] = id[i] >= lo && id[i] < hi ? id[i] : -1;
      t.z[k] = x[i];
    }
  }
  for (int i = me; i < (hi - lo + 127) / 128; i += kHelpers) seen[i] = make_uint4(0, 0, 0, 0);
  any = __any_sync(kFullMask, any);
  if (!a.teacher_lse) most = warp_max(most);
  if (lane == 0) {
    totals.any[warp] = any;
    totals.most[warp] = most;
  }
  if (me == 0) totals.twice = 0;
  helpers_wait<kHelpers>();
  // an id's entries are joined at whichever of them comes first here
  for (int k = me; k < a.k; k += kHelpers) {
    const int at = t.at[k] - lo;
    if (at < 0) continue;
    if (atomicOr(reinterpret_cast<uint32_t*>(seen) + at / 32, 1u << at % 32) >> at % 32 & 1u) {
      t.at[k] = -2 - t.at[k];
      totals.twice = 1;
    }
  }
  float lse;
  if (a.teacher_lse) {
    lse = a.teacher_lse[row];
    helpers_wait<kHelpers>();
  } else {
    most = totals.most[0];
#pragma unroll
    for (int i = 1; i < helper_warps<kHelpers>(); ++i) most = fmaxf(most, totals.most[i]);
    if (most == -INFINITY) most = 0.f;  // no entry: L is not used
    float s = 0.f;
    for (int k = me; k < a.k; k += kHelpers) {
      const float x = (t.t[k] - most) * inv_t;
      t.t[k] = x;
      s += exp2_ftz(x * kLog2e);
    }
    s = warp_sum(s);
    if (lane == 0) totals.exps[warp] = s;
    helpers_wait<kHelpers>();
    s = totals.exps[0];
#pragma unroll
    for (int i = 1; i < helper_warps<kHelpers>(); ++i) s += totals.exps[i];
    lse = logf(s);
  }
  if (me == 0) totals.lse = lse;
  const auto p_of = [&](int k) { return t.t[k] == -INFINITY ? 0.f : exp2_ftz((t.t[k] - lse) * kLog2e); };
  float mass = 0.f;
  for (int k = me; k < a.k; k += kHelpers) {
    const float p = p_of(k);
    mass += p;
    t.sum[k] = p;
  }
  mass = warp_sum(mass);
  if (lane == 0) totals.mass[warp] = mass;
  if (totals.twice == 0) return;
  // ids that came again: their bits are taken out, which tells the entries that stand for them, and a warp looks
  // for an id's entries together (4096 x 32,000 with 1024 entries, one of them twice: 234 us; 3740 where every entry
  // looked for others by itself, 184 without one)
  for (int k = me; k < a.k; k += kHelpers) {
    const int at = -2 - t.at[k] - lo;
    if (t.at[k] < -1) atomicAnd(reinterpret_cast<uint32_t*>(seen) + at / 32, ~(1u << at % 32));
  }
  helpers_wait<kHelpers>();
  for (int k0 = me - lane; k0 < a.k; k0 += kHelpers) {
    const int k = k0 + lane, id = k < a.k ? t.at[k] : -1, at = id - lo;
    unsigned again =
        __ballot_sync(kFullMask, id >= 0 && !(reinterpret_cast<const uint32_t*>(seen)[at / 32] >> at % 32 & 1u));
    for (; again != 0; again &= again - 1u) {
      const int which = __ffs(again) - 1, wanted = __shfl_sync(kFullMask, id, which);
      float sum = 0.f;  // over places, whichever entry stands for the id
      for (int j = lane; j < a.k; j += 32)
        if (a.ids[row * a.teacher_ld + j] == wanted) sum += p_of(j);
      sum = warp_sum(sum);
      if (lane == which) t.sum[k] = sum;
    }
  }
}

// 16-byte packs of shared memory for a part's values, and for a bit for each of them and of a row's edges.
template <typename T>
__host__ __device__ constexpr int held_packs(int64_t vocab, int pieces) {
  return (int)(vocab * (int64_t)sizeof(T) / 16) / pieces + 1;
}
template <typename T>
__host__ __device__ constexpr int seen_packs(int held) {
  return (held * (16 / (int)sizeof(T)) + 32 + 127) / 128;
}
template <typename T>
__host__ __device__ constexpr int held_shared(int32_t k, int64_t vocab, int pieces) {
  return 2 * teacher_bytes(k) + 16 * (held_packs<T>(vocab, pieces) + seen_packs<T>(held_packs<T>(vocab, pieces)));
}

// A block's part of a row.
template <typename T, int kWorkers>
struct Part {
  static constexpr int E = 16 / (int)sizeof(T);
  const T* z;
  int head;        // values of the row before its first whole pack
  int p_lo, p_hi;  // the part's packs: pack p holds values head + p E and the E - 1 after it
  int lo, hi;      // the part's values, the row's edges included
  int n;           // this thread's packs: p_lo + threadIdx.x, + kWorkers, ...

  __device__ __forceinline__ Part(const DistillationArgs& a, int64_t row, int piece, int pieces) {
    const int vocab = (int)a.vocab;
    z = static_cast<const T*>(a.logits) + row * a.ld;
    head = min((int)((16 - (uintptr_t)z % 16) % 16 / sizeof(T)), vocab);
    const int packs = (vocab - head) / E;
    p_lo = packs / pieces * piece + min(piece, packs % pieces);
    p_hi = packs / pieces * (piece + 1) + min(piece + 1, packs % pieces);
    lo = piece == 0 ? 0 : head + p_lo * E;
    hi = piece == pieces - 1 ? vocab : head + p_hi * E;
    const int left = p_hi - p_lo - (int)threadIdx.x;
    n = threadIdx.x < kWorkers && left > 0 ? (left + kWorkers - 1) / kWorkers : 0;
  }
  __device__ __forceinline__ int first_value() const { return head + (p_lo + (int)threadIdx.x) * E; }
  // the value at the part's edges that this lane of the first helper warp holds, or -1
  __device__ __forceinline__ int edge_value() const {
    const int lane = threadIdx.x & 31, before = head + p_lo * E - lo, after = hi - (head + p_hi * E);
    if (lane < 16) return lane < before ? lane : -1;
    return lane - 16 < after ? hi - after + lane - 16 : -1;
  }
};

// Writes gradient_of(i), this thread's pack i, for every i: value by value where the gradient's rows are aligned
// otherwise than the logits' (4096 x 32,000 bf16 306 us, 89 where they are alike).
template <typename T, int kWorkers, typename F>
__device__ __forceinline__ void put_all(const Part<T, kWorkers>& part, T* dz, F&& gradient_of) {
  constexpr int E = Part<T, kWorkers>::E;
  T* to = dz + part.first_value();
  if (((uintptr_t)dz ^ (uintptr_t)part.z) % 16 == 0) {
#pragma unroll 4
    for (int i = 0; i < part.n; ++i) __stcs(reinterpret_cast<uint4*>(to) + i * kWorkers, gradient_of(i));
    return;
  }
  for (int i = 0; i < part.n; ++i) {
    const uint4 v = gradient_of(i);
#pragma unroll
    for (int j = 0; j < E; ++j) to[i * kWorkers * E + j] = reinterpret_cast<const T*>(&v)[j];
  }
}

// Helper threads of a block: twice as many for many teacher entries.
constexpr int helpers(int workers, bool many) { return (workers == 256 ? 64 : 32) * (many ? 2 : 1); }

template <typename T, DistillationWay kWay, int kWorkers, bool kMany>
__global__ void __launch_bounds__(kWorkers + helpers(kWorkers, kMany), 1024 / (kWorkers + helpers(kWorkers, kMany)))
    distillation_kernel(DistillationArgs a, int pieces) {
  dq_pdl_enter();
  // this block runs: others of its cluster wait for that before they write into its shared memory
  const bool exchanges = kWay != DistillationWay::kBackward && pieces > 1;
  if (exchanges) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  using P = Packs<T>;
  using Mine = Part<T, kWorkers>;
  constexpr int E = P::E, kWarps = kWorkers / 32;  // of workers
  constexpr bool kStats = kWay != DistillationWay::kBackward, kGradient = kWay != DistillationWay::kForward;
  extern __shared__ __align__(16) unsigned char dynamic[];
  // (maximum, sum) of every warp of the cluster; a block may write a row's while another reads the row before's
  __shared__ float2 pairs[2][kStats ? 8 * (kWarps + 1) : 1];
  constexpr int kHelpers = helpers(kWorkers, kMany);
  __shared__ TeacherTotals<kHelpers> totals[2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const bool works = warp < kWarps, first_helper = warp == kWarps;
  const int piece = blockIdx.x % pieces;
  const int64_t first_row = blockIdx.x / pieces, stride = gridDim.x / pieces;
  const auto teacher = [&](int parity) {
    Teacher t;
    t.t = reinterpret_cast<float*>(dynamic + parity * teacher_bytes(a.k));
    t.z = t.t + a.k;
    t.sum = t.z + a.k;
    t.at = reinterpret_cast<int32_t*>(t.sum + a.k);
    return t;
  };
  uint4* const seen = reinterpret_cast<uint4*>(dynamic + 2 * teacher_bytes(a.k));
  uint4* const held = seen + seen_packs<T>(held_packs<T>(a.vocab, pieces)) + threadIdx.x;  // this thread's packs
  const float inv_t = 1.f / a.temperature;

  // the weights of this cluster's next 32 rows, a lane each
  float some_weights = 0.f;
  int64_t weights_at = -1;  // the first of those rows, by the cluster's count
  const auto weight_of = [&](int64_t turn) {
    if (!a.weights) return 1.f;
    if (weights_at < 0 || turn - weights_at >= 32) {
      weights_at = turn;
      const int64_t row = first_row + (turn + lane) * stride;
      some_weights = row < a.rows ? a.weights[row] : 0.f;
    }
    return __shfl_sync(kFullMask, some_weights, (int)(turn - weights_at));
  };
  // the next row from `turn` on that counts; those before it get their zeros
  float next_c = 1.f;
  const auto advance = [&](int64_t turn) {
    for (;; ++turn) {
      const int64_t row = first_row + turn * stride;
      if (row >= a.rows) return turn;
      next_c = weight_of(turn);
      if (next_c != 0.f) return turn;
      if (kStats && piece == 0 && threadIdx.x == 0) {
        a.loss[row] = 0.f;
        if (a.lse) a.lse[row] = 0.f;
      }
      if (kGradient) {
        const Mine part(a, row, piece, pieces);
        T* const dz = static_cast<T*>(a.dlogits) + row * a.dld;
        put_all(part, dz, [](int) { return make_uint4(0, 0, 0, 0); });
        if (first_helper && part.edge_value() >= 0) dz[part.edge_value()] = from_float<T>(0.f);
      }
    }
  };
  float edge = 0.f, next_edge = 0.f;  // first helper warp: the lane's value at the part's edges
  const auto prepare = [&](const Mine& part, int64_t row, int parity) {
    next_edge = part.edge_value() >= 0 ? to_float(part.z[part.edge_value()]) : -INFINITY;
    prepare_teacher<T, kHelpers>(a, row, teacher(parity), totals[parity], seen, (int)threadIdx.x - kWorkers, part.lo, part.hi,
                                 kStats && piece == 0, part.z);
  };

  const auto all_run = [&] {
    __syncwarp();
    if (exchanges) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  };
  int64_t turn = advance(0);
  if (first_row + turn * stride >= a.rows) {  // as the whole cluster does
    all_run();
    return;
  }
  Mine part(a, first_row + turn * stride, piece, pieces);
  if (works) {
#pragma unroll 4
    for (int i = 0; i < part.n; ++i)
      copy16_async(held + i * kWorkers, reinterpret_cast<const uint4*>(part.z + part.first_value()) + i * kWorkers, 16);
  } else {
    prepare(part, first_row + turn * stride, 0);
  }
  all_run();
  for (int parity = 0;; parity ^= 1) {
    const int64_t row = first_row + turn * stride;
    const float c = next_c;
    T* const dz = kGradient ? static_cast<T*>(a.dlogits) + row * a.dld : nullptr;
    // the row after this one: its packs follow into this one's places
    const int64_t next_turn = advance(turn + 1);
    const bool last = first_row + next_turn * stride >= a.rows;
    const Mine next(a, last ? row : first_row + next_turn * stride, piece, pieces);
    const int next_n = last ? 0 : next.n;
    const uint4* const next_from = reinterpret_cast<const uint4*>(next.z + next.first_value());
    const auto follow = [&](int i) {
      if (i < next_n) copy16_async(held + i * kWorkers, next_from + i * kWorkers, 16);
    };

    // a value's q: exp2((v * mul + add) * by) * (1 / sum), in that order: the difference first, so that
    // the type's lowest values do not overflow
    float mul = 1.f, add = 0.f, by = inv_t * kLog2e, inv_sum = 1.f, log_sum = 0.f, top = -INFINITY, sum = 0.f;
    if (works) {
      asm volatile("cp.async.wait_all;" ::: "memory");
      if (kStats) {
#pragma unroll 4
        for (int i = 0; i < part.n; ++i) top = fmaxf(top, P::max_of(held[i * kWorkers]));
        top = warp_max(top);
        const float2 at = both(top == -INFINITY ? 0.f : -top);  // nothing but -inf in this warp: a sum of 0
        float2 s = both(0.f);
#pragma unroll 4
        for (int i = 0; i < part.n; ++i) {
          const uint4 x = held[i * kWorkers];
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            const float2 y = mul2(add2(pair_of<T>(x, e), at), both(by));
            s = add2(s, make_float2(exp2_ftz(y.x), exp2_ftz(y.y)));
          }
          if (!kGradient) follow(i);
        }
        sum = warp_sum(s.x + s.y);
      }
    } else if (kStats) {
      edge = next_edge;
      top = warp_max(edge);
      sum = warp_sum(exp2_ftz((edge - (top == -INFINITY ? 0.f : top)) * by));
    } else {
      edge = next_edge;
    }
    if (kStats) {
      if (pieces == 1) {
        if (lane == 0 && warp <= kWarps) pairs[parity][warp] = make_float2(top, sum);
        __syncthreads();
      } else {
        if (lane < pieces && warp <= kWarps) {
          const uint32_t mine = smem_addr(&pairs[parity][piece * (kWarps + 1) + warp]);
          uint32_t there;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(lane));
          asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(top), "f"(sum) : "memory");
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
      }
      // every warp joins the pairs, in the same order
      const int all = pieces * (kWarps + 1);
      float most = -INFINITY;
      for (int i = lane; i < all; i += 32) most = fmaxf(most, pairs[parity][i].x);
      top = warp_max(most);
      float total = 0.f;
      for (int i = lane; i < all; i += 32) {
        const float2 pair = pairs[parity][i];
        // a sum of 0 stays out: its maximum is -inf; a NaN goes in
        if (pair.y != 0.f) total = fmaf(pair.y, exp2_ftz((pair.x - top) * by), total);
      }
      total = warp_sum(total);
      add = -top;
      inv_sum = 1.f / total;
      log_sum = logf(total);
      if (top == -INFINITY) inv_sum = log_sum = NAN;
    } else {
      __syncthreads();
      mul = inv_t;
      add = -a.lse[row];
      by = kLog2e;
    }
    float mass = totals[parity].mass[0];
    int any = totals[parity].any[0];
#pragma unroll
    for (int i = 1; i < helper_warps<kHelpers>(); ++i) {
      mass += totals[parity].mass[i];
      any |= totals[parity].any[i];
    }
    const bool none = any == 0;
    const float factor = a.scale * c * a.temperature, coef = factor * mass * inv_sum;
    if (works) {
      if (kGradient) {
        if (none) {
          put_all(part, dz, [](int) { return make_uint4(0, 0, 0, 0); });
          for (int i = 0; i < part.n; ++i) follow(i);
        } else {
          put_all(part, dz, [&](int i) {
            uint4 v = held[i * kWorkers];
#pragma unroll
            for (int e = 0; e < E; e += 2) {
              const float2 y = mul2(fma2(pair_of<T>(v, e), both(mul), both(add)), both(by));
              set_pair<T>(v, e, mul2(make_float2(exp2_ftz(y.x), exp2_ftz(y.y)), both(coef)));
            }
            follow(i);
            return v;
          });
        }
        __syncwarp();
        asm volatile("bar.arrive 1, %0;" ::"n"(kWorkers + kHelpers) : "memory");
      }
      for (int i = part.n; i < next_n; ++i) follow(i);
    } else {
      const Teacher t = teacher(parity);
      if (kStats && piece == 0 && first_helper) {
        float loss = 0.f;
        const float lse_t = totals[parity].lse;
        if (!none)
          for (int k = lane; k < a.k; k += 32) {
            const float logp = t.t[k] - lse_t;
            const float p = exp2_ftz(logp * kLog2e);
            if (p != 0.f) loss = fmaf(p, logp - ((t.z[k] - top) * inv_t - log_sum), loss);
          }
        loss = warp_sum(loss);
        if (lane == 0) {
          a.loss[row] = none ? 0.f : c * a.temperature * a.temperature * loss;
          if (a.lse) a.lse[row] = none ? 0.f : fmaf(top, inv_t, log_sum);
        }
      }
      const int at_edge = first_helper ? part.edge_value() : -1;
      if (kGradient && at_edge >= 0)
        dz[at_edge] = from_float<T>(none ? 0.f : exp2_ftz(fmaf(edge, mul, add) * by) * coef);
      if (!last) prepare(next, first_row + next_turn * stride, parity ^ 1);
      if (kGradient) {
        // the entries' own gradients over what the workers wrote there
        __syncwarp();
        asm volatile("bar.sync 1, %0;" ::"n"(kWorkers + kHelpers) : "memory");
        if (!none)
          for (int k = (int)threadIdx.x - kWorkers; k < a.k; k += kHelpers)
            if (t.at[k] >= 0)
              dz[t.at[k]] = from_float<T>(fmaf(exp2_ftz(fmaf(t.z[k], mul, add) * by), coef, -factor * t.sum[k]));
      }
    }
    if (last) return;
    turn = next_turn;
    part = next;
  }
}

// Clusters of `pieces` blocks that fit on the GPU at once.  Asked of the runtime
// when the sizes differ from the last call's (a few microseconds).
template <typename K>
cudaError_t resident_clusters(K kern, int threads, int shared, int pieces, std::atomic<uint64_t> (&kept)[kKeptDevices],
                              int* clusters) {
  int dev = 0;
  cudaError_t st = cudaGetDevice(&dev);
  if (st != cudaSuccess) return st;
  if (dev < 0 || dev >= kKeptDevices) return cudaErrorInvalidDevice;
  const uint64_t key = (uint64_t)shared << 8 | (uint64_t)pieces, seen = kept[dev].load(std::memory_order_acquire);
  if (seen >> 24 == key) {
    *clusters = (int)(seen & 0xffffffu);
    return cudaSuccess;
  }
  if ((st = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared)) != cudaSuccess)
    return st;
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)pieces;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  lc.gridDim = dim3((unsigned)pieces);
  lc.blockDim = dim3((unsigned)threads);
  lc.dynamicSmemBytes = (size_t)shared;
  lc.attrs = attr;
  lc.numAttrs = 1;
  int n = 0;
  if ((st = cudaOccupancyMaxActiveClusters(&n, kern, &lc)) != cudaSuccess) return st;
  *clusters = n > 0 ? n : 1;
  kept[dev].store(key << 24 | (uint64_t)*clusters, std::memory_order_release);
  return cudaSuccess;
}

template <typename T, DistillationWay kWay, int kWorkers, bool kMany>
cudaError_t launch_held(const DistillationArgs& a, int pieces, cudaStream_t stream) {
  constexpr int kThreadsHeld = kWorkers + helpers(kWorkers, kMany);
  const auto kern = distillation_kernel<T, kWay, kWorkers, kMany>;
  static std::atomic<uint64_t> kept[kKeptDevices];
  const int shared = held_shared<T>(a.k, a.vocab, pieces);
  const int cluster = kWay == DistillationWay::kBackward ? 1 : pieces;  // its pieces exchange nothing
  int clusters = 0;
  const cudaError_t st = resident_clusters(kern, kThreadsHeld, shared, cluster, kept, &clusters);
  if (st != cudaSuccess) return st;
  const int64_t at_once = min64(a.rows, max64((int64_t)clusters * cluster / pieces, 1));
  return launch_pdl_cluster(kern, cluster, dim3((unsigned)(at_once * pieces)), dim3(kThreadsHeld), (size_t)shared, stream,
                            a, pieces);
}

template <typename T, DistillationWay kWay>
cudaError_t launch(const DistillationArgs& a, cudaStream_t stream) {
  const int packs = held_packs<T>(a.vocab, 1);
  // 2300 bf16 values, 8000 rows, us with the lesser and the greater number of helpers: 8 entries 37 | 39, 184
  // entries 72 | 54
  const auto many = [&](int w) { return a.k > (w == kMostWorkers ? 128 : 64); };
  int workers = 32, pieces = 1;
  if (packs <= 64 * 16) {
    // 4096 rows of 4000 bf16 values: 28 us with 64 workers, 38 with 32
    if (packs > 32 * 8) workers = 64;
  } else {
    // What counts is the rows on their way on an SM, as far as registers (launch bounds) and shared memory let
    // blocks onto it, and next the warps: 4096 rows, % of the measured copy bandwidth by (workers, pieces):
    // 50,000 bf16 values (256, 1) 200 KB on an SM: 89, (256, 2) 150 KB: 72; 80,000 (128, 4) 200 KB: 78, (256, 3)
    // 160 KB: 73; 128,000 (256, 4) 192 KB: 84, (128, 4) 192 KB: 79.
    int64_t best = 0;
    const int64_t sms = device_sms();
    for (int w = 128; w <= kMostWorkers; w *= 2)
      for (int p = 1; p <= 8; ++p) {
        const int shared = held_shared<T>(a.k, a.vocab, p), threads = w + helpers(w, many(w));
        if (shared > kMostShared || packs < p * w * 8) continue;
        // the gradient alone, whose pieces exchange nothing: 1023 x 50,001 fp32 values in 4 pieces 67 us, in 2 74
        if (kWay == DistillationWay::kBackward && packs > p * 4096 && p < 8) continue;
        const int64_t blocks = min64(1024 / threads, (226 << 10) / (shared + (3 << 10)));
        // (one block alone has nothing to do between its phases); the last turn may leave clusters idle
        const int64_t at_once = max64(blocks * sms / p, 1), turns = ceil_div(a.rows, at_once);
        const int64_t busy = a.rows <= at_once ? 100 : 100 * a.rows / (turns * at_once);
        const int64_t score =
            min64(blocks * (packs / p) * 16, 200 << 10) * (w == kMostWorkers ? 11 : 10) * (blocks > 1 ? 10 : 7) * busy + blocks;
        if (score <= best) continue;
        best = score;
        workers = w;
        pieces = p;
      }
  }
  if (held_shared<T>(a.k, a.vocab, pieces) > kMostShared)
    return launch_pdl(distillation_long_kernel<T, kWay>, dim3((unsigned)a.rows), dim3(kThreads), 0, stream, a);
  // few rows: more, smaller pieces, down to a pack a thread, while SMs are idle
  while (pieces < 8 && a.rows * (pieces + 1) <= device_sms() && packs > workers * pieces) ++pieces;
  const auto go = [&](auto of) {
    constexpr int kWorkers = decltype(of)::value;
    return many(kWorkers) ? launch_held<T, kWay, kWorkers, true>(a, pieces, stream)
                          : launch_held<T, kWay, kWorkers, false>(a, pieces, stream);
  };
  switch (workers) {
    case 32: return go(std::integral_constant<int, 32>{});
    case 64: return go(std::integral_constant<int, 64>{});
    case 128: return go(std::integral_constant<int, 128>{});
  }
  return go(std::integral_constant<int, kMostWorkers>{});
}

}  // namespace

cudaError_t launch_distillation(const DistillationArgs& a, DistillationWay way, cudaStream_t stream,
                                uint64_t* launches) {
  if (a.rows == 0) return cudaSuccess;
  ++*launches;
  return with_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    switch (way) {
      case DistillationWay::kForward: return launch<T, DistillationWay::kForward>(a, stream);
      case DistillationWay::kBackward: return launch<T, DistillationWay::kBackward>(a, stream);
      case DistillationWay::kStep: return launch<T, DistillationWay::kStep>(a, stream);
    }
    return cudaErrorInvalidValue;
  });
}

}  // namespace dq
