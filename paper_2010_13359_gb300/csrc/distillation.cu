// Distillation from a teacher's top logits: the loss of each row, and its
// gradient with respect to the student's logits.
//
//   p_k = exp(t_k / T - L), q = softmax(z / T), P = sum p_k
//   loss = c T^2 sum p_k (log p_k - log q_id_k), dz = scale c T (P q - p at the ids)
#include <cmath>

#include "device_common.cuh"
#include "operators.cuh"

namespace dq {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxEntries = 1024;

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

// One block per row.
template <typename T, typename E, DistillationWay kWay>
__global__ void __launch_bounds__(kThreads) distillation_kernel(DistillationArgs a) {
  dq_pdl_enter();
  __shared__ float shared[32];
  __shared__ int32_t id[kMaxEntries];
  __shared__ float p[kMaxEntries], fix[kMaxEntries];
  const int64_t row = blockIdx.x;
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  T* dz = kWay == DistillationWay::kForward ? nullptr : static_cast<T*>(a.dlogits) + row * a.dld;
  const float c = a.weights ? a.weights[row] : 1.f;
  const float inv_t = 1.f / a.temperature;

  // the teacher's entries: p holds t / T, then the probabilities
  float most = -INFINITY;
  for (int k = threadIdx.x; k < a.k; k += kThreads) {
    const int32_t v = a.ids[row * a.teacher_ld + k];
    const float t = to_float(static_cast<const E*>(a.values)[row * a.teacher_ld + k]) * inv_t;
    const bool there = v >= 0 && v < a.vocab && t != -INFINITY;
    id[k] = there ? v : -1;
    p[k] = there ? t : -INFINITY;
    if (there) most = fmaxf(most, t);
  }
  const bool any = __syncthreads_or(most > -INFINITY ? 1 : 0);
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
    lse_t = a.teacher_lse[row];
  } else {
    most = block_max(most, shared);
    float s = 0.f;
    for (int k = threadIdx.x; k < a.k; k += kThreads)
      if (id[k] >= 0) s += expf(p[k] - most);
    lse_t = most + logf(block_sum(s, shared));
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
      const float logp = p[k] - lse_t;
      const float pk = expf(logp);
      if (pk > 0.f) loss += pk * (logp - ((to_float(z[id[k]]) - top) * inv_t - log_sum));
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

template <typename T, typename E>
cudaError_t launch(const DistillationArgs& a, DistillationWay way, cudaStream_t stream) {
  auto kernel = way == DistillationWay::kForward    ? distillation_kernel<T, E, DistillationWay::kForward>
                : way == DistillationWay::kBackward ? distillation_kernel<T, E, DistillationWay::kBackward>
                                                    : distillation_kernel<T, E, DistillationWay::kStep>;
  return launch_pdl(kernel, dim3((unsigned)a.rows), dim3(kThreads), 0, stream, a);
}

}  // namespace

cudaError_t launch_distillation(const DistillationArgs& a, DistillationWay way, cudaStream_t stream,
                                uint64_t* launches) {
  if (a.rows == 0) return cudaSuccess;
  ++*launches;
  return with_dtype(a.dtype, [&](auto t) {
    return with_dtype(a.teacher_dtype, [&](auto e) { return launch<decltype(t), decltype(e)>(a, way, stream); });
  });
}

}  // namespace dq
