// Layer norm over the rows of W workers, and its gradient.
//
//   mu = mean(x), s^2 = mean((x - mu)^2), r = 1 / sqrt(s^2 + eps), h = (x - mu) r
//   y = h weight + bias
//   a = dy weight, dx = r (a - mean(a) - h mean(a h)), dweight = sum dy h, dbias = sum dy
#include "device_common.cuh"
#include "operators.cuh"

namespace dq {
namespace {

constexpr int kThreads = 256;

// One block per row: three passes over it, the later ones out of the caches.
template <typename T>
__global__ void __launch_bounds__(kThreads) layer_norm_forward_kernel(LayerNormArgs a) {
  dq_pdl_enter();
  __shared__ float shared[32];
  const int64_t row = blockIdx.x;
  const int64_t m = row / a.rows;
  const T* x = static_cast<const T*>(a.x) + row * a.x_ld;
  T* y = static_cast<T*>(a.out) + row * a.out_ld;
  const float* weight = a.weight ? a.weight + m * a.p_stride : nullptr;
  const float* bias = a.bias ? a.bias + m * a.p_stride : nullptr;
  float s = 0.f;
  for (int64_t c = threadIdx.x; c < a.width; c += kThreads) s += to_float(x[c]);
  const float mean = block_sum(s, shared) / (float)a.width;
  s = 0.f;
  for (int64_t c = threadIdx.x; c < a.width; c += kThreads) {
    const float d = to_float(x[c]) - mean;
    s = fmaf(d, d, s);
  }
  const float rstd = 1.f / sqrtf(block_sum(s, shared) / (float)a.width + a.eps);
  for (int64_t c = threadIdx.x; c < a.width; c += kThreads) {
    const float h = (to_float(x[c]) - mean) * rstd;
    y[c] = from_float<T>(fmaf(h, weight ? weight[c] : 1.f, bias ? bias[c] : 0.f));
  }
  if (threadIdx.x == 0 && a.mean) {
    a.mean[row] = mean;
    a.rstd[row] = rstd;
  }
}

// dx: one block per row.
template <typename T>
__global__ void __launch_bounds__(kThreads) layer_norm_dx_kernel(LayerNormArgs a) {
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
  for (int64_t c = threadIdx.x; c < a.width; c += kThreads) {
    const float g = to_float(dy[c]) * (weight ? weight[c] : 1.f);
    s1 += g;
    s2 = fmaf(g, (to_float(x[c]) - mean) * rstd, s2);
  }
  const float c1 = block_sum(s1, shared) / (float)a.width;
  const float c2 = block_sum(s2, shared) / (float)a.width;
  for (int64_t c = threadIdx.x; c < a.width; c += kThreads) {
    const float g = to_float(dy[c]) * (weight ? weight[c] : 1.f);
    const float h = (to_float(x[c]) - mean) * rstd;
    dx[c] = from_float<T>(rstd * (g - c1 - h * c2));
  }
}

// dweight and dbias: a block takes 32 columns of one worker; its 8 warps take
// every eighth row and their sums are added in order.
template <typename T>
__global__ void __launch_bounds__(kThreads) layer_norm_dparams_kernel(LayerNormArgs a) {
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

}  // namespace

size_t layer_norm_scratch_bytes(int64_t, int32_t) { return 0; }

cudaError_t launch_layer_norm_forward(const LayerNormArgs& a, cudaStream_t stream, uint64_t* launches) {
  const int64_t rows = a.rows * a.workers;
  if (rows == 0) return cudaSuccess;
  ++*launches;
  return with_dtype(a.dtype, [&](auto t) {
    return launch_pdl(layer_norm_forward_kernel<decltype(t)>, dim3((unsigned)rows), dim3(kThreads), 0, stream, a);
  });
}

cudaError_t launch_layer_norm_backward(const LayerNormArgs& a, cudaStream_t stream, uint64_t* launches) {
  const int64_t rows = a.rows * a.workers;
  return with_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    // the parameters' gradients first: dx may be dy
    if (a.dweight || a.dbias) {
      ++*launches;
      const cudaError_t st = launch_pdl(layer_norm_dparams_kernel<T>, dim3((unsigned)ceil_div(a.width, 32), a.workers),
                                        dim3(kThreads), 0, stream, a);
      if (st != cudaSuccess) return st;
    }
    if (!a.out || rows == 0) return cudaSuccess;
    ++*launches;
    return launch_pdl(layer_norm_dx_kernel<T>, dim3((unsigned)rows), dim3(kThreads), 0, stream, a);
  });
}

}  // namespace dq
