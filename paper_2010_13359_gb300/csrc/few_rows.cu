// Products of a few rows a worker, without tiles: what bounds them is the bytes of the weights (read once) and of their
// gradients (written once).  fp32 sums of products of the values as they are, without parts.
#include <type_traits>

#include "device_common.cuh"
#include "products.cuh"

namespace dq {

namespace {

// Sums over a warp's lanes of kValues values each (a power of two, at most 32): lane l gets one of them.  Each step sends
// half of what is left to the lane that keeps that half.
template <int kValues>
__device__ __forceinline__ int sum_over_lanes(float (&x)[kValues], int lane) {
  int which = 0;
  int d = 16;
#pragma unroll
  for (int h = kValues / 2; h > 0; h /= 2, d /= 2) {
    const bool upper = lane & d;
    if (upper) which += h;
#pragma unroll
    for (int i = 0; i < h; ++i) {
      const float send = upper ? x[i] : x[i + h], keep = upper ? x[i + h] : x[i];
      x[i] = keep + __shfl_xor_sync(kFullMask, send, d);
    }
  }
  for (; d > 0; d /= 2) x[0] += __shfl_xor_sync(kFullMask, x[0], d);
  return which;
}

// A few rows: what bounds them is the weights' bytes, each read once.  A warp takes four rows of W, 16 bytes (32 of fp32) a
// lane at a time, and kRows rows of x beside them from L1; 1, 2, 4 or 8 warps share the inputs.  fp32 sums of
// products of the values as they are, without parts.  4096 x 4096 in bf16: 8.9 us for one row (5.0 at the copy's
// bandwidth), 14 for two, 17 for four, 23 for eight; the tiles need 16.4 for any number up to 128.  1024 x 4096: 3.4, 4.6,
// 7.8, 9.0 and 8.9; 8192 x 1024: 6.1, 6.8, 8.3, 11.8 and 14.2.  Up to four rows of a forward pass come here, and up to eight
// where the tiles would have to split fp32 weights first.
template <typename T, typename E, typename O, int kRows, bool kPacks>
__global__ void __launch_bounds__(256) few_rows_kernel(const T* x, int64_t x_ld, const E* weight, int64_t p_stride, int64_t inputs,
                                                       int64_t outputs, int rows, int sharing, const StoreArgs store) {
  dq_pdl_enter();
  constexpr int kOut = 4, kValues = kOut * kRows;
  __shared__ float part[8][kValues];
  const int warp = (int)threadIdx.x / 32, lane = (int)threadIdx.x & 31;
  const int64_t worker = blockIdx.y, group = (int64_t)blockIdx.x * (8 / sharing) + warp / sharing, first = group * kOut;
  const int share = warp % sharing;
  x += worker * rows * x_ld;
  weight += worker * p_stride;
  // rows beyond the last are the last's, and not stored
  const E* w[kOut];
#pragma unroll
  for (int o = 0; o < kOut; ++o) w[o] = weight + min64(first + o, outputs - 1) * inputs;
  float2 sum[kValues] = {};
  if (first < outputs) {
    if constexpr (kPacks) {
#pragma unroll 2
      for (int64_t k = share * 256 + lane * 8; k < inputs; k += 256 * sharing) {  // whole packs: inputs is a multiple of eight
        float a[kOut][8];
#pragma unroll
        for (int o = 0; o < kOut; ++o) read8(w[o] + k, 8, true, a[o]);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          float v[8];
          read8(x + min(r, rows - 1) * x_ld + k, 8, true, v);
#pragma unroll
          for (int o = 0; o < kOut; ++o)
#pragma unroll
            for (int i = 0; i < 8; i += 2)
              sum[o * kRows + r] = fma2(make_float2(a[o][i], a[o][i + 1]), make_float2(v[i], v[i + 1]), sum[o * kRows + r]);
        }
      }
    } else {
#pragma unroll 2
      for (int64_t k = share * 32 + lane; k < inputs; k += 32 * sharing) {
        float a[kOut];
#pragma unroll
        for (int o = 0; o < kOut; ++o) a[o] = to_float(w[o][k]);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          const float v = to_float(x[min(r, rows - 1) * x_ld + k]);
#pragma unroll
          for (int o = 0; o < kOut; ++o) sum[o * kRows + r].x = fmaf(a[o], v, sum[o * kRows + r].x);
        }
      }
    }
  }
  float one[kValues];
#pragma unroll
  for (int i = 0; i < kValues; ++i) one[i] = sum[i].x + sum[i].y;
  const int which = sum_over_lanes(one, lane);
  part[warp][which] = one[0];  // equal lanes write equal values
  __syncthreads();
  // the shares of a group's sums in order
  const int t = (int)threadIdx.x;
  if (t < 8 / sharing * kValues) {
    const int g = t / kValues, i = t % kValues, r = i % kRows;
    const int64_t column = ((int64_t)blockIdx.x * (8 / sharing) + g) * kOut + i / kRows;
    float s = 0.f;
    for (int w = 0; w < sharing; ++w) s += part[g * sharing + w][i];
    if (column < outputs && r < rows)
      store_value<O>(store, (int)worker, r, column, s, store.bias ? store.bias[worker * store.bias_batch + column] : 0.f);
  }
}

template <typename T, typename E, typename O>
cudaError_t few_rows(const MatrixArgs& x, const MatrixArgs& w, const StoreArgs& store, cudaStream_t stream, uint64_t* launches) {
  const auto on_packs = [](const void* p, int64_t ld, int64_t batch, int64_t size) {
    return ((uintptr_t)p & 15) == 0 && ld * size % 16 == 0 && batch * size % 16 == 0;
  };
  const int64_t inputs = x.columns, outputs = w.rows;
  const bool packs = inputs % 8 == 0 && on_packs(x.data, x.ld, 0, sizeof(T)) && on_packs(w.data, w.ld, w.batch, sizeof(E));
  // as many warps as have something to do, 256 inputs (32 without packs) each
  const int64_t steps = ceil_div(inputs, packs ? 256 : 32);
  const int sharing = steps >= 8 ? 8 : steps >= 4 ? 4 : steps >= 2 ? 2 : 1;
  const auto run = [&](auto rows, auto in_packs) {
    ++*launches;
    return launch_pdl(few_rows_kernel<T, E, O, decltype(rows)::value, decltype(in_packs)::value>,
                      dim3((unsigned)ceil_div(outputs, 32 / sharing), (unsigned)x.workers), dim3(256), 0, stream,
                      static_cast<const T*>(x.data), x.ld, static_cast<const E*>(w.data), w.batch, inputs, outputs, (int)x.rows,
                      sharing, store);
  };
  const auto by_rows = [&](auto in_packs) {
    return x.rows == 1   ? run(std::integral_constant<int, 1>{}, in_packs)
           : x.rows == 2 ? run(std::integral_constant<int, 2>{}, in_packs)
           : x.rows <= 4 ? run(std::integral_constant<int, 4>{}, in_packs)
                         : run(std::integral_constant<int, kFewRows>{}, in_packs);
  };
  return packs ? by_rows(std::true_type{}) : by_rows(std::false_type{});
}

// du of a few rows in fp32, and the sums over the rows.
template <typename T>
__global__ void __launch_bounds__(256) few_slopes_kernel(const T* dy, int64_t dy_ld, const T* pre, int64_t pre_ld, int activation,
                                                         int rows, int64_t columns, float* du, float* dbias, int64_t g_stride,
                                                         int accumulate) {
  dq_pdl_enter();
  const int64_t j = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, worker = blockIdx.y;
  if (j >= columns) return;
  float x[kFewRows], u[kFewRows] = {}, sum = 0.f;
#pragma unroll
  for (int r = 0; r < kFewRows; ++r) {
    const int64_t row = worker * rows + min(r, rows - 1);
    x[r] = to_float(dy[row * dy_ld + j]);
    if (pre) u[r] = to_float(pre[row * pre_ld + j]);
  }
  if (pre) scale_by_slope<sizeof(T) == 4>(x, u, activation);
#pragma unroll
  for (int r = 0; r < kFewRows; ++r)
    if (r < rows) {
      sum += x[r];
      du[(worker * rows + r) * columns + j] = x[r];
    }
  if (dbias) {
    float* const to = dbias + worker * g_stride + j;
    *to = accumulate ? *to + sum : sum;
  }
}

constexpr int kFewColumns = 1024;  // of a block, four a thread
constexpr int kFewRun = 256;       // most rows of W that one fp32 sum runs over
constexpr int kFewOutputs = 64;    // rows of the weights' gradient that a block writes

// dW = d^T x of a few rows: a thread keeps four columns of x's rows and writes them times d's values.  With the two kernels
// below it makes the gradient of 8 x 5 bf16 rows of 4722 x 1314 150 us, where the tiles need 284.
template <typename T, int kRows, bool kPacks>
__global__ void __launch_bounds__(256) few_outer_kernel(const float* d, const MatrixArgs x, int64_t outputs, float* out, int64_t batch,
                                                        int accumulate) {
  dq_pdl_enter();
  __shared__ float factors[kRows][kFewOutputs];
  const int64_t worker = blockIdx.z, first = (int64_t)blockIdx.y * kFewOutputs, base = (int64_t)blockIdx.x * kFewColumns;
  const int rows = (int)x.rows, outs = (int)min64(kFewOutputs, outputs - first);
  // few columns: the block's threads share out the outputs
  const int shares = x.columns <= 128 ? 8 : x.columns <= 256 ? 4 : x.columns <= 512 ? 2 : 1;
  const int across = 256 / shares, thread = (int)threadIdx.x % across, n0 = (int)threadIdx.x / across;
  for (int i = (int)threadIdx.x; i < kRows * kFewOutputs; i += 256) {
    const int r = i / kFewOutputs, n = i % kFewOutputs;
    factors[r][n] = r < rows && n < outs ? d[(worker * rows + r) * outputs + first + n] : 0.f;
  }
  float v[kRows][4];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int64_t row = worker * rows + min(r, rows - 1);
    const bool counts = r < rows && row_counts(x, row);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t k = base + (kPacks ? thread * 4 + i : thread + across * i);
      v[r][i] = counts && k < x.columns ? to_float(static_cast<const T*>(x.data)[row * x.ld + k]) : 0.f;
    }
  }
  __syncthreads();
  for (int n = n0; n < outs; n += shares) {
    float s[4] = {};
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = fmaf(factors[r][n], v[r][i], s[i]);
    float* const to = out + worker * batch + (first + n) * x.columns + base;
    if constexpr (kPacks) {  // x.columns is a multiple of four
      const int k = thread * 4;
      if (base + k < x.columns) {
        float4 sum = make_float4(s[0], s[1], s[2], s[3]);
        if (accumulate) {
          const float4 old = *reinterpret_cast<const float4*>(to + k);
          sum = make_float4(sum.x + old.x, sum.y + old.y, sum.z + old.z, sum.w + old.w);
        }
        *reinterpret_cast<float4*>(to + k) = sum;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = thread + across * i;
        if (base + k < x.columns) to[k] = accumulate ? to[k] + s[i] : s[i];
      }
    }
  }
}

// dx = d W of a few rows: a block takes a run of W's rows and 1024 columns; its sums, or with several runs their place among
// [run][worker][row][columns].
template <typename E, int kRows, bool kPacks>
__global__ void __launch_bounds__(256) few_across_kernel(const float* d, const MatrixArgs w, int rows, int per_run, float* sums) {
  dq_pdl_enter();
  extern __shared__ float run_factors[];  // [per_run][kRows]
  const int64_t worker = blockIdx.z, first = (int64_t)blockIdx.y * per_run, base = (int64_t)blockIdx.x * kFewColumns;
  const int count = (int)min64(per_run, w.rows - first);
  for (int i = (int)threadIdx.x; i < per_run * kRows; i += 256) {
    const int n = i / kRows, r = i % kRows;
    run_factors[i] = n < count && r < rows ? d[(worker * rows + r) * w.rows + first + n] : 0.f;
  }
  __syncthreads();
  float s[kRows][4] = {};
  const E* const from = static_cast<const E*>(w.data) + worker * w.batch + first * w.ld + base;
#pragma unroll 4
  for (int n = 0; n < count; ++n) {
    float v[4];
    if constexpr (kPacks) {  // four values on a boundary of as many: 8 or 16 bytes
      const int k = (int)threadIdx.x * 4;
      const bool in = base + k < w.columns;
      if constexpr (sizeof(E) == 4) {
        const float4 pack = in ? *reinterpret_cast<const float4*>(from + n * w.ld + k) : make_float4(0.f, 0.f, 0.f, 0.f);
        v[0] = pack.x, v[1] = pack.y, v[2] = pack.z, v[3] = pack.w;
      } else {
        const uint2 pack = in ? *reinterpret_cast<const uint2*>(from + n * w.ld + k) : make_uint2(0, 0);
        const E* const e = reinterpret_cast<const E*>(&pack);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = to_float(e[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = (int)threadIdx.x + 256 * i;
        v[i] = base + k < w.columns ? to_float(from[n * w.ld + k]) : 0.f;
      }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[r][i] = fmaf(run_factors[n * kRows + r], v[i], s[r][i]);
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (r >= rows) break;
    float* const to = sums + (((int64_t)blockIdx.y * gridDim.z + worker) * rows + r) * w.columns + base;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = kPacks ? (int)threadIdx.x * 4 + i : (int)threadIdx.x + 256 * i;
      if (base + k < w.columns) to[k] = s[r][i];
    }
  }
}

// The runs' sums: eight warps in turn, and then in order.  0 in x's rows that do not count.
template <typename T>
__global__ void __launch_bounds__(256) few_join_kernel(const float* sums, int runs, int64_t rows, int64_t columns, const MatrixArgs x, T* dx,
                                                       int64_t dx_ld) {
  dq_pdl_enter();
  __shared__ float part[8][32];
  const int warp = (int)threadIdx.x / 32, lane = (int)threadIdx.x & 31;
  const int64_t j = (int64_t)blockIdx.x * 32 + lane, r = blockIdx.y;
  float s = 0.f;
  if (j < columns) {
#pragma unroll 8
    for (int i = warp; i < runs; i += 8) s += sums[(i * rows + r) * columns + j];
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp > 0 || j >= columns) return;
  for (int w = 1; w < 8; ++w) s += part[w][lane];
  dx[r * dx_ld + j] = from_float<T>(row_counts(x, r) ? s : 0.f);
}

// A row's lse and loss from its logits, and their gradient in their place.
__global__ void __launch_bounds__(1024) few_loss_kernel(float* z, const MatrixArgs x, float scale, bool forward, bool backward, float* loss,
                                                        float* lse) {
  dq_pdl_enter();
  __shared__ float shared[32];
  const int64_t r = blockIdx.x;
  float* const row = z + r * x.vocab;
  const bool counts = row_counts(x, r);
  const float c = x.weights ? x.weights[r] : 1.f;
  float all = 0.f;
  if (forward) {
    float most = -INFINITY, sum = 0.f;
    for (int64_t v = threadIdx.x; v < x.vocab; v += 1024) most = fmaxf(most, row[v]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(kFullMask, most, o));
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x / 32] = most;
    __syncthreads();
    for (int i = 0; i < 32; ++i) most = fmaxf(most, shared[i]);
    const float from = most == -INFINITY ? 0.f : most;
    for (int64_t v = threadIdx.x; v < x.vocab; v += 1024) sum += expf(row[v] - from);
    all = most + logf(block_sum(sum, shared));
    if (threadIdx.x == 0) {
      loss[r] = counts ? c * (all - row[token_at(x.targets, x.token_bits, r)]) : 0.f;
      if (lse) lse[r] = counts ? all : 0.f;
    }
  } else {
    all = lse[r];
  }
  if (!backward) return;
  __syncthreads();  // the target's logit has been read
  const int64_t t = counts ? token_at(x.targets, x.token_bits, r) : -1;
  for (int64_t v = threadIdx.x; v < x.vocab; v += 1024) {
    const float q = expf(at_most_0(row[v] - all));
    row[v] = counts ? scale * c * (v == t ? q - 1.f : q) : 0.f;
  }
}

template <typename F>
cudaError_t with_rows(int64_t rows, F&& f) {
  return rows == 1   ? f(std::integral_constant<int, 1>{})
         : rows == 2 ? f(std::integral_constant<int, 2>{})
         : rows <= 4 ? f(std::integral_constant<int, 4>{})
                     : f(std::integral_constant<int, kFewRows>{});
}

}  // namespace

cudaError_t launch_few_rows(const MatrixArgs& x, const MatrixArgs& w, const StoreArgs& store, cudaStream_t stream, uint64_t* launches) {
  return with_dtype(x.dtype, [&](auto t) {
    using T = decltype(t);
    const auto by_out = [&](auto o) {
      using O = decltype(o);
      return w.dtype == DQGAN_F32 ? few_rows<T, float, O>(x, w, store, stream, launches) : few_rows<T, T, O>(x, w, store, stream, launches);
    };
    return store.out_dtype == DQGAN_F32 ? by_out(float{}) : by_out(t);
  });
}

cudaError_t launch_few_slopes(const MatrixArgs& dy, const void* pre, int64_t pre_ld, int activation, float* du, float* dbias,
                              int64_t g_stride, int accumulate, cudaStream_t stream, uint64_t* launches) {
  ++*launches;
  return with_dtype(dy.dtype, [&](auto t) {
    using T = decltype(t);
    return launch_pdl(few_slopes_kernel<T>, dim3((unsigned)ceil_div(dy.columns, 256), (unsigned)dy.workers), dim3(256), 0, stream,
                      static_cast<const T*>(dy.data), dy.ld, static_cast<const T*>(pre), pre_ld, activation, (int)dy.rows, dy.columns, du,
                      dbias, g_stride, accumulate);
  });
}

cudaError_t launch_few_outer(const float* d, const MatrixArgs& x, int64_t outputs, float* out, int64_t batch, int accumulate,
                             cudaStream_t stream, uint64_t* launches) {
  const bool packs = ((uintptr_t)out & 15) == 0 && x.columns % 4 == 0 && (x.workers == 1 || batch % 4 == 0);
  const dim3 grid((unsigned)ceil_div(x.columns, kFewColumns), (unsigned)ceil_div(outputs, kFewOutputs), (unsigned)x.workers);
  ++*launches;
  return with_dtype(x.dtype, [&](auto t) {
    using T = decltype(t);
    return with_rows(x.rows, [&](auto rows) {
      constexpr int R = decltype(rows)::value;
      return packs ? launch_pdl(few_outer_kernel<T, R, true>, grid, dim3(256), 0, stream, d, x, outputs, out, batch, accumulate)
                   : launch_pdl(few_outer_kernel<T, R, false>, grid, dim3(256), 0, stream, d, x, outputs, out, batch, accumulate);
    });
  });
}

cudaError_t launch_few_across(const float* d, const MatrixArgs& w, const MatrixArgs& x, int64_t rows, void* dx, int64_t dx_ld, int32_t dx_dtype,
                              void* scratch, cudaStream_t stream, uint64_t* launches) {
  const int sms = device_sms();
  if (sms <= 0) return cudaErrorInvalidDevice;
  const int64_t wide = ceil_div(w.columns, kFewColumns), one = (int64_t)w.workers * rows * w.columns * 4;
  // four blocks an SM, and sums that are quickly joined; all runs' sums stay within the scratch
  int64_t runs = min64(ceil_div((int64_t)sms * 4, wide * w.workers), sms);
  runs = min64(runs, max64(1, (int64_t)kProductScratch / one));
  runs = max64(runs, ceil_div(w.rows, kFewRun));
  const int per_run = (int)ceil_div(w.rows, runs);
  runs = ceil_div(w.rows, per_run);
  if (runs * one > (int64_t)kProductScratch || runs > 65535) return cudaErrorInvalidValue;
  const bool packs = w.columns % 4 == 0 && ((uintptr_t)w.data & 15) == 0 && (w.workers == 1 || w.batch % 4 == 0);
  const dim3 grid((unsigned)wide, (unsigned)runs, (unsigned)w.workers);
  float* const sums = static_cast<float*>(scratch);
  ++*launches;
  cudaError_t st = with_dtype(w.dtype, [&](auto e) {
    using E = decltype(e);
    return with_rows(rows, [&](auto n) {
      constexpr int R = decltype(n)::value;
      const size_t smem = (size_t)per_run * R * 4;
      return packs ? launch_pdl(few_across_kernel<E, R, true>, grid, dim3(256), smem, stream, d, w, (int)rows, per_run, sums)
                   : launch_pdl(few_across_kernel<E, R, false>, grid, dim3(256), smem, stream, d, w, (int)rows, per_run, sums);
    });
  });
  if (st != cudaSuccess) return st;
  ++*launches;
  return with_dtype(dx_dtype, [&](auto t) {
    using T = decltype(t);
    return launch_pdl(few_join_kernel<T>, dim3((unsigned)ceil_div(w.columns, 32), (unsigned)(rows * w.workers)), dim3(256), 0, stream,
                      (const float*)sums, (int)runs, rows * w.workers, w.columns, x, static_cast<T*>(dx), dx_ld);
  });
}

int64_t most_few_rows(int32_t workers, int64_t w_rows, int64_t w_columns, int64_t rows) {
  if (w_rows > (int64_t)65535 * kFewOutputs) return 0;
  const int64_t one_row = ceil_div(w_rows, kFewRun) * workers * w_columns * 4;
  return min64(min64(rows, kFewRows), (int64_t)kProductScratch / one_row);
}

cudaError_t launch_few_loss(float* z, const MatrixArgs& x, float scale, bool forward, bool backward, float* loss, float* lse,
                            cudaStream_t stream, uint64_t* launches) {
  ++*launches;
  return launch_pdl(few_loss_kernel, dim3((unsigned)(x.rows * x.workers)), dim3(1024), 0, stream, z, x, scale, forward, backward, loss, lse);
}

}  // namespace dq
