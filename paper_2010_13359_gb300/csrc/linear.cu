// Linear layers of the workers: y = act(x W^T + b) + r, and the gradients of x, W and b.
//
//   u = x W^T + b;  y = act(u) + r
//   du = dy act'(u);  dx = du W;  dW = du^T x;  db = sum over rows of du   (dr = dy)
//
// Three products a layer (2 rows inputs outputs operations each), bound by the
// tensor cores where there are some hundred rows, by the weights' bytes below.
// How many 16-bit parts an operand has follows from the result's type.  What has
// 32 bits (fp32 weights, and du where the slope is not 0 or 1) is two parts in a result of 16 bits and three in
// fp32 gradients and all of fp32 layers, so that 2^-16 or 2^-24 of it is left out beside the result's own rounding.  (In
// one part du would be rounded a second time, and weights at a lookahead point would be those at the point itself
// wherever they differ by less than 2^-9 of them.  The gradient of 8 x 2048 bf16 rows of 1024 x 4096 with
// GELU: 538 us, 359 with du as one part in dx and two in dW, whose errors were 1.4 and 7 times larger;
// the forward pass with fp32 weights 242 us, 154 with one part of them and an error 1.4 times larger.)
// f16 values that do not lie as f16 in memory are two bf16 parts
// (all of their 11 bits, at any exponent).
#include "device_common.cuh"
#include "products.cuh"

namespace dq {

namespace {

int act_parts(int dtype) { return dtype == DQGAN_F32 ? 3 : dtype == DQGAN_F16 ? 2 : 1; }
int weight_parts(const LinearShape& s) {
  return s.dtype == DQGAN_F32 ? 3 : s.dtype == DQGAN_F16 || s.weight_dtype == DQGAN_F32 ? 2 : 1;
}
bool exact_slope(int activation) { return activation == DQGAN_NONE || activation == DQGAN_RELU; }  // du has dy's values
int grad_parts(const LinearShape& s) {
  return s.dtype == DQGAN_F32 || !exact_slope(s.activation) ? 3 : s.dtype == DQGAN_F16 ? 2 : 1;
}
bool half_forward(const LinearShape& s) { return s.dtype == DQGAN_F16 && s.weight_dtype == DQGAN_F16; }
bool half_backward(const LinearShape& s) { return half_forward(s) && exact_slope(s.activation); }

constexpr int kGradColumns = 256;   // of a block of slope_kernel
constexpr int kGradBlocks = 152 * 8;
// Blocks of a worker's rows: what fills the GPU eight times, of eight rows at least.
int64_t most_row_blocks(const LinearShape& s) {
  return ceil_div(kGradBlocks, ceil_div(s.outputs, kGradColumns) * s.workers);
}

struct Scratch {
  uint32_t* err;
  void* products;
  void *x, *w, *d;
  float *sums, *few;
  size_t bytes;
};

Scratch scratch_of(const LinearShape& s, void* base) {
  Scratch c{};
  size_t at = 0;
  const auto take = [&](int64_t bytes) {
    void* p = static_cast<char*>(base) + at;
    at += (size_t)ceil_div(bytes, 1024) * 1024;
    return p;
  };
  c.err = static_cast<uint32_t*>(take(1024));
  c.products = take(kProductScratch);
  const int64_t rows = (int64_t)s.workers * s.max_rows;
  c.x = take(rows * round8(s.inputs) * 2 * act_parts(s.dtype));
  c.w = take((int64_t)s.workers * s.outputs * round8(s.inputs) * 2 * weight_parts(s));
  c.d = take(rows * round8(s.outputs) * 2 * grad_parts(s));
  c.sums = static_cast<float*>(take(s.workers * most_row_blocks(s) * s.outputs * 4));
  c.few = static_cast<float*>(take(s.workers * most_few_rows(s.workers, s.outputs, s.inputs, s.max_rows) * s.outputs * 4));
  c.bytes = at;
  return c;
}

struct SlopeArgs {
  const void* dy;
  int64_t dy_ld;
  const void* pre;
  int64_t pre_ld;
  void* to;  // du in parts, or nullptr
  int64_t ld, part;
  int32_t parts;
  bool half;
  float* sums;  // [worker][block of rows][outputs], or nullptr
  int64_t rows, columns;
  int32_t block_rows;
  int32_t activation;
  bool dy_packs, pre_packs;
};

// du of a block of rows and 256 columns, in parts, and the columns' sums.  Bound by memory: 10 bytes a value in bf16 with
// GELU (dy, u, three parts).  Where rows are on 16-byte boundaries four of them a warp are on their way at once.
template <typename T, bool kSlope>
__global__ void __launch_bounds__(256, 3) slope_kernel(const SlopeArgs a) {
  dq_pdl_enter();
  __shared__ float turn[8][kGradColumns];
  constexpr int kAhead = 4, E = 16 / (int)sizeof(T), kPacks = 8 / E;
  const int warp = (int)threadIdx.x / 32, lane = (int)threadIdx.x & 31;
  const int64_t column = (int64_t)blockIdx.x * kGradColumns + lane * 8;
  const int64_t worker = blockIdx.z;
  const int64_t first = (int64_t)blockIdx.y * a.block_rows, last = min(first + a.block_rows, a.rows);
  const int count = (int)max((int64_t)0, min((int64_t)8, a.columns - column));
  float sum[8] = {};
  const T* const dy = static_cast<const T*>(a.dy) + worker * a.rows * a.dy_ld + column;
  const T* const pre = kSlope ? static_cast<const T*>(a.pre) + worker * a.rows * a.pre_ld + column : nullptr;
  const auto row = [&](int64_t r, float (&x)[8], const float (&u)[8]) {
    if constexpr (kSlope) scale_by_slope<sizeof(T) == 4>(x, u, a.activation);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i >= count) x[i] = 0.f;
      sum[i] += x[i];
    }
    if (a.to) write_parts<sizeof(T) == 4>(x, a.to, (worker * a.rows + r) * a.ld + column, a.part, a.parts, a.half);
  };
  const auto unpack = [](const uint4 (&packs)[kPacks], float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float2 v = pair_of<T>(packs[i / E], i % E);
      x[i] = v.x;
      x[i + 1] = v.y;
    }
  };
  int64_t r = first + warp;
  const bool packs = a.dy_packs && (!kSlope || a.pre_packs);
  if (packs && count == 8) {
    for (; r + 8 * (kAhead - 1) < last; r += 8 * kAhead) {
      uint4 d[kAhead][kPacks], p[kAhead][kPacks];
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
#pragma unroll
        for (int q = 0; q < kPacks; ++q) {
          d[k][q] = reinterpret_cast<const uint4*>(dy + (r + 8 * k) * a.dy_ld)[q];
          if constexpr (kSlope) p[k][q] = reinterpret_cast<const uint4*>(pre + (r + 8 * k) * a.pre_ld)[q];
        }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        float x[8], u[8] = {};
        unpack(d[k], x);
        if constexpr (kSlope) unpack(p[k], u);
        row(r + 8 * k, x, u);
      }
    }
  }
  if (packs) {
    if (count > 0)
      for (; r < last; r += 8) {
        float x[8], u[8] = {};
        read8(dy + r * a.dy_ld, count, true, x);
        if constexpr (kSlope) read8(pre + r * a.pre_ld, count, true, u);
        row(r, x, u);
      }
  } else {
    const int64_t rows = (int64_t)gridDim.z * a.rows - 1;
    const T* const dy_end = static_cast<const T*>(a.dy) + rows * a.dy_ld + a.columns;
    const T* const pre_end = kSlope ? static_cast<const T*>(a.pre) + rows * a.pre_ld + a.columns : nullptr;
    if (count > 0)
#pragma unroll 2
      for (; r < last; r += 8) {
        float x[8], u[8] = {};
        read8_near(dy + r * a.dy_ld, count, a.dy, dy_end, x);
        if constexpr (kSlope) read8_near(pre + r * a.pre_ld, count, a.pre, pre_end, u);
        row(r, x, u);
      }
  }
  if (a.sums) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn[warp][lane * 8 + i] = sum[i];
    __syncthreads();
    const int64_t j = (int64_t)blockIdx.x * kGradColumns + threadIdx.x;
    if (j < a.columns) {
      float s = 0.f;
      for (int w = 0; w < 8; ++w) s += turn[w][threadIdx.x];
      a.sums[((worker * gridDim.y) + blockIdx.y) * a.columns + j] = s;
    }
  }
}

// db: the blocks' sums, eight warps in turn and then in order.
__global__ void __launch_bounds__(256) bias_kernel(const float* sums, int blocks, int64_t columns, float* dbias,
                                                   int64_t g_stride, int accumulate) {
  dq_pdl_enter();
  __shared__ double part[8][32];
  const int warp = (int)threadIdx.x / 32, lane = (int)threadIdx.x & 31;
  const int64_t j = (int64_t)blockIdx.x * 32 + lane, worker = blockIdx.y;
  double s = 0.;
  if (j < columns) {
#pragma unroll 4
    for (int b = warp; b < blocks; b += 8) s += sums[(worker * blocks + b) * columns + j];
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp > 0 || j >= columns) return;
  for (int w = 1; w < 8; ++w) s += part[w][lane];
  float* const to = dbias + worker * g_stride + j;
  *to = accumulate ? *to + (float)s : (float)s;
}

bool has_few_rows(const LinearShape& s, int64_t rows) { return rows <= (s.weight_dtype == DQGAN_F32 ? kFewRows : kFewRows / 2); }

}  // namespace

size_t linear_scratch_bytes(const LinearShape& s) { return scratch_of(s, nullptr).bytes; }

cudaError_t launch_linear_forward(const LinearArgs& a, cudaStream_t stream, uint64_t* launches) {
  const LinearShape& s = a.shape;
  const Scratch c = scratch_of(s, a.scratch);
  const bool half = half_forward(s);
  StoreArgs out{};
  out.out = a.y;
  out.out_ld = a.y_ld;
  out.out_batch = a.rows * a.y_ld;
  out.out_dtype = s.dtype;
  out.pre = a.pre_out;
  out.pre_ld = a.pre_ld;
  out.pre_batch = a.rows * a.pre_ld;
  out.residual = a.residual;
  out.residual_ld = a.residual_ld;
  out.residual_batch = a.rows * a.residual_ld;
  out.bias = a.bias;
  out.bias_batch = a.b_stride;
  out.activation = s.activation;
  const MatrixArgs x{a.x, a.x_ld, a.rows * a.x_ld, s.dtype, a.rows, s.inputs, s.workers};
  const MatrixArgs w{a.weight, s.inputs, a.p_stride, s.weight_dtype, s.outputs, s.inputs, s.workers};
  if (has_few_rows(s, a.rows))
    return launch_few_rows(x, w, out, stream, launches);
  Product p;
  p.rows = a.rows;
  p.columns = s.outputs;
  p.depth = s.inputs;
  p.workers = s.workers;
  Splits splits{stream, launches};
  cudaError_t st = make_operand(x, half ? 1 : act_parts(s.dtype), half, c.x, splits, &p.a);
  if (st == cudaSuccess) st = make_operand(w, half ? 1 : weight_parts(s), half, c.w, splits, &p.b);
  if (st == cudaSuccess) st = splits.flush();
  if (st != cudaSuccess) return st;
  p.terms = product_terms(p.a.parts, p.b.parts);
  return launch_product_store(p, out, c.products, c.err, stream, launches);
}

cudaError_t launch_linear_backward(const LinearArgs& a, cudaStream_t stream, uint64_t* launches) {
  const LinearShape& s = a.shape;
  const Scratch c = scratch_of(s, a.scratch);
  cudaError_t st = cudaSuccess;
  if (a.rows == 0) {  // gradients of nothing
    if (a.accumulate) return st;
    for (int m = 0; m < s.workers && st == cudaSuccess; ++m) {
      if (a.dweight) st = cudaMemsetAsync(a.dweight + m * a.g_stride, 0, (size_t)s.outputs * s.inputs * 4, stream);
      if (a.dbias && st == cudaSuccess) st = cudaMemsetAsync(a.dbias + m * a.g_stride, 0, (size_t)s.outputs * 4, stream);
    }
    return st;
  }
  const MatrixArgs few_w{a.weight, s.inputs, a.p_stride, s.weight_dtype, s.outputs, s.inputs, s.workers};
  if (few_rows_fit(few_w, a.rows)) {
    const MatrixArgs few_dy{a.dy, a.dy_ld, a.rows * a.dy_ld, s.dtype, a.rows, s.outputs, s.workers};
    const MatrixArgs few_x{a.x, a.x_ld, a.rows * a.x_ld, s.dtype, a.rows, s.inputs, s.workers};
    st = launch_few_slopes(few_dy, s.activation == DQGAN_NONE ? nullptr : a.pre, a.pre_ld, s.activation, c.few, a.dbias, a.g_stride,
                           a.accumulate, stream, launches);
    if (st == cudaSuccess && a.dx)
      st = launch_few_across(c.few, few_w, few_x, a.rows, a.dx, a.dx_ld, s.dtype, c.products, stream, launches);
    if (st == cudaSuccess && a.dweight)
      st = launch_few_outer(c.few, few_x, s.outputs, a.dweight, a.g_stride, a.accumulate, stream, launches);
    return st;
  }
  const bool half = half_backward(s);
  const int parts = half ? 1 : grad_parts(s);
  const MatrixArgs dy{a.dy, a.dy_ld, a.rows * a.dy_ld, s.dtype, a.rows, s.outputs, s.workers};
  const bool direct = s.activation == DQGAN_NONE && (half || (s.dtype == DQGAN_BF16 && parts == 1)) &&
                      operand_in_place(a.dy, a.dy_ld, a.rows * a.dy_ld);
  ProductOperand d, weight, x;
  Splits splits{stream, launches};
  if (direct) st = make_operand(dy, parts, half, c.d, splits, &d);
  if (st == cudaSuccess && a.dx) {
    const MatrixArgs w{a.weight, s.inputs, a.p_stride, s.weight_dtype, s.outputs, s.inputs, s.workers};
    st = make_operand(w, half ? 1 : weight_parts(s), half, c.w, splits, &weight);
  }
  if (st == cudaSuccess && a.dweight) {
    const MatrixArgs rows{a.x, a.x_ld, a.rows * a.x_ld, s.dtype, a.rows, s.inputs, s.workers};
    st = make_operand(rows, half ? 1 : act_parts(s.dtype), half, c.x, splits, &x);
  }
  if (st == cudaSuccess) st = splits.flush();
  if (st == cudaSuccess && (!direct || a.dbias)) {
    const int size = s.dtype == DQGAN_F32 ? 4 : 2;
    SlopeArgs k{};
    k.dy = a.dy;
    k.dy_ld = a.dy_ld;
    k.dy_packs = ((uintptr_t)a.dy & 15) == 0 && a.dy_ld * size % 16 == 0;
    if (s.activation != DQGAN_NONE) {
      k.pre = a.pre;
      k.pre_ld = a.pre_ld;
      k.pre_packs = ((uintptr_t)a.pre & 15) == 0 && a.pre_ld * size % 16 == 0;
    }
    k.ld = round8(s.outputs);
    k.part = k.ld * a.rows * s.workers;
    k.parts = parts;
    k.half = half;
    k.rows = a.rows;
    k.columns = s.outputs;
    k.activation = s.activation;
    k.to = direct ? nullptr : c.d;
    k.sums = a.dbias ? c.sums : nullptr;
    const int64_t wide = ceil_div(s.outputs, kGradColumns);
    k.block_rows = (int32_t)(ceil_div(ceil_div(a.rows, most_row_blocks(s)), 8) * 8);
    const int64_t blocks = ceil_div(a.rows, k.block_rows);
    ++*launches;
    st = with_dtype(s.dtype, [&](auto t) {
      const dim3 grid((unsigned)wide, (unsigned)blocks, (unsigned)s.workers);
      return k.pre ? launch_pdl(slope_kernel<decltype(t), true>, grid, dim3(256), 0, stream, k)
                   : launch_pdl(slope_kernel<decltype(t), false>, grid, dim3(256), 0, stream, k);
    });
    if (st == cudaSuccess && a.dbias) {
      ++*launches;
      st = launch_pdl(bias_kernel, dim3((unsigned)ceil_div(s.outputs, 32), (unsigned)s.workers), dim3(256), 0, stream,
                      (const float*)c.sums, (int)blocks, s.outputs, a.dbias, a.g_stride, a.accumulate);
    }
    if (!direct) {
      d.data = c.d;
      d.ld = k.ld;
      d.batch = k.ld * a.rows;
      d.part = k.part;
      d.parts = parts;
      d.half = half;
    }
  }
  if (st != cudaSuccess) return st;
  if (a.dx) {
    Product p;
    p.rows = a.rows;
    p.columns = s.inputs;
    p.depth = s.outputs;
    p.workers = s.workers;
    p.a = d;
    if (s.dtype != DQGAN_F32 && p.a.parts > 2) p.a.parts = 2;
    p.b = weight;
    p.b.across = true;
    p.terms = product_terms(p.a.parts, p.b.parts);
    StoreArgs out{};
    out.out = a.dx;
    out.out_ld = a.dx_ld;
    out.out_batch = a.rows * a.dx_ld;
    out.out_dtype = s.dtype;
    st = launch_product_store(p, out, c.products, c.err, stream, launches);
  }
  if (st == cudaSuccess && a.dweight) {
    Product p;
    p.rows = s.outputs;
    p.columns = s.inputs;
    p.depth = a.rows;
    p.workers = s.workers;
    p.a = d;
    p.b = x;
    p.a.across = p.b.across = true;
    p.terms = product_terms(p.a.parts, p.b.parts);
    StoreArgs out{};
    out.out = a.dweight;
    out.out_ld = s.inputs;
    out.out_batch = a.g_stride;
    out.out_dtype = DQGAN_F32;
    if (a.accumulate) {
      out.add = a.dweight;
      out.add_ld = s.inputs;
      out.add_batch = a.g_stride;
    }
    st = launch_product_store(p, out, c.products, c.err, stream, launches);
  }
  return st;
}

}  // namespace dq
