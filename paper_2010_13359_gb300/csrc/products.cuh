// Matrix products of the token-model operators on the tensor cores (not part
// of the C-ABI): what a product is, and its launchers.
//
// A product is D[i][j] = sum over k of A[i][k] B[j][k] for every worker, with
// 16-bit operands, fp32 sums, and an epilogue.  Operands in 32 bits, and
// values computed in 32 bits, come as a sum of parts of 16 bits (x = x0 + x1 +
// ..., each the rounding of what the ones before leave), and the product as
// the sum over pairs of parts that matter ("terms").
#pragma once

#include "operators.cuh"

namespace dq {

// A 16-bit operand as it lies in memory.  Element (i, k) of worker m and part
// p is data[p * part + m * batch + i * ld + k], or with `across` data[p * part +
// m * batch + k * ld + i].  Base and strides are multiples of 16 bytes.
struct ProductOperand {
  const void* data = nullptr;
  int64_t ld = 0, batch = 0, part = 0;
  int32_t parts = 1;
  bool across = false;
  bool shared = false;  // one matrix for all workers
  bool half = false;    // f16; else bf16 (both operands alike)
};

struct ProductTerms {
  int32_t count = 1;
  uint8_t a[6] = {}, b[6] = {};
};
// All pairs of parts whose product is above the rounding of the last part: of
// (2, 1), (2, 2) and (3, 3) parts those with i + j < max.
ProductTerms product_terms(int a_parts, int b_parts);

// What is done with the sums.  Row i and column j of worker m.
struct StoreArgs {
  void* out;             // out + m * out_batch + i * out_ld + j
  int64_t out_batch, out_ld;
  int32_t out_dtype;
  void* pre;             // the sum with the bias, of the same type, or nullptr
  int64_t pre_batch, pre_ld;
  const void* residual;  // of the same type, added last, or nullptr
  int64_t residual_batch, residual_ld;
  const float* bias;     // bias + m * bias_batch + j, or nullptr
  int64_t bias_batch;
  const float* add;      // fp32 values added to the sum (add + m * add_batch + i * add_ld + j), or nullptr; may be out
  int64_t add_batch, add_ld;
  int32_t activation;
  // Rows that do not count are stored as 0, whatever their sums are (0 times what is not finite); as in SplitArgs.
  const void* targets;
  const float* weights;
  int32_t token_bits;
  int64_t vocab;
};

struct SoftmaxArgs {
  const void* targets;    // one a row, worker m's at + m * m_rows
  int32_t token_bits;
  const float* weights;   // one a row, or nullptr
  int64_t first;          // the first column's place in the vocabulary
  int64_t vocab;
  float2* stats;          // forward: (maximum, sum of exp(z - maximum)) of row r's columns in slot s at [(m * slots + s) * rows + r]
  int32_t slots, slot;    // slots of a row; the first of this product's
  float* target_logit;    // forward: one a row
  const float* lse;       // gradient
  float scale;
  void* grad;             // gradient in bf16 parts: [part][worker][row][grad_ld]
  int64_t grad_ld, grad_part;
  int32_t grad_parts;
};

struct ProductArgs {
  CUtensorMap a, b;
  CUtensorMap out, pre;     // results, where TMA can write them (pre: of StoreArgs)
  int64_t rows, columns;    // of D, per worker
  int32_t workers;
  int32_t kblocks;          // blocks of 64 of the contracted index
  int32_t group;            // blocks whose products go to one accumulator in tensor memory, one pair of parts after another
  int32_t chunk;            // their terms: group * terms.count
  int32_t pieces;           // of the contracted index, that are summed apart in the tiles from `whole` on
  int64_t whole;
  int32_t tiles_m, tiles_n;
  ProductTerms terms;
  uint8_t a_across, b_across, a_shared, b_shared, half;
  float* partial;           // the pieces' sums
  uint32_t* err;
  StoreArgs store;
  SoftmaxArgs softmax;
};

struct Product {
  ProductOperand a, b;
  int64_t rows, columns, depth;
  int32_t workers;
  ProductTerms terms;
};

// How a product is cut: tiles of 256 x 256 for pairs of blocks, or of 128 x 64 for single ones; and of the tiles
// that do not fill the GPU for a last time, those from `whole` on, the contracted index in pieces.
struct Cut {
  int width;
  int64_t whole;
  int pieces;
};
// For `slots` SMs; `only`: tiles of that width, 0: of either.
Cut cut_product(const Product& p, int64_t slots, int only);

// Scratch of the products of one operator: the sums of pieces.
constexpr size_t kProductScratch = (size_t)80 << 20;

// scratch: kProductScratch bytes.
cudaError_t launch_product_store(const Product& p, const StoreArgs& store, void* scratch, uint32_t* err,
                                 cudaStream_t stream, uint64_t* launches);
// Rows of a matrix turned into 16-bit parts, [part][worker][row][ld] with ld a
// multiple of 8; the columns up to ld are 0.
struct SplitArgs {
  const void* from;       // worker m's row r at + m * batch + r * from_ld
  int64_t batch, from_ld;
  int32_t dtype;          // of the values
  void* to;
  int64_t ld, part;       // elements
  int32_t parts;
  bool half;              // to f16 (one part, from f16); else bf16
  int64_t rows, columns;
  int32_t workers;
  // Rows that do not count become 0: those whose target is outside [0, vocab) or whose weight is 0.
  const void* targets;    // or nullptr: all rows count
  const float* weights;   // or nullptr
  int32_t token_bits;
  int64_t vocab;
  bool packs;             // rows can be read 16 bytes at a time (set by Splits)
};
// Matrices that are to be split, two of one type to a launch.  What is added has to be flushed before it is read.
struct Splits {
  cudaStream_t stream;
  uint64_t* launches;
  SplitArgs pending[2] = {};
  int count = 0;
  cudaError_t add(const SplitArgs& a);
  cudaError_t flush();
};

// Whether a matrix of a 16-bit type can be an operand as it lies.
inline bool operand_in_place(const void* p, int64_t ld, int64_t batch) {
  return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && batch % 8 == 0 && ld < ((int64_t)1 << 38) && batch < ((int64_t)1 << 38);
}

__device__ __forceinline__ int64_t token_at(const void* ids, int bits, int64_t r) {
  return bits == 32 ? (int64_t) static_cast<const int32_t*>(ids)[r] : static_cast<const int64_t*>(ids)[r];
}
// Whether row r counts: where there are targets, if its target is in the vocabulary and its weight is not 0.
template <typename Args>
__device__ __forceinline__ bool row_counts(const Args& a, int64_t r) {
  if (!a.targets) return true;
  const int64_t t = token_at(a.targets, a.token_bits, r);
  return t >= 0 && t < a.vocab && !(a.weights && a.weights[r] == 0.f);
}

__device__ __forceinline__ float exp2_approx(float x) {  // 2 units; below 2^-126: 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float reciprocal_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// min(x, 0); NaN stays NaN.
__device__ __forceinline__ float at_most_0(float x) {
  float y;
  asm("min.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(x));
  return y;
}

// Phi(u) and exp(-u^2 / 2).  For results of 16 bits: Abramowitz and Stegun 7.1.26, erfc(x) = t (a1 + t (a2 + ...)) exp(-x^2)
// with t = 1 / (1 + p x), off by at most 1.5e-7, which is a fifth of erff's instructions.
template <bool kExact>
__device__ __forceinline__ float2 normal_cdf(float u) {
  if constexpr (kExact) return make_float2(0.5f * erfcf(u * -0.70710678118654752f), expf(-0.5f * u * u));
  const float x = fabsf(u) * 0.70710678118654752f;
  const float e = exp2_approx(u * u * -0.72134752044448170f);
  const float t = reciprocal_approx(fmaf(0.3275911f, x, 1.f));
  const float tail = 0.5f * e * t *
                     fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
  return make_float2(u > 0.f ? 1.f - tail : tail, e);
}
template <bool kExact>
__device__ __forceinline__ float logistic(float u) {
  if constexpr (kExact) return 1.f / (1.f + expf(-u));
  return reciprocal_approx(1.f + exp2_approx(u * -1.4426950408889634f));
}

// act(u), and its slope.
template <bool kExact>
__device__ __forceinline__ float activate(float u, int activation) {
  switch (activation) {
    case DQGAN_RELU: return u > 0.f ? u : (u != u ? u : 0.f);
    case DQGAN_GELU: return u * normal_cdf<kExact>(u).x;
    case DQGAN_SILU: return u * logistic<kExact>(u);
  }
  return u;
}
// 1 - Phi(|u|) and exp(-u^2 / 2) of two values as normal_cdf<false>, two fp32 operations to an instruction.
__device__ __forceinline__ void normal_tails(float2 u, float2 x, float2* tail, float2* e) {
  const float2 d = fma2(x, both(0.3275911f * 0.70710678118654752f), both(1.f));
  const float2 t = make_float2(reciprocal_approx(d.x), reciprocal_approx(d.y));
  const float2 power = mul2(mul2(u, u), both(-0.72134752044448170f));
  *e = make_float2(exp2_approx(power.x), exp2_approx(power.y));
  float2 f = fma2(t, both(0.5f * 1.061405429f), both(0.5f * -1.453152027f));
  f = fma2(f, t, both(0.5f * 1.421413741f));
  f = fma2(f, t, both(0.5f * -0.284496736f));
  f = fma2(f, t, both(0.5f * 0.254829592f));
  *tail = mul2(mul2(f, t), *e);
}
__device__ __forceinline__ float2 gelu2(float2 u) {
  const float2 x = make_float2(fabsf(u.x), fabsf(u.y));
  float2 tail, e;
  normal_tails(u, x, &tail, &e);
  tail = mul2(tail, x);  // what u Phi(u) is less than max(u, 0)
  return make_float2(fmaxf(u.x, 0.f) - tail.x, fmaxf(u.y, 0.f) - tail.y);
}
__device__ __forceinline__ float2 gelu_slope2(float2 u) {
  const float2 x = make_float2(fabsf(u.x), fabsf(u.y));
  float2 tail, e;
  normal_tails(u, x, &tail, &e);
  // u phi(u) - (1 - Phi(u)) for u > 0, and the slopes at u and -u add up to 1
  const float2 h = fma2(mul2(x, both(0.39894228040143268f)), e, make_float2(-tail.x, -tail.y));
  return make_float2(u.x > 0.f ? 1.f + h.x : -h.x, u.y > 0.f ? 1.f + h.y : -h.y);
}

template <bool kExact, int N>
__device__ __forceinline__ void activate_all(float (&x)[N], int activation) {
  if (activation == DQGAN_GELU && !kExact) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 y = gelu2(make_float2(x[i], x[i + 1]));
      x[i] = y.x;
      x[i + 1] = y.y;
    }
  } else if (activation == DQGAN_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = activate<kExact>(x[i], DQGAN_GELU);
  } else if (activation == DQGAN_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = activate<kExact>(x[i], DQGAN_SILU);
  } else if (activation == DQGAN_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = activate<kExact>(x[i], DQGAN_RELU);
  }
}
template <bool kExact>
__device__ __forceinline__ float activation_slope(float u, int activation) {
  switch (activation) {
    case DQGAN_RELU: return u > 0.f ? 1.f : (u != u ? u : 0.f);
    case DQGAN_GELU: {
      const float2 f = normal_cdf<kExact>(u);
      return fmaf(u * 0.39894228040143268f, f.y, f.x);
    }
    case DQGAN_SILU: {
      const float s = logistic<kExact>(u);
      return s * fmaf(u, 1.f - s, 1.f);
    }
  }
  return 1.f;
}

// x times the slope at u.
template <bool kExact, int N>
__device__ __forceinline__ void scale_by_slope(float (&x)[N], const float (&u)[N], int activation) {
  if (activation == DQGAN_GELU && !kExact) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 s = gelu_slope2(make_float2(u[i], u[i + 1]));
      x[i] *= s.x;
      x[i + 1] *= s.y;
    }
  } else if (activation == DQGAN_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] *= activation_slope<kExact>(u[i], DQGAN_GELU);
  } else if (activation == DQGAN_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] *= activation_slope<kExact>(u[i], DQGAN_SILU);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] *= activation_slope<kExact>(u[i], DQGAN_RELU);
  }
}

// x's rounding to bf16, and what it leaves.  A finite value stays finite; a value that is not leaves nothing.
__device__ __forceinline__ __nv_bfloat16 take_part(float& x) {
  __nv_bfloat16 h = __float2bfloat16_rn(x);
  float back = __bfloat162float(h);
  if (isinf(back) && !isinf(x)) {
    h = __float2bfloat16_rz(x);
    back = __bfloat162float(h);
  }
  x = isfinite(back) ? x - back : 0.f;
  return h;
}

// The same of two values, in a few instructions: one that is not finite, or rounds to what is not, leaves NaN.
__device__ __forceinline__ uint32_t take_parts2(float2& x) {
  const __nv_bfloat162 h = __float22bfloat162_rn(x);
  const uint32_t bits = reinterpret_cast<const uint32_t&>(h);
  x = add2(x, make_float2(-__uint_as_float(bits << 16), -__uint_as_float(bits & 0xffff0000u)));
  return bits;
}

// kSafe: as take_part.
template <bool kSafe>
__device__ __forceinline__ void write_parts(float (&x)[8], void* to, int64_t at, int64_t part, int parts, bool half) {
  if (half) {
    uint4 pack;
#pragma unroll
    for (int i = 0; i < 8; i += 2) set_pair<__half>(pack, i, make_float2(x[i], x[i + 1]));
    *reinterpret_cast<uint4*>(static_cast<__half*>(to) + at) = pack;
    return;
  }
  for (int q = 0; q < parts; ++q) {
    uint4 pack;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      if constexpr (kSafe) {
        __nv_bfloat162 h;
        h.x = take_part(x[i]);
        h.y = take_part(x[i + 1]);
        reinterpret_cast<__nv_bfloat162*>(&pack)[i / 2] = h;
      } else {
        float2 v = make_float2(x[i], x[i + 1]);
        reinterpret_cast<uint32_t*>(&pack)[i / 2] = take_parts2(v);
        x[i] = v.x;
        x[i + 1] = v.y;
      }
    }
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(to) + q * part + at) = pack;
  }
}

// One result: the sum of a product, and what is done with it.
template <typename T>
__device__ __forceinline__ void store_value(const StoreArgs& s, int worker, int64_t row, int64_t column, float x, float bias) {
  if (s.add) x += s.add[worker * s.add_batch + row * s.add_ld + column];
  x += bias;
  if (s.pre) static_cast<T*>(s.pre)[worker * s.pre_batch + row * s.pre_ld + column] = from_float<T>(x);
  x = activate<sizeof(T) == 4>(x, s.activation);
  if (s.residual)
    x += to_float(static_cast<const T*>(s.residual)[worker * s.residual_batch + row * s.residual_ld + column]);
  static_cast<T*>(s.out)[worker * s.out_batch + row * s.out_ld + column] = from_float<T>(x);
}

// A matrix of the caller's: worker m's row r at data + m * batch + r * ld.
struct MatrixArgs {
  const void* data;
  int64_t ld, batch;  // batch 0: one for all workers
  int32_t dtype;
  int64_t rows, columns;
  int32_t workers;
  const void* targets = nullptr;  // as in SplitArgs
  const float* weights = nullptr;
  int32_t token_bits = 32;
  int64_t vocab = 0;
};
// The operand that it is: as it lies, or split into `buffer`.
cudaError_t make_operand(const MatrixArgs& m, int parts, bool half, void* buffer, Splits& splits, ProductOperand* out);

// Products of up to kFewRows rows a worker (few_rows.cu).  x: rows; w: weights, w.rows x w.columns; d: fp32, [worker][row][w.rows].
constexpr int kFewRows = 8;
// x W^T, and what is done with it; the result has x's type or fp32.
cudaError_t launch_few_rows(const MatrixArgs& x, const MatrixArgs& w, const StoreArgs& store, cudaStream_t stream, uint64_t* launches);
// du = dy act'(pre) (pre: nullptr for no activation), and its sums over the rows (or dbias nullptr).
cudaError_t launch_few_slopes(const MatrixArgs& dy, const void* pre, int64_t pre_ld, int activation, float* du, float* dbias,
                              int64_t g_stride, int accumulate, cudaStream_t stream, uint64_t* launches);
// d^T x, outputs x x.columns, worker m's at out + m * batch.  x's rows that do not count are left out.
cudaError_t launch_few_outer(const float* d, const MatrixArgs& x, int64_t outputs, float* out, int64_t batch, int accumulate,
                             cudaStream_t stream, uint64_t* launches);
// Most rows a worker, up to `rows` and kFewRows, that the kernels' scratch and grids hold; 0: none.
int64_t most_few_rows(int32_t workers, int64_t w_rows, int64_t w_columns, int64_t rows);
inline bool few_rows_fit(const MatrixArgs& w, int64_t rows) {
  return rows <= kFewRows && most_few_rows(w.workers, w.rows, w.columns, rows) == rows;
}
// d W; 0 in x's rows that do not count.  scratch: kProductScratch bytes.
cudaError_t launch_few_across(const float* d, const MatrixArgs& w, const MatrixArgs& x, int64_t rows, void* dx, int64_t dx_ld, int32_t dx_dtype,
                              void* scratch, cudaStream_t stream, uint64_t* launches);
// loss and lse of rows of x.vocab logits (forward), and the gradient in their place (backward; without forward: from lse).
cudaError_t launch_few_loss(float* z, const MatrixArgs& x, float scale, bool forward, bool backward, float* loss, float* lse,
                            cudaStream_t stream, uint64_t* launches);

}  // namespace dq
