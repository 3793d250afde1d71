// Softmax cross entropy of the workers' output layers over a large vocabulary,
// without keeping the logits.
//
//   z = x W^T;  lse = log sum_v exp z_v;  loss = c (lse - z_t)
//   dz = scale c (exp(z - lse) - [v = t]);  dx = dz W;  dW = dz^T x
//
// The forward pass leaves of each row's 128 (or 32) logits their maximum and the sum of their
// exponentials, in the product's epilogue; a second kernel joins them in order.
// The gradient takes the vocabulary in pieces: a piece's logits are computed
// again, their epilogue writes dz in three bf16 parts into scratch, and two products
// take it from there, dW's all of it and dx's of 16 bits two parts.  In products of rows vocab width, bf16 rows and weights: the logits
// twice, dx 2, dW 3; with fp32 weights 3 + 3, 3, 3; f16 1 + 1, 3, 5, with fp32 weights 5 + 5, 3, 5; fp32 four times 6.
// The step of 4 x 1024 bf16 rows of 32,000 x 1024: 1356 us, 987 with one part of dz in dx
// and two in dW, whose errors were 1.4 and 6.5 times larger.
#include "product_kernel.cuh"

namespace dq {

namespace {

int act_parts(int dtype) { return dtype == DQGAN_F32 ? 3 : dtype == DQGAN_F16 ? 2 : 1; }
// Of the weights: in the logits, whose loss and lse are fp32, and in dx.  Three parts keep 2^-24 of a value, two 2^-16.
int logit_weight_parts(const TokenLossShape& s) { return s.weight_dtype == DQGAN_F32 ? 3 : s.dtype == DQGAN_F16 ? 2 : 1; }
int grad_weight_parts(const TokenLossShape& s) {
  return s.dtype == DQGAN_F32 ? 3 : s.dtype == DQGAN_F16 || s.weight_dtype == DQGAN_F32 ? 2 : 1;
}
// Of dz: in dW, which is fp32, and in dx.
constexpr int kGradParts = 3;
int dx_grad_parts(const TokenLossShape& s) { return s.dtype == DQGAN_F32 ? 3 : 2; }
bool half_logits(const TokenLossShape& s) { return s.dtype == DQGAN_F16 && s.weight_dtype == DQGAN_F16; }

constexpr int64_t kGradBytes = (int64_t)1 << 30, kWeightBytes = (int64_t)1 << 30;
constexpr int kFewTiles = 76;  // below: narrow tiles

// Columns of a piece of the vocabulary, a multiple of 256.
int64_t piece_of(const TokenLossShape& s) {
  const int64_t by_grad = kGradBytes / ((int64_t)s.workers * s.max_rows * 2 * kGradParts);
  const int64_t by_weight = kWeightBytes / (s.workers * round8(s.width) * 2 * logit_weight_parts(s));
  const int64_t most = by_grad < by_weight ? by_grad : by_weight;
  const int64_t whole = ceil_div(s.vocab, 256) * 256;
  return most < 256 ? 256 : most < whole ? most / 256 * 256 : whole;
}

bool narrow(int64_t rows, int32_t workers, int64_t columns) {
  return ceil_div(rows, kTileRows) * ceil_div(columns, 256) * workers < kFewTiles;
}

// Slots that the scratch space has for a row: those of wide tiles, and of narrow ones where a vocabulary is small enough
// for them (in pieces a large one's could have narrow tiles too).
constexpr int64_t wide_slots(int64_t vocab) { return 2 * ceil_div(vocab, 256); }
constexpr int64_t thin_slots(int64_t vocab) { return 2 * ceil_div(vocab, 64); }
bool thin_fits(int64_t vocab) { return thin_slots(vocab) <= 8 * kFewTiles; }
int64_t most_slots(int64_t vocab) { return thin_fits(vocab) ? thin_slots(vocab) : wide_slots(vocab); }

struct Scratch {
  uint32_t* err;
  void* products;
  void *x, *x_half, *w, *grad;
  float2* stats;
  float *target_logit, *lse, *dx, *few;
  size_t bytes;
};

Scratch scratch_of(const TokenLossShape& s, void* base) {
  Scratch c{};
  size_t at = 0;
  const auto take = [&](int64_t bytes) {
    void* p = static_cast<char*>(base) + at;
    at += (size_t)ceil_div(bytes, 1024) * 1024;
    return p;
  };
  const int64_t rows = (int64_t)s.workers * s.max_rows, piece = piece_of(s);
  c.err = static_cast<uint32_t*>(take(1024));
  c.products = take(kProductScratch);
  c.x = take(rows * round8(s.width) * 2 * act_parts(s.dtype));
  c.x_half = take(half_logits(s) ? rows * round8(s.width) * 2 : 0);
  c.w = take((int64_t)s.workers * piece * round8(s.width) * 2 * logit_weight_parts(s));
  c.grad = take(rows * piece * 2 * kGradParts);
  c.stats = static_cast<float2*>(take(rows * most_slots(s.vocab) * 8));
  c.target_logit = static_cast<float*>(take(rows * 4));
  c.lse = static_cast<float*>(take(rows * 4));
  c.dx = static_cast<float*>(take(piece < s.vocab ? rows * s.width * 4 : 0));
  c.few = static_cast<float*>(take(s.workers * most_few_rows(s.workers, s.vocab, s.width, s.max_rows) * s.vocab * 4));
  c.bytes = at;
  return c;
}

__device__ __forceinline__ int64_t counting_target(const SoftmaxArgs& s, int64_t r) {
  return row_counts(s, r) ? token_at(s.targets, s.token_bits, r) : -1;
}

constexpr float kLog2e = 1.4426950408889634f;

struct StatsEpilogue {
  static constexpr int kWarps = 8;
  template <int BN, typename S = ProductShape<BN, kWarps>>
  static __device__ __forceinline__ void run(const ProductArgs& p, const ProductTile& tile, int64_t row, int64_t column,
                                             float (&v)[S::kWidth], TurnStore<S::kBuffers>& store) {
    constexpr int kWidth = S::kWidth;
    const SoftmaxArgs& s = p.softmax;
    const int lane = store.lane;
    if (row + lane >= p.rows) return;
    const int64_t r = tile.worker * p.rows + row + lane;
    const int valid = (int)max64(0, min64(kWidth, p.columns - column));
    if (valid < kWidth) {
#pragma unroll
      for (int j = 0; j < kWidth; ++j)
        if (j >= valid) v[j] = -INFINITY;
    }
    float four[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < kWidth; ++j) four[j & 3] = fmaxf(four[j & 3], v[j]);
    const float most = fmaxf(fmaxf(four[0], four[1]), fmaxf(four[2], four[3]));
    const int64_t place = counting_target(s, r) - s.first - column;
    const int t = place >= 0 && place < valid ? (int)place : -1;
    if (t >= 0) {  // one row of 250 here, where the vocabulary has 32,000 entries
      float z = 0.f;
#pragma unroll
      for (int j = 0; j < kWidth; ++j) z += t == j ? v[j] : 0.f;
      s.target_logit[r] = z;
    }
    // the differences first: they are exact where they matter, whatever the logits' size
    const float from = most == -INFINITY ? 0.f : -most;
    float2 sums[2] = {};
#pragma unroll
    for (int j = 0; j < kWidth; j += 4) {
      const float2 a = mul2(add2(make_float2(v[j], v[j + 1]), both(from)), both(kLog2e));
      const float2 b = mul2(add2(make_float2(v[j + 2], v[j + 3]), both(from)), both(kLog2e));
      sums[0] = add2(sums[0], make_float2(exp2_approx(a.x), exp2_approx(a.y)));
      sums[1] = add2(sums[1], make_float2(exp2_approx(b.x), exp2_approx(b.y)));
    }
    const float2 sum = add2(sums[0], sums[1]);
    const int slot = s.slot + (int)(column / kWidth);
    s.stats[((int64_t)tile.worker * s.slots + slot) * p.rows + row + lane] = make_float2(most, sum.x + sum.y);
  }
};

// The gradient of the logits, in parts.
struct GradEpilogue {
  static constexpr int kWarps = 8;
  template <int BN, typename S = ProductShape<BN, kWarps>>
  static __device__ __forceinline__ void run(const ProductArgs& p, const ProductTile& tile, int64_t row, int64_t column,
                                             float (&v)[S::kWidth], TurnStore<S::kBuffers>& store) {
    constexpr int kWidth = S::kWidth;
    const SoftmaxArgs& s = p.softmax;
    const int lane = store.lane;
    const int64_t first = tile.worker * p.rows + row;
    int64_t target = -1;
    float lse = 0.f, factor = 0.f;
    if (row >= p.rows) return;
    if (row + lane < p.rows) {
      target = counting_target(s, first + lane);
      lse = s.lse[first + lane];
      factor = s.weights ? s.scale * s.weights[first + lane] : s.scale;
    }
    if (target < 0) factor = 0.f;  // the row does not count: see below where its logits are not finite
    const int64_t place = target - s.first - column;
    const int t = target >= 0 && place >= 0 && place < kWidth ? (int)place : -1;
#pragma unroll
    for (int g = 0; g < kWidth; g += 32) {
      if (column + g >= p.columns) break;
      float2 x[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        // no probability is above 1: a logit's own rounding, which may be large, does not lift it over lse
        const float2 d = add2(make_float2(v[g + 2 * j], v[g + 2 * j + 1]), both(-lse));
        const float2 e = mul2(make_float2(at_most_0(d.x), at_most_0(d.y)), both(kLog2e));
        x[j] = mul2(make_float2(exp2_approx(e.x), exp2_approx(e.y)), both(factor));
      }
      if (__any_sync(kFullMask, target < 0 || (t >= g && t < g + 32))) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (t == g + 2 * j) x[j].x -= factor;
          if (t == g + 2 * j + 1) x[j].y -= factor;
          if (target < 0) x[j] = make_float2(0.f, 0.f);
        }
      }
      for (int part = 0; part < s.grad_parts; ++part) {
        uint4 packs[4];
#pragma unroll
        for (int j = 0; j < 16; ++j) reinterpret_cast<uint32_t*>(&packs[j / 4])[j % 4] = take_parts2(x[j]);
        store.put(packs, &p.out, (int)column + g, (int)row, tile.worker, part);
      }
    }
  }
};

// A row's lse and loss from its slots: eight warps take 32 rows' slots in turn, eight loads at once, joined in order.
__global__ void __launch_bounds__(256) join_stats_kernel(const SoftmaxArgs s, int64_t rows, int32_t workers, float* loss,
                                                         float* lse) {
  dq_pdl_enter();
  __shared__ float2 part[8][32];
  constexpr int kAhead = 8;
  const int warp = (int)threadIdx.x / 32, lane = (int)threadIdx.x & 31;
  const int64_t r = (int64_t)blockIdx.x * 32 + lane;
  float most = -INFINITY, sum = 0.f;
  // sums of exponentials from one maximum to another's; of -inf nothing has been added
  const auto scale = [](float from, float to) { return from == to ? 1.f : exp2_approx((from - to) * kLog2e); };
  const auto join = [&](float2 x) {
    const float top = fmaxf(most, x.x);
    sum = sum * scale(most, top) + x.y * scale(x.x, top);
    most = top;
  };
  if (r < rows * workers) {
    const int64_t worker = r / rows, row = r - worker * rows;
    const float2* const from = s.stats + worker * s.slots * rows + row;
    for (int i = warp; i < s.slots; i += 8 * kAhead) {
      float2 x[kAhead];
      float top = most;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) x[k] = i + 8 * k < s.slots ? from[(i + 8 * k) * rows] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) top = fmaxf(top, x[k].x);
      sum *= scale(most, top);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) sum = fmaf(x[k].y, scale(x[k].x, top), sum);
      most = top;
    }
  }
  part[warp][lane] = make_float2(most, sum);
  __syncthreads();
  if (warp > 0 || r >= rows * workers) return;
  for (int w = 1; w < 8; ++w) join(part[w][lane]);
  const bool counts = counting_target(s, r) >= 0;
  const float all = most + logf(sum);
  const float c = s.weights ? s.weights[r] : 1.f;
  if (loss) loss[r] = counts ? c * (all - s.target_logit[r]) : 0.f;
  if (lse) lse[r] = counts ? all : 0.f;
}

template <typename Epilogue>
cudaError_t softmax_product(const Product& p, const SoftmaxArgs& softmax, bool thin, const Scratch& c, cudaStream_t stream,
                            uint64_t* launches) {
  ProductArgs args{};
  const int chunk = p.terms.count == 6 ? 12 : 16;
  if (!(thin ? product_args<64>(p, chunk, c.err, &args) : product_args<256>(p, chunk, c.err, &args))) return cudaErrorInvalidValue;
  args.softmax = softmax;
  const int sms = device_sms();
  if (sms <= 1) return cudaErrorInvalidDevice;
  const Cut cut = cut_product(p, sms, thin ? 64 : 256);
  args.whole = cut.whole;
  args.pieces = cut.pieces;
  args.partial = static_cast<float*>(c.products);
  if (softmax.grad && !encode_result(softmax.grad, DQGAN_BF16, p.columns, p.rows, p.workers, softmax.grad_parts, softmax.grad_ld,
                                     p.rows * softmax.grad_ld, softmax.grad_part, &args.out))
    return cudaErrorInvalidValue;
  return thin ? launch_product<64, Epilogue>(args, stream, launches) : launch_product<256, Epilogue>(args, stream, launches);
}

}  // namespace

size_t token_loss_scratch_bytes(const TokenLossShape& s) { return scratch_of(s, nullptr).bytes; }

cudaError_t launch_token_loss(const TokenLossArgs& a, cudaStream_t stream, uint64_t* launches) {
  const TokenLossShape& s = a.shape;
  const Scratch c = scratch_of(s, a.scratch);
  const bool half = half_logits(s);
  const int64_t wsize = s.weight_dtype == DQGAN_F32 ? 4 : 2, piece = piece_of(s);
  cudaError_t st = cudaSuccess;
  if (a.rows == 0) {  // gradients of nothing
    for (int m = 0; m < s.workers && st == cudaSuccess; ++m)
      if (a.backward && a.dweight && !a.accumulate)
        st = cudaMemsetAsync(a.dweight + m * a.g_stride, 0, (size_t)(s.vocab * s.width) * 4, stream);
    return st;
  }

  SoftmaxArgs soft{};
  soft.targets = a.targets;
  soft.token_bits = s.token_bits;
  soft.weights = a.weights;
  soft.vocab = s.vocab;
  soft.stats = c.stats;
  soft.target_logit = c.target_logit;
  soft.lse = a.lse ? a.lse : c.lse;
  soft.scale = a.scale;

  // A few rows: without tiles, their logits and those's gradient in scratch.
  const MatrixArgs few_w{a.weight, s.width, a.p_stride, s.weight_dtype, s.vocab, s.width, s.workers};
  if (few_rows_fit(few_w, a.rows)) {
    MatrixArgs few_x{a.x, a.x_ld, a.rows * a.x_ld, s.dtype, a.rows, s.width, s.workers};
    few_x.targets = a.targets;
    few_x.weights = a.weights;
    few_x.token_bits = s.token_bits;
    few_x.vocab = s.vocab;
    StoreArgs z{};
    z.out = c.few;
    z.out_ld = s.vocab;
    z.out_batch = a.rows * s.vocab;
    z.out_dtype = DQGAN_F32;
    const bool backward = a.backward && (a.dx || a.dweight);
    if (!a.forward && !backward) return st;
    st = launch_few_rows(few_x, few_w, z, stream, launches);
    if (st == cudaSuccess) st = launch_few_loss(c.few, few_x, a.scale, a.forward, backward, a.loss, a.lse, stream, launches);
    if (st == cudaSuccess && backward && a.dx)
      st = launch_few_across(c.few, few_w, few_x, a.rows, a.dx, a.dx_ld, s.dtype, c.products, stream, launches);
    if (st == cudaSuccess && backward && a.dweight)
      st = launch_few_outer(c.few, few_x, s.vocab, a.dweight, a.g_stride, a.accumulate, stream, launches);
    return st;
  }

  // x: of the gradient, the rows that do not count as zeros, whatever they hold
  ProductOperand x_logits, x_grad;
  Splits splits{stream, launches};
  MatrixArgs x{a.x, a.x_ld, a.rows * a.x_ld, s.dtype, a.rows, s.width, s.workers};
  if (a.forward || a.dx || a.dweight) {
    if (half) st = make_operand(x, 1, true, c.x_half, splits, &x_logits);
    if (a.backward) {
      x.targets = a.targets;
      x.weights = a.weights;
      x.token_bits = s.token_bits;
      x.vocab = s.vocab;
    }
    if (st == cudaSuccess && (!half || a.backward))
      st = make_operand(x, act_parts(s.dtype), false, c.x, splits, &x_grad);
    if (!half) x_logits = x_grad;
    if (st != cudaSuccess) return st;
  }

  // columns [first, first + count) of the vocabulary as an operand
  const auto weights = [&](int64_t first, int64_t count, int parts, bool as_half, ProductOperand* out) {
    const MatrixArgs w{static_cast<const char*>(a.weight) + first * s.width * wsize, s.width, a.p_stride, s.weight_dtype,
                       count, s.width, s.workers};
    const cudaError_t made = make_operand(w, parts, as_half, c.w, splits, out);
    return made == cudaSuccess ? splits.flush() : made;  // with what x needs, the first time
  };
  Product logits;
  logits.rows = a.rows;
  logits.depth = s.width;
  logits.workers = s.workers;
  logits.a = x_logits;
  const int logit_parts = half ? 1 : logit_weight_parts(s);
  // Both passes take the same pieces in tiles of the same width, and so sum each logit in the same order: of a row whose
  // largest logit is far above the others the gradient is 0 only if that logit has the bits that lse was made of.
  const bool thin = thin_fits(s.vocab) && narrow(a.rows, s.workers, piece < s.vocab ? piece : s.vocab);

  if (a.forward) {
    const int64_t columns = thin ? ProductShape<64>::kWidth : ProductShape<256>::kWidth;  // of a slot
    soft.slots = (int32_t)(thin ? thin_slots(s.vocab) : wide_slots(s.vocab));
    for (int64_t first = 0; first < s.vocab && st == cudaSuccess; first += piece) {
      logits.columns = s.vocab - first < piece ? s.vocab - first : piece;
      if ((st = weights(first, logits.columns, logit_parts, half, &logits.b)) != cudaSuccess) break;
      logits.terms = product_terms(logits.a.parts, logits.b.parts);
      soft.first = first;
      soft.slot = (int32_t)(first / columns);
      st = softmax_product<StatsEpilogue>(logits, soft, thin, c, stream, launches);
    }
    if (st != cudaSuccess) return st;
    ++*launches;
    st = launch_pdl(join_stats_kernel, dim3((unsigned)ceil_div(a.rows * s.workers, 32)), dim3(256), 0, stream, soft, a.rows,
                    s.workers, a.loss, const_cast<float*>(soft.lse));
    if (st != cudaSuccess) return st;
  }

  if (!a.backward || (!a.dx && !a.dweight)) return st;
  for (int64_t first = 0; first < s.vocab && st == cudaSuccess; first += piece) {
    const int64_t count = s.vocab - first < piece ? s.vocab - first : piece;
    logits.columns = count;
    if ((st = weights(first, count, logit_parts, half, &logits.b)) != cudaSuccess) return st;
    logits.terms = product_terms(logits.a.parts, logits.b.parts);
    soft.first = first;
    soft.grad = c.grad;
    soft.grad_ld = piece;
    soft.grad_part = (int64_t)s.workers * a.rows * piece;
    soft.grad_parts = kGradParts;
    st = softmax_product<GradEpilogue>(logits, soft, thin, c, stream, launches);
    if (st != cudaSuccess) return st;
    ProductOperand d;
    d.data = c.grad;
    d.ld = piece;
    d.batch = a.rows * piece;
    d.part = soft.grad_part;
    d.parts = soft.grad_parts;
    if (a.dweight) {
      Product p;
      p.rows = count;
      p.columns = s.width;
      p.depth = a.rows;
      p.workers = s.workers;
      p.a = d;
      p.b = x_grad;
      p.a.across = p.b.across = true;
      p.terms = product_terms(p.a.parts, p.b.parts);
      StoreArgs out{};
      float* const to = a.dweight + first * s.width;
      out.out = to;
      out.out_ld = s.width;
      out.out_batch = a.g_stride;
      out.out_dtype = DQGAN_F32;
      if (a.accumulate) {
        out.add = to;
        out.add_ld = s.width;
        out.add_batch = a.g_stride;
      }
      if ((st = launch_product_store(p, out, c.products, c.err, stream, launches)) != cudaSuccess) return st;
    }
    if (a.dx) {
      Product p;
      p.rows = a.rows;
      p.columns = s.width;
      p.depth = count;
      p.workers = s.workers;
      p.a = d;
      p.a.parts = dx_grad_parts(s);
      // the logits' parts serve where they are bf16 (their first ones)
      p.b = logits.b;
      if (half) st = weights(first, count, grad_weight_parts(s), false, &p.b);
      if (st != cudaSuccess) return st;
      p.b.parts = grad_weight_parts(s);
      p.b.across = true;
      p.terms = product_terms(p.a.parts, p.b.parts);
      StoreArgs out{};
      const int64_t dense = a.rows * s.width;
      if (first > 0) {
        out.add = c.dx;
        out.add_ld = s.width;
        out.add_batch = dense;
      }
      const bool last = first + count == s.vocab;
      if (last) {
        out.targets = a.targets;
        out.weights = a.weights;
        out.token_bits = s.token_bits;
        out.vocab = s.vocab;
      }
      out.out = last ? a.dx : c.dx;
      out.out_ld = last ? a.dx_ld : s.width;
      out.out_batch = last ? a.rows * a.dx_ld : dense;
      out.out_dtype = last ? s.dtype : DQGAN_F32;
      st = launch_product_store(p, out, c.products, c.err, stream, launches);
    }
  }
  return st;
}

}  // namespace dq
