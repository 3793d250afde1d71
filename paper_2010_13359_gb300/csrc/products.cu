// Matrix products that are stored: with bias, activation, residual, or added to
// what is there; and the splitting of operands into 16-bit parts.
#include <initializer_list>

#include "product_kernel.cuh"

namespace dq {

ProductTerms product_terms(int a_parts, int b_parts) {
  ProductTerms t;
  t.count = 0;
  const int parts = a_parts > b_parts ? a_parts : b_parts;
  for (int order = parts - 1; order >= 0; --order)  // the smallest first
    for (int i = 0; i <= order; ++i)
      if (i < a_parts && order - i < b_parts) {
        t.a[t.count] = (uint8_t)i;
        t.b[t.count++] = (uint8_t)(order - i);
      }
  return t;
}

namespace {

// 32 values of a row, 16 bytes at a time, up to `count`.
template <typename T>
__device__ __forceinline__ void add32(const T* from, int64_t count, float (&x)[32]) {
  constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < 32; i += E) {
    if (i + E <= count) {
      const uint4 pack = *reinterpret_cast<const uint4*>(from + i);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 v = pair_of<T>(pack, e);
        x[i + e] += v.x;
        x[i + e + 1] += v.y;
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (i + e < count) x[i + e] += to_float(from[i + e]);
    }
  }
}

// A warp's 32 rows, by TMA.
template <typename T, int kSumWarps>
struct StoreEpilogue {
  static constexpr int kWarps = kSumWarps;
  template <int BN, typename S = ProductShape<BN, kWarps>>
  static __device__ __forceinline__ void run(const ProductArgs& p, const ProductTile& tile, int64_t row, int64_t column,
                                             const float (&v)[S::kWidth], TurnStore<S::kBuffers>& store) {
    const StoreArgs& s = p.store;
    const int lane = store.lane;
    const int rows = (int)min64(32, p.rows - row);
    if (rows <= 0) return;
    const float* const bias = s.bias ? s.bias + tile.worker * s.bias_batch : nullptr;
    const bool counts = lane >= rows || row_counts(s, tile.worker * p.rows + row + lane);
#pragma unroll
    for (int g = 0; g < S::kWidth; g += 32) {
      const int64_t j = column + g, count = p.columns - j;
      if (count <= 0) break;
      float x[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) x[i] = v[g + i];
      const float b = bias && lane < count ? bias[j + lane] : 0.f;
      if (s.add && lane < rows) add32(s.add + tile.worker * s.add_batch + (row + lane) * s.add_ld + j, count, x);
      if (bias) {
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] += __shfl_sync(kFullMask, b, i);
      }
      if (s.pre) store.template put32<T>(x, &p.pre, (int)j, (int)row, tile.worker);
      activate_all<sizeof(T) == 4>(x, s.activation);
      if (s.residual && lane < rows)
        add32(static_cast<const T*>(s.residual) + tile.worker * s.residual_batch + (row + lane) * s.residual_ld + j, count, x);
      if (!counts) {
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = 0.f;
      }
      store.template put32<T>(x, &p.out, (int)j, (int)row, tile.worker);
    }
  }
};

}  // namespace

// By the time that the busiest block needs, in units of a block of 64 of the contracted index of a 256 x 256 tile (0.3 us).  A
// tile's end costs as much as 12 of them (3 of a narrow tile, whose blocks take 0.6: 24 KB to load instead of 32); pieces
// cost a second kernel, 10, their sums' way through memory, 0.3 each, and one load after another there, 1 for each of a tile's.
Cut cut_product(const Product& p, int64_t slots, int only) {
  const int64_t depth = ceil_div(p.depth, kBlockDepth), length = depth * p.terms.count;
  Cut best{256, 0, 1};
  double least = 1e300;
  for (int width = 64; width <= 256; width += 192) {
    if (only != 0 && width != only) continue;
    const bool wide = width == 256;
    const int64_t tiles = ceil_div(p.rows, wide ? 256 : 128) * ceil_div(p.columns, width) * p.workers;
    const int64_t at_once = wide ? slots / 2 : slots, rest = tiles % at_once, whole = tiles - rest;
    const double block = wide ? 1. : 0.6, end = wide ? 12. : 3., sums = wide ? 0.3 : 0.04;
    for (const int pieces : {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 16, 24, 32}) {
      const int64_t items = rest * pieces;
      if (pieces > 1 && (rest == 0 || pieces > depth || (size_t)items * (wide ? 1 << 18 : 1 << 15) > kProductScratch)) break;
      double time = (double)(whole / at_once) * (length * block + end) +
                    (double)ceil_div(items, at_once) * (ceil_div(depth, pieces) * p.terms.count * block + end);
      if (pieces > 1) time += 10. + items * sums + pieces;
      if (time < least) {
        least = time;
        best = {width, pieces > 1 ? whole : tiles, pieces};
      }
    }
  }
  return best;
}

namespace {

template <int BN>
cudaError_t store_product(const Product& p, const StoreArgs& store, const Cut& cut, void* scratch, uint32_t* err,
                          cudaStream_t stream, uint64_t* launches) {
  ProductArgs args{};
  const int chunk = p.terms.count == 6 ? 12 : store.out_dtype == DQGAN_F32 ? 16 : store.out_dtype == DQGAN_F16 ? 32 : 128;
  if (!product_args<BN>(p, chunk, err, &args)) return cudaErrorInvalidValue;
  args.store = store;
  args.whole = cut.whole;
  args.pieces = cut.pieces;
  args.partial = static_cast<float*>(scratch);
  const int64_t size = store.out_dtype == DQGAN_F32 ? 4 : 2;
  const auto packs = [&](const void* at, int64_t ld, int64_t batch, int64_t of) {
    return !at || (((uintptr_t)at & 15) == 0 && ld * of % 16 == 0 && ld * of < ((int64_t)1 << 40) &&
                   (p.workers == 1 || (batch * of % 16 == 0 && batch * of < ((int64_t)1 << 40))));
  };
  const bool by_tma = p.columns * size % 16 == 0 && packs(store.out, store.out_ld, store.out_batch, size) && packs(store.pre, store.pre_ld, store.pre_batch, size) &&
                     packs(store.residual, store.residual_ld, store.residual_batch, size) &&
                     packs(store.add, store.add_ld, store.add_batch, 4);
  if (!by_tma) return launch_product_rows<BN>(args, stream, launches);
  if (!(encode_result(store.out, store.out_dtype, p.columns, p.rows, p.workers, 1, store.out_ld, store.out_batch, 0, &args.out) &&
        (!store.pre || encode_result(store.pre, store.out_dtype, p.columns, p.rows, p.workers, 1, store.pre_ld, store.pre_batch, 0,
                                     &args.pre))))
    return cudaErrorInvalidValue;
  return with_dtype(store.out_dtype, [&](auto t) {
    return BN == 256 && store.activation != DQGAN_NONE ? launch_product<BN, StoreEpilogue<decltype(t), BN == 256 ? 16 : 8>>(args, stream, launches)
                                                       : launch_product<BN, StoreEpilogue<decltype(t), 8>>(args, stream, launches);
  });
}

}  // namespace

cudaError_t launch_product_store(const Product& p, const StoreArgs& store, void* scratch, uint32_t* err,
                                 cudaStream_t stream, uint64_t* launches) {
  if (p.rows == 0 || p.columns == 0) return cudaSuccess;
  const int sms = device_sms();
  if (sms <= 1) return cudaErrorInvalidDevice;
  const Cut cut = cut_product(p, sms, 0);
  return cut.width == 256 ? store_product<256>(p, store, cut, scratch, err, stream, launches)
                          : store_product<64>(p, store, cut, scratch, err, stream, launches);
}

// ---- parts ----
namespace {

// 8 values of one of two matrices a thread; the second one's follow the first one's.
template <typename T>
__global__ void __launch_bounds__(256) split_kernel(const SplitArgs first, const SplitArgs second) {
  dq_pdl_enter();
  const int64_t of_first = first.ld / 8 * first.rows * first.workers, total = of_first + second.ld / 8 * second.rows * second.workers;
  for (int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; at < total; at += (int64_t)gridDim.x * blockDim.x) {
    const SplitArgs& a = at < of_first ? first : second;
    const int64_t i = at < of_first ? at : at - of_first, across = a.ld / 8;
    const int64_t r = i / across;
    const int column = (int)(i - r * across) * 8;
    const int64_t worker = r / a.rows, row = r - worker * a.rows;
    float x[8] = {};
    if (row_counts(a, r)) {
      const T* const from = static_cast<const T*>(a.from) + worker * a.batch + row * a.from_ld + column;
      const int count = (int)min64(8, a.columns - column);
      if (a.packs)
        read8(from, count, true, x);
      else
        read8_near(from, count, a.from, static_cast<const T*>(a.from) + (a.workers - 1) * a.batch + (a.rows - 1) * a.from_ld + a.columns, x);
    }
    write_parts<true>(x, a.to, r * a.ld + column, a.part, a.parts, a.half);
  }
}

}  // namespace

cudaError_t Splits::add(const SplitArgs& a) {
  cudaError_t st = cudaSuccess;
  if (a.rows == 0 || a.workers == 0) return st;
  if (count == 2 || (count == 1 && pending[0].dtype != a.dtype)) st = flush();
  pending[count] = a;
  const int64_t size = a.dtype == DQGAN_F32 ? 4 : 2;
  pending[count++].packs = ((uintptr_t)a.from & 15) == 0 && a.from_ld * size % 16 == 0 && (a.workers == 1 || a.batch * size % 16 == 0);
  return st;
}

cudaError_t Splits::flush() {
  if (count == 0) return cudaSuccess;
  const SplitArgs first = pending[0], second = count == 2 ? pending[1] : SplitArgs{};
  count = 0;
  const int64_t total = first.ld / 8 * first.rows * first.workers + second.ld / 8 * second.rows * second.workers;
  const int sms = device_sms();
  if (sms <= 0) return cudaErrorInvalidDevice;
  ++*launches;
  const dim3 grid((unsigned)min64(ceil_div(total, 256), (int64_t)sms * 8));
  return with_dtype(first.dtype, [&](auto t) { return launch_pdl(split_kernel<decltype(t)>, grid, dim3(256), 0, stream, first, second); });
}

cudaError_t make_operand(const MatrixArgs& m, int parts, bool half, void* buffer, Splits& splits, ProductOperand* out) {
  const bool as_is = !m.targets && (half ? m.dtype == DQGAN_F16 : m.dtype == DQGAN_BF16 && parts == 1);
  out->shared = m.batch == 0 && m.workers > 1;
  out->half = half;
  out->across = false;
  if (as_is && operand_in_place(m.data, m.ld, m.workers > 1 ? m.batch : 0)) {
    out->data = m.data;
    out->ld = m.ld;
    out->batch = m.batch;
    out->parts = 1;
    out->part = 0;
    return cudaSuccess;
  }
  SplitArgs s{};
  s.from = m.data;
  s.batch = m.batch;
  s.from_ld = m.ld;
  s.dtype = m.dtype;
  s.to = buffer;
  s.ld = round8(m.columns);
  s.rows = m.rows;
  s.columns = m.columns;
  s.workers = out->shared ? 1 : m.workers;
  s.part = s.ld * s.rows * s.workers;
  s.parts = parts;
  s.half = half;
  s.targets = m.targets;
  s.weights = m.weights;
  s.token_bits = m.token_bits;
  s.vocab = m.vocab;
  out->data = buffer;
  out->ld = s.ld;
  out->batch = s.ld * s.rows;
  out->part = s.part;
  out->parts = parts;
  return splits.add(s);
}

}  // namespace dq
