// Products whose results TMA cannot write: rows that are not on 16-byte boundaries, or do not end on one.
#include "product_kernel.cuh"

namespace dq {

namespace {

// A warp's 32 rows, turned in shared memory so that its lanes hold neighbouring columns, and stored by single values.
template <typename T>
struct RowsEpilogue {
  static constexpr int kWarps = 8;
  template <int BN, typename S = ProductShape<BN, kWarps>>
  static __device__ __forceinline__ void run(const ProductArgs& p, const ProductTile& tile, int64_t row, int64_t column,
                                             const float (&v)[S::kWidth], TurnStore<S::kBuffers>& store) {
    const StoreArgs& s = p.store;
    const int lane = store.lane;
    const int rows = (int)min64(32, p.rows - row);
    if (rows <= 0) return;
    const float* const bias = s.bias ? s.bias + tile.worker * s.bias_batch : nullptr;
#pragma unroll
    for (int g = 0; g < S::kWidth; g += 32) {
      const int64_t j = column + g + lane;
      if (column + g >= p.columns) break;
      store.turn(v + g);
      if (j >= p.columns) continue;
      const float b = bias ? bias[j] : 0.f;
      const T* const residual = s.residual ? static_cast<const T*>(s.residual) + tile.worker * s.residual_batch + row * s.residual_ld + j : nullptr;
      const float* const add = s.add ? s.add + tile.worker * s.add_batch + row * s.add_ld + j : nullptr;
      T* const pre = s.pre ? static_cast<T*>(s.pre) + tile.worker * s.pre_batch + row * s.pre_ld + j : nullptr;
      T* const out = static_cast<T*>(s.out) + tile.worker * s.out_batch + row * s.out_ld + j;
      // Eight rows at a time, all loads before their use.  Rows beyond the last are the last's and not stored: branches
      // around the loads would make each wait for itself.
#pragma unroll 1
      for (int i = 0; i < rows; i += 8) {
        float x[8];
        T more[8];
        if (residual) {
#pragma unroll
          for (int k = 0; k < 8; ++k) more[k] = residual[min(i + k, rows - 1) * s.residual_ld];
        }
        if (add) {
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] = add[min(i + k, rows - 1) * s.add_ld];
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] += store.turned(i + k);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] = store.turned(i + k);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] += b;
        if (pre) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (i + k < rows) pre[(i + k) * s.pre_ld] = from_float<T>(x[k]);
        }
        activate_all<sizeof(T) == 4>(x, s.activation);
        if (residual) {
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] += to_float(more[k]);
        }
        if (s.targets) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (!row_counts(s, tile.worker * p.rows + row + min(i + k, rows - 1))) x[k] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (i + k < rows) out[(i + k) * s.out_ld] = from_float<T>(x[k]);
      }
    }
  }
};

}  // namespace

template <int BN>
cudaError_t launch_product_rows(const ProductArgs& args, cudaStream_t stream, uint64_t* launches) {
  return with_dtype(args.store.out_dtype, [&](auto t) { return launch_product<BN, RowsEpilogue<decltype(t)>>(args, stream, launches); });
}
template cudaError_t launch_product_rows<256>(const ProductArgs& args, cudaStream_t stream, uint64_t* launches);
template cudaError_t launch_product_rows<64>(const ProductArgs& args, cudaStream_t stream, uint64_t* launches);

}  // namespace dq
