// Declarations of the token-model operators (not part of the C-ABI): argument
// blocks, launchers, and the element types' conversions.  Their arithmetic is
// fp32; unlike the compress and server kernels they may use fused
// multiply-adds (written out as fmaf: the library is built without contraction).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.cuh"

namespace dq {

struct LayerNormArgs {
  const void* x;        // worker m's row r at x + (m * rows + r) * x_ld elements
  const void* dy;       // backward
  void* out;            // y, or dx (backward; may be nullptr)
  int64_t x_ld, dy_ld, out_ld;
  const float* weight;  // worker m's at + m * p_stride, or nullptr (ones)
  const float* bias;    // forward; nullptr: zeros
  int64_t p_stride;
  float* mean;          // one a row (forward: or nullptr)
  float* rstd;
  float* dweight;       // backward; worker m's at + m * g_stride, or nullptr
  float* dbias;
  int64_t g_stride;
  float* scratch;       // backward: layer_norm_scratch_bytes
  int64_t rows;         // per worker
  int64_t width;
  int32_t workers;
  int32_t dtype;
  float eps;
  int32_t accumulate;
};

struct EmbeddingArgs {
  const void* ids;      // worker m's at + m * tokens, int32 or int64
  const void* table;    // forward; worker m's at + m * p_stride elements
  int64_t p_stride;
  void* y;              // forward
  const void* dy;       // backward
  int64_t ld;           // row stride of y or dy
  float* dtable;        // backward; worker m's at + m * g_stride
  int64_t g_stride;
  void* scratch;        // backward: embedding_scratch_bytes
  int64_t tokens;       // per worker
  int64_t vocab;
  int64_t width;
  int32_t workers;
  int32_t table_dtype;
  int32_t dtype;
  int32_t token_bits;
  float scale;
  int32_t accumulate;
};

struct DistillationArgs {
  const void* logits;       // row r at + r * ld
  int64_t ld;
  void* dlogits;            // backward and step
  int64_t dld;
  const int32_t* ids;       // row r's k entries at + r * teacher_ld
  const void* values;
  int64_t teacher_ld;
  const float* teacher_lse; // or nullptr
  const float* weights;     // or nullptr
  float* loss;              // forward and step
  float* lse;               // forward and step: written, or nullptr; backward: read
  int64_t rows;
  int64_t vocab;
  int32_t k;
  int32_t dtype;
  int32_t teacher_dtype;
  float temperature;
  float scale;
};

enum class DistillationWay { kForward, kBackward, kStep };

size_t layer_norm_scratch_bytes(int64_t width, int32_t workers);
cudaError_t launch_layer_norm_forward(const LayerNormArgs& a, cudaStream_t stream, uint64_t* launches);
cudaError_t launch_layer_norm_backward(const LayerNormArgs& a, cudaStream_t stream, uint64_t* launches);

size_t embedding_scratch_bytes(int64_t vocab, int64_t width, int64_t max_tokens, int32_t workers);
cudaError_t launch_embedding_forward(const EmbeddingArgs& a, cudaStream_t stream, uint64_t* launches);
cudaError_t launch_embedding_backward(const EmbeddingArgs& a, cudaStream_t stream, uint64_t* launches);

cudaError_t launch_distillation(const DistillationArgs& a, DistillationWay way, cudaStream_t stream,
                                uint64_t* launches);

__host__ __device__ constexpr int64_t ceil_div(int64_t x, int64_t m) { return (x + m - 1) / m; }

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) {
  return x;
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}
template <>
__device__ __forceinline__ __half from_float<__half>(float x) {
  return __float2half_rn(x);
}

// Two fp32 operations in one instruction, each rounded as the single one.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<const uint64_t&>(a)), "l"(reinterpret_cast<const uint64_t&>(b)),
        "l"(reinterpret_cast<const uint64_t&>(c)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<const uint64_t&>(a)), "l"(reinterpret_cast<const uint64_t&>(b)));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<const uint64_t&>(a)), "l"(reinterpret_cast<const uint64_t&>(b)));
  return d;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// Elements (e, e + 1) of a pack, and back.
template <typename T>
__device__ __forceinline__ float2 pair_of(const uint4& p, int e);
template <>
__device__ __forceinline__ float2 pair_of<float>(const uint4& p, int e) {
  const float* v = reinterpret_cast<const float*>(&p);
  return make_float2(v[e], v[e + 1]);
}
template <>
__device__ __forceinline__ float2 pair_of<__nv_bfloat16>(const uint4& p, int e) {
  const uint32_t v = reinterpret_cast<const uint32_t*>(&p)[e / 2];  // a bf16 is the upper half of an fp32
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
template <>
__device__ __forceinline__ float2 pair_of<__half>(const uint4& p, int e) {
  return __half22float2(reinterpret_cast<const __half2*>(&p)[e / 2]);
}

template <typename T>
__device__ __forceinline__ void set_pair(uint4& p, int e, float2 v);
template <>
__device__ __forceinline__ void set_pair<float>(uint4& p, int e, float2 v) {
  float* to = reinterpret_cast<float*>(&p);
  to[e] = v.x;
  to[e + 1] = v.y;
}
template <>
__device__ __forceinline__ void set_pair<__nv_bfloat16>(uint4& p, int e, float2 v) {
  reinterpret_cast<__nv_bfloat162*>(&p)[e / 2] = __float22bfloat162_rn(v);
}
template <>
__device__ __forceinline__ void set_pair<__half>(uint4& p, int e, float2 v) {
  reinterpret_cast<__half2*>(&p)[e / 2] = __float22half2_rn(v);
}

// Bytes [s, s + 16) of the 32 in (a, b); s < 16, a multiple of 2.
__device__ __forceinline__ uint4 funnel16(const uint4& a, const uint4& b, int s) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint32_t t[6], u[5];
#pragma unroll
  for (int k = 0; k < 6; ++k) t[k] = s & 8 ? w[k + 2] : w[k];
#pragma unroll
  for (int k = 0; k < 5; ++k) u[k] = s & 4 ? t[k + 1] : t[k];
  const int bits = (s & 3) * 8;
  return make_uint4(__funnelshift_r(u[0], u[1], bits), __funnelshift_r(u[1], u[2], bits),
                    __funnelshift_r(u[2], u[3], bits), __funnelshift_r(u[3], u[4], bits));
}

// Rows that do not start or end on 16-byte boundaries are read as the aligned packs of 16 bytes that hold them.  Gaps
// between rows may be read along, but nothing before the first row's first value or after the last row's last: those of
// worker m's rows whose packs stay clear of that.  near: the rows from either end whose packs may not; heads: a pack
// may begin before its row does; tails: it may end after it.
struct Rows {
  int begin, end;
};
__host__ __device__ constexpr int rows_near(int64_t ld_bytes) { return ld_bytes < 16 ? (int)ceil_div(16, ld_bytes) : 1; }
__host__ __device__ constexpr Rows rows_inside(int rows, int workers, int m, int near, bool heads, bool tails) {
  const int64_t before = near - (int64_t)m * rows, after = near - (int64_t)(workers - 1 - m) * rows;
  const int begin = !heads || before < 0 ? 0 : before < rows ? (int)before : rows;
  const int end = rows - (!tails || after < 0 ? 0 : after < rows - begin ? (int)after : rows - begin);
  return {begin, end};
}

// Copies `bytes` (at most 16) bytes and zeros the rest of the 16, asynchronously.
__device__ __forceinline__ void copy16_async(void* to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_begun() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void wait_copies() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

// Calls f with a value of the element type that `dtype` names.
template <typename F>
inline cudaError_t with_dtype(int32_t dtype, F&& f) {
  switch (dtype) {
    case DQGAN_F32: return f(float{});
    case DQGAN_BF16: return f(__nv_bfloat16{});
    case DQGAN_F16: return f(__half{});
  }
  return cudaErrorInvalidValue;
}

// Sum over the block in a fixed order (warp butterflies, then the warps' sums
// in order); every thread gets it.  `shared`: 32 floats, reused by the next call.
__device__ __forceinline__ float block_sum(float x, float* shared) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(kFullMask, x, o);
  const int warps = (int)(blockDim.x + 31) / 32;
  __syncthreads();
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x / 32] = x;
  __syncthreads();
  float s = shared[0];
  for (int i = 1; i < warps; ++i) s += shared[i];
  return s;
}

}  // namespace dq
