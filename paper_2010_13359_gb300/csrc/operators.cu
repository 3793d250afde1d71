// C-ABI of the token-model operators (declared in include/dqgan.h): argument
// checking, ownership of the scratch space and dispatch to the kernels.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>

#include <nvtx3/nvToolsExt.h>

#include "operators.cuh"

namespace {

enum class Kind { kLayerNorm, kEmbedding, kDistillation };

}  // namespace

struct dqgan_operator {
  Kind kind;
  dqgan_layer_norm_config norm{};
  dqgan_embedding_config embedding{};
  dqgan_distillation_config distillation{};
  cudaStream_t stream = nullptr;
  void* scratch = nullptr;
  uint64_t launches = 0;
  char err[256] = "";
};

namespace {

constexpr int64_t kMaxWidth = 65536, kMaxWorkers = 4096, kMaxVocab = 1 << 24, kMaxTokens = 1 << 24;
constexpr int64_t kMaxBatch = 1 << 28;          // workers * tokens, workers * vocab
constexpr int64_t kMaxRows = (int64_t)1 << 30;  // rows of one call, over all workers
constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr int kMaxEntries = 1024;

struct NvtxRange {
  explicit NvtxRange(const char* name) { nvtxRangePushA(name); }
  ~NvtxRange() { nvtxRangePop(); }
  NvtxRange(const NvtxRange&) = delete;
  NvtxRange& operator=(const NvtxRange&) = delete;
};

thread_local char tl_operator_err[256] = "";

int fail(dqgan_operator* op, int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(op ? op->err : tl_operator_err, sizeof tl_operator_err, fmt, ap);
  va_end(ap);
  return code;
}

int invalid(dqgan_operator* op, const char* what) { return fail(op, DQGAN_ERR_INVALID_ARG, "%s", what); }

int launched(dqgan_operator* op, cudaError_t st, const char* what) {
  if (st == cudaSuccess) return DQGAN_OK;
  return fail(op, DQGAN_ERR_CUDA, "%s launch: %s", what, cudaGetErrorString(st));
}

bool known_dtype(int32_t t) { return t == DQGAN_F32 || t == DQGAN_BF16 || t == DQGAN_F16; }
uintptr_t dtype_size(int32_t t) { return t == DQGAN_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool stride_ok(int64_t stride, int64_t least) { return stride >= least && stride <= kMaxStride; }

int create(Kind kind, void* stream, size_t scratch_bytes, dqgan_operator** out) {
  dq::arm_device_allocation();
  dqgan_operator* op = new (std::nothrow) dqgan_operator();
  if (!op) return fail(nullptr, DQGAN_ERR_OOM, "host allocation failed");
  op->kind = kind;
  op->stream = reinterpret_cast<cudaStream_t>(stream);
  if (scratch_bytes > 0) {
    const cudaError_t st = dq::device_allocate(&op->scratch, scratch_bytes);
    if (st != cudaSuccess) {
      cudaGetLastError();
      delete op;
      return fail(nullptr, st == cudaErrorMemoryAllocation ? DQGAN_ERR_OOM : DQGAN_ERR_CUDA, "allocating scratch: %s",
                  cudaGetErrorString(st));
    }
  }
  *out = op;
  return DQGAN_OK;
}

int check(dqgan_operator* op, Kind kind, const char* name) {
  if (!op) return invalid(nullptr, "operator is NULL");
  if (op->kind != kind) return fail(op, DQGAN_ERR_INVALID_ARG, "the operator is not %s", name);
  return DQGAN_OK;
}

// Rows per worker: the call's over all workers stay below kMaxRows.
int check_rows(dqgan_operator* op, const char* what, int64_t rows, int64_t workers) {
  if (rows < 0 || rows * (double)workers > (double)kMaxRows)
    return fail(op, DQGAN_ERR_INVALID_ARG, "%s = %lld outside [0, %lld]", what, (long long)rows,
                (long long)(kMaxRows / workers));
  return DQGAN_OK;
}

}  // namespace

extern "C" {

int dqgan_layer_norm_create(const dqgan_layer_norm_config* cfg, dqgan_operator** out) {
  if (!out) return invalid(nullptr, "out is NULL");
  *out = nullptr;
  if (!cfg) return invalid(nullptr, "config is NULL");
  if (cfg->width < 1 || cfg->width > kMaxWidth) return invalid(nullptr, "width outside [1, 65536]");
  if (cfg->workers < 1 || cfg->workers > kMaxWorkers) return invalid(nullptr, "workers outside [1, 4096]");
  if (!known_dtype(cfg->dtype)) return invalid(nullptr, "unknown dtype");
  if (!std::isfinite(cfg->eps) || cfg->eps < 0.f) return invalid(nullptr, "eps is negative or not finite");
  if (cfg->reserved != 0) return invalid(nullptr, "reserved is not 0");
  const int st = create(Kind::kLayerNorm, cfg->cuda_stream, dq::layer_norm_scratch_bytes(cfg->width, cfg->workers), out);
  if (st == DQGAN_OK) (*out)->norm = *cfg;
  return st;
}

int dqgan_embedding_create(const dqgan_embedding_config* cfg, dqgan_operator** out) {
  if (!out) return invalid(nullptr, "out is NULL");
  *out = nullptr;
  if (!cfg) return invalid(nullptr, "config is NULL");
  if (cfg->vocab < 1 || cfg->vocab > kMaxVocab) return invalid(nullptr, "vocab outside [1, 2^24]");
  if (cfg->width < 1 || cfg->width > kMaxWidth) return invalid(nullptr, "width outside [1, 65536]");
  if (cfg->max_tokens < 1 || cfg->max_tokens > kMaxTokens) return invalid(nullptr, "max_tokens outside [1, 2^24]");
  if (cfg->workers < 1 || cfg->workers > kMaxWorkers) return invalid(nullptr, "workers outside [1, 4096]");
  if (cfg->workers * cfg->max_tokens > kMaxBatch || cfg->workers * cfg->vocab > kMaxBatch)
    return invalid(nullptr, "workers * max_tokens or workers * vocab above 2^28");
  if (!known_dtype(cfg->table_dtype) || !known_dtype(cfg->dtype)) return invalid(nullptr, "unknown dtype");
  if (cfg->token_bits != 32 && cfg->token_bits != 64) return invalid(nullptr, "token_bits not in {32, 64}");
  if (!std::isfinite(cfg->scale)) return invalid(nullptr, "scale is not finite");
  if (cfg->reserved != 0) return invalid(nullptr, "reserved is not 0");
  const int st = create(Kind::kEmbedding, cfg->cuda_stream,
                        dq::embedding_scratch_bytes(cfg->vocab, cfg->width, cfg->max_tokens, cfg->workers), out);
  if (st == DQGAN_OK) (*out)->embedding = *cfg;
  return st;
}

int dqgan_distillation_create(const dqgan_distillation_config* cfg, dqgan_operator** out) {
  if (!out) return invalid(nullptr, "out is NULL");
  *out = nullptr;
  if (!cfg) return invalid(nullptr, "config is NULL");
  if (cfg->vocab < 1 || cfg->vocab > kMaxVocab) return invalid(nullptr, "vocab outside [1, 2^24]");
  if (cfg->k < 1 || cfg->k > kMaxEntries) return invalid(nullptr, "k outside [1, 1024]");
  if (!known_dtype(cfg->dtype) || !known_dtype(cfg->teacher_dtype)) return invalid(nullptr, "unknown dtype");
  if (!std::isnormal(cfg->temperature) || !(cfg->temperature > 0.f))  // of a subnormal one 1 / T overflows
    return invalid(nullptr, "temperature is not a positive normal number");
  if (cfg->reserved[0] != 0 || cfg->reserved[1] != 0) return invalid(nullptr, "reserved is not 0");
  const int st = create(Kind::kDistillation, cfg->cuda_stream, 0, out);
  if (st == DQGAN_OK) (*out)->distillation = *cfg;
  return st;
}

int dqgan_operator_destroy(dqgan_operator* op) {
  if (!op) return DQGAN_OK;
  cudaStreamSynchronize(op->stream);
  if (op->scratch) cudaFree(op->scratch);
  delete op;
  const cudaError_t st = cudaGetLastError();
  if (st != cudaSuccess) return fail(nullptr, DQGAN_ERR_CUDA, "destroy: %s", cudaGetErrorString(st));
  return DQGAN_OK;
}

int dqgan_operator_synchronize(dqgan_operator* op) {
  if (!op) return invalid(nullptr, "operator is NULL");
  const cudaError_t st = cudaStreamSynchronize(op->stream);
  if (st != cudaSuccess) return fail(op, DQGAN_ERR_CUDA, "synchronize: %s", cudaGetErrorString(st));
  return DQGAN_OK;
}

uint64_t dqgan_operator_launch_count(const dqgan_operator* op) { return op ? op->launches : 0; }

const char* dqgan_operator_last_error(const dqgan_operator* op) { return op ? op->err : tl_operator_err; }

int dqgan_layer_norm_forward(dqgan_operator* op, int64_t rows, const void* x, int64_t x_stride, const float* weight,
                             const float* bias, int64_t p_stride, void* y, int64_t y_stride, float* mean, float* rstd) {
  if (int r = check(op, Kind::kLayerNorm, "a layer norm")) return r;
  const dqgan_layer_norm_config& c = op->norm;
  if (int r = check_rows(op, "rows", rows, c.workers)) return r;
  if (rows == 0) return DQGAN_OK;
  if (!x || !y) return invalid(op, "NULL x or y");
  if ((mean == nullptr) != (rstd == nullptr)) return invalid(op, "mean and rstd: both or neither");
  if (!stride_ok(x_stride, c.width) || !stride_ok(y_stride, c.width)) return invalid(op, "a row stride is below the width");
  if (p_stride != 0 && !stride_ok(p_stride, c.width)) return invalid(op, "p_stride is neither 0 nor at least the width");
  if (!aligned(x, dtype_size(c.dtype)) || !aligned(y, dtype_size(c.dtype)) || !aligned(weight, 4) || !aligned(bias, 4) ||
      !aligned(mean, 4) || !aligned(rstd, 4))
    return invalid(op, "a pointer is not aligned to its element");
  NvtxRange range("dqgan layer norm forward");
  dq::LayerNormArgs a{};
  a.x = x;
  a.out = y;
  a.x_ld = x_stride;
  a.out_ld = y_stride;
  a.weight = weight;
  a.bias = bias;
  a.p_stride = p_stride;
  a.mean = mean;
  a.rstd = rstd;
  a.rows = rows;
  a.width = c.width;
  a.workers = c.workers;
  a.dtype = c.dtype;
  a.eps = c.eps;
  return launched(op, dq::launch_layer_norm_forward(a, op->stream, &op->launches), "layer norm forward");
}

int dqgan_layer_norm_backward(dqgan_operator* op, int64_t rows, const void* dy, int64_t dy_stride, const void* x,
                              int64_t x_stride, const float* weight, int64_t p_stride, const float* mean,
                              const float* rstd, void* dx, int64_t dx_stride, float* dweight, float* dbias,
                              int64_t g_stride, int32_t accumulate) {
  if (int r = check(op, Kind::kLayerNorm, "a layer norm")) return r;
  const dqgan_layer_norm_config& c = op->norm;
  if (int r = check_rows(op, "rows", rows, c.workers)) return r;
  if (!dx && !dweight && !dbias) return DQGAN_OK;
  if (rows > 0) {
    if (!dy || !x || !mean || !rstd) return invalid(op, "NULL dy, x, mean or rstd");
    if (!stride_ok(dy_stride, c.width) || !stride_ok(x_stride, c.width) || (dx && !stride_ok(dx_stride, c.width)))
      return invalid(op, "a row stride is below the width");
  }
  if (p_stride != 0 && !stride_ok(p_stride, c.width)) return invalid(op, "p_stride is neither 0 nor at least the width");
  if ((dweight || dbias) && c.workers > 1 && !stride_ok(g_stride, c.width))
    return invalid(op, "g_stride is below the width");
  const uintptr_t size = dtype_size(c.dtype);
  if (!aligned(dy, size) || !aligned(x, size) || !aligned(dx, size) || !aligned(weight, 4) || !aligned(mean, 4) ||
      !aligned(rstd, 4) || !aligned(dweight, 4) || !aligned(dbias, 4))
    return invalid(op, "a pointer is not aligned to its element");
  NvtxRange range("dqgan layer norm backward");
  dq::LayerNormArgs a{};
  a.x = x;
  a.dy = dy;
  a.out = dx;
  a.x_ld = x_stride;
  a.dy_ld = dy_stride;
  a.out_ld = dx_stride;
  a.weight = weight;
  a.p_stride = p_stride;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dweight = dweight;
  a.dbias = dbias;
  a.g_stride = c.workers > 1 ? g_stride : 0;
  a.scratch = static_cast<float*>(op->scratch);
  a.rows = rows;
  a.width = c.width;
  a.workers = c.workers;
  a.dtype = c.dtype;
  a.accumulate = accumulate != 0;
  return launched(op, dq::launch_layer_norm_backward(a, op->stream, &op->launches), "layer norm backward");
}

int dqgan_embedding_forward(dqgan_operator* op, int64_t tokens, const void* ids, const void* table, int64_t p_stride,
                            void* y, int64_t y_stride) {
  if (int r = check(op, Kind::kEmbedding, "an embedding")) return r;
  const dqgan_embedding_config& c = op->embedding;
  if (tokens < 0 || tokens > c.max_tokens) return invalid(op, "tokens outside [0, max_tokens]");
  if (tokens == 0) return DQGAN_OK;
  if (!ids || !table || !y) return invalid(op, "NULL ids, table or y");
  if (!stride_ok(y_stride, c.width)) return invalid(op, "the row stride is below the width");
  if (p_stride != 0 && !stride_ok(p_stride, c.vocab * c.width))
    return invalid(op, "p_stride is neither 0 nor at least vocab * width");
  if (!aligned(ids, c.token_bits / 8) || !aligned(table, dtype_size(c.table_dtype)) || !aligned(y, dtype_size(c.dtype)))
    return invalid(op, "a pointer is not aligned to its element");
  NvtxRange range("dqgan embedding forward");
  dq::EmbeddingArgs a{};
  a.ids = ids;
  a.table = table;
  a.p_stride = p_stride;
  a.y = y;
  a.ld = y_stride;
  a.tokens = tokens;
  a.vocab = c.vocab;
  a.width = c.width;
  a.workers = c.workers;
  a.table_dtype = c.table_dtype;
  a.dtype = c.dtype;
  a.token_bits = c.token_bits;
  a.scale = c.scale;
  return launched(op, dq::launch_embedding_forward(a, op->stream, &op->launches), "embedding forward");
}

int dqgan_embedding_backward(dqgan_operator* op, int64_t tokens, const void* ids, const void* dy, int64_t dy_stride,
                             float* dtable, int64_t g_stride, int32_t accumulate) {
  if (int r = check(op, Kind::kEmbedding, "an embedding")) return r;
  const dqgan_embedding_config& c = op->embedding;
  if (tokens < 0 || tokens > c.max_tokens) return invalid(op, "tokens outside [0, max_tokens]");
  if (tokens == 0 && accumulate) return DQGAN_OK;
  if (!dtable) return invalid(op, "NULL dtable");
  if (tokens > 0) {
    if (!ids || !dy) return invalid(op, "NULL ids or dy");
    if (!stride_ok(dy_stride, c.width)) return invalid(op, "the row stride is below the width");
  }
  if (c.workers > 1 && !stride_ok(g_stride, c.vocab * c.width)) return invalid(op, "g_stride is below vocab * width");
  if (!aligned(ids, c.token_bits / 8) || !aligned(dy, dtype_size(c.dtype)) || !aligned(dtable, 4))
    return invalid(op, "a pointer is not aligned to its element");
  NvtxRange range("dqgan embedding backward");
  dq::EmbeddingArgs a{};
  a.ids = ids;
  a.dy = dy;
  a.ld = dy_stride;
  a.dtable = dtable;
  a.g_stride = c.workers > 1 ? g_stride : 0;
  a.scratch = op->scratch;
  a.tokens = tokens;
  a.vocab = c.vocab;
  a.width = c.width;
  a.workers = c.workers;
  a.dtype = c.dtype;
  a.token_bits = c.token_bits;
  a.scale = c.scale;
  a.accumulate = accumulate != 0;
  return launched(op, dq::launch_embedding_backward(a, op->stream, &op->launches), "embedding backward");
}

}  // extern "C"

namespace {

// What the three distillation calls share: checks, and the argument block.
int distillation(dqgan_operator* op, dq::DistillationWay way, int64_t rows, const void* logits, int64_t logits_stride,
                 const int32_t* ids, const void* values, int64_t teacher_stride, const float* teacher_lse,
                 const float* weights, float scale, float* loss, float* lse, void* dlogits, int64_t dlogits_stride) {
  using Way = dq::DistillationWay;
  if (int r = check(op, Kind::kDistillation, "a distillation")) return r;
  const dqgan_distillation_config& c = op->distillation;
  if (int r = check_rows(op, "rows", rows, 1)) return r;
  if (rows == 0) return DQGAN_OK;
  if (!logits || !ids || !values) return invalid(op, "NULL logits, ids or values");
  if (way != Way::kBackward && !loss) return invalid(op, "NULL loss");
  if (way == Way::kBackward && !lse) return invalid(op, "NULL lse");
  if (way != Way::kForward && !dlogits) return invalid(op, "NULL dlogits");
  if (!stride_ok(logits_stride, c.vocab) || (way != Way::kForward && !stride_ok(dlogits_stride, c.vocab)))
    return invalid(op, "a row stride is below the vocabulary");
  if (!stride_ok(teacher_stride, c.k)) return invalid(op, "teacher_stride is below k");
  if (!std::isfinite(scale)) return invalid(op, "scale is not finite");
  const uintptr_t size = dtype_size(c.dtype);
  if (!aligned(logits, size) || !aligned(dlogits, size) || !aligned(ids, 4) ||
      !aligned(values, dtype_size(c.teacher_dtype)) || !aligned(teacher_lse, 4) || !aligned(weights, 4) ||
      !aligned(loss, 4) || !aligned(lse, 4))
    return invalid(op, "a pointer is not aligned to its element");
  NvtxRange range(way == Way::kForward    ? "dqgan distillation forward"
                  : way == Way::kBackward ? "dqgan distillation backward"
                                          : "dqgan distillation step");
  dq::DistillationArgs a{};
  a.logits = logits;
  a.ld = logits_stride;
  a.dlogits = dlogits;
  a.dld = dlogits_stride;
  a.ids = ids;
  a.values = values;
  a.teacher_ld = teacher_stride;
  a.teacher_lse = teacher_lse;
  a.weights = weights;
  a.loss = loss;
  a.lse = lse;
  a.rows = rows;
  a.vocab = c.vocab;
  a.k = c.k;
  a.dtype = c.dtype;
  a.teacher_dtype = c.teacher_dtype;
  a.temperature = c.temperature;
  a.scale = scale;
  return launched(op, dq::launch_distillation(a, way, op->stream, &op->launches), "distillation");
}

}  // namespace

extern "C" {

int dqgan_distillation_forward(dqgan_operator* op, int64_t rows, const void* logits, int64_t logits_stride,
                               const int32_t* ids, const void* values, int64_t teacher_stride,
                               const float* teacher_lse, const float* weights, float* loss, float* lse) {
  return distillation(op, dq::DistillationWay::kForward, rows, logits, logits_stride, ids, values, teacher_stride,
                      teacher_lse, weights, 0.f, loss, lse, nullptr, 0);
}

int dqgan_distillation_backward(dqgan_operator* op, int64_t rows, const void* logits, int64_t logits_stride,
                                const float* lse, const int32_t* ids, const void* values, int64_t teacher_stride,
                                const float* teacher_lse, const float* weights, float scale, void* dlogits,
                                int64_t dlogits_stride) {
  return distillation(op, dq::DistillationWay::kBackward, rows, logits, logits_stride, ids, values, teacher_stride,
                      teacher_lse, weights, scale, nullptr, const_cast<float*>(lse), dlogits, dlogits_stride);
}

int dqgan_distillation_step(dqgan_operator* op, int64_t rows, const void* logits, int64_t logits_stride,
                            const int32_t* ids, const void* values, int64_t teacher_stride, const float* teacher_lse,
                            const float* weights, float scale, float* loss, float* lse, void* dlogits,
                            int64_t dlogits_stride) {
  return distillation(op, dq::DistillationWay::kStep, rows, logits, logits_stride, ids, values, teacher_stride,
                      teacher_lse, weights, scale, loss, lse, dlogits, dlogits_stride);
}

}  // extern "C"
