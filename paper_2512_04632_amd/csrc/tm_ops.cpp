// C entry points of the operators beside the orthogonalizer: argument checks,
// workspace layout and launches.  Nothing is enqueued for a refused call, and
// no exception leaves an entry point.
#include <new>
#include <string>

#include "tm_ops.h"

namespace {

using tmk::fail_with;

tm_status refuse(tm_status s, const std::string& msg) { return fail_with(s, msg.c_str()); }

bool misaligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

tm_status check_dtype(const char* name, int dtype) {
  if (dtype != TM_DTYPE_BF16 && dtype != TM_DTYPE_F32)
    return refuse(TM_ERR_INVALID_ARG, std::string(name) + " " + std::to_string(dtype) + " is neither TM_DTYPE_BF16 nor TM_DTYPE_F32");
  return TM_OK;
}

size_t size_of(int dtype) { return dtype == TM_DTYPE_BF16 ? 2u : 4u; }

tm_status check_range(const char* name, int64_t v, int64_t lo, int64_t hi) {
  if (v < lo || v > hi)
    return refuse(TM_ERR_INVALID_ARG, std::string(name) + " " + std::to_string(v) + " out of range [" +
                                          std::to_string(lo) + ", " + std::to_string(hi) + "]");
  return TM_OK;
}

// A device array that a call needs: there, aligned to its elements.
struct Ptr {
  const char* name;
  const void* p;
  size_t align;
  bool optional;
};
// Rows of `width` elements with a stride.
struct Stride {
  const char* name;
  int64_t ld, width;
};

template <size_t N>
tm_status check_pointers(const Ptr (&ps)[N]) {
  for (const Ptr& q : ps) {
    if (q.p == nullptr && !q.optional) return refuse(TM_ERR_INVALID_ARG, std::string(q.name) + " is NULL");
    if (misaligned(q.p, q.align))
      return refuse(TM_ERR_UNSUPPORTED, std::string(q.name) + " is not aligned to its elements");
  }
  return TM_OK;
}

constexpr int64_t kMaxStride = int64_t(1) << 40;

template <size_t N>
tm_status check_strides(const Stride (&ss)[N]) {
  for (const Stride& s : ss)
    if (s.ld < s.width || s.ld > kMaxStride)
      return refuse(TM_ERR_INVALID_ARG, std::string(s.name) + " " + std::to_string(s.ld) + " out of range [" +
                                            std::to_string(s.width) + ", 2^40]");
  return TM_OK;
}

#define TM_CHECK(call)                 \
  do {                                 \
    const tm_status s_ = (call);       \
    if (s_ != TM_OK) return s_;        \
  } while (0)

template <class F>
struct EnqueueFn : tmk::Enqueue {
  F f;
  explicit EnqueueFn(F g) : f(g) {}
  hipError_t operator()(char* ws, hipStream_t st) const override { return f(ws, st); }
};

template <class F>
tm_status run_op(int phase, size_t bytes, void* stream, F f) {
  return tmk::run_op(phase, bytes, static_cast<hipStream_t>(stream), EnqueueFn<F>(f));
}

// Runs an entry point's body; what it throws (memory for a message) becomes a status.
template <class F>
tm_status guarded(F body) noexcept {
  try {
    tmk::clear_error();
    return body();
  } catch (const std::bad_alloc&) {
    return TM_ERR_NO_MEMORY;
  } catch (...) {
    return TM_ERR_HIP;
  }
}

tm_status layer_norm(const void* x, int64_t ldx, const float* weight, const float* bias, void* y, int64_t ldy,
                     float* mean, float* rstd, int64_t rows, int64_t d, float eps, int dtype, void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_range("rows", rows, 0, TM_MAX_ROWS));
  TM_CHECK(check_range("d", d, 1, TM_MAX_DIM));
  if (!(eps >= 0.f)) return refuse(TM_ERR_INVALID_ARG, "eps must not be negative");
  if (rows == 0) return TM_OK;
  const size_t esz = size_of(dtype);
  TM_CHECK(check_strides({{"ldx", ldx, d}, {"ldy", ldy, d}}));
  TM_CHECK(check_pointers({{"x", x, esz, false}, {"weight", weight, 4, true}, {"bias", bias, 4, true},
                           {"y", y, esz, false}, {"mean", mean, 4, false}, {"rstd", rstd, 4, false}}));
  tmk::NormArgs A{};
  A.x = static_cast<const char*>(x);
  A.out = static_cast<char*>(y);
  A.weight = weight;
  A.bias = bias;
  A.mean = mean;
  A.rstd = rstd;
  A.ldx = ldx;
  A.ldo = ldy;
  A.rows = int32_t(rows);
  A.d = int32_t(d);
  A.eps = eps;
  return run_op(TM_PHASE_LAYER_NORM, 0, stream,
                [&](char*, hipStream_t st) { return tmk::launch_norm(A, dtype == TM_DTYPE_F32, st); });
}

tm_status layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* weight,
                              const float* mean, const float* rstd, void* dx, int64_t lddx, float* dweight,
                              float* dbias, int64_t rows, int64_t d, int dtype, void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_range("rows", rows, 0, TM_MAX_ROWS));
  TM_CHECK(check_range("d", d, 1, TM_MAX_DIM));
  const size_t esz = size_of(dtype);
  const bool empty = rows == 0;
  if (empty && dweight == nullptr && dbias == nullptr) return TM_OK;
  if (!empty) TM_CHECK(check_strides({{"lddy", lddy, d}, {"ldx", ldx, d}, {"lddx", lddx, d}}));
  TM_CHECK(check_pointers({{"dy", dy, esz, empty}, {"x", x, esz, empty}, {"weight", weight, 4, true},
                           {"mean", mean, 4, empty}, {"rstd", rstd, 4, empty}, {"dx", dx, esz, empty},
                           {"dweight", dweight, 4, true}, {"dbias", dbias, 4, true}}));
  tmk::NormArgs A{};
  A.x = static_cast<const char*>(x);
  A.dy = static_cast<const char*>(dy);
  A.out = static_cast<char*>(dx);
  A.weight = weight;
  A.mean = const_cast<float*>(mean);
  A.rstd = const_cast<float*>(rstd);
  A.ldx = ldx;
  A.lddy = lddy;
  A.ldo = lddx;
  A.rows = int32_t(rows);
  A.d = int32_t(d);
  A.dweight = dweight;
  A.dbias = dbias;
  const int blocks = tmk::norm_blocks(rows, d, dtype == TM_DTYPE_F32);
  const bool params = (dweight != nullptr || dbias != nullptr) && (blocks != 1 || d > tmk::kNormMaxFused);
  const size_t bytes = params ? size_t(blocks) * 2u * size_t(d) * 4u : 0u;
  return run_op(TM_PHASE_LAYER_NORM_BACKWARD, bytes, stream, [&](char* ws, hipStream_t st) {
    A.part = params ? reinterpret_cast<float*>(ws) : nullptr;
    hipError_t e = hipSuccess;
    if (!empty) e = tmk::launch_norm_backward(A, dtype == TM_DTYPE_F32, blocks, st);
    if (e == hipSuccess && params) e = tmk::launch_norm_params(A.part, blocks, A.d, dweight, dbias, st);
    return e;
  });
}

tm_status check_expert_sizes(int64_t rows, int64_t experts, int64_t k, int64_t n) {
  TM_CHECK(check_range("rows", rows, 0, TM_MAX_ROWS));
  TM_CHECK(check_range("experts", experts, 1, TM_MAX_EXPERTS));
  TM_CHECK(check_range("k", k, 1, TM_MAX_DIM));
  return check_range("n", n, 1, TM_MAX_DIM);
}

tm_status expert_matmul(const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t stride_w,
                        const int32_t* ends, void* y, int64_t ldy, int64_t rows, int64_t experts, int64_t k,
                        int64_t n, int transposed, int dtype, void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_expert_sizes(rows, experts, k, n));
  if (rows == 0) return TM_OK;
  const size_t esz = size_of(dtype);
  const int64_t wrows = transposed ? n : k, wcols = transposed ? k : n;
  TM_CHECK(check_strides({{"ldx", ldx, k}, {"ldw", ldw, wcols}, {"ldy", ldy, n}}));
  if (stride_w < 0 || stride_w > kMaxStride || (experts > 1 && stride_w < (wrows - 1) * ldw + wcols))
    return refuse(TM_ERR_INVALID_ARG, "stride_w " + std::to_string(stride_w) + " is less than a matrix or over 2^40");
  TM_CHECK(check_pointers({{"x", x, esz, false}, {"w", w, esz, false}, {"ends", ends, 4, false}, {"y", y, esz, false}}));
  tmk::ExpertArgs A{};
  A.a = static_cast<const char*>(x);
  A.b = static_cast<const char*>(w);
  A.out = static_cast<char*>(y);
  A.ends = ends;
  A.lda = ldx;
  A.ldb = ldw;
  A.ldo = ldy;
  A.stride_b = stride_w;
  A.rows = int32_t(rows);
  A.experts = int32_t(experts);
  A.k = int32_t(k);
  A.n = int32_t(n);
  const bool f32 = dtype == TM_DTYPE_F32, trans = transposed != 0;
  const tmk::ExpertPlan P = tmk::plan_expert_matmul(A, f32, trans);
  return run_op(TM_PHASE_EXPERT_MATMUL, size_t(P.bytes), stream,
                [&](char* ws, hipStream_t st) { return tmk::launch_expert_matmul(A, P, f32, trans, ws, st); });
}

tm_status expert_wgrad(const void* x, int64_t ldx, const void* dy, int64_t lddy, const int32_t* ends, void* dw,
                       int64_t lddw, int64_t stride_dw, int64_t rows, int64_t experts, int64_t k, int64_t n,
                       int dtype, int out_dtype, void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_dtype("out_dtype", out_dtype));
  if (dtype == TM_DTYPE_F32 && out_dtype != TM_DTYPE_F32)
    return refuse(TM_ERR_UNSUPPORTED, "the product of fp32 rows is fp32");
  TM_CHECK(check_expert_sizes(rows, experts, k, n));
  const size_t esz = size_of(dtype);
  const bool empty = rows == 0;
  if (!empty) TM_CHECK(check_strides({{"ldx", ldx, k}, {"lddy", lddy, n}}));
  TM_CHECK(check_strides({{"lddw", lddw, n}}));
  if (stride_dw < 0 || stride_dw > kMaxStride || (experts > 1 && stride_dw < (k - 1) * lddw + n))
    return refuse(TM_ERR_INVALID_ARG, "stride_dw " + std::to_string(stride_dw) + " is less than a matrix or over 2^40");
  TM_CHECK(check_pointers({{"x", x, esz, empty}, {"dy", dy, esz, empty}, {"ends", ends, 4, false},
                           {"dw", dw, size_of(out_dtype), false}}));
  tmk::ExpertArgs A{};
  A.a = static_cast<const char*>(x);
  A.b = static_cast<const char*>(dy);
  A.out = static_cast<char*>(dw);
  A.ends = ends;
  A.lda = ldx;
  A.ldb = lddy;
  A.ldo = lddw;
  A.stride_b = stride_dw;
  A.rows = int32_t(rows);
  A.experts = int32_t(experts);
  A.k = int32_t(k);
  A.n = int32_t(n);
  const bool f32 = dtype == TM_DTYPE_F32, out_f32 = out_dtype == TM_DTYPE_F32;
  const tmk::ExpertPlan P = tmk::plan_expert_wgrad(A, f32);
  return run_op(TM_PHASE_EXPERT_WGRAD, size_t(P.bytes), stream,
                [&](char* ws, hipStream_t st) { return tmk::launch_expert_wgrad(A, P, f32, out_f32, ws, st); });
}

tm_status check_temperature(float t) {
  const float inv = 1.f / t;
  if (!(t > 0.f) || !(inv > 0.f) || !(inv <= 3.0e38f))
    return refuse(TM_ERR_INVALID_ARG, "temperature must be positive, and so must be its inverse in fp32");
  return TM_OK;
}

tm_status check_blocks(int64_t rows, int64_t chunks, uint64_t threads) {
  if (!tmk::launchable(uint64_t(rows) * uint64_t(chunks), threads))
    return refuse(TM_ERR_UNSUPPORTED, "too many blocks in one launch");
  return TM_OK;
}

// Length of a chunk: whole 16-byte vectors of either type.
int64_t chunk_length(int64_t vocab, int64_t chunks) { return ((vocab + chunks - 1) / chunks + 7) / 8 * 8; }

// A workgroup of the elementwise gradient takes this many bytes of a row: 3000 x
// 32001 fp32 109 us, 129 with half, 121 with four times as many; 8192 x 131072 bf16 539,
// 623 with half, 595 with twice as many.
constexpr int64_t kGradBytes = 8192;

tm_status policy_loss(const void* logits, int64_t ld, const int64_t* targets, const float* old_logp,
                      const float* advantages, const float* weights, const float* ref_logp, float clip_low,
                      float clip_high, float kl, float temperature, float* loss, float* logp, float* lse,
                      float* slope, void* dlogits, int64_t ldd, int64_t rows, int64_t vocab, int dtype,
                      void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_range("rows", rows, 0, TM_MAX_ROWS));
  TM_CHECK(check_range("vocab", vocab, 1, TM_MAX_VOCAB));
  TM_CHECK(check_temperature(temperature));
  if (!(clip_low >= 0.f && clip_low <= 1.f) || !(clip_high >= 0.f) || !(kl >= 0.f))
    return refuse(TM_ERR_INVALID_ARG, "need 0 <= clip_low <= 1, clip_high >= 0 and kl >= 0");
  const size_t esz = size_of(dtype);
  const bool empty = rows == 0, grad = dlogits != nullptr;
  if (!empty) TM_CHECK(check_strides({{"ld", ld, vocab}}));
  if (!empty && grad) TM_CHECK(check_strides({{"ld_dlogits", ldd, vocab}}));
  TM_CHECK(check_pointers({{"logits", logits, esz, empty}, {"targets", targets, 8, empty},
                           {"old_logp", old_logp, 4, empty}, {"advantages", advantages, 4, empty},
                           {"weights", weights, 4, empty}, {"ref_logp", ref_logp, 4, true},
                           {"loss", loss, 4, false}, {"logp", logp, 4, empty}, {"lse", lse, 4, true},
                           {"slope", slope, 4, true}, {"dlogits", dlogits, esz, true}}));
  tmk::LossArgs A{};
  A.logits = static_cast<const char*>(logits);
  A.targets = targets;
  A.old_logp = old_logp;
  A.advantages = advantages;
  A.weights = weights;
  A.ref_logp = ref_logp;
  A.loss = loss;
  A.logp = logp;
  A.dlogits = static_cast<char*>(dlogits);
  A.ld = ld;
  A.ldd = ldd;
  A.rows = int32_t(rows);
  A.vocab = int32_t(vocab);
  A.clip_low = clip_low;
  A.clip_high = clip_high;
  A.kl = kl;
  A.inv_temp = 1.f / temperature;
  const int64_t chunks = empty ? 1 : tmk::loss_chunks(rows, vocab);
  // threads of a row at most (launch_rows)
  const int64_t line_bytes = vocab * int64_t(esz);
  TM_CHECK(check_blocks(rows, chunks, line_bytes <= 4096 ? 64 : line_bytes <= 48 * 1024 ? 256 : 1024));
  A.chunks = int32_t(chunks);
  A.chunk = int32_t(chunk_length(vocab, chunks));
  // workspace: the rows' shares of the loss, lse and slope where the caller
  // keeps none, the chunks' maxima and sums, and those of their rows
  const size_t line = size_t(tmk::align256(uint64_t(rows) * 4u));
  const size_t bytes = 3u * line + (chunks > 1 ? size_t(rows) * size_t(chunks + 1) * sizeof(float2) : 0u) + 256u;
  return run_op(TM_PHASE_POLICY_LOSS, bytes, stream, [&](char* ws, hipStream_t st) {
    A.row_loss = reinterpret_cast<float*>(ws);
    A.lse = lse != nullptr ? lse : reinterpret_cast<float*>(ws + line);
    A.slope = slope != nullptr ? slope : reinterpret_cast<float*>(ws + 2u * line);
    A.part = reinterpret_cast<float2*>(ws + 3u * line);
    A.stats = A.part + rows * chunks;
    return tmk::launch_loss(A, dtype == TM_DTYPE_F32, st);
  });
}

tm_status policy_loss_backward(const void* logits, int64_t ld, const int64_t* targets, const float* lse,
                               const float* slope, const float* grad, float temperature, void* dlogits,
                               int64_t ldd, int64_t rows, int64_t vocab, int dtype, void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_range("rows", rows, 0, TM_MAX_ROWS));
  TM_CHECK(check_range("vocab", vocab, 1, TM_MAX_VOCAB));
  TM_CHECK(check_temperature(temperature));
  if (rows == 0) return TM_OK;
  const size_t esz = size_of(dtype);
  TM_CHECK(check_strides({{"ld", ld, vocab}, {"ld_dlogits", ldd, vocab}}));
  TM_CHECK(check_pointers({{"logits", logits, esz, false}, {"targets", targets, 8, false}, {"lse", lse, 4, false},
                           {"slope", slope, 4, false}, {"grad", grad, 4, true}, {"dlogits", dlogits, esz, false}}));
  tmk::LossArgs A{};
  A.logits = static_cast<const char*>(logits);
  A.targets = targets;
  A.grad = grad;
  A.lse = const_cast<float*>(lse);
  A.slope = const_cast<float*>(slope);
  A.dlogits = static_cast<char*>(dlogits);
  A.ld = ld;
  A.ldd = ldd;
  A.rows = int32_t(rows);
  A.vocab = int32_t(vocab);
  A.inv_temp = 1.f / temperature;
  const int64_t chunks = (vocab * int64_t(esz) + kGradBytes - 1) / kGradBytes;
  TM_CHECK(check_blocks(rows, chunks, 256));
  A.chunks = int32_t(chunks);
  A.chunk = int32_t(chunk_length(vocab, chunks));
  return run_op(TM_PHASE_POLICY_LOSS_BACKWARD, 0, stream,
                [&](char*, hipStream_t st) { return tmk::launch_loss_backward(A, dtype == TM_DTYPE_F32, st); });
}

}  // namespace

extern "C" {

tm_status tm_layer_norm(const void* x, int64_t ldx, const float* weight, const float* bias, void* y, int64_t ldy,
                        float* mean, float* rstd, int64_t rows, int64_t d, float eps, int dtype, void* stream) {
  return guarded([&] { return layer_norm(x, ldx, weight, bias, y, ldy, mean, rstd, rows, d, eps, dtype, stream); });
}

tm_status tm_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* weight,
                                 const float* mean, const float* rstd, void* dx, int64_t lddx, float* dweight,
                                 float* dbias, int64_t rows, int64_t d, int dtype, void* stream) {
  return guarded([&] {
    return layer_norm_backward(dy, lddy, x, ldx, weight, mean, rstd, dx, lddx, dweight, dbias, rows, d, dtype, stream);
  });
}

tm_status tm_expert_matmul(const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t stride_w,
                           const int32_t* ends, void* y, int64_t ldy, int64_t rows, int64_t experts, int64_t k,
                           int64_t n, int transposed, int dtype, void* stream) {
  return guarded([&] {
    return expert_matmul(x, ldx, w, ldw, stride_w, ends, y, ldy, rows, experts, k, n, transposed, dtype, stream);
  });
}

tm_status tm_expert_wgrad(const void* x, int64_t ldx, const void* dy, int64_t lddy, const int32_t* ends, void* dw,
                          int64_t lddw, int64_t stride_dw, int64_t rows, int64_t experts, int64_t k, int64_t n,
                          int dtype, int out_dtype, void* stream) {
  return guarded([&] {
    return expert_wgrad(x, ldx, dy, lddy, ends, dw, lddw, stride_dw, rows, experts, k, n, dtype, out_dtype, stream);
  });
}

tm_status tm_policy_loss(const void* logits, int64_t ld, const int64_t* targets, const float* old_logp,
                         const float* advantages, const float* weights, const float* ref_logp, float clip_low,
                         float clip_high, float kl, float temperature, float* loss, float* logp, float* lse,
                         float* slope, void* dlogits, int64_t ld_dlogits, int64_t rows, int64_t vocab, int dtype,
                         void* stream) {
  return guarded([&] {
    return policy_loss(logits, ld, targets, old_logp, advantages, weights, ref_logp, clip_low, clip_high, kl,
                       temperature, loss, logp, lse, slope, dlogits, ld_dlogits, rows, vocab, dtype, stream);
  });
}

tm_status tm_policy_loss_backward(const void* logits, int64_t ld, const int64_t* targets, const float* lse,
                                  const float* slope, const float* grad, float temperature, void* dlogits,
                                  int64_t ld_dlogits, int64_t rows, int64_t vocab, int dtype, void* stream) {
  return guarded([&] {
    return policy_loss_backward(logits, ld, targets, lse, slope, grad, temperature, dlogits, ld_dlogits, rows,
                                vocab, dtype, stream);
  });
}

}  // extern "C"
