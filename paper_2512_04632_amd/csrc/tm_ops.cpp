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
    if (e == hipSuccess && params) e = tmk::launch_norm_params(A.part, blocks, 2, A.d, dweight, dbias, st);
    return e;
  });
}

tm_status rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* weight, void* sum,
                   int64_t lds, void* y, int64_t ldy, float* rstd, int64_t rows, int64_t d, float eps, int dtype,
                   void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_range("rows", rows, 0, TM_MAX_ROWS));
  TM_CHECK(check_range("d", d, 1, TM_MAX_DIM));
  if (!(eps >= 0.f)) return refuse(TM_ERR_INVALID_ARG, "eps must not be negative");
  if (rows == 0) return TM_OK;
  const size_t esz = size_of(dtype);
  const bool res = residual != nullptr;
  TM_CHECK(check_strides({{"ldx", ldx, d}, {"ldy", ldy, d}}));
  if (res) TM_CHECK(check_strides({{"ldr", ldr, d}, {"lds", lds, d}}));
  TM_CHECK(check_pointers({{"x", x, esz, false}, {"residual", residual, esz, true}, {"weight", weight, 4, true},
                           {"sum", sum, esz, !res}, {"y", y, esz, false}, {"rstd", rstd, 4, false}}));
  if (res && sum == y) return refuse(TM_ERR_INVALID_ARG, "sum and y are the same array");
  tmk::RmsArgs A{};
  A.x = static_cast<const char*>(x);
  A.residual = static_cast<const char*>(residual);
  A.sum = static_cast<char*>(sum);
  A.out = static_cast<char*>(y);
  A.weight = weight;
  A.rstd = rstd;
  A.ldx = ldx;
  A.ldr = ldr;
  A.lds = lds;
  A.ldo = ldy;
  A.rows = int32_t(rows);
  A.d = int32_t(d);
  A.eps = eps;
  return run_op(TM_PHASE_RMS_NORM, 0, stream,
                [&](char*, hipStream_t st) { return tmk::launch_rms(A, dtype == TM_DTYPE_F32, st); });
}

tm_status rms_norm_backward(const void* dy, int64_t lddy, const void* s, int64_t lds, const float* weight,
                            const float* rstd, const void* dsum, int64_t lddsum, void* ds, int64_t ldds,
                            float* dweight, int64_t rows, int64_t d, int dtype, void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_range("rows", rows, 0, TM_MAX_ROWS));
  TM_CHECK(check_range("d", d, 1, TM_MAX_DIM));
  const size_t esz = size_of(dtype);
  const bool empty = rows == 0;
  if (empty && dweight == nullptr) return TM_OK;
  if (!empty) TM_CHECK(check_strides({{"lddy", lddy, d}, {"lds", lds, d}, {"ldds", ldds, d}}));
  if (!empty && dsum != nullptr) TM_CHECK(check_strides({{"lddsum", lddsum, d}}));
  TM_CHECK(check_pointers({{"dy", dy, esz, empty}, {"s", s, esz, empty}, {"weight", weight, 4, true},
                           {"rstd", rstd, 4, empty}, {"dsum", dsum, esz, true}, {"ds", ds, esz, empty},
                           {"dweight", dweight, 4, true}}));
  tmk::RmsArgs A{};
  A.x = static_cast<const char*>(s);
  A.residual = static_cast<const char*>(dsum);
  A.dy = static_cast<const char*>(dy);
  A.out = static_cast<char*>(ds);
  A.weight = weight;
  A.rstd = const_cast<float*>(rstd);
  A.ldx = lds;
  A.ldr = lddsum;
  A.lddy = lddy;
  A.ldo = ldds;
  A.rows = int32_t(rows);
  A.d = int32_t(d);
  A.dweight = dweight;
  const int blocks = tmk::rms_backward_blocks(rows, d, dtype == TM_DTYPE_F32);
  const bool params = dweight != nullptr && (blocks != 1 || d > tmk::kNormMaxFused);
  const size_t bytes = params ? size_t(blocks) * size_t(d) * 4u : 0u;
  return run_op(TM_PHASE_RMS_NORM_BACKWARD, bytes, stream, [&](char* ws, hipStream_t st) {
    A.part = params ? reinterpret_cast<float*>(ws) : nullptr;
    hipError_t e = hipSuccess;
    if (!empty) e = tmk::launch_rms_backward(A, dtype == TM_DTYPE_F32, blocks, st);
    if (e == hipSuccess && params) e = tmk::launch_norm_params(A.part, blocks, 1, A.d, dweight, nullptr, st);
    return e;
  });
}

tm_status check_route_sizes(int64_t rows, int64_t experts, int64_t top, float scale) {
  TM_CHECK(check_range("rows", rows, 0, TM_MAX_ROWS));
  TM_CHECK(check_range("experts", experts, 1, TM_MAX_EXPERTS));
  TM_CHECK(check_range("top", top, 1, experts < TM_MAX_TOP ? experts : TM_MAX_TOP));
  TM_CHECK(check_range("rows top", rows * top, 0, TM_MAX_ROWS));
  if (!(scale - scale == 0.f)) return refuse(TM_ERR_INVALID_ARG, "scale must be finite");
  return TM_OK;
}

tm_status expert_route(const void* logits, int64_t ld, const uint8_t* active, int renormalize, float scale,
                       int32_t* chosen, float* weights, int32_t* slots, int32_t* ends, float* balance,
                       int64_t rows, int64_t experts, int64_t top, int dtype, void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_route_sizes(rows, experts, top, scale));
  const size_t esz = size_of(dtype);
  const bool empty = rows == 0;
  if (!empty) TM_CHECK(check_strides({{"ld", ld, experts}}));
  TM_CHECK(check_pointers({{"logits", logits, esz, empty}, {"chosen", chosen, 4, empty}, {"weights", weights, 4, empty},
                           {"slots", slots, 4, empty}, {"ends", ends, 4, false}, {"balance", balance, 4, false}}));
  tmk::RouteArgs A{};
  A.logits = static_cast<const char*>(logits);
  A.active = active;
  A.chosen = chosen;
  A.weights = weights;
  A.slots = slots;
  A.ends = ends;
  A.balance = balance;
  A.ld = ld;
  A.rows = int32_t(rows);
  A.experts = int32_t(experts);
  A.top = int32_t(top);
  A.renormalize = renormalize != 0;
  A.scale = scale;
  tmk::plan_route(A);
  // workspace: the blocks' counts and sums of probabilities, lines of whole vectors; none for a single block
  const uint64_t entries = uint64_t(A.blocks) * ((uint64_t(experts) + 7u) / 8u * 8u);
  const uint64_t dots = 256u + tmk::align256(uint64_t(A.blocks) * sizeof(double)), counts = tmk::align256(entries * sizeof(uint16_t));
  const uint64_t bytes = A.blocks > 1 ? dots + counts + entries * sizeof(float) : 0u;
  return run_op(TM_PHASE_EXPERT_ROUTE, size_t(bytes), stream, [&](char* ws, hipStream_t st) {
    A.arrived = reinterpret_cast<int32_t*>(ws);
    A.dots = reinterpret_cast<double*>(ws + 256u);
    A.counts = reinterpret_cast<uint16_t*>(ws + dots);
    A.shares = reinterpret_cast<float*>(ws + dots + counts);
    return tmk::launch_route(A, dtype == TM_DTYPE_F32, st);
  });
}

tm_status expert_route_backward(const void* logits, int64_t ld, const int32_t* chosen, const int32_t* ends,
                                const float* dweights, const float* dbalance, int renormalize, float scale,
                                void* dlogits, int64_t ldd, int64_t rows, int64_t experts, int64_t top, int dtype,
                                void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_route_sizes(rows, experts, top, scale));
  if (rows == 0) return TM_OK;
  const size_t esz = size_of(dtype);
  TM_CHECK(check_strides({{"ld", ld, experts}, {"ldd", ldd, experts}}));
  TM_CHECK(check_pointers({{"logits", logits, esz, false}, {"chosen", chosen, 4, false}, {"ends", ends, 4, false},
                           {"dweights", dweights, 4, true}, {"dbalance", dbalance, 4, true},
                           {"dlogits", dlogits, esz, false}}));
  tmk::RouteGradArgs A{};
  A.logits = static_cast<const char*>(logits);
  A.chosen = chosen;
  A.ends = ends;
  A.dweights = dweights;
  A.dbalance = dbalance;
  A.dlogits = static_cast<char*>(dlogits);
  A.ld = ld;
  A.ldd = ldd;
  A.rows = int32_t(rows);
  A.experts = int32_t(experts);
  A.top = int32_t(top);
  A.renormalize = renormalize != 0;
  A.scale = scale;
  return run_op(TM_PHASE_EXPERT_ROUTE_BACKWARD, 0, stream,
                [&](char*, hipStream_t st) { return tmk::launch_route_backward(A, dtype == TM_DTYPE_F32, st); });
}

tm_status check_rows_sizes(int64_t count, int64_t rows, int64_t top, int64_t d) {
  TM_CHECK(check_range("count", count, 0, TM_MAX_ROWS));
  TM_CHECK(check_range("rows", rows, 0, TM_MAX_ROWS));
  TM_CHECK(check_range("top", top, 1, TM_MAX_TOP));
  return check_range("d", d, 1, TM_MAX_DIM);
}

tmk::RowsArgs rows_args(const int32_t* slots, int64_t count, int64_t rows, int64_t top, int64_t d) {
  tmk::RowsArgs A{};
  A.slots = slots;
  A.count = count;
  A.rows = int32_t(rows);
  A.top = int32_t(top);
  A.d = int32_t(d);
  return A;
}

tm_status expert_gather(const void* x, int64_t ldx, const int32_t* slots, const int32_t* used, void* out,
                        int64_t ldo, int64_t count, int64_t rows, int64_t top, int64_t d, int dtype, void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_rows_sizes(count, rows, top, d));
  if (count == 0) return TM_OK;
  const size_t esz = size_of(dtype);
  const bool empty = rows == 0;
  if (!empty) TM_CHECK(check_strides({{"ldx", ldx, d}}));
  TM_CHECK(check_strides({{"ldo", ldo, d}}));
  TM_CHECK(check_pointers({{"x", x, esz, empty}, {"slots", slots, 4, empty}, {"used", used, 4, true}, {"out", out, esz, false}}));
  tmk::RowsArgs A = rows_args(slots, count, rows, top, d);
  A.x = static_cast<const char*>(x);
  A.used = used;
  A.out = static_cast<char*>(out);
  A.ldx = ldx;
  A.ldo = ldo;
  return run_op(TM_PHASE_EXPERT_GATHER, 0, stream,
                [&](char*, hipStream_t st) { return tmk::launch_gather(A, dtype == TM_DTYPE_F32, st); });
}

tm_status expert_combine(const void* y, int64_t ldy, const int32_t* slots, const int32_t* used, const float* weights,
                         const void* residual, int64_t ldr, void* out, int64_t ldo, int64_t count, int64_t rows,
                         int64_t top, int64_t d, int dtype, void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_rows_sizes(count, rows, top, d));
  if (rows == 0) return TM_OK;
  const size_t esz = size_of(dtype);
  if (count > 0) TM_CHECK(check_strides({{"ldy", ldy, d}}));
  TM_CHECK(check_strides({{"ldo", ldo, d}}));
  if (residual != nullptr) TM_CHECK(check_strides({{"ldr", ldr, d}}));
  TM_CHECK(check_pointers({{"y", y, esz, count == 0}, {"slots", slots, 4, false}, {"used", used, 4, true},
                           {"weights", weights, 4, true}, {"residual", residual, esz, true}, {"out", out, esz, false}}));
  tmk::RowsArgs A = rows_args(slots, count, rows, top, d);
  A.used = used;
  A.x = static_cast<const char*>(residual);
  A.y = static_cast<const char*>(y);
  A.weights = weights;
  A.out = static_cast<char*>(out);
  A.ldx = ldr;
  A.ldy = ldy;
  A.ldo = ldo;
  return run_op(TM_PHASE_EXPERT_COMBINE, 0, stream,
                [&](char*, hipStream_t st) { return tmk::launch_combine(A, dtype == TM_DTYPE_F32, st); });
}

tm_status expert_combine_backward(const void* dout, int64_t lddout, const void* y, int64_t ldy, const int32_t* slots,
                                  const int32_t* used, const float* weights, void* dy, int64_t lddy, float* dweights,
                                  int64_t count, int64_t rows, int64_t top, int64_t d, int dtype, void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_rows_sizes(count, rows, top, d));
  const size_t esz = size_of(dtype);
  const bool empty = rows == 0, reads = !empty && count > 0 && dweights != nullptr;
  if (count == 0 && (empty || dweights == nullptr)) return TM_OK;
  if (!empty) TM_CHECK(check_strides({{"lddout", lddout, d}}));
  if (reads) TM_CHECK(check_strides({{"ldy", ldy, d}}));
  if (count > 0) TM_CHECK(check_strides({{"lddy", lddy, d}}));
  TM_CHECK(check_pointers({{"dout", dout, esz, empty}, {"y", y, esz, !reads}, {"slots", slots, 4, empty},
                           {"used", used, 4, true}, {"weights", weights, 4, true}, {"dy", dy, esz, count == 0},
                           {"dweights", dweights, 4, true}}));
  tmk::RowsArgs A = rows_args(slots, count, rows, top, d);
  A.x = static_cast<const char*>(dout);
  A.y = static_cast<const char*>(y);
  A.used = used;
  A.weights = weights;
  A.out = static_cast<char*>(dy);
  A.dweights = dweights;
  A.ldx = lddout;
  A.ldy = ldy;
  A.ldo = lddy;
  return run_op(TM_PHASE_EXPERT_COMBINE_BACKWARD, 0, stream,
                [&](char*, hipStream_t st) { return tmk::launch_combine_backward(A, dtype == TM_DTYPE_F32, st); });
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

// Rows of a wave each, four to a workgroup, the last of which counts in full.
tm_status check_quads(int64_t rows) { return check_blocks((rows + 3) / 4, 1, 256); }

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
  // threads of a row at most (launch_rows); short ones go four to a workgroup
  const int64_t line_bytes = vocab * int64_t(esz);
  TM_CHECK(line_bytes <= 4096 ? check_quads(rows) : check_blocks(rows, chunks, line_bytes <= 48 * 1024 ? 256 : 1024));
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

// A temperature whose inverse stays finite as the factor of an exponent of 2.
tm_status check_exponent(float t) {
  TM_CHECK(check_temperature(t));
  if (!(1.f / t <= 2.0e38f)) return refuse(TM_ERR_INVALID_ARG, "temperature must be 5e-39 or more");
  return TM_OK;
}

tm_status token_logp(const void* logits, int64_t ld, const int64_t* targets, float temperature, float* logp,
                     float* entropy, float* stats, int64_t top, float* top_logp, int64_t* top_ids, int64_t rows,
                     int64_t vocab, int dtype, void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_range("rows", rows, 0, TM_MAX_ROWS));
  TM_CHECK(check_range("vocab", vocab, 1, TM_MAX_VOCAB));
  TM_CHECK(check_range("top", top, 0, vocab < TM_MAX_TOP ? vocab : TM_MAX_TOP));
  TM_CHECK(check_exponent(temperature));
  if (rows == 0) return TM_OK;
  const size_t esz = size_of(dtype);
  TM_CHECK(check_strides({{"ld", ld, vocab}}));
  TM_CHECK(check_pointers({{"logits", logits, esz, false}, {"targets", targets, 8, false}, {"logp", logp, 4, false},
                           {"entropy", entropy, 4, false}, {"stats", stats, 8, false},
                           {"top_logp", top_logp, 4, top == 0}, {"top_ids", top_ids, 8, top == 0}}));
  tmk::LogpArgs A{};
  A.logits = static_cast<const char*>(logits);
  A.targets = targets;
  A.logp = logp;
  A.entropy = entropy;
  A.stats = reinterpret_cast<float2*>(stats);
  A.top_logp = top_logp;
  A.top_ids = top_ids;
  A.ld = ld;
  A.rows = int32_t(rows);
  A.vocab = int32_t(vocab);
  A.top = int32_t(top);
  A.inv_temp = 1.f / temperature;
  tmk::plan_logp(A, dtype == TM_DTYPE_F32);
  const int threads = tmk::logp_threads(A, dtype == TM_DTYPE_F32);   // 0: a wave holds a row
  TM_CHECK(threads == 0 ? check_quads(rows) : check_blocks(rows, A.chunks, uint64_t(threads)));
  const uint64_t chunks = A.chunks > 1 ? uint64_t(rows) * uint64_t(A.chunks) : 0u;
  return run_op(TM_PHASE_TOKEN_LOGP, size_t(chunks * (sizeof(float4) + uint64_t(top) * 8u)), stream,
                [&](char* ws, hipStream_t st) {
                  A.part = reinterpret_cast<float4*>(ws);
                  A.keys = reinterpret_cast<uint64_t*>(ws + chunks * sizeof(float4));
                  return tmk::launch_logp(A, dtype == TM_DTYPE_F32, st);
                });
}

tm_status token_logp_backward(const void* logits, int64_t ld, const int64_t* targets, const float* stats,
                              const float* entropy, const float* dlogp, const float* dentropy, float temperature,
                              void* dlogits, int64_t ldd, int64_t rows, int64_t vocab, int dtype, void* stream) {
  TM_CHECK(check_dtype("dtype", dtype));
  TM_CHECK(check_range("rows", rows, 0, TM_MAX_ROWS));
  TM_CHECK(check_range("vocab", vocab, 1, TM_MAX_VOCAB));
  TM_CHECK(check_exponent(temperature));
  if (rows == 0) return TM_OK;
  const size_t esz = size_of(dtype);
  TM_CHECK(check_strides({{"ld", ld, vocab}, {"ld_dlogits", ldd, vocab}}));
  TM_CHECK(check_pointers({{"logits", logits, esz, false}, {"targets", targets, 8, false}, {"stats", stats, 8, false},
                           {"entropy", entropy, 4, false}, {"dlogp", dlogp, 4, true},
                           {"dentropy", dentropy, 4, true}, {"dlogits", dlogits, esz, false}}));
  tmk::LogpArgs A{};
  A.logits = static_cast<const char*>(logits);
  A.targets = targets;
  A.stats = reinterpret_cast<float2*>(const_cast<float*>(stats));
  A.entropy = const_cast<float*>(entropy);
  A.dlogp = dlogp;
  A.dentropy = dentropy;
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
  return run_op(TM_PHASE_TOKEN_LOGP_BACKWARD, 0, stream,
                [&](char*, hipStream_t st) { return tmk::launch_logp_backward(A, dtype == TM_DTYPE_F32, st); });
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

tm_status tm_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* weight,
                      void* sum, int64_t lds, void* y, int64_t ldy, float* rstd, int64_t rows, int64_t d,
                      float eps, int dtype, void* stream) {
  return guarded([&] {
    return rms_norm(x, ldx, residual, ldr, weight, sum, lds, y, ldy, rstd, rows, d, eps, dtype, stream);
  });
}

tm_status tm_rms_norm_backward(const void* dy, int64_t lddy, const void* s, int64_t lds, const float* weight,
                               const float* rstd, const void* dsum, int64_t lddsum, void* ds, int64_t ldds,
                               float* dweight, int64_t rows, int64_t d, int dtype, void* stream) {
  return guarded([&] {
    return rms_norm_backward(dy, lddy, s, lds, weight, rstd, dsum, lddsum, ds, ldds, dweight, rows, d, dtype,
                             stream);
  });
}

tm_status tm_expert_route(const void* logits, int64_t ld, const uint8_t* active, int renormalize, float scale,
                          int32_t* chosen, float* weights, int32_t* slots, int32_t* ends, float* balance,
                          int64_t rows, int64_t experts, int64_t top, int dtype, void* stream) {
  return guarded([&] {
    return expert_route(logits, ld, active, renormalize, scale, chosen, weights, slots, ends, balance, rows,
                        experts, top, dtype, stream);
  });
}

tm_status tm_expert_route_backward(const void* logits, int64_t ld, const int32_t* chosen, const int32_t* ends,
                                   const float* dweights, const float* dbalance, int renormalize, float scale,
                                   void* dlogits, int64_t ldd, int64_t rows, int64_t experts, int64_t top,
                                   int dtype, void* stream) {
  return guarded([&] {
    return expert_route_backward(logits, ld, chosen, ends, dweights, dbalance, renormalize, scale, dlogits,
                                 ldd, rows, experts, top, dtype, stream);
  });
}

tm_status tm_expert_gather(const void* x, int64_t ldx, const int32_t* slots, const int32_t* used, void* out,
                           int64_t ldo, int64_t count, int64_t rows, int64_t top, int64_t d, int dtype,
                           void* stream) {
  return guarded([&] { return expert_gather(x, ldx, slots, used, out, ldo, count, rows, top, d, dtype, stream); });
}

tm_status tm_expert_combine(const void* y, int64_t ldy, const int32_t* slots, const int32_t* used,
                            const float* weights, const void* residual, int64_t ldr, void* out, int64_t ldo,
                            int64_t count, int64_t rows, int64_t top, int64_t d, int dtype, void* stream) {
  return guarded([&] {
    return expert_combine(y, ldy, slots, used, weights, residual, ldr, out, ldo, count, rows, top, d, dtype, stream);
  });
}

tm_status tm_expert_combine_backward(const void* dout, int64_t lddout, const void* y, int64_t ldy,
                                     const int32_t* slots, const int32_t* used, const float* weights, void* dy,
                                     int64_t lddy, float* dweights, int64_t count, int64_t rows, int64_t top,
                                     int64_t d, int dtype, void* stream) {
  return guarded([&] {
    return expert_combine_backward(dout, lddout, y, ldy, slots, used, weights, dy, lddy, dweights, count,
                                   rows, top, d, dtype, stream);
  });
}

tm_status tm_token_logp(const void* logits, int64_t ld, const int64_t* targets, float temperature, float* logp,
                        float* entropy, float* stats, int64_t top, float* top_logp, int64_t* top_ids, int64_t rows,
                        int64_t vocab, int dtype, void* stream) {
  return guarded([&] {
    return token_logp(logits, ld, targets, temperature, logp, entropy, stats, top, top_logp, top_ids, rows,
                      vocab, dtype, stream);
  });
}

tm_status tm_token_logp_backward(const void* logits, int64_t ld, const int64_t* targets, const float* stats,
                                 const float* entropy, const float* dlogp, const float* dentropy,
                                 float temperature, void* dlogits, int64_t ld_dlogits, int64_t rows, int64_t vocab,
                                 int dtype, void* stream) {
  return guarded([&] {
    return token_logp_backward(logits, ld, targets, stats, entropy, dlogp, dentropy, temperature, dlogits,
                               ld_dlogits, rows, vocab, dtype, stream);
  });
}

}  // extern "C"
