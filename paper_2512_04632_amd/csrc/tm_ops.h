// Descriptors of the operators beside the orthogonalizer (layer norm, expert
// products, policy loss), shared between their entry points (tm_ops.cpp) and
// their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tm_internal.h"
#include "turbomuon.h"

namespace tmk {

// ---------------------------------------------------------------- layer norm
struct NormArgs {
  const char* x;        // rows x d, row stride ldx elements
  const char* dy;       // backward only
  char* out;            // y, or dx
  const float* weight;  // nullptr: ones
  const float* bias;    // nullptr: zeros
  float* mean;          // forward: written; backward: read
  float* rstd;
  float* part;          // backward: column sums of each block, [blocks][2][d]; nullptr: one block, or none wanted
  float *dweight, *dbias;   // where a single block puts them
  int64_t ldx, lddy, ldo;
  int32_t rows, d;
  float eps;
};

// Widest row that a workgroup keeps in registers.
constexpr int kNormMaxFused = 16384;

hipError_t launch_norm(const NormArgs& A, bool f32, hipStream_t st);
// Blocks (and so column sums in `part`) of a backward launch.
int norm_blocks(int64_t rows, int64_t d, bool f32);
hipError_t launch_norm_backward(const NormArgs& A, bool f32, int blocks, hipStream_t st);
// dweight, dbias (either may be nullptr) = sums of `blocks` partial sums.
hipError_t launch_norm_params(const float* part, int blocks, int d, float* dweight, float* dbias,
                              hipStream_t st);

// ---------------------------------------------------------------- expert products
// Whether a launch's threads fit the 32 bits that the dispatch packet has for them.
inline bool launchable(uint64_t blocks, uint64_t threads) { return blocks * threads < (uint64_t(1) << 32); }

struct ExpertArgs {
  const char* a;        // x (rows x k), or x of a weight gradient
  const char* b;        // the experts' matrices, or dy of a weight gradient (rows x n)
  char* out;            // rows x n, or experts x k x n
  const int32_t* ends;  // device: rows up to the last of each expert
  int64_t lda, ldb, ldo;
  int64_t stride_b;     // elements from one expert's matrix to the next (b, or out of a weight gradient)
  int32_t rows, experts, k, n;
  int32_t slices;       // matmul: of the summed index, each with a result of its own:
  int64_t slice_out;    // elements from one slice's result to the next
  int32_t chunk;        // weight gradient: rows of an expert that are summed into one matrix (0: all of them)
};

// How a call is run: by which tiles, and over how many slices of the summed index.
struct ExpertPlan {
  bool staged;          // through registers: fp32, operands that are not 16-byte aligned, groups of a few rows
  int tile, slices, chunk;
  uint64_t bytes;       // workspace: the slices' or chunks' results
};

ExpertPlan plan_expert_matmul(const ExpertArgs& A, bool f32, bool transposed);
ExpertPlan plan_expert_wgrad(const ExpertArgs& A, bool f32);
hipError_t launch_expert_matmul(const ExpertArgs& A, const ExpertPlan& P, bool f32, bool transposed, char* ws,
                                hipStream_t st);
hipError_t launch_expert_wgrad(const ExpertArgs& A, const ExpertPlan& P, bool f32, bool out_f32, char* ws,
                               hipStream_t st);
// The launches that these are made of.
hipError_t launch_rows_tiles(const ExpertArgs& A, const ExpertPlan& P, bool transposed, hipStream_t st);
hipError_t launch_wgrad_tiles(const ExpertArgs& A, const ExpertPlan& P, bool out_f32, hipStream_t st);
hipError_t launch_rows_staged(const ExpertArgs& A, const ExpertPlan& P, bool f32, bool transposed, hipStream_t st);
hipError_t launch_wgrad_staged(const ExpertArgs& A, const ExpertPlan& P, bool f32, bool out_f32, hipStream_t st);

// ---------------------------------------------------------------- policy loss
struct LossArgs {
  const char* logits;        // rows x vocab, row stride ld elements
  const int64_t* targets;
  const float *old_logp, *advantages, *weights, *ref_logp;   // ref_logp: nullptr without the KL term
  const float* grad;         // backward: the loss's own gradient on the device (nullptr: 1)
  float *loss, *logp, *lse, *slope;
  char* dlogits;             // nullptr: no gradient
  float* row_loss;           // workspace: each row's share of the loss
  float2* part;              // workspace: (max, sum of exponentials) of each chunk, [rows][chunks]
  float2* stats;             // workspace: (max, 1 / sum) of each row that is cut into chunks
  int64_t ld, ldd;
  int32_t rows, vocab;
  int32_t chunks, chunk;     // chunks of a row and their length
  float clip_low, clip_high, kl, inv_temp;
};

// Chunks of a row where there are too few rows to fill the chip with one workgroup each (1: whole rows).
int loss_chunks(int64_t rows, int64_t vocab);
hipError_t launch_loss(const LossArgs& A, bool f32, hipStream_t st);
hipError_t launch_loss_backward(const LossArgs& A, bool f32, hipStream_t st);

// ---------------------------------------------------------------- host side (tm_api.cpp)
tm_status fail_with(tm_status s, const char* msg);
void clear_error();
// Runs `enqueue` on the current device with `bytes` of the stream's operator
// workspace, timed as one record of `phase` while the timing hooks are on.
struct Enqueue {
  virtual hipError_t operator()(char* ws, hipStream_t st) const = 0;
};
tm_status run_op(int phase, size_t bytes, hipStream_t st, const Enqueue& enqueue);

}  // namespace tmk
