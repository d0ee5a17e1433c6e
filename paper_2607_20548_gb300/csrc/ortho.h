// Internal declarations of the stand-alone orthogonalisation (include/muon.h, muon_orthogonalize).
#pragma once

#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace soap {
namespace ortho {

constexpr int kMaxSteps = 64;
constexpr int kDoneExtra = 3;  // words after the matrices' counters

// One Newton-Schulz step on scaled fp16 intermediates (the scales are powers of two):
//   S = s_alpha t^2 X X^T,  B = b_alpha S S + b_beta S,  X' = t (x_alpha B X + x_beta X)
// with t applied in the first step only.
struct StepCoef {
  float s_alpha, b_alpha, b_beta, x_alpha, x_beta;
};

// What steps_kernel works on. X: batch matrices of rows x cols (row-major, leading dimension ld_x, a
// multiple of 8), twice; S and B: batch r x r matrices, r = min(rows, cols). With `split`, every
// matrix is a hi + lo pair: matrix b's hi plane at index b, its lo plane at index batch + b. The
// first X is the input; the last step writes the caller's matrices.
struct Steps {
  int rows, cols, batch, steps;
  bool split;
  __half *x[2], *s, *b;
  int ld_x, ld_s;
  const float* t;  // per matrix
  int* done;       // per matrix, then kDoneExtra: the list's next place, CTAs that are through, whether a wait gave up
  void* out;       // out_type (soap_dtype_t), leading dimension, elements between matrices
  int out_type;
  int64_t ld_out, stride_out;
  int out_exp;     // the last step's result carries 2^out_exp (run_steps: 0)
  int* status;
  uint64_t wait_ns;  // bound of the waits, and a flag to wait for first (soap_wait_limit)
  const int* hold;
  StepCoef coef[kMaxSteps];
};

cudaError_t run_steps(const Steps& p, cudaStream_t s);

// Matrices with a side of up to 128 that a cluster of CTAs can hold on chip, in one launch from the caller's
// matrices M (leading dimension ld, elements between matrices) to p.out; of p's buffers it uses none. sx: the
// scale of the first X. small_cluster: the CTAs per matrix, 0 if it does not fit.
int small_cluster(int rows, int cols, int batch, bool split);
cudaError_t run_small(const Steps& p, int cluster, const void* M, int64_t ld, int64_t stride, float eps, int sx,
                      cudaStream_t s);

}  // namespace ortho
}  // namespace soap
