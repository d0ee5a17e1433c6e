// Internal declarations of the stand-alone orthogonalisation (include/muon.h, muon_orthogonalize).
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace soap {
namespace ortho {

// A batch of row-major fp16 matrices with a leading dimension that is a multiple of 8, scaled by a
// power of two. Split operands hold x = hi + lo as two planes: matrix b's hi part at index b, its
// lo part at index batch + b. The columns between cols and ld hold nothing that counts.
struct Mat {
  __half* p;
  int rows, cols, ld;
  int64_t stride;  // elements between matrices (and planes)
  CUtensorMap map; // boxes of 64 x 64 elements, 128-byte swizzle
};

// How an operand's M (or N) x K elements are stored.
enum Major : int { kRowsK = 0 /* row m, column k */, kRowsM = 1 /* row k, column m */ };

struct Product {
  int M, N, K, batch;
  bool split;      // operands (and an internal result) are hi + lo pairs
  bool symmetric;  // M = N and the result is symmetric: tiles below the diagonal, mirrored
  Major a_major, b_major;
  float alpha, beta;      // out = t^t_pow (alpha A B^T + beta cin)
  const Mat* cin;         // same rows and columns as the result, or nullptr
  const float* t;         // per matrix
  int t_pow;              // 0, 1 or 2
  const Mat* out;         // internal result, or
  void* user;             // the caller's matrix: type, leading dimension, stride between matrices
  int user_type;
  int64_t user_ld, user_stride;
  int* status;
};

bool make_map(Mat& m, int planes);
cudaError_t product(const Product& p, const Mat& a, const Mat& b, cudaStream_t s);

}  // namespace ortho
}  // namespace soap
