// Internal declarations of the gated feed-forward block (include/layer.h, layer_ffn_*).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace soap {
namespace ffn {

constexpr int kMaxGroups = 1024;
constexpr int kSms = 152;           // that a product's parts are shared out among, one or a pair for each
constexpr int kMinParted = 24;      // fewer slices of 64 products (fp32: times 6) stay in one part
constexpr int kMaxSlices = 1024;    // most slices that one accumulator adds up

// Maps that end at a group's last row, so that loads of its rows give 0 beyond it and stores leave the rows behind it
// alone: results (boxes of 32 x 32) and factors of the weights' gradients (boxes of 64 x 64).
enum Clip { kH, kY, kDG, kDU, kInX, kInDY, kInH, kInDG, kInDU, kClips };

struct Maps {
  CUtensorMap a0;           // factors of 128 rows: x or dy
  CUtensorMap a1[2];        // h, or dg and du
  CUtensorMap w0[2];        // gate and up, or down
  CUtensorMap w1[2];        // down, or gate and up
  CUtensorMap dw[3];        // results: the weights' gradients
  CUtensorMap clip[kClips]; // dense: up to the last row; groups: what their own are made from
};

// Tiles of a call: rows, columns per phase; units at a time; of a part's sums the fp32 elements and the blocks that are
// counted.
struct Tiles {
  int rows, cols[3], pool, partial, blocks;
};

// What is made on the device before the products run.
struct Plan {
  int next, through, gave_up;  // the list's next place; CTAs that are through; whether a wait gave up
  int total;                   // units in the list
  int first[3];                // of the phases
  int tiles[2], splits[2];     // of the row phases
  int bounds[kMaxGroups + 1];  // the groups' rows
  int row_tiles[kMaxGroups + 1];  // tiles of rows before each group
  int blocks[kMaxGroups + 1];     // blocks of 32 rows before each group
  int parts[kMaxGroups + 1];      // parts along the rows (of the weights' gradients) before each group
  int slots[kMaxGroups + 1];      // of them those of groups with more than one
};

struct Args {
  Plan* plan;
  int *done_row, *done_group;   // stored blocks of 32 x 32 of h (or dg, du and h), per row tile and per group
  int *count[3];                // parts that are there, per block of a tile, per phase
  float* partial[3];
  const CUtensorMap* clips;     // [groups][kClips], or nullptr: those in Maps (dense, few rows)
  int backward, params;
  int groups, rows, hidden, width;
  int row_tile, col_tile[3], pool;
  int narrow[3];                // whether a phase's tiles have half the columns (g's and u's 64 each, others' 128)
  int each[3];                  // tiles of a group's weights' gradients
  int stored;                   // blocks that the first phase stores for a row tile
  void* h;                      // few rows: where the first phase's results go
  int64_t ld_h, h_plane;
  int plane_bits;               // log2 of the planes of h, dg and du (16-bit types)
  int b_columns[2];             // whether the second factor of a row phase has its K dimension outermost
  int kblocks[2];               // slices of a factor pair, per row phase
  int products;                 // of planes, per slice
  int slices[2];                // of a tile, per row phase: of all pairs and planes that are added
  int wa[3], wb[3];             // Clip of the factors of the weights' gradients
  int wrows[3], wcols[3];       // sides of the weights' gradients as they are stored
  int act;
  float* pre;
  int64_t pre_elems;
  void* y;                      // y or dx
  int64_t ld_y;
  int y_tma;
  void* dw[3];
  int64_t ld_dw[3], stride_dw[3];
  int dw_tma[3];
  int* status;
  uint64_t wait_ns;
  const int* hold;
  const int32_t* offsets;       // the caller's
  int done_words;               // to zero, from done_row on
};

// Copies of operands with rows of whole 16-byte units: 16-bit elements as they are, fp32 ones as three bf16 planes
// that add up to the element (8 bits of its significand each).
//
// Every plane is multiplied by planes of the other operand, of which one may be infinite: a lower plane that is 0 (one in
// 256 of them, and all of bf16 values') would make NaN of what is an infinity. So a plane is at least kLeast of what the
// plane before it was taken from, with its sign: 2^-32 of the element, 2^-8 of an fp32 rounding. That is a bf16 value for
// elements from 2^-62 on; all of an infinity's planes are infinite, all of a zero's 0 (0 x inf is NaN).
constexpr float kLeast = 2.3283064365386963e-10f;  // 2^-32
struct CopyJob {
  const void* src;
  int64_t ld, stride;   // of rows and of matrices
  int64_t rows;         // of a matrix
  int inner, ld_out;
  int64_t matrices;
  int of_groups;        // whether they are the groups'
  uint16_t* dst;
  int64_t plane;
};
struct CopyJobs {
  CopyJob job[5];
  int n;
};

// type: soap_dtype_t. units: no more than this many are ever in the list.
cudaError_t run(const Maps& maps, const Args& a, int type, int64_t units, cudaStream_t s);
// The same for few rows of 16-bit types, forward.
cudaError_t run_few(const Maps& maps, const Args& a, int type, int64_t units, cudaStream_t s);
// The plan, the groups' maps, zeros for rows of no group and for the gradients of groups without rows, and the copies
// (`chunks`: of 8 elements, in the largest of them).
cudaError_t prepare(const Maps& maps, const Args& a, const CopyJobs& jobs, int64_t chunks, int type, cudaStream_t s);

// (a 64-bit division takes a scout longer than its loads)
template <typename A, typename B>
inline __host__ __device__ int up_div(A a, B b) {
  if constexpr (sizeof(A) <= 4 && sizeof(B) <= 4)
    return (int)((uint32_t)(a + b - 1) / (uint32_t)b);
  else
    return (int)(((int64_t)a + b - 1) / b);
}

}  // namespace ffn
}  // namespace soap
