// What the routing kernels share (route.cu: a group of lanes per token; route_tile.cu: two lanes per token):
// the logits' order as keys, exponentials, and the way from CTAs' column sums to the totals.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/layer.h"
#include "types.h"

namespace soap {
namespace route {

constexpr int kCluster = 8;
constexpr int kTileCluster = 2;  // with two lanes per token: clusters of 8 left a quarter of the SMs' time idle
constexpr int kMaxParts = 228;   // clusters, and partial rows, of a forward launch

struct Forward {
  const void* logits;
  int64_t ld;
  const uint8_t* mask;
  int64_t tokens;
  int experts, k, normalize;
  int32_t* indices;
  float* gates;
  float2* stats;
  float* part_p;
  int* part_c;
  int* status;
};
struct Totals {
  int32_t* counts;
  int32_t* live;
  float *mean_probs, *loss;
  float coef;
};
struct Backward {
  const void* logits;
  int64_t ld;
  const uint8_t* mask;
  int64_t tokens;
  int experts, k, normalize;
  float scale;  // of counts / n^2
  const int32_t* indices;
  const float2* stats;
  const int32_t *counts, *live;
  const float* dgates;
  void* dlogits;
  int64_t ld_d;
};

// The kernels with two lanes per token: whether they take a call, and the launches. forward_ctas: whole
// clusters.
constexpr int64_t kFewTokens = 152 * 96;  // below: an SM would have only a few warps
bool tile_fits(int64_t tokens, int experts, int k, int32_t type);
int tile_forward_ctas(int64_t tokens, int experts, int k, int32_t type);
cudaError_t tile_forward(const Forward& f, const Totals& out, int32_t type, cudaStream_t s);
cudaError_t tile_backward(const Backward& b, int32_t type, cudaStream_t s);

// Keys in the order of the logits. A NaN's is above +inf's: adding 0 makes every NaN the positive one
// (and -0 a +0). 0 stands for "none".
constexpr uint32_t kKeyNegInf = 0x007fffffu, kKeyInf = 0xff800000u;
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// 16-bit logits differ in the upper 19 bits of their fp32 key (their 13 low mantissa bits are zero, in a
// negative one's key ones): the complemented index goes below.
constexpr uint32_t kLow = 0x1fffu;
__device__ __forceinline__ uint32_t pack_key(uint32_t key, int idx) { return (key & ~kLow) | (kLow - (uint32_t)idx); }
__device__ __forceinline__ uint32_t unpack_key(uint32_t b) { return b & 0x80000000u ? b & ~kLow : b | kLow; }
__device__ __forceinline__ int packed_index(uint32_t b) { return (int)(kLow - (b & kLow)); }

// e^x for x <= 0: one multiplication and the hardware's 2^x (relative error 2^-22 and |x| 2^-24).
__device__ __forceinline__ float exp_neg(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.4426950408889634f));
  return r;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// The word at p's place in the shared memory of the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t peer_word(const void* p, uint32_t rank) {
  const uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(p));
  uint32_t r, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(r) : "memory");
  return v;
}

// A sum over a CTA in a fixed order. (fp32, as everything here: an SM's fp64 rate is so low that the few
// dozen fp64 operations of a thread took 17 us of a launch.)
__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  v = 0.f;
  for (int w = 0; w < (int)blockDim.x / 32; ++w) v += red[w];
  return v;
}

// coef E / (k n) sum_e counts_e mean_e, from the sum.
__device__ __forceinline__ float loss_of(float sum, int n, int experts, int k, float coef) {
  return n > 0 ? coef * (float)experts / (float)k * (sum / (float)n) : 0.f;
}

// The end of a forward kernel: the CTA's warps have left their column sums in shared[warp][experts], and
// counts[experts + 1] holds its choices and the tokens counted. Adds the cluster's CTAs in order, each CTA
// some of the columns; one cluster finishes by itself, several leave a partial row each. `red`: kWarps + 1
// floats.
template <int kWarps>
__device__ __forceinline__ void finish_columns(float* shared, int* counts, float* red, int experts, int k,
                                               float* part_p, int* part_c, const Totals& out) {
  constexpr int kThreads = 32 * kWarps;
  __syncthreads();
  for (int c = threadIdx.x; c < experts; c += kThreads) {
    float v = shared[c];
    for (int w = 1; w < kWarps; ++w) v += shared[w * experts + c];
    shared[c] = v;
  }
  // the cluster's CTAs in order, each CTA some of the columns
  cluster_sync();
  const uint32_t rank = cluster_rank(), size = cluster_size();
  const bool alone = gridDim.x == size;  // one cluster: the totals are complete
  const int64_t part = blockIdx.x / size;
  int n = 0;
  for (uint32_t q = 0; q < size; ++q) n += (int)peer_word(&counts[experts], q);
  float dot = 0.f;
  for (int c = rank * kThreads + threadIdx.x; c < experts; c += size * kThreads) {
    float v = 0.f;
    int cnt = 0;
    for (uint32_t q = 0; q < size; ++q) {
      v += __uint_as_float(peer_word(&shared[c], q));
      cnt += (int)peer_word(&counts[c], q);
    }
    if (alone) {
      const float mean = n > 0 ? v / (float)n : 0.f;
      out.counts[c] = cnt;
      if (out.mean_probs) out.mean_probs[c] = mean;
      dot = fmaf((float)cnt, mean, dot);
    } else {
      part_p[part * experts + c] = v;
      part_c[part * (experts + 1) + c] = cnt;
    }
  }
  if (!alone) {
    if (rank == 0 && threadIdx.x == 0) part_c[part * (experts + 1) + experts] = n;
  } else {
    dot = block_sum(dot, red);
    if (threadIdx.x == 0) red[kWarps] = dot;
    __syncthreads();
  }
  cluster_sync();
  if (alone && rank == 0 && threadIdx.x == 0) {
    dot = 0.f;
    for (uint32_t q = 0; q < size; ++q) dot += __uint_as_float(peer_word(&red[kWarps], q));
    *out.live = n;
    *out.loss = loss_of(dot, n, experts, k, out.coef);
  }
  if (alone) cluster_sync();  // the first CTA has read the others
}

}  // namespace route
}  // namespace soap
