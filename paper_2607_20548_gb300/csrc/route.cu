// A mixture-of-experts router's decision and its gradient (include/layer.h).
//
//   p = softmax(z); the k largest (z, lower index first); gates; counts_e; P_e = sum_t p_te
//   loss = coef E / (k n) sum_e counts_e P_e / n
//   dz_e = p_e (u_e - sum_j p_j u_j),  u = coef dloss E / (k n^2) counts + (d gates -> p)
//
// A group of G lanes (8, 16 or 32) takes a token; lane l holds the logits l, l + G, ... in NE
// registers. The choice runs on 32-bit keys in the logits' order: each lane keeps its keys
// sorted, and k times the group's largest head is found and popped by its owner. Column sums of
// p stay in registers over all of a warp's tokens, counts in shared memory, and both leave the
// CTA as one partial row that a second kernel adds in a fixed order.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/layer.h"
#include "profile.h"
#include "types.h"

namespace soap {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxExperts = 1024;
constexpr int kMaxCtas = 152 * 4;  // most partial rows

// Keys in the order of the logits: finite values map to 1 .. 2^32 - 1, -inf and "no logit" to 0.
__device__ __forceinline__ uint32_t order_key(float z) {
  if (z == -INFINITY) return 0u;
  const uint32_t u = __float_as_uint(z + 0.f);  // -0 counts as +0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <int G>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  if constexpr (G == 32) {
    return __reduce_max_sync(0xffffffffu, v);
  } else {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  }
}
template <int G>
__device__ __forceinline__ uint32_t group_min(uint32_t v) {
  return ~group_max<G>(~v);
}

// One token's softmax: z in registers -> e = exp(z - max) with zero for -inf and absent logits.
// Returns false for a row that is not counted (no finite logit); bad: it holds a NaN or +inf.
template <int G, int NE>
__device__ __forceinline__ bool softmax_row(const float (&z)[NE], float (&e)[NE], float& top, float& sum, bool& bad) {
  float m = -INFINITY;
  int odd = 0;
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    m = fmaxf(m, z[i]);
    odd |= !(z[i] < INFINITY);
  }
  const uint32_t top_key = group_max<G>(order_key(m));
  bad = group_max<G>((uint32_t)odd) != 0;
  top = key_value(top_key);
  sum = 0.f;
  if (top_key == 0) return false;
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    e[i] = __expf(z[i] - top);
    sum += e[i];
  }
  return true;
}

template <typename T, int G, int NE>
__device__ __forceinline__ void load_row(const T* row, int experts, int lane, float (&z)[NE]) {
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const int c = lane + i * G;
    z[i] = c < experts ? to_f32(row[c]) : -INFINITY;
  }
}

template <typename T, int G, int NE>
__global__ void __launch_bounds__(kThreads)
    route_fwd_kernel(const T* logits, int64_t ld, const uint8_t* mask, int64_t tokens, int experts, int k,
                     int normalize, int32_t* indices, float* gates, float* part_p, int* part_c, int* status) {
  extern __shared__ int counts[];             // [experts + 1]: the choices, and the tokens counted
  __shared__ float sums[kThreads / 32][33];
  const int lane = threadIdx.x % G;
  for (int c = threadIdx.x; c <= experts; c += kThreads) counts[c] = 0;
  __syncthreads();
  float acc[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) acc[i] = 0.f;
  const int64_t groups = (int64_t)gridDim.x * (kThreads / G);
  const int64_t passes = (tokens + groups - 1) / groups;
  for (int64_t pass = 0; pass < passes; ++pass) {
    const int64_t t = pass * groups + (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
    const bool live = t < tokens && (!mask || mask[t] != 0);
    float z[NE], e[NE];
    if (live) {
      load_row<T, G, NE>(logits + t * ld, experts, lane, z);
    } else {
#pragma unroll
      for (int i = 0; i < NE; ++i) z[i] = -INFINITY;
    }
    float top, sum;
    bool bad;
    const bool counted = softmax_row<G, NE>(z, e, top, sum, bad);
    sum = group_sum<G>(counted ? sum : 0.f);
    const float inv = 1.f / sum;
    if (bad) {
#pragma unroll
      for (int i = 0; i < NE; ++i) acc[i] = NAN;
      if (status && lane == 0) atomicOr(status, SOAP_STATUS_NONFINITE);
    } else if (counted) {
#pragma unroll
      for (int i = 0; i < NE; ++i) acc[i] = fmaf(e[i], inv, acc[i]);
    }
    if (lane == 0 && (counted || bad)) atomicAdd(&counts[experts], 1);
    // the choice: few keys per lane are kept sorted (falling, equal ones by rising index, i.e. in
    // place), so that a pop is a shift; more are scanned again after each pop
    constexpr bool kSorted = NE <= 8;
    uint32_t key[NE];
    int idx[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      key[i] = bad ? 0u : order_key(z[i]);
      idx[i] = lane + i * G;
    }
    if (kSorted) {
#pragma unroll
      for (int i = 1; i < NE; ++i)
#pragma unroll
        for (int j = i; j > 0; --j) {
          const bool up = key[j] > key[j - 1];
          const uint32_t hi = up ? key[j] : key[j - 1], lo = up ? key[j - 1] : key[j];
          const int ih = up ? idx[j] : idx[j - 1], il = up ? idx[j - 1] : idx[j];
          key[j - 1] = hi;
          key[j] = lo;
          idx[j - 1] = ih;
          idx[j] = il;
        }
    }
    int my_idx = -1;
    float my_gate = 0.f;
    for (int r = 0; r < k; ++r) {
      uint32_t head = key[0];
      int head_idx = idx[0];
      if (!kSorted) {
#pragma unroll
        for (int i = 1; i < NE; ++i)
          if (key[i] > head) {
            head = key[i];
            head_idx = idx[i];
          }
      }
      const uint32_t best = group_max<G>(head);
      const uint32_t at = group_min<G>(head == best ? (uint32_t)head_idx : 0xffffffffu);
      const bool some = best != 0;
      if (some && lane == r) {
        my_idx = (int)at;
        my_gate = __expf(key_value(best) - top) * inv;
      }
      if (some && head == best && (uint32_t)head_idx == at) {
        atomicAdd(&counts[at], 1);
        if (kSorted) {
#pragma unroll
          for (int i = 1; i < NE; ++i) {
            key[i - 1] = key[i];
            idx[i - 1] = idx[i];
          }
          key[NE - 1] = 0u;
        } else {
#pragma unroll
          for (int i = 0; i < NE; ++i)
            if ((uint32_t)idx[i] == at) key[i] = 0u;
        }
      }
    }
    if (normalize) {
      const float total = group_sum<G>(my_gate);
      if (total > 0.f) my_gate /= total;
    }
    if (bad) my_gate = NAN;
    if (t < tokens && lane < k) {
      indices[t * k + lane] = my_idx;
      gates[t * k + lane] = my_gate;
    }
  }
  // column sums: the groups of a warp by shuffles, the warps through shared memory in order
  const int warp = threadIdx.x / 32, wl = threadIdx.x % 32;
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    float v = acc[i];
#pragma unroll
    for (int o = G; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    sums[warp][wl] = v;
    __syncthreads();
    const int c = threadIdx.x + i * G;
    if (threadIdx.x < G && c < experts) {
      float s = 0.f;
      for (int w = 0; w < kThreads / 32; ++w) s += sums[w][threadIdx.x];
      part_p[(int64_t)blockIdx.x * experts + c] = s;
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c <= experts; c += kThreads) part_c[(int64_t)blockIdx.x * (experts + 1) + c] = counts[c];
}

// Adds the CTAs' partial rows in a fixed order, a warp to a column; the loss. One CTA of 1024 threads.
__global__ void __launch_bounds__(1024)
    route_sum_kernel(const float* part_p, const int* part_c, int parts, int experts, int k, float coef,
                     int32_t* counts, int32_t* live, float* mean_probs, float* loss) {
  __shared__ double red[32];
  __shared__ int total;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (warp == 0) {
    int n = 0;
    for (int p = lane; p < parts; p += 32) n += part_c[(int64_t)p * (experts + 1) + experts];
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) total = n;
  }
  __syncthreads();
  const int n = total;
  double dot = 0.0;
  for (int c = warp; c < experts; c += 32) {
    int cnt = 0;
    double s = 0.0;
    for (int p = lane; p < parts; p += 32) {
      cnt += part_c[(int64_t)p * (experts + 1) + c];
      s += (double)part_p[(int64_t)p * experts + c];
    }
    cnt = __reduce_add_sync(0xffffffffu, cnt);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const double mean = n > 0 ? s / n : 0.0;
    dot += (double)cnt * mean;
    if (lane == 0) {
      counts[c] = cnt;
      if (mean_probs) mean_probs[c] = (float)mean;
    }
  }
  if (lane == 0) red[warp] = dot;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < 32; ++w) t += red[w];
    *live = n;
    *loss = n > 0 ? (float)((double)coef * experts / ((double)k * n) * t) : 0.f;
  }
}

template <typename T, int G, int NE>
__global__ void __launch_bounds__(kThreads)
    route_bwd_kernel(const T* logits, int64_t ld, const uint8_t* mask, int64_t tokens, int experts, int k,
                     int normalize, double scale, const int32_t* indices, const int32_t* counts, const int32_t* live_n,
                     const float* dgates, T* dlogits, int64_t ld_d) {
  const int lane = threadIdx.x % G;
  const int n = *live_n;
  const double per = n > 0 ? scale / ((double)n * n) : 0.0;
  float up[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const int c = lane + i * G;
    up[i] = c < experts ? (float)(per * counts[c]) : 0.f;
  }
  const int64_t groups = (int64_t)gridDim.x * (kThreads / G);
  const int64_t passes = (tokens + groups - 1) / groups;
  for (int64_t pass = 0; pass < passes; ++pass) {
    const int64_t t = pass * groups + (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
    const bool live = t < tokens && (!mask || mask[t] != 0);
    float z[NE], e[NE];
    const T* row = logits + t * ld;
    if (live) {
      load_row<T, G, NE>(row, experts, lane, z);
    } else {
#pragma unroll
      for (int i = 0; i < NE; ++i) z[i] = -INFINITY;
    }
    float top, sum;
    bool bad;
    const bool counted = softmax_row<G, NE>(z, e, top, sum, bad);
    sum = group_sum<G>(counted ? sum : 0.f);
    const float inv = 1.f / sum;
    // the gates' gradient at the chosen logits: lane r holds choice r
    float d = 0.f;
    int at = -1;
    float pc = 0.f;
    if (dgates && live && lane < k) {
      at = indices[t * k + lane];
      if (at >= 0 && at < experts) {
        d = dgates[t * k + lane];
        pc = __expf(to_f32(row[at]) - top) * inv;
      } else {
        at = -1;
      }
    }
    if (dgates && normalize) {  // gate_r = p_r / S: d p_r = (d gate_r - sum_j d gate_j gate_j) / S
      const float S = group_sum<G>(pc);
      const float dg = group_sum<G>(d * pc);
      if (at >= 0) d = (d - dg / S) / S;
    }
    float dot = pc * d;
    if (counted) {
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        e[i] *= inv;
        dot = fmaf(e[i], up[i], dot);
      }
    }
    dot = group_sum<G>(dot);
    if (t < tokens) {
      T* out = dlogits + t * ld_d;
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        const int c = lane + i * G;
        if (c < experts) out[c] = from_f32<T>(bad ? NAN : counted ? e[i] * (up[i] - dot) : 0.f);
      }
    }
    if (dgates) {  // the chosen ones again, with the gates' part (ordered after the row's stores)
      __syncwarp();
      if (at >= 0)
        dlogits[t * ld_d + at] = from_f32<T>(pc * ((float)(per * counts[at]) + d - dot));
    }
  }
}

// ---- launches ------------------------------------------------------------------------------

// f(group size, registers per lane) for a number of experts: a group just wide enough up to 32.
template <typename F>
cudaError_t with_shape(int experts, F&& f) {
  using std::integral_constant;
  if (experts <= 8) return f(integral_constant<int, 8>(), integral_constant<int, 1>());
  if (experts <= 16) return f(integral_constant<int, 16>(), integral_constant<int, 1>());
  if (experts <= 32) return f(integral_constant<int, 32>(), integral_constant<int, 1>());
  if (experts <= 64) return f(integral_constant<int, 32>(), integral_constant<int, 2>());
  if (experts <= 128) return f(integral_constant<int, 32>(), integral_constant<int, 4>());
  if (experts <= 256) return f(integral_constant<int, 32>(), integral_constant<int, 8>());
  if (experts <= 512) return f(integral_constant<int, 32>(), integral_constant<int, 16>());
  return f(integral_constant<int, 32>(), integral_constant<int, 32>());
}

template <typename F>
cudaError_t with_type(int32_t type, F&& f) {
  if (type == SOAP_F32) return f(float());
  return type == SOAP_BF16 ? f(__nv_bfloat16()) : f(__half());
}

int group_of(int experts) { return experts <= 8 ? 8 : experts <= 16 ? 16 : 32; }

int ctas_for(int64_t tokens, int experts) {
  const int per = kThreads / group_of(experts);
  return (int)std::max<int64_t>(1, std::min<int64_t>(kMaxCtas, (tokens + per - 1) / per));
}

bool bad_ptr(const void* p, size_t size) { return !p || reinterpret_cast<uintptr_t>(p) % size; }

bool bad_route(int64_t tokens, int32_t experts, int32_t k, const void* logits, int64_t ld, int32_t type, float coef) {
  if (tokens < 0 || tokens > INT32_MAX || experts < 1 || experts > kMaxExperts) return true;
  if (k < 1 || k > experts || k > 32 || type < SOAP_F32 || type > SOAP_F16 || !std::isfinite(coef)) return true;
  return tokens > 0 && (bad_ptr(logits, dtype_size(type)) || ld < experts);
}

}  // namespace
}  // namespace soap

using namespace soap;

extern "C" {

size_t layer_route_workspace_bytes(int64_t tokens, int32_t experts) {
  if (tokens < 0 || tokens > INT32_MAX || experts < 1 || experts > kMaxExperts) return 0;
  return (size_t)ctas_for(tokens, experts) * (2 * (size_t)experts + 1) * 4;
}

soap_status_t layer_route_forward(int64_t tokens, int32_t experts, int32_t k, const void* logits, int64_t ld,
                                  int32_t type, const uint8_t* mask, int32_t normalize, float coef,
                                  int32_t* indices, float* gates, int32_t* counts, int32_t* live,
                                  float* mean_probs, float* loss, int32_t* status, void* workspace,
                                  size_t workspace_bytes, soap_stream_t stream) {
  if (bad_route(tokens, experts, k, logits, ld, type, coef)) return SOAP_ERR_INVALID_ARG;
  if (tokens > 0 && (bad_ptr(indices, 4) || bad_ptr(gates, 4))) return SOAP_ERR_INVALID_ARG;
  if (bad_ptr(counts, 4) || bad_ptr(live, 4) || bad_ptr(loss, 4) || (mean_probs && bad_ptr(mean_probs, 4)) ||
      (status && bad_ptr(status, 4)) || bad_ptr(workspace, 16) ||
      workspace_bytes < layer_route_workspace_bytes(tokens, experts))
    return SOAP_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  const int parts = ctas_for(tokens, experts);
  float* part_p = static_cast<float*>(workspace);
  int* part_c = reinterpret_cast<int*>(part_p + (size_t)parts * experts);
  const double n = (double)tokens * experts;
  ProfScope prof(kFamElementwise, 6.0 * n, n * dtype_size(type) + 8.0 * tokens * k, s);
  const cudaError_t e = with_type(type, [&](auto t) {
    using T = decltype(t);
    return with_shape(experts, [&](auto g, auto ne) {
      route_fwd_kernel<T, decltype(g)::value, decltype(ne)::value><<<parts, kThreads, (experts + 1) * 4, s>>>(
          static_cast<const T*>(logits), ld, mask, tokens, experts, k, normalize, indices, gates, part_p, part_c,
          status);
      const cudaError_t le = cudaGetLastError();
      if (le != cudaSuccess) return le;
      route_sum_kernel<<<1, 1024, 0, s>>>(part_p, part_c, parts, experts, k, coef, counts, live, mean_probs, loss);
      return cudaGetLastError();
    });
  });
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

soap_status_t layer_route_backward(int64_t tokens, int32_t experts, int32_t k, const void* logits, int64_t ld,
                                   int32_t type, const uint8_t* mask, int32_t normalize, float coef, float dloss,
                                   const int32_t* indices, const int32_t* counts, const int32_t* live,
                                   const float* dgates, void* dlogits, int64_t ld_d, soap_stream_t stream) {
  if (bad_route(tokens, experts, k, logits, ld, type, coef) || !std::isfinite(dloss)) return SOAP_ERR_INVALID_ARG;
  if (tokens == 0) return SOAP_OK;
  if (bad_ptr(counts, 4) || bad_ptr(live, 4) || bad_ptr(dlogits, dtype_size(type)) || ld_d < experts ||
      (dgates && (bad_ptr(dgates, 4) || bad_ptr(indices, 4))))
    return SOAP_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  const int ctas = ctas_for(tokens, experts);
  const double n = (double)tokens * experts;
  const double scale = (double)coef * dloss * experts / k;
  ProfScope prof(kFamElementwise, 6.0 * n, 2.0 * n * dtype_size(type) + 12.0 * tokens * k, s);
  const cudaError_t e = with_type(type, [&](auto t) {
    using T = decltype(t);
    return with_shape(experts, [&](auto g, auto ne) {
      route_bwd_kernel<T, decltype(g)::value, decltype(ne)::value><<<ctas, kThreads, 0, s>>>(
          static_cast<const T*>(logits), ld, mask, tokens, experts, k, normalize, scale, indices, counts, live, dgates,
          static_cast<T*>(dlogits), ld_d);
      return cudaGetLastError();
    });
  });
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

}  // extern "C"
