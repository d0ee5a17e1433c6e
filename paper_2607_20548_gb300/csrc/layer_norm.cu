// Layer norm of rows and its backward pass (include/layer.h).
//
//   mu = mean(x), rstd = 1 / sqrt(mean((x - mu)^2) + eps), y = (x - mu) rstd w + b
//   g = dy w, xh = (x - mu) rstd, dx = rstd (g - mean(g) - xh mean(g xh)),
//   dw = sum_rows dy xh, db = sum_rows dy
//
// Bound by memory: x is read and y written once (backward: x and dy read, dx written once). A
// group of threads holds a row in registers, so that the variance is a second pass over registers
// (not E[x^2] - mu^2, which cancels) and nothing is read twice. CTAs are persistent: each thread
// keeps its columns' weights (backward: and their gradients' sums) in registers over all its rows
// (read again for every row, fp32 weights are four times the traffic of a bf16 x through L1: 3.1
// TB/s at 32768 x 8192), and its rows come in kDepth ahead by cp.async into slots that only it reads,
// so no barrier waits for them.
#include <algorithm>
#include <atomic>
#include <cstdint>

#include "../../include/layer.h"
#include "profile.h"
#include "types.h"

namespace soap {
namespace {

constexpr int kMaxThreads = 512;  // of the kernels for rows too wide to be held
// A CTA's threads by the elements of a row that each holds: few registers, all of an SM's threads.
constexpr int threads_for(int elems) { return elems <= 8 ? 1024 : 512; }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// One barrier among a row group's threads (blockDim.x of them, more than a warp).
__device__ __forceinline__ void group_barrier() {
  asm volatile("bar.sync %0, %1;" ::"r"((int)threadIdx.y + 1), "r"((int)blockDim.x) : "memory");
}

// What a row group's warps exchange: two values per warp, in two halves used in turn, so that one
// barrier per exchange is enough (a half is written again only after the barrier of the exchange
// between).
struct Exchange {
  float2* buf;  // [2][blockDim.y][blockDim.x / 32]
  int half = 0;
  // Afterwards lane l holds warp l's values ((0, 0) from the last warp on).
  __device__ __forceinline__ float2 all(float x, float y) {
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    float2* p = buf + (half * blockDim.y + threadIdx.y) * warps;
    half ^= 1;
    if (lane == 0) p[threadIdx.x >> 5] = make_float2(x, y);
    group_barrier();
    return lane < warps ? p[lane] : make_float2(0.f, 0.f);
  }
};

// N bytes from global to shared memory, asynchronously.
template <int N>
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
  const uint32_t d = static_cast<uint32_t>(__cvta_generic_to_shared(dst));
  if constexpr (N == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(d), "l"(src), "n"(N) : "memory");
}

// A thread's part of the rows of a matrix, NV packs of V elements per row, kDepth rows in flight.
// Packs of less than 4 bytes cannot be copied asynchronously and are loaded when they are used.
template <typename T, int V, int NV, int DEPTH, bool FULL>
struct Rows {
  static constexpr bool kAsync = V * sizeof(T) >= 4;
  static constexpr int kSlot = kAsync ? V * sizeof(T) : 0;
  const T* base;
  int64_t ld;
  uint8_t* ring;  // this thread's slots: pack i of stage s at ((s * NV + i) * threads) * kSlot

  __device__ __forceinline__ uint8_t* slot(int s, int i) const {
    return ring + (size_t)((s * NV + i) * blockDim.x * blockDim.y) * kSlot;
  }
  __device__ __forceinline__ void request(int64_t row, int s, int width) const {
    if constexpr (kAsync) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * V;
        if (FULL || c < width) copy_async<V * sizeof(T)>(slot(s, i), base + row * ld + c);
      }
    }
  }
  // The row's packs, zero beyond its end.
  __device__ __forceinline__ void get(int64_t row, int s, int width, Pack<T, V> (&p)[NV]) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * V;
      if (FULL || c < width) {
        p[i] = kAsync ? *reinterpret_cast<const Pack<T, V>*>(slot(s, i))
                      : *reinterpret_cast<const Pack<T, V>*>(base + row * ld + c);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) p[i].v[e] = from_f32<T>(0.f);
      }
    }
  }
};

// Elements 2 k and 2 k + 1 of a thread's packs as fp32.
template <typename T, int V, int NV>
__device__ __forceinline__ float2 values(const Pack<T, V> (&p)[NV], int k) {
  if constexpr (V == 1)
    return make_float2(to_f32(p[2 * k].v[0]), to_f32(p[2 * k + 1].v[0]));
  else
    return to_pair(p[2 * k / V].v + 2 * k % V);
}

// A row's results in pack i (V == 1: packs i and i + 1), rounded once.
template <typename T, int V, bool FULL>
__device__ __forceinline__ void put(T* row, int width, int i, const float2* v) {
#pragma unroll
  for (int j = 0; j < (V == 1 ? 2 : 1); ++j) {
    const int c = ((i + j) * blockDim.x + threadIdx.x) * V;
    if (!FULL && c >= width) break;
    Pack<T, V> o;
    if constexpr (V == 1) {
      o.v[0] = from_f32<T>(j ? v[0].y : v[0].x);
    } else {
#pragma unroll
      for (int e = 0; e < V; e += 2) from_pair(v[e / 2], o.v + e);
    }
    *reinterpret_cast<Pack<T, V>*>(row + c) = o;
  }
}

// A thread's columns of a vector as fp32 pairs (`none` beyond the width, or everywhere without one).
template <typename W, int V, int NV>
__device__ __forceinline__ void columns(const W* w, float none, int width, float2 (&v)[NV * V / 2]) {
#pragma unroll
  for (int k = 0; k < NV * V; ++k) {
    const int c = ((k / V) * blockDim.x + threadIdx.x) * V + k % V;
    const float x = w && c < width ? to_f32(w[c]) : none;
    if (k % 2)
      v[k / 2].y = x;
    else
      v[k / 2].x = x;
  }
}

__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void arrived() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// ---- forward: a group of blockDim.x threads per row, NV packs of V elements each ------------

// FULL: the group's threads have exactly the row's elements.
template <typename T, typename W, int V, int NV, int DEPTH, bool FULL>
__global__ void __launch_bounds__(threads_for(NV * V))
    norm_fwd_kernel(const T* x, int64_t ld_x, const W* weight, const W* bias, float eps, T* y, int64_t ld_y,
                    float* mean, float* rstd, int64_t rows, int width) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float2 buf[2 * 32];
  constexpr int P = NV * V / 2, kPer = V == 1 ? 2 : 1;
  using R = Rows<T, V, NV, DEPTH, FULL>;
  const int tid = threadIdx.y * blockDim.x + threadIdx.x, lane = threadIdx.x & 31;
  const R in{x, ld_x, smem + (size_t)tid * R::kSlot};
  Exchange ex{buf};
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
#pragma unroll
  for (int s = 0; s < DEPTH - 1; ++s) {
    if (row + s * step < rows) in.request(row + s * step, s, width);
    commit();
  }
  float2 w[P], b[P];
  columns<W, V, NV>(weight, 1.f, width, w);
  columns<W, V, NV>(bias, 0.f, width, b);
  // elements of the row in this thread's warp, and in the group's warp `lane`
  auto warp_count = [&](int warp) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) n += max(0, min(32 * V, width - (int)(i * blockDim.x + warp * 32) * V));
    return (float)n;
  };
  const float here = warp_count(threadIdx.x >> 5), inv = 1.f / (float)width;
  const float there = lane < (int)blockDim.x / 32 ? warp_count(lane) : 0.f;
  const float inv_here = here > 0.f ? 1.f / here : 0.f, inv_there = there > 0.f ? 1.f / there : 0.f;
  // whether this thread's element k is one of the row's
  auto has = [&](int k) { return ((k / V) * (int)blockDim.x + (int)threadIdx.x) * V + k % V < width; };
  int s = 0;
  for (; row < rows; row += step) {
    const int64_t ahead = row + (DEPTH - 1) * step;
    if (ahead < rows) in.request(ahead, s == 0 ? DEPTH - 1 : s - 1, width);
    commit();
    arrived<DEPTH - 1>();
    float2 v[P];
    Pack<T, V> raw[NV];
    in.get(row, s, width, raw);
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = values(raw, i);
    s = s + 1 == DEPTH ? 0 : s + 1;
    // sum and spread of the warp's elements about the warp's mean, then over the warps
    float2 acc = pair(0.f);
#pragma unroll
    for (int i = 0; i < P; ++i) acc = add2(acc, v[i]);
    float sum = warp_sum(acc.x + acc.y);
    float mu = sum * inv_here;
    acc = pair(0.f);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      float2 d = add2(v[i], pair(-mu));
      if constexpr (!FULL) {
        if (!has(2 * i)) d.x = 0.f;
        if (!has(2 * i + 1)) d.y = 0.f;
      }
      acc = fma2(d, d, acc);
    }
    float q = warp_sum(acc.x + acc.y);
    if (blockDim.x > 32) {
      const float2 o = ex.all(sum, q);
      mu = warp_sum(o.x) * inv;
      const float d = o.x * inv_there - mu;
      q = warp_sum(fmaf(there * d, d, o.y));
    }
    const float rs = rsqrtf(q * inv + eps);
    if (threadIdx.x == 0) {
      if (mean) mean[row] = mu;
      if (rstd) rstd[row] = rs;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = fma2(mul2(add2(v[i], pair(-mu)), pair(rs)), w[i], b[i]);
#pragma unroll
    for (int i = 0; i < NV; i += kPer) put<T, V, FULL>(y + row * ld_y, width, i, v + i * V / 2);
  }
  arrived<0>();
}

// Sum over a one-row CTA's threads, for the kernels that do not hold a row.
template <int N>
__device__ __forceinline__ void block_sum(float (&v)[N], float* buf) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
  __syncthreads();
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) buf[(threadIdx.x >> 5) * N + i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.f;
  for (int j = 0; j < (int)blockDim.x / 32; ++j)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += buf[j * N + i];
}

// Rows too wide for registers: one CTA per row, three passes over the row.
template <typename T, typename W>
__global__ void __launch_bounds__(kMaxThreads)
    norm_fwd_wide_kernel(const T* x, int64_t ld_x, const W* weight, const W* bias, float eps, T* y, int64_t ld_y,
                         float* mean, float* rstd, int64_t width) {
  __shared__ float buf[32];
  const int64_t row = blockIdx.x;
  const T* xr = x + row * ld_x;
  T* yr = y + row * ld_y;
  float s[1] = {0.f}, q[1] = {0.f};
  for (int64_t c = threadIdx.x; c < width; c += blockDim.x) s[0] += to_f32(xr[c]);
  block_sum(s, buf);
  const float mu = s[0] / (float)width;
  for (int64_t c = threadIdx.x; c < width; c += blockDim.x) {
    const float d = to_f32(xr[c]) - mu;
    q[0] = fmaf(d, d, q[0]);
  }
  block_sum(q, buf);
  const float rs = rsqrtf(q[0] / (float)width + eps);
  if (threadIdx.x == 0) {
    if (mean) mean[row] = mu;
    if (rstd) rstd[row] = rs;
  }
  for (int64_t c = threadIdx.x; c < width; c += blockDim.x)
    yr[c] = from_f32<T>(fmaf((to_f32(xr[c]) - mu) * rs, weight ? to_f32(weight[c]) : 1.f,
                             bias ? to_f32(bias[c]) : 0.f));
}

// ---- backward ------------------------------------------------------------------------------
// Persistent CTAs walk the rows; each thread keeps its columns' sums of dy xh and dy in
// registers, the CTA adds its groups' sums at the end and writes one partial row per sum, and
// norm_cols_kernel adds the partial rows in order (no atomics: the result does not depend on
// which CTA finishes first).

// R rows of a group go through an iteration side by side, so that one's chain of sums and exchanges
// fills the other's waits. A thread keeps a row's packs and converts them twice. kSmemW: weights in
// shared memory (fp32, at their columns), where registers would not hold them beside both sums.
template <typename T, typename W, int V, int NV, int R, int DEPTH, bool FULL>
__global__ void __launch_bounds__(threads_for(NV * V))
    norm_bwd_kernel(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, const float* mean, const float* rstd,
                    const W* weight, T* dx, int64_t ld_dx, float* part, int64_t rows, int width) {
  extern __shared__ __align__(16) uint8_t smem[];  // the rings (and weights); afterwards the groups' column sums
  __shared__ float4 buf[2 * 32];
  constexpr int E = NV * V, P = E / 2, kPer = V == 1 ? 2 : 1;
  constexpr bool kSmemW = E > 16;
  using S = Rows<T, V, NV, DEPTH * R, FULL>;
  const int threads = blockDim.x * blockDim.y, tid = threadIdx.y * blockDim.x + threadIdx.x;
  const S rx{x, ld_x, smem + (size_t)tid * S::kSlot};
  const S rg{dy, ld_dy, smem + (size_t)(DEPTH * R * NV * threads + tid) * S::kSlot};
  float* const weights = reinterpret_cast<float*>(smem + (size_t)2 * DEPTH * R * NV * threads * S::kSlot);
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  auto request = [&](int64_t first, int stage) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (first + r * step < rows) {
        rx.request(first + r * step, stage * R + r, width);
        rg.request(first + r * step, stage * R + r, width);
      }
    commit();
  };
#pragma unroll
  for (int s = 0; s < DEPTH - 1; ++s) request(row + s * R * step, s);
  float2 w[kSmemW ? 1 : P], aw[P], ab[P];
  if constexpr (kSmemW) {
    for (int c = tid; c < width; c += threads) weights[c] = weight ? to_f32(weight[c]) : 1.f;
    __syncthreads();
  } else {
    columns<W, V, NV>(weight, 1.f, width, w);
  }
#pragma unroll
  for (int i = 0; i < P; ++i) aw[i] = ab[i] = pair(0.f);
  // weights of elements 2 k and 2 k + 1 (beyond the row's end any finite value: dy is zero there)
  auto weight_of = [&](int k) {
    if constexpr (!kSmemW) {
      return w[k];
    } else {
      const int c = ((2 * k / V) * blockDim.x + threadIdx.x) * V + 2 * k % V;
      if (V == 1) return make_float2(weights[min(c, width - 1)], weights[min(c + (int)blockDim.x, width - 1)]);
      return FULL || c < width ? *reinterpret_cast<const float2*>(weights + c) : pair(0.f);
    }
  };
  const float inv = 1.f / (float)width;
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  float mu[R], rs[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    mu[r] = rs[r] = 0.f;
    if (row + r * step < rows) {
      mu[r] = mean[row + r * step];
      rs[r] = rstd[row + r * step];
    }
  }
  int s = 0, half = 0;
  for (; row < rows; row += R * step) {
    request(row + (DEPTH - 1) * R * step, s == 0 ? DEPTH - 1 : s - 1);
    arrived<DEPTH - 1>();
    Pack<T, V> px[R][NV], pg[R][NV];
    float sum[R][2];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + r * step < rows) {
        rx.get(row + r * step, s * R + r, width, px[r]);
        rg.get(row + r * step, s * R + r, width, pg[r]);
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < V; ++e) px[r][i].v[e] = pg[r][i].v[e] = from_f32<T>(0.f);
      }
      // beyond the row's end dy is zero, so whatever xh is there counts nowhere
      float2 a0 = pair(0.f), a1 = pair(0.f);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const float2 xh = mul2(add2(values(px[r], k), pair(-mu[r])), pair(rs[r]));
        float2 g = values(pg[r], k);
        aw[k] = fma2(g, xh, aw[k]);
        ab[k] = add2(ab[k], g);
        g = mul2(g, weight_of(k));
        a0 = add2(a0, g);
        a1 = fma2(g, xh, a1);
      }
      sum[r][0] = a0.x + a0.y;
      sum[r][1] = a1.x + a1.y;
    }
    s = s + 1 == DEPTH ? 0 : s + 1;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int r = 0; r < 2 * R; ++r) sum[r / 2][r % 2] += __shfl_xor_sync(0xffffffffu, sum[r / 2][r % 2], o);
    if (warps > 1) {  // the halves of the buffer in turn, as in Exchange
      float4* p = buf + (half * blockDim.y + threadIdx.y) * warps;
      half ^= 1;
      if (lane == 0) p[threadIdx.x >> 5] = make_float4(sum[0][0], sum[0][1], sum[R - 1][0], sum[R - 1][1]);
      group_barrier();
      const float4 o = lane < warps ? p[lane] : make_float4(0.f, 0.f, 0.f, 0.f);
      sum[R - 1][0] = o.z;
      sum[R - 1][1] = o.w;
      sum[0][0] = o.x;
      sum[0][1] = o.y;
#pragma unroll
      for (int q = 16; q > 0; q >>= 1)
#pragma unroll
        for (int r = 0; r < 2 * R; ++r) sum[r / 2][r % 2] += __shfl_xor_sync(0xffffffffu, sum[r / 2][r % 2], q);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t here = row + r * step;
      if (here < rows) {
        const float2 m1 = pair(-sum[r][0] * inv * rs[r]), m2 = pair(-sum[r][1] * inv * rs[r]);
        T* to = dx + here * ld_dx;
#pragma unroll
        for (int i = 0; i < NV; i += kPer) {
          float2 g[kPer * V / 2];
#pragma unroll
          for (int j = 0; j < kPer * V / 2; ++j) {
            const int k = i * V / 2 + j;
            const float2 xh = mul2(add2(values(px[r], k), pair(-mu[r])), pair(rs[r]));
            g[j] = fma2(xh, m2, fma2(mul2(values(pg[r], k), weight_of(k)), pair(rs[r]), m1));
          }
          put<T, V, FULL>(to, width, i, g);
        }
      }
      const int64_t next = here + R * step;
      if (next < rows) {
        mu[r] = mean[next];
        rs[r] = rstd[next];
      }
    }
  }
  arrived<0>();
  if (!part) return;
  // add the groups in order, first dweight's sums, then dbias's
  float* sums = reinterpret_cast<float*>(smem);
  const int lanes = blockDim.x * E;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const float2 a = k == 0 ? aw[j / 2] : ab[j / 2];
      sums[threadIdx.y * lanes + ((j / V) * blockDim.x + threadIdx.x) * V + j % V] = j % 2 ? a.y : a.x;
    }
    __syncthreads();
    float* out = part + ((int64_t)blockIdx.x * 2 + k) * width;
    for (int c = tid; c < width; c += threads) {
      float t = 0.f;
      for (int gq = 0; gq < (int)blockDim.y; ++gq) t += sums[gq * lanes + c];
      out[c] = t;
    }
  }
}

// Rows too wide for registers: dx by one CTA per row in two passes ...
template <typename T, typename W>
__global__ void __launch_bounds__(kMaxThreads)
    norm_bwd_wide_kernel(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, const float* mean, const float* rstd,
                         const W* weight, T* dx, int64_t ld_dx, int64_t width) {
  __shared__ float buf[32 * 2];
  const int64_t row = blockIdx.x;
  const T *xr = x + row * ld_x, *gr = dy + row * ld_dy;
  T* dr = dx + row * ld_dx;
  const float mu = mean[row], rs = rstd[row];
  float s[2] = {0.f, 0.f};
  for (int64_t c = threadIdx.x; c < width; c += blockDim.x) {
    const float g = to_f32(gr[c]) * (weight ? to_f32(weight[c]) : 1.f);
    s[0] += g;
    s[1] = fmaf(g, (to_f32(xr[c]) - mu) * rs, s[1]);
  }
  block_sum(s, buf);
  const float m1 = s[0] / (float)width, m2 = s[1] / (float)width;
  for (int64_t c = threadIdx.x; c < width; c += blockDim.x) {
    const float g = to_f32(gr[c]) * (weight ? to_f32(weight[c]) : 1.f);
    dr[c] = from_f32<T>(rs * (g - m1 - (to_f32(xr[c]) - mu) * rs * m2));
  }
}

// ... and the column sums by threads that own a column each (run before the kernel above, which
// may write over dy or x).
template <typename T>
__global__ void __launch_bounds__(kMaxThreads)
    norm_cols_wide_kernel(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, const float* mean, const float* rstd,
                          float* part, int64_t rows, int64_t width) {
  const int64_t c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= width) return;
  float aw = 0.f, ab = 0.f;
  for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
    const float d = to_f32(dy[row * ld_dy + c]);
    aw = fmaf(d, (to_f32(x[row * ld_x + c]) - mean[row]) * rstd[row], aw);
    ab += d;
  }
  part[((int64_t)blockIdx.y * 2) * width + c] = aw;
  part[((int64_t)blockIdx.y * 2 + 1) * width + c] = ab;
}

// dweight and dbias from `parts` partial rows each: 32 columns per CTA, 32 row lanes.
__global__ void norm_cols_kernel(const float* part, int parts, int64_t width, float* dweight, float* dbias) {
  __shared__ float red[32][33];
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the launch overlaps the end of the kernel before
  const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x;
  float* out = blockIdx.y == 0 ? dweight : dbias;
  if (!out) return;
  float t = 0.f;
  if (c < width)
    for (int p = threadIdx.y; p < parts; p += 32) t += part[((int64_t)p * 2 + blockIdx.y) * width + c];
  red[threadIdx.y][threadIdx.x] = t;
  __syncthreads();
  t = red[threadIdx.x][threadIdx.y];  // column threadIdx.y's 32 sums across a warp
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  const int64_t oc = (int64_t)blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && oc < width) out[oc] = t;
}

// ---- launch choice -------------------------------------------------------------------------

constexpr int kSms = 152;
constexpr int kParts = 2 * kSms;  // most CTAs, and partial rows

struct NormShape {
  int nv, tx;  // accesses per thread and row, threads per row
};

// Threads for a row of `width` elements in accesses of v: a warp where 16 elements per thread are
// enough, else the fewest that give a thread no more than `elems` elements, or more up to `most` where
// the row needs it. nv = 0: too wide for that.
NormShape norm_shape(int64_t width, int v, int elems, int most) {
  const int64_t packs = (width + v - 1) / v;
  for (int nv = v == 1 ? 2 : 1; nv * v <= 16; nv *= 2)
    if (packs <= 32 * nv) return {nv, 32};
  for (int e = elems; e <= most; e *= 2)
    for (int tx = 64; tx <= threads_for(e); tx *= 2)
      if (packs * v <= (int64_t)tx * e) return {e / v, tx};
  return {0, 0};
}

// With few rows per SM a row's own time counts: 8 elements per thread and many threads. With many, rows
// side by side in an SM hide each other's chains of sums: more elements per thread, so that more rows
// fit (forward, 32768 x 8192 bf16: 258 us with 8, 260 with 16, 200 with 32).
bool many_rows(int64_t rows) { return rows >= 16 * kSms; }

int norm_threads(const NormShape& n, int v) { return n.tx >= 128 ? threads_for(n.nv * v) : 512; }

// Rows per CTA: full CTAs, unless the rows would then not reach every SM.
int norm_groups(int64_t rows, const NormShape& n, int v) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(norm_threads(n, v) / n.tx, (rows + kSms - 1) / kSms));
}

// CTAs: two per SM where one does not fill it.
int norm_ctas(int64_t rows, const NormShape& n, int v, int ty) {
  const int most = n.tx * ty <= 512 && n.nv * v <= 8 ? kParts : kSms;
  return (int)std::min<int64_t>(most, (rows + ty - 1) / ty);
}

template <typename F>
cudaError_t with_nv(int nv, F&& f) {
  switch (nv) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 4: return f(std::integral_constant<int, 4>());
    case 8: return f(std::integral_constant<int, 8>());
    case 16: return f(std::integral_constant<int, 16>());
    default: return f(std::integral_constant<int, 32>());
  }
}

// f(elements per access) for rows whose addresses and lengths in bytes, ORed, are `bytes`: 16 bytes, else
// 8, else 4, else an element.
template <typename T, typename F>
cudaError_t with_access(uintptr_t bytes, F&& f) {
  if (bytes % 16 == 0) return f(std::integral_constant<int, 16 / sizeof(T)>());
  if (bytes % 8 == 0) return f(std::integral_constant<int, 8 / sizeof(T)>());
  if (sizeof(T) == 2 && bytes % 4 == 0) return f(std::integral_constant<int, sizeof(T) == 2 ? 2 : 1>());
  return f(std::integral_constant<int, 1>());
}

// f(whether the row has exactly the group's elements): told apart for the widest accesses.
template <int V, typename F>
cudaError_t with_full(bool full, F&& f) {
  if (V >= 4 && full) return f(std::integral_constant<bool, (V >= 4)>());
  return f(std::integral_constant<bool, false>());
}

uintptr_t address(const void* p) { return reinterpret_cast<uintptr_t>(p); }

// One bit per device on which the kernel has its shared-memory attribute.
template <typename K>
cudaError_t allow_smem(K kernel, int bytes, std::atomic<uint64_t>& set) {
  if (bytes <= 48 * 1024 - 4096) return cudaSuccess;  // beside the static part
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t(1) << dev : 0;
  if (bit && (set.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
  if (e == cudaSuccess) set.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

template <typename T, typename W, int V>
cudaError_t fwd_v(int64_t rows, int64_t width, const T* x, int64_t ld_x, const W* w, const W* b, float eps, T* y,
                  int64_t ld_y, float* mean, float* rstd, cudaStream_t s) {
  const NormShape n = norm_shape(width, V, many_rows(rows) ? 32 : 8, 32);
  if (n.nv == 0) {
    norm_fwd_wide_kernel<T, W><<<(unsigned)rows, kMaxThreads, 0, s>>>(x, ld_x, w, b, eps, y, ld_y, mean, rstd, width);
    return cudaGetLastError();
  }
  const int ty = norm_groups(rows, n, V);
  const unsigned grid = (unsigned)norm_ctas(rows, n, V, ty);
  return with_nv(n.nv, [&](auto nv) {
    constexpr int NV = decltype(nv)::value, DEPTH = NV * V * sizeof(T) > 64 ? 3 : 4;
    if constexpr (NV * V <= 32 && NV * V > 1) {
      const int smem = DEPTH * NV * n.tx * ty * Rows<T, V, NV, DEPTH, false>::kSlot;
      return with_full<V>(width == (int64_t)n.tx * NV * V, [&](auto full) {
        static std::atomic<uint64_t> set{0};
        const auto kernel = norm_fwd_kernel<T, W, V, NV, DEPTH, decltype(full)::value>;
        const cudaError_t e = allow_smem(kernel, smem, set);
        if (e != cudaSuccess) return e;
        kernel<<<grid, dim3(n.tx, ty), smem, s>>>(x, ld_x, w, b, eps, y, ld_y, mean, rstd, rows, (int)width);
        return cudaGetLastError();
      });
    }
    return cudaErrorInvalidValue;
  });
}

template <typename T, typename W>
cudaError_t fwd_t(int64_t rows, int64_t width, const void* x, int64_t ld_x, const void* w, const void* b, float eps,
                  void* y, int64_t ld_y, float* mean, float* rstd, cudaStream_t s) {
  const uintptr_t bytes = address(x) | address(y) | (ld_x | ld_y | width) * sizeof(T);
  return with_access<T>(bytes, [&](auto v) {
    return fwd_v<T, W, decltype(v)::value>(rows, width, static_cast<const T*>(x), ld_x, static_cast<const W*>(w),
                                           static_cast<const W*>(b), eps, static_cast<T*>(y), ld_y, mean, rstd, s);
  });
}

template <typename T, typename W, int V>
cudaError_t bwd_v(int64_t rows, int64_t width, const T* dy, int64_t ld_dy, const T* x, int64_t ld_x,
                  const float* mean, const float* rstd, const W* w, T* dx, int64_t ld_dx, float* dw, float* db,
                  float* part, cudaStream_t s) {
  const NormShape n = norm_shape(width, V, many_rows(rows) ? 16 : 8, sizeof(T) == 2 ? 32 : 16);
  float* p = dw || db ? part : nullptr;
  int parts = (int)std::min<int64_t>(kSms, rows);
  cudaError_t e;
  if (n.nv == 0) {
    if (p)
      norm_cols_wide_kernel<T><<<dim3((unsigned)((width + 255) / 256), parts), 256, 0, s>>>(dy, ld_dy, x, ld_x, mean,
                                                                                           rstd, p, rows, width);
    norm_bwd_wide_kernel<T, W><<<(unsigned)rows, kMaxThreads, 0, s>>>(dy, ld_dy, x, ld_x, mean, rstd, w, dx, ld_dx,
                                                                     width);
    e = cudaGetLastError();
  } else {
    const int ty = norm_groups(rows, n, V);
    parts = norm_ctas(rows, n, V, ty);
    e = with_nv(n.nv, [&](auto nv) {
      constexpr int NV = decltype(nv)::value, E = NV * V;
      if constexpr (E <= (sizeof(T) == 2 ? 32 : 16) && E > 1) {
        // two rows at a time where a CTA has few threads per SM and registers for them; at most 192 KB of rows
        constexpr int R = E == 16 && sizeof(T) == 2 ? 2 : 1;
        constexpr int kStage = threads_for(E) * E * (int)sizeof(T) * 2 * R;
        constexpr int DEPTH = E > 16 ? 2 : std::min(4, 192 * 1024 / kStage);
        const int threads = n.tx * ty;
        const int ring = 2 * DEPTH * R * NV * threads * Rows<T, V, NV, DEPTH, false>::kSlot;
        const int smem = std::max(ring + (E > 16 ? (int)width * 4 : 0), threads * E * 4);
        return with_full<V>(width == (int64_t)n.tx * NV * V, [&](auto full) {
          static std::atomic<uint64_t> set{0};
          const auto kernel = norm_bwd_kernel<T, W, V, NV, R, DEPTH, decltype(full)::value>;
          const cudaError_t ae = allow_smem(kernel, smem, set);
          if (ae != cudaSuccess) return ae;
          kernel<<<parts, dim3(n.tx, ty), smem, s>>>(dy, ld_dy, x, ld_x, mean, rstd, w, dx, ld_dx, p, rows, (int)width);
          return cudaGetLastError();
        });
      }
      return cudaErrorInvalidValue;
    });
  }
  if (e != cudaSuccess || !p) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)((width + 31) / 32), 2);
  cfg.blockDim = dim3(32, 32);
  cfg.stream = s;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, norm_cols_kernel, static_cast<const float*>(p), parts, width, dw, db);
}

template <typename T, typename W>
cudaError_t bwd_t(int64_t rows, int64_t width, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x,
                  const float* mean, const float* rstd, const void* w, void* dx, int64_t ld_dx, float* dw, float* db,
                  void* part, cudaStream_t s) {
  const uintptr_t bytes = address(x) | address(dy) | address(dx) | (ld_x | ld_dy | ld_dx | width) * sizeof(T);
  return with_access<T>(bytes, [&](auto v) {
    return bwd_v<T, W, decltype(v)::value>(rows, width, static_cast<const T*>(dy), ld_dy, static_cast<const T*>(x), ld_x,
                                           mean, rstd, static_cast<const W*>(w), static_cast<T*>(dx), ld_dx, dw, db,
                                           static_cast<float*>(part), s);
  });
}

// f(T(), W()) for an activation and a weight type.
template <typename F>
cudaError_t with_types(int32_t xt, int32_t wt, F&& f) {
  if (xt == SOAP_F32) return f(float(), float());
  if (xt == SOAP_BF16)
    return wt == SOAP_F32 ? f(__nv_bfloat16(), float()) : f(__nv_bfloat16(), __nv_bfloat16());
  return wt == SOAP_F32 ? f(__half(), float()) : f(__half(), __half());
}

bool bad_ptr(const void* p, size_t size) { return p && reinterpret_cast<uintptr_t>(p) % size; }

bool bad_norm(int64_t rows, int64_t width, int32_t xt, const void* w, const void* b, int32_t wt) {
  if (rows < 0 || width < 1 || rows > INT32_MAX || width > INT32_MAX) return true;
  if (xt < SOAP_F32 || xt > SOAP_F16 || (wt != SOAP_F32 && wt != xt)) return true;
  return bad_ptr(w, dtype_size(wt)) || bad_ptr(b, dtype_size(wt));
}

bool bad_rows(const void* p, int64_t ld, int64_t rows, int64_t width, int32_t t) {
  return rows > 0 && (!p || bad_ptr(p, dtype_size(t)) || ld < width);
}

}  // namespace
}  // namespace soap

using namespace soap;

extern "C" {

soap_status_t layer_norm_forward(int64_t rows, int64_t width, const void* x, int64_t ld_x, int32_t x_type,
                                 const void* weight, const void* bias, int32_t w_type, float eps, void* y,
                                 int64_t ld_y, float* mean, float* rstd, soap_stream_t stream) {
  if (bad_norm(rows, width, x_type, weight, bias, w_type) || !(eps >= 0.f)) return SOAP_ERR_INVALID_ARG;
  if (bad_rows(x, ld_x, rows, width, x_type) || bad_rows(y, ld_y, rows, width, x_type)) return SOAP_ERR_INVALID_ARG;
  if (bad_ptr(mean, 4) || bad_ptr(rstd, 4)) return SOAP_ERR_INVALID_ARG;
  if (rows == 0) return SOAP_OK;
  const double n = (double)rows * width;
  ProfScope prof(kFamElementwise, 8.0 * n, 2.0 * n * dtype_size(x_type), (cudaStream_t)stream);
  const cudaError_t e = with_types(x_type, w_type, [&](auto t, auto w) {
    return fwd_t<decltype(t), decltype(w)>(rows, width, x, ld_x, weight, bias, eps, y, ld_y, mean, rstd,
                                           (cudaStream_t)stream);
  });
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

size_t layer_norm_workspace_bytes(int64_t rows, int64_t width) {
  if (rows <= 0 || width <= 0 || rows > INT32_MAX || width > INT32_MAX) return 0;
  return (size_t)std::min<int64_t>(kParts, rows) * 2 * (size_t)width * sizeof(float);
}

soap_status_t layer_norm_backward(int64_t rows, int64_t width, const void* dy, int64_t ld_dy, const void* x,
                                  int64_t ld_x, int32_t x_type, const float* mean, const float* rstd,
                                  const void* weight, int32_t w_type, void* dx, int64_t ld_dx, float* dweight,
                                  float* dbias, void* workspace, size_t workspace_bytes, soap_stream_t stream) {
  if (bad_norm(rows, width, x_type, weight, nullptr, w_type)) return SOAP_ERR_INVALID_ARG;
  if (bad_rows(dy, ld_dy, rows, width, x_type) || bad_rows(x, ld_x, rows, width, x_type) ||
      bad_rows(dx, ld_dx, rows, width, x_type))
    return SOAP_ERR_INVALID_ARG;
  if (bad_ptr(mean, 4) || bad_ptr(rstd, 4) || bad_ptr(dweight, 4) || bad_ptr(dbias, 4)) return SOAP_ERR_INVALID_ARG;
  if (rows > 0 && (!mean || !rstd)) return SOAP_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  if (rows == 0) {
    cudaError_t e = cudaSuccess;
    if (dweight) e = cudaMemsetAsync(dweight, 0, (size_t)width * 4, s);
    if (e == cudaSuccess && dbias) e = cudaMemsetAsync(dbias, 0, (size_t)width * 4, s);
    return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
  }
  if ((dweight || dbias) && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 ||
                             workspace_bytes < layer_norm_workspace_bytes(rows, width)))
    return SOAP_ERR_INVALID_ARG;
  const double n = (double)rows * width;
  ProfScope prof(kFamElementwise, 12.0 * n, 3.0 * n * dtype_size(x_type), s);
  const cudaError_t e = with_types(x_type, w_type, [&](auto t, auto w) {
    return bwd_t<decltype(t), decltype(w)>(rows, width, dy, ld_dy, x, ld_x, mean, rstd, weight, dx, ld_dx, dweight,
                                           dbias, workspace, s);
  });
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

}  // extern "C"
