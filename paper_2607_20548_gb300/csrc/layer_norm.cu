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

constexpr int kMaxThreads = 512;
constexpr int kElems = 16;  // most elements of a row per thread

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
  float2* buf;  // [2][blockDim.y][16]
  int half = 0;
  // Afterwards lane l holds warp l's values ((0, 0) from the last warp on).
  __device__ __forceinline__ float2 all(float x, float y) {
    float2* p = buf + (half * blockDim.y + threadIdx.y) * 16;
    half ^= 1;
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
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
template <typename T, int V, int NV, int DEPTH>
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
        if (c < width) copy_async<V * sizeof(T)>(slot(s, i), base + row * ld + c);
      }
    }
  }
  __device__ __forceinline__ void get(int64_t row, int s, int width, Pack<T, V> (&p)[NV]) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * V;
      if (c < width)
        p[i] = kAsync ? *reinterpret_cast<const Pack<T, V>*>(slot(s, i))
                      : *reinterpret_cast<const Pack<T, V>*>(base + row * ld + c);
    }
  }
};

__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void arrived() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// ---- forward: a group of blockDim.x threads per row, NV packs of V elements each ------------

template <typename T, typename W, int V, int NV, int DEPTH>
__global__ void __launch_bounds__(kMaxThreads)
    norm_fwd_kernel(const T* x, int64_t ld_x, const W* weight, const W* bias, float eps, T* y, int64_t ld_y,
                    float* mean, float* rstd, int64_t rows, int width) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float2 buf[2 * 16 * 16];
  constexpr int E = NV * V;
  using R = Rows<T, V, NV, DEPTH>;
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
  float w[E], b[E];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      w[i * V + e] = weight && c < width ? to_f32(weight[c + e]) : 1.f;
      b[i * V + e] = bias && c < width ? to_f32(bias[c + e]) : 0.f;
    }
  }
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
  int s = 0;
  for (; row < rows; row += step) {
    const int64_t ahead = row + (DEPTH - 1) * step;
    if (ahead < rows) in.request(ahead, s == 0 ? DEPTH - 1 : s - 1, width);
    commit();
    arrived<DEPTH - 1>();
    Pack<T, V> p[NV];
    in.get(row, s, width, p);
    s = s + 1 == DEPTH ? 0 : s + 1;
    // sum and spread of the warp's elements about the warp's mean, then over the warps
    float v[E], sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const bool in_row = (int)(i * blockDim.x + threadIdx.x) * V < width;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        v[i * V + e] = in_row ? to_f32(p[i].v[e]) : 0.f;
        sum += v[i * V + e];
      }
    }
    sum = warp_sum(sum);
    float mu = sum * inv_here, q = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const bool in_row = (int)(i * blockDim.x + threadIdx.x) * V < width;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = v[i * V + e] - mu;
        if (in_row) q = fmaf(d, d, q);
      }
    }
    q = warp_sum(q);
    if (blockDim.x > 32) {
      const float2 o = ex.all(sum, q);
      mu = warp_sum(o.x) * inv;
      const float d = o.x * inv_there - mu;
      q = warp_sum(fmaf(there * d, d, o.y));
    }
    const float rs = 1.f / sqrtf(q * inv + eps);
    if (threadIdx.x == 0) {
      if (mean) mean[row] = mu;
      if (rstd) rstd[row] = rs;
    }
    T* yr = y + row * ld_y;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * V;
      if (c >= width) break;
      Pack<T, V> o;
#pragma unroll
      for (int e = 0; e < V; ++e) o.v[e] = from_f32<T>(fmaf((v[i * V + e] - mu) * rs, w[i * V + e], b[i * V + e]));
      *reinterpret_cast<Pack<T, V>*>(yr + c) = o;
    }
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
  const float rs = 1.f / sqrtf(q[0] / (float)width + eps);
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

template <typename T, typename W, int V, int NV, int DEPTH>
__global__ void __launch_bounds__(kMaxThreads)
    norm_bwd_kernel(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, const float* mean, const float* rstd,
                    const W* weight, T* dx, int64_t ld_dx, float* part, int64_t rows, int width) {
  extern __shared__ __align__(16) uint8_t smem[];  // the rings; afterwards the groups' column sums
  __shared__ float2 buf[2 * 16 * 16];
  constexpr int E = NV * V;
  using R = Rows<T, V, NV, DEPTH>;
  const int threads = blockDim.x * blockDim.y, tid = threadIdx.y * blockDim.x + threadIdx.x;
  const R rx{x, ld_x, smem + (size_t)tid * R::kSlot};
  const R rg{dy, ld_dy, smem + (size_t)(DEPTH * NV * threads + tid) * R::kSlot};
  Exchange ex{buf};
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
#pragma unroll
  for (int s = 0; s < DEPTH - 1; ++s) {
    if (row + s * step < rows) {
      rx.request(row + s * step, s, width);
      rg.request(row + s * step, s, width);
    }
    commit();
  }
  float w[E], aw[E], ab[E];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      w[i * V + e] = weight && c < width ? to_f32(weight[c + e]) : 1.f;
      aw[i * V + e] = ab[i * V + e] = 0.f;
    }
  }
  const float inv = 1.f / (float)width;
  float mu = 0.f, rs = 0.f;
  if (row < rows) {
    mu = mean[row];
    rs = rstd[row];
  }
  int s = 0;
  while (row < rows) {
    const int64_t ahead = row + (DEPTH - 1) * step;
    if (ahead < rows) {
      const int to = s == 0 ? DEPTH - 1 : s - 1;
      rx.request(ahead, to, width);
      rg.request(ahead, to, width);
    }
    commit();
    arrived<DEPTH - 1>();
    Pack<T, V> px[NV], pg[NV];
    rx.get(row, s, width, px);
    rg.get(row, s, width, pg);
    s = s + 1 == DEPTH ? 0 : s + 1;
    const int64_t next = row + step;
    float mu_next = 0.f, rs_next = 0.f;
    if (next < rows) {
      mu_next = mean[next];
      rs_next = rstd[next];
    }
    float xh[E], g[E], s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const bool in_row = (int)(i * blockDim.x + threadIdx.x) * V < width;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int k = i * V + e;
        const float d = in_row ? to_f32(pg[i].v[e]) : 0.f;
        xh[k] = in_row ? (to_f32(px[i].v[e]) - mu) * rs : 0.f;
        g[k] = d * w[k];
        s0 += g[k];
        s1 = fmaf(g[k], xh[k], s1);
        aw[k] = fmaf(d, xh[k], aw[k]);
        ab[k] += d;
      }
    }
    s0 = warp_sum(s0);
    s1 = warp_sum(s1);
    if (blockDim.x > 32) {
      const float2 o = ex.all(s0, s1);
      s0 = warp_sum(o.x);
      s1 = warp_sum(o.y);
    }
    const float m1 = s0 * inv, m2 = s1 * inv;
    T* dr = dx + row * ld_dx;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * V;
      if (c >= width) break;
      Pack<T, V> o;
#pragma unroll
      for (int e = 0; e < V; ++e) o.v[e] = from_f32<T>(rs * (g[i * V + e] - m1 - xh[i * V + e] * m2));
      *reinterpret_cast<Pack<T, V>*>(dr + c) = o;
    }
    row = next;
    mu = mu_next;
    rs = rs_next;
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
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e)
        sums[threadIdx.y * lanes + (i * blockDim.x + threadIdx.x) * V + e] = k == 0 ? aw[i * V + e] : ab[i * V + e];
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

constexpr int kParts = 152;  // most partial rows: one CTA per SM

struct NormShape {
  int nv, tx;  // accesses per thread and row, threads per row
};

// Threads for a row of `width` elements in accesses of v: at most 16 elements per thread, so that a
// thread's columns and both of their sums stay in registers; nv = 0: too wide for that. Rows that a
// warp or two can hold take fewer elements per thread.
NormShape norm_shape(int64_t width, int v) {
  const int64_t packs = (width + v - 1) / v;
  const int most = kElems / v;
  for (int nv = 1; nv <= most; nv *= 2)
    for (int tx = 32; tx <= kMaxThreads; tx *= 2)
      if (packs <= (int64_t)tx * nv && (nv == most || tx <= 64)) return {nv, tx};
  return {0, 0};
}

// Rows per CTA: full CTAs, unless the rows would then not reach every SM.
int norm_groups(int64_t rows, int tx) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(kMaxThreads / tx, (rows + kParts - 1) / kParts));
}

template <typename F>
cudaError_t with_nv(int nv, F&& f) {
  switch (nv) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 4: return f(std::integral_constant<int, 4>());
    case 8: return f(std::integral_constant<int, 8>());
    default: return f(std::integral_constant<int, 16>());
  }
}

// f(elements per access): the widest access of up to 16 bytes that `bytes` (an OR of all addresses and
// row lengths in bytes) divides into.
template <typename T, typename F>
cudaError_t with_access(uintptr_t bytes, F&& f) {
  if (bytes % 16 == 0) return f(std::integral_constant<int, 16 / sizeof(T)>());
  if (bytes % 8 == 0) return f(std::integral_constant<int, 8 / sizeof(T)>());
  if (sizeof(T) < 4 && bytes % 4 == 0) return f(std::integral_constant<int, std::max<int>(1, 4 / sizeof(T))>());
  return f(std::integral_constant<int, 1>());
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
  const NormShape n = norm_shape(width, V);
  if (n.nv == 0) {
    norm_fwd_wide_kernel<T, W><<<(unsigned)rows, kMaxThreads, 0, s>>>(x, ld_x, w, b, eps, y, ld_y, mean, rstd, width);
    return cudaGetLastError();
  }
  const int ty = norm_groups(rows, n.tx);
  const unsigned grid = (unsigned)std::min<int64_t>(kParts, (rows + ty - 1) / ty);
  return with_nv(n.nv, [&](auto nv) {
    constexpr int NV = decltype(nv)::value, DEPTH = 4;
    if constexpr (NV * V <= kElems) {
      static std::atomic<uint64_t> set{0};
      const int smem = DEPTH * NV * n.tx * ty * Rows<T, V, NV, DEPTH>::kSlot;
      const cudaError_t e = allow_smem(norm_fwd_kernel<T, W, V, NV, DEPTH>, smem, set);
      if (e != cudaSuccess) return e;
      norm_fwd_kernel<T, W, V, NV, DEPTH>
          <<<grid, dim3(n.tx, ty), smem, s>>>(x, ld_x, w, b, eps, y, ld_y, mean, rstd, rows, (int)width);
    }
    return cudaGetLastError();
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
  const NormShape n = norm_shape(width, V);
  float* p = dw || db ? part : nullptr;
  int parts = (int)std::min<int64_t>(kParts, rows);
  cudaError_t e;
  if (n.nv == 0) {
    if (p)
      norm_cols_wide_kernel<T><<<dim3((unsigned)((width + 255) / 256), parts), 256, 0, s>>>(dy, ld_dy, x, ld_x, mean,
                                                                                           rstd, p, rows, width);
    norm_bwd_wide_kernel<T, W><<<(unsigned)rows, kMaxThreads, 0, s>>>(dy, ld_dy, x, ld_x, mean, rstd, w, dx, ld_dx,
                                                                     width);
    e = cudaGetLastError();
  } else {
    const int ty = norm_groups(rows, n.tx);
    parts = (int)std::min<int64_t>(kParts, (rows + ty - 1) / ty);
    e = with_nv(n.nv, [&](auto nv) {
      constexpr int NV = decltype(nv)::value, DEPTH = sizeof(T) == 4 ? 3 : 4;
      if constexpr (NV * V <= kElems) {
        static std::atomic<uint64_t> set{0};
        const int threads = n.tx * ty;
        const int smem = threads * NV * std::max<int>(2 * DEPTH * Rows<T, V, NV, DEPTH>::kSlot, V * 4);
        const cudaError_t ae = allow_smem(norm_bwd_kernel<T, W, V, NV, DEPTH>, smem, set);
        if (ae != cudaSuccess) return ae;
        norm_bwd_kernel<T, W, V, NV, DEPTH><<<parts, dim3(n.tx, ty), smem, s>>>(dy, ld_dy, x, ld_x, mean, rstd, w, dx,
                                                                                ld_dx, p, rows, (int)width);
      }
      return cudaGetLastError();
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
