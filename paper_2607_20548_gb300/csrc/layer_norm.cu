// Layer norm of rows and its backward pass (include/layer.h).
//
//   mu = mean(x), rstd = 1 / sqrt(mean((x - mu)^2) + eps), y = (x - mu) rstd w + b
//   g = dy w, xh = (x - mu) rstd, dx = rstd (g - mean(g) - xh mean(g xh)),
//   dw = sum_rows dy xh, db = sum_rows dy
//
// Bound by memory: x is read and y written once (backward: x and dy read, dx written once). A
// group of threads holds a row in registers, so that the variance is a second pass over
// registers (not E[x^2] - mu^2, which cancels) and nothing is read twice.
#include <algorithm>
#include <cstdint>

#include "../../include/layer.h"
#include "profile.h"
#include "types.h"

namespace soap {
namespace {

constexpr int kMaxThreads = 512;

// Sum over a row group's threads (blockDim.x of them, a multiple of 32 when more than a warp).
// `slot` alternates between the two halves of `buf`, so that one barrier per call is enough: a
// thread writes a half again only after the barrier of the call in between.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* buf, int& slot) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if (blockDim.x <= 32) return;
  const int nw = blockDim.x >> 5, w = threadIdx.x >> 5;
  float* p = buf + ((slot * blockDim.y + threadIdx.y) * 32) * N;
  slot ^= 1;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) p[w * N + i] = v[i];
  asm volatile("bar.sync %0, %1;" ::"r"((int)threadIdx.y + 1), "r"((int)blockDim.x) : "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.f;
  for (int j = 0; j < nw; ++j)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += p[j * N + i];
}

// ---- forward: a group of blockDim.x threads per row, NV packs of V elements each ------------

template <typename T, typename W, int V, int NV>
__global__ void __launch_bounds__(kMaxThreads)
    norm_fwd_kernel(const T* x, int64_t ld_x, const W* weight, const W* bias, float eps, T* y, int64_t ld_y,
                    float* mean, float* rstd, int64_t rows, int width) {
  __shared__ float buf[2 * 16 * 32];
  int slot = 0;
  const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= rows) return;
  const T* xr = x + row * ld_x;
  float v[NV * V];
  float s[1] = {0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * V;
    Pack<T, V> p;
    if (c < width) p = *reinterpret_cast<const Pack<T, V>*>(xr + c);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      v[i * V + e] = c < width ? to_f32(p.v[e]) : 0.f;
      s[0] += v[i * V + e];
    }
  }
  group_sum(s, buf, slot);
  const float mu = s[0] / (float)width;
  float q[1] = {0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const bool in = (i * blockDim.x + threadIdx.x) * V < width;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      v[i * V + e] -= mu;
      if (in) q[0] = fmaf(v[i * V + e], v[i * V + e], q[0]);
    }
  }
  group_sum(q, buf, slot);
  const float rs = 1.f / sqrtf(q[0] / (float)width + eps);
  if (threadIdx.x == 0) {
    if (mean) mean[row] = mu;
    if (rstd) rstd[row] = rs;
  }
  T* yr = y + row * ld_y;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * V;
    if (c >= width) break;
    Pack<W, V> w, b;
    if (weight) w = *reinterpret_cast<const Pack<W, V>*>(weight + c);
    if (bias) b = *reinterpret_cast<const Pack<W, V>*>(bias + c);
    Pack<T, V> o;
#pragma unroll
    for (int e = 0; e < V; ++e)
      o.v[e] = from_f32<T>(fmaf(v[i * V + e] * rs, weight ? to_f32(w.v[e]) : 1.f, bias ? to_f32(b.v[e]) : 0.f));
    *reinterpret_cast<Pack<T, V>*>(yr + c) = o;
  }
}

// Rows too wide for registers: one CTA per row, three passes over the row.
template <typename T, typename W>
__global__ void __launch_bounds__(kMaxThreads)
    norm_fwd_wide_kernel(const T* x, int64_t ld_x, const W* weight, const W* bias, float eps, T* y, int64_t ld_y,
                         float* mean, float* rstd, int64_t width) {
  __shared__ float buf[2 * 32];
  int slot = 0;
  const int64_t row = blockIdx.x;
  const T* xr = x + row * ld_x;
  T* yr = y + row * ld_y;
  float s[1] = {0.f}, q[1] = {0.f};
  for (int64_t c = threadIdx.x; c < width; c += blockDim.x) s[0] += to_f32(xr[c]);
  group_sum(s, buf, slot);
  const float mu = s[0] / (float)width;
  for (int64_t c = threadIdx.x; c < width; c += blockDim.x) {
    const float d = to_f32(xr[c]) - mu;
    q[0] = fmaf(d, d, q[0]);
  }
  group_sum(q, buf, slot);
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

template <typename T, typename W, int V, int NV>
__global__ void __launch_bounds__(kMaxThreads)
    norm_bwd_kernel(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, const float* mean, const float* rstd,
                    const W* weight, T* dx, int64_t ld_dx, float* part, int64_t rows, int width) {
  extern __shared__ float sums[];  // one float per thread and element: the groups' column sums
  __shared__ float buf[2 * 16 * 32 * 2];
  constexpr int E = NV * V;
  int slot = 0;
  float w[E], aw[E], ab[E];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      w[i * V + e] = c < width ? (weight ? to_f32(weight[c + e]) : 1.f) : 0.f;
      aw[i * V + e] = ab[i * V + e] = 0.f;
    }
  }
  const float inv = 1.f / (float)width;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  for (int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y; row < rows; row += step) {
    const T *xr = x + row * ld_x, *gr = dy + row * ld_dy;
    Pack<T, V> px[NV], pg[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * V;
      if (c < width) {
        px[i] = *reinterpret_cast<const Pack<T, V>*>(xr + c);
        pg[i] = *reinterpret_cast<const Pack<T, V>*>(gr + c);
      }
    }
    const float mu = mean[row], rs = rstd[row];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const bool in = (i * blockDim.x + threadIdx.x) * V < width;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = in ? to_f32(pg[i].v[e]) : 0.f;
        const float xh = in ? (to_f32(px[i].v[e]) - mu) * rs : 0.f;
        const float g = d * w[i * V + e];
        s[0] += g;
        s[1] = fmaf(g, xh, s[1]);
        aw[i * V + e] = fmaf(d, xh, aw[i * V + e]);
        ab[i * V + e] += d;
      }
    }
    group_sum(s, buf, slot);
    const float m1 = s[0] * inv, m2 = s[1] * inv;
    T* dr = dx + row * ld_dx;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * V;
      if (c >= width) break;
      Pack<T, V> o;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float xh = (to_f32(px[i].v[e]) - mu) * rs;
        o.v[e] = from_f32<T>(rs * (to_f32(pg[i].v[e]) * w[i * V + e] - m1 - xh * m2));
      }
      *reinterpret_cast<Pack<T, V>*>(dr + c) = o;
    }
  }
  if (!part) return;
  // add the groups in order, first dweight's sums, then dbias's
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
    for (int c = threadIdx.y * blockDim.x + threadIdx.x; c < width; c += blockDim.x * blockDim.y) {
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
  __shared__ float buf[2 * 32 * 2];
  int slot = 0;
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
  group_sum(s, buf, slot);
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
  int v, nv, tx, ty;  // elements per access, accesses per thread, threads per row, rows per CTA
};

// Threads for a row of `width` elements in accesses of v: at most 16 elements per thread, so that a
// thread's columns and both of their sums stay in registers; nv = 0: too wide for that.
NormShape norm_shape(int64_t width, int v) {
  const int64_t packs = (width + v - 1) / v;
  const int most = 16 / v;
  for (int nv = 1; nv <= most; nv *= 2)
    for (int tx = 32; tx <= kMaxThreads; tx *= 2)
      if (packs <= (int64_t)tx * nv && (nv == most || tx <= 64)) return {v, nv, tx, std::max(1, 256 / tx)};
  return {v, 0, 0, 0};
}

template <typename F>
auto with_nv(int nv, F&& f) {
  switch (nv) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 4: return f(std::integral_constant<int, 4>());
    case 8: return f(std::integral_constant<int, 8>());
    default: return f(std::integral_constant<int, 16>());
  }
}

bool aligned(const void* p, int64_t ld, size_t size) {
  return (reinterpret_cast<uintptr_t>(p) % 16) == 0 && ((size_t)ld * size) % 16 == 0;
}

template <typename T, typename W, int V>
cudaError_t fwd_v(int64_t rows, int64_t width, const T* x, int64_t ld_x, const W* w, const W* b, float eps, T* y,
                  int64_t ld_y, float* mean, float* rstd, cudaStream_t s) {
  const NormShape n = norm_shape(width, V);
  if (n.nv == 0) {
    norm_fwd_wide_kernel<T, W><<<(unsigned)rows, kMaxThreads, 0, s>>>(x, ld_x, w, b, eps, y, ld_y, mean, rstd, width);
    return cudaGetLastError();
  }
  const unsigned grid = (unsigned)((rows + n.ty - 1) / n.ty);
  const dim3 block(n.tx, n.ty);
  return with_nv(n.nv, [&](auto nv) {
    constexpr int NV = decltype(nv)::value;
    if constexpr (NV * V <= 16)
      norm_fwd_kernel<T, W, V, NV><<<grid, block, 0, s>>>(x, ld_x, w, b, eps, y, ld_y, mean, rstd, rows, (int)width);
    return cudaGetLastError();
  });
}

template <typename T, typename W>
cudaError_t fwd_t(int64_t rows, int64_t width, const void* x, int64_t ld_x, const void* w, const void* b, float eps,
                  void* y, int64_t ld_y, float* mean, float* rstd, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = width % V == 0 && aligned(x, ld_x, sizeof(T)) && aligned(y, ld_y, sizeof(T)) && aligned(w, 0, 1) &&
                   aligned(b, 0, 1);
  const T* xt = static_cast<const T*>(x);
  const W *wt = static_cast<const W*>(w), *bt = static_cast<const W*>(b);
  if (vec) return fwd_v<T, W, V>(rows, width, xt, ld_x, wt, bt, eps, static_cast<T*>(y), ld_y, mean, rstd, s);
  return fwd_v<T, W, 1>(rows, width, xt, ld_x, wt, bt, eps, static_cast<T*>(y), ld_y, mean, rstd, s);
}

int norm_parts(int64_t rows, int ty) {
  return (int)std::min<int64_t>(kParts, (rows + ty - 1) / ty);
}

template <typename T, typename W, int V>
cudaError_t bwd_v(int64_t rows, int64_t width, const T* dy, int64_t ld_dy, const T* x, int64_t ld_x,
                  const float* mean, const float* rstd, const W* w, T* dx, int64_t ld_dx, float* dw, float* db,
                  float* part, cudaStream_t s) {
  NormShape n = norm_shape(width, V);
  float* p = dw || db ? part : nullptr;
  int parts;
  if (n.nv == 0) {
    parts = norm_parts(rows, 1);
    if (p)
      norm_cols_wide_kernel<T><<<dim3((unsigned)((width + 255) / 256), parts), 256, 0, s>>>(dy, ld_dy, x, ld_x, mean,
                                                                                           rstd, p, rows, width);
    norm_bwd_wide_kernel<T, W><<<(unsigned)rows, kMaxThreads, 0, s>>>(dy, ld_dy, x, ld_x, mean, rstd, w, dx, ld_dx,
                                                                     width);
  } else {
    n.ty = std::max(1, kMaxThreads / n.tx);
    parts = norm_parts(rows, n.ty);
    with_nv(n.nv, [&](auto nv) {
      constexpr int NV = decltype(nv)::value;
      if constexpr (NV * V <= 16)
        norm_bwd_kernel<T, W, V, NV><<<parts, dim3(n.tx, n.ty), n.tx * n.ty * NV * V * sizeof(float), s>>>(
            dy, ld_dy, x, ld_x, mean, rstd, w, dx, ld_dx, p, rows, (int)width);
      return 0;
    });
  }
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || !p) return e;
  norm_cols_kernel<<<dim3((unsigned)((width + 31) / 32), 2), dim3(32, 32), 0, s>>>(p, parts, width, dw, db);
  return cudaGetLastError();
}

template <typename T, typename W>
cudaError_t bwd_t(int64_t rows, int64_t width, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x,
                  const float* mean, const float* rstd, const void* w, void* dx, int64_t ld_dx, float* dw, float* db,
                  void* part, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = width % V == 0 && aligned(x, ld_x, sizeof(T)) && aligned(dy, ld_dy, sizeof(T)) &&
                   aligned(dx, ld_dx, sizeof(T));
  const T *xt = static_cast<const T*>(x), *gt = static_cast<const T*>(dy);
  const W* wt = static_cast<const W*>(w);
  T* dt = static_cast<T*>(dx);
  float* pt = static_cast<float*>(part);
  if (vec) return bwd_v<T, W, V>(rows, width, gt, ld_dy, xt, ld_x, mean, rstd, wt, dt, ld_dx, dw, db, pt, s);
  return bwd_v<T, W, 1>(rows, width, gt, ld_dy, xt, ld_x, mean, rstd, wt, dt, ld_dx, dw, db, pt, s);
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
  return (size_t)norm_parts(rows, 1) * 2 * (size_t)width * sizeof(float);
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
