// Layer norm of rows (include/layer.h).
//
//   mu = mean(x), rstd = 1 / sqrt(mean((x - mu)^2) + eps), y = (x - mu) rstd w + b
#include "layer_norm.h"

namespace soap {
namespace {

// ---- forward: a group of blockDim.x threads per row, NV packs of V elements each ------------

// FULL: the group's threads have exactly the row's elements.
template <typename T, typename W, int V, int NV, int DEPTH, bool FULL, bool RING>
__global__ void __launch_bounds__(threads_for(NV * V), 1)
    norm_fwd_kernel(const T* x, int64_t ld_x, const W* weight, const W* bias, float eps, T* y, int64_t ld_y,
                    float* mean, float* rstd, int rows, int width, int* status, const WaitLimit wait) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float2 buf[2 * 32];
  __shared__ uint64_t full[kMaxGroups][DEPTH];
  constexpr int P = NV * V / 2, kPer = V == 1 ? 2 : 1;
  using Feed = Rows<T, V, NV, 1, DEPTH, FULL, RING>;
  const int lane = threadIdx.x & 31;
  Exchange ex{buf};
  const int step = gridDim.x * blockDim.y;
  int row = blockIdx.x * blockDim.y + threadIdx.y;
  Feed in{{x}, {ld_x}, rows, step, width, smem + threadIdx.y * Feed::ring_bytes(blockDim.x), full[threadIdx.y], status, wait};
  in.start(row);
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
  for (; row < rows; row += step) {
    Pack<T, V> raw[1][NV];
    in.get(row, raw);
    float2 v[P];
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = values(raw[0], i);
    // sum and spread of the warp's elements about the warp's mean, then over the warps
    float2 acc = pair(0.f);
#pragma unroll
    for (int i = 0; i < P; ++i) acc = add2(acc, v[i]);
    float sum = warp_sum(in.dead() ? NAN : acc.x + acc.y);
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
    } else {
      __syncwarp();
    }
    in.refill(row);
    const float rs = rsqrtf(q * inv + eps);
    if (threadIdx.x == 0) {
      if (mean) mean[row] = mu;
      if (rstd) rstd[row] = rs;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = fma2(mul2(add2(v[i], pair(-mu)), pair(rs)), w[i], b[i]);
#pragma unroll
    for (int i = 0; i < NV; i += kPer) put<T, V, FULL>(y + (int64_t)row * ld_y, width, i, v + i * V / 2);
  }
  in.finish();
}

// Rows too wide for registers: one CTA per row, three passes over the row.
template <typename T, typename W>
__global__ void __launch_bounds__(kMaxThreads)
    norm_fwd_wide_kernel(const T* x, int64_t ld_x, const W* weight, const W* bias, float eps, T* y, int64_t ld_y,
                         float* mean, float* rstd, int64_t width) {
  __shared__ float buf[32];
  const int64_t row = blockIdx.x;
  const T* xr = x + row * ld_x;
  T* yr = y + (int64_t)row * ld_y;
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

template <typename T, typename W, int V>
cudaError_t fwd_v(int64_t rows, int64_t width, const T* x, int64_t ld_x, const W* w, const W* b, float eps, T* y,
                  int64_t ld_y, float* mean, float* rstd, int* status, cudaStream_t s) {
  const NormShape n = norm_shape(width, V, !many_rows(rows) ? 8 : V * sizeof(T) == 16 ? 32 : 16, 32);
  if (n.nv == 0) {
    norm_fwd_wide_kernel<T, W><<<(unsigned)rows, kMaxThreads, 0, s>>>(x, ld_x, w, b, eps, y, ld_y, mean, rstd, width);
    return cudaGetLastError();
  }
  const int ty = norm_groups(rows, n, V);
  const unsigned grid = (unsigned)norm_ctas(rows, n, V, ty);
  return with_nv(n.nv, [&](auto nv) {
    constexpr int NV = decltype(nv)::value, DEPTH = NV * V * sizeof(T) > 64 ? 3 : 4;
    if constexpr (NV * V <= 32 && NV * V > 1) {
      return with_full<V, NV * V>(width == (int64_t)n.tx * NV * V, n.tx, [&](auto full, auto ring) {
        static std::atomic<uint64_t> set{0};
        constexpr bool kFull = decltype(full)::value, kRing = decltype(ring)::value;
        const int smem = ty * Rows<T, V, NV, 1, DEPTH, kFull, kRing>::ring_bytes(n.tx);
        const auto kernel = norm_fwd_kernel<T, W, V, NV, DEPTH, kFull, kRing>;
        const cudaError_t e = allow_smem(kernel, smem, set);
        if (e != cudaSuccess) return e;
        kernel<<<grid, dim3(n.tx, ty), smem, s>>>(x, ld_x, w, b, eps, y, ld_y, mean, rstd, (int)rows, (int)width,
                                                  status, wait_limit());
        return cudaGetLastError();
      });
    }
    return cudaErrorInvalidValue;
  });
}

template <typename T, typename W>
cudaError_t fwd_t(int64_t rows, int64_t width, const void* x, int64_t ld_x, const void* w, const void* b, float eps,
                  void* y, int64_t ld_y, float* mean, float* rstd, int* status, cudaStream_t s) {
  const uintptr_t bytes = address(x) | address(y) | (ld_x | ld_y | width) * sizeof(T);
  return with_access<T>(bytes, [&](auto v) {
    return fwd_v<T, W, decltype(v)::value>(rows, width, static_cast<const T*>(x), ld_x, static_cast<const W*>(w),
                                           static_cast<const W*>(b), eps, static_cast<T*>(y), ld_y, mean, rstd, status,
                                           s);
  });
}

}  // namespace
}  // namespace soap

using namespace soap;

extern "C" {

soap_status_t layer_norm_forward(int64_t rows, int64_t width, const void* x, int64_t ld_x, int32_t x_type,
                                 const void* weight, const void* bias, int32_t w_type, float eps, void* y,
                                 int64_t ld_y, float* mean, float* rstd, int32_t* status,
                                 soap_stream_t stream) {
  if (bad_norm(rows, width, x_type, weight, bias, w_type) || !(eps >= 0.f)) return SOAP_ERR_INVALID_ARG;
  if (bad_rows(x, ld_x, rows, width, x_type) || bad_rows(y, ld_y, rows, width, x_type)) return SOAP_ERR_INVALID_ARG;
  if (bad_ptr(mean, 4) || bad_ptr(rstd, 4) || bad_ptr(status, 4)) return SOAP_ERR_INVALID_ARG;
  if (rows == 0) return SOAP_OK;
  const double n = (double)rows * width;
  ProfScope prof(kFamElementwise, 8.0 * n, 2.0 * n * dtype_size(x_type), (cudaStream_t)stream);
  const cudaError_t e = with_types(x_type, w_type, [&](auto t, auto w) {
    return fwd_t<decltype(t), decltype(w)>(rows, width, x, ld_x, weight, bias, eps, y, ld_y, mean, rstd, status,
                                           (cudaStream_t)stream);
  });
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

}  // extern "C"
