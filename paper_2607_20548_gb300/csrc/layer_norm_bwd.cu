// The backward pass of layer norm (include/layer.h).
//
//   g = dy w, xh = (x - mu) rstd, dx = rstd (g - mean(g) - xh mean(g xh)),
//   dw = sum_rows dy xh, db = sum_rows dy
#include "layer_norm.h"

namespace soap {
namespace {

// ---- backward ------------------------------------------------------------------------------
// Persistent CTAs walk the rows; each thread keeps its columns' sums of dy xh and dy in
// registers, the CTA adds its groups' sums at the end and writes one partial row per sum, and
// norm_cols_kernel adds the partial rows in order (no atomics: the result does not depend on
// which CTA finishes first).

// A thread keeps its row's packs and converts them twice. Weights that registers would not hold beside
// both sums (more than 16 elements per thread) are in shared memory. (Two rows per iteration spilled
// registers: 360 us in place of 258 at 32768 x 8192.)
template <typename T, typename W, int V, int NV, int DEPTH, bool FULL, bool RING>
__global__ void __launch_bounds__(threads_for(NV * V), 1)
    norm_bwd_kernel(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, const float* mean, const float* rstd,
                    const W* weight, T* dx, int64_t ld_dx, float* part, int rows, int width,
                    int* status, const WaitLimit wait) {
  extern __shared__ __align__(16) uint8_t smem[];  // the rings (and weights); afterwards the groups' column sums
  __shared__ float2 buf[2 * 32];
  __shared__ uint64_t full[kMaxGroups][DEPTH];
  constexpr int E = NV * V, P = E / 2, kPer = V == 1 ? 2 : 1;
  constexpr bool kSmemW = E > 16;
  using Feed = Rows<T, V, NV, 2, DEPTH, FULL, RING>;
  const int threads = blockDim.x * blockDim.y, tid = threadIdx.y * blockDim.x + threadIdx.x;
  // [P][blockDim.x]
  float2* const weights = reinterpret_cast<float2*>(smem + blockDim.y * Feed::ring_bytes(blockDim.x));
  const int step = gridDim.x * blockDim.y;
  int row = blockIdx.x * blockDim.y + threadIdx.y;
  Feed in{{x, dy},    {ld_x, ld_dy}, rows,
          step,       width,         smem + threadIdx.y * Feed::ring_bytes(blockDim.x),
          full[threadIdx.y], status, wait};
  in.start(row);
  Exchange ex{buf};
  float2 w[kSmemW ? 1 : P], aw[P], ab[P];
  if constexpr (kSmemW) {
    if (threadIdx.y == 0) {
      float2 t[P];
      columns<W, V, NV>(weight, 1.f, width, t);
#pragma unroll
      for (int i = 0; i < P; ++i) weights[i * blockDim.x + threadIdx.x] = t[i];
    }
    __syncthreads();
  } else {
    columns<W, V, NV>(weight, 1.f, width, w);
  }
#pragma unroll
  for (int i = 0; i < P; ++i) aw[i] = ab[i] = pair(0.f);
  // weights of elements 2 k and 2 k + 1
  auto weight_of = [&](int k) {
    if constexpr (kSmemW)
      return weights[k * blockDim.x + threadIdx.x];
    else
      return w[k];
  };
  const float inv = 1.f / (float)width;
  float mu = 0.f, rs = 0.f;
  if (row < rows) {
    mu = mean[row];
    rs = rstd[row];
  }
  while (row < rows) {
    const int next = row + step;
    float mu_next = 0.f, rs_next = 0.f;
    if (next < rows) {
      mu_next = mean[next];
      rs_next = rstd[next];
    }
    Pack<T, V> p[2][NV];  // x, dy
    in.get(row, p);
    // beyond the row's end dy is zero, so whatever xh is there counts nowhere
    float2 a0 = pair(0.f), a1 = pair(0.f);
#pragma unroll
    for (int k = 0; k < P; ++k) {
      const float2 xh = mul2(add2(values(p[0], k), pair(-mu)), pair(rs));
      float2 g = values(p[1], k);
      aw[k] = fma2(g, xh, aw[k]);
      ab[k] = add2(ab[k], g);
      g = mul2(g, weight_of(k));
      a0 = add2(a0, g);
      a1 = fma2(g, xh, a1);
    }
    float s0 = warp_sum(in.dead() ? NAN : a0.x + a0.y), s1 = warp_sum(a1.x + a1.y);
    if (blockDim.x > 32) {
      const float2 o = ex.all(s0, s1);
      s0 = warp_sum(o.x);
      s1 = warp_sum(o.y);
    } else {
      __syncwarp();
    }
    in.refill(row);
    const float2 m1 = pair(-s0 * inv * rs), m2 = pair(-s1 * inv * rs);
#pragma unroll
    for (int i = 0; i < NV; i += kPer) {
      float2 g[kPer * V / 2];
#pragma unroll
      for (int j = 0; j < kPer * V / 2; ++j) {
        const int k = i * V / 2 + j;
        const float2 xh = mul2(add2(values(p[0], k), pair(-mu)), pair(rs));
        g[j] = fma2(xh, m2, fma2(mul2(values(p[1], k), weight_of(k)), pair(rs), m1));
      }
      put<T, V, FULL>(dx + (int64_t)row * ld_dx, width, i, g);
    }
    row = next;
    mu = mu_next;
    rs = rs_next;
  }
  in.finish();
  if (!part) return;
  // add the groups in order, first dweight's sums, then dbias's
  float* sums = reinterpret_cast<float*>(smem);
  const int lanes = blockDim.x * E;
  const bool none = __syncthreads_or(in.dead());  // (the rings have been read)
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
      out[c] = none ? NAN : t;
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
  asm volatile("griddepcontrol.wait;" ::: "memory");  // launched ahead: it starts as the last CTAs of the kernel before exit
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

template <typename T, typename W, int V>
cudaError_t bwd_v(int64_t rows, int64_t width, const T* dy, int64_t ld_dy, const T* x, int64_t ld_x,
                  const float* mean, const float* rstd, const W* w, T* dx, int64_t ld_dx, float* dw, float* db,
                  float* part, int* status, cudaStream_t s) {
  constexpr int kMost = V == 8 ? 32 : 16;  // elements per thread: beyond, registers spill
  const NormShape n = norm_shape(width, V, many_rows(rows) ? 16 : 8, kMost);
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
      if constexpr (E <= kMost && E > 1) {
        constexpr int kStage = threads_for(E) * E * (int)sizeof(T) * 2;
        constexpr int DEPTH = E > 16 ? 2 : std::min(4, 192 * 1024 / kStage);  // at most 192 KB of rows
        const int threads = n.tx * ty;
        return with_full<V, E>(width == (int64_t)n.tx * NV * V, n.tx, [&](auto full, auto in_ring) {
          static std::atomic<uint64_t> set{0};
          constexpr bool kFull = decltype(full)::value, kRing = decltype(in_ring)::value;
          const int ring = ty * Rows<T, V, NV, 2, DEPTH, kFull, kRing>::ring_bytes(n.tx);
          const int smem = std::max(ring + (E > 16 ? n.tx * E * 4 : 0), threads * E * 4);
          const auto kernel = norm_bwd_kernel<T, W, V, NV, DEPTH, kFull, kRing>;
          const cudaError_t ae = allow_smem(kernel, smem, set);
          if (ae != cudaSuccess) return ae;
          kernel<<<parts, dim3(n.tx, ty), smem, s>>>(dy, ld_dy, x, ld_x, mean, rstd, w, dx, ld_dx, p, (int)rows,
                                                     (int)width, status, wait_limit());
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
                  void* part, int* status, cudaStream_t s) {
  const uintptr_t bytes = address(x) | address(dy) | address(dx) | (ld_x | ld_dy | ld_dx | width) * sizeof(T);
  return with_access<T>(bytes, [&](auto v) {
    return bwd_v<T, W, decltype(v)::value>(rows, width, static_cast<const T*>(dy), ld_dy, static_cast<const T*>(x),
                                           ld_x, mean, rstd, static_cast<const W*>(w), static_cast<T*>(dx), ld_dx, dw,
                                           db, static_cast<float*>(part), status, s);
  });
}

}  // namespace
}  // namespace soap

using namespace soap;

extern "C" {

size_t layer_norm_workspace_bytes(int64_t rows, int64_t width) {
  if (rows <= 0 || width <= 0 || rows > kMaxRows || width > INT32_MAX) return 0;
  return (size_t)std::min<int64_t>(kParts, rows) * 2 * (size_t)width * sizeof(float);
}

soap_status_t layer_norm_backward(int64_t rows, int64_t width, const void* dy, int64_t ld_dy, const void* x,
                                  int64_t ld_x, int32_t x_type, const float* mean, const float* rstd,
                                  const void* weight, int32_t w_type, void* dx, int64_t ld_dx, float* dweight,
                                  float* dbias, void* workspace, size_t workspace_bytes, int32_t* status,
                                  soap_stream_t stream) {
  if (bad_norm(rows, width, x_type, weight, nullptr, w_type)) return SOAP_ERR_INVALID_ARG;
  if (bad_rows(dy, ld_dy, rows, width, x_type) || bad_rows(x, ld_x, rows, width, x_type) ||
      bad_rows(dx, ld_dx, rows, width, x_type))
    return SOAP_ERR_INVALID_ARG;
  if (bad_ptr(mean, 4) || bad_ptr(rstd, 4) || bad_ptr(dweight, 4) || bad_ptr(dbias, 4) || bad_ptr(status, 4))
    return SOAP_ERR_INVALID_ARG;
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
                                           dbias, workspace, status, s);
  });
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

}  // extern "C"
