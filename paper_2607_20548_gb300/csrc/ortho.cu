// Stand-alone orthogonalisation by Newton-Schulz products (include/muon.h, muon_orthogonalize):
//
//   X_0 = M / max(||M||_F, eps),   X' = a X + B X,  B = b S + c S^2,  S = X X^T
//
// (X B with S = X^T X for tall matrices: the Gram matrix is always the smaller side's). The steps
// run on X itself, not on S alone: S = X X^T formed afresh stays positive semidefinite to rounding,
// while a recursion in S would square the condition number and let small eigenvalues turn negative,
// where the odd polynomials grow.
//
// Precision. Intermediates are fp16 times a power of two. For bf16 results (8 bits) one fp16 value
// (11 bits) per element leaves the iteration's error below the result's own rounding; fp16 and fp32
// results take hi + lo pairs (22 bits). M enters scaled by a power of two only, which is exact for
// bf16 and fp16 inputs; the remaining factor t in (1, 2] of 1 / max(||M||_F, eps) is applied in
// fp32 in the first step's results.
//
// Range. With sigma <= u before a step, S <= u^2, |B| <= max |b s + c s^2| on [0, u^2] and
// sigma <= max |sigma (a + b sigma^2 + c sigma^4)| after it, all at the ends or at the roots of a
// derivative: each intermediate's scale is the power of two that keeps its bound (twice) inside fp16.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/muon.h"
#include "ortho.h"
#include "profile.h"
#include "soap_internal.h"
#include "types.h"

namespace soap {
namespace ortho {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxParts = 1216;  // partial sums of squares: 8 CTAs per SM, dealt to the matrices

// Squares of a pack's elements: in fp32 where no square underflows and no sum of 2^31 of them
// overflows (or the pack is zero), else in fp64, whose rate is so low that nothing else here uses
// it. NaN and inf come out as such either way.
template <typename T, int V>
__device__ __forceinline__ void add_squares(const Pack<T, V>& p, float& s, double& d) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < V; ++e) m = fmaxf(m, fabsf(to_f32(p.v[e])));
  if (sizeof(T) == 2 && std::is_same<T, __half>::value) m = 1.f;  // no fp16 square leaves fp32's range
  if (m == 0.f || (m > 0x1p-40f && m < 0x1p48f)) {
#pragma unroll
    for (int e = 0; e < V; ++e) s = fmaf(to_f32(p.v[e]), to_f32(p.v[e]), s);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) d += (double)to_f32(p.v[e]) * to_f32(p.v[e]);
  }
}

// Partial sums of squares, gridDim.x of them for each matrix (gridDim.y): in part_f, and in part_d; where
// fp32's range did not do, part_f's is NaN. Rows are dealt to warps; a thread adds runs of 4 packs.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads)
    norm_kernel(const T* M, int64_t ld, int64_t stride, int64_t rows, int64_t cols, float* part_f, double* part_d) {
  __shared__ float red[kThreads / 32];
  __shared__ double red_d[kThreads / 32];
  const T* m = M + (int64_t)blockIdx.y * stride;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  float total = 0.f;
  double d = 0.0;
  for (int64_t r = (int64_t)blockIdx.x * (kThreads / 32) + warp; r < rows; r += (int64_t)gridDim.x * (kThreads / 32)) {
    const T* row = m + r * ld;
    for (int64_t c0 = lane * V; c0 < cols; c0 += 4 * 32 * V) {
      Pack<T, V> p[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t c = c0 + u * 32 * V;
        if (c < cols) {
          p[u] = *reinterpret_cast<const Pack<T, V>*>(row + c);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) p[u].v[e] = from_f32<T>(0.f);
        }
      }
      float s = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) add_squares(p[u], s, d);
      total += s;
    }
  }
  const int64_t at = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  const bool wide = __syncthreads_or(!(d == 0.0));
  float w = total;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
  if (lane == 0) red[warp] = w;
  if (wide) {
    d += (double)total;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
    if (lane == 0) red_d[warp] = d;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int q = 1; q < kThreads / 32; ++q) w += red[q];
    if (wide)
      for (int q = 1; q < kThreads / 32; ++q) d += red_d[q];
    part_f[at] = wide ? NAN : w;
    part_d[at] = wide ? d : (double)w;
  }
}

// X = M 2^(e + sx) in fp16 (hi, and lo if split), with 1 / max(||M||_F, eps) = t 2^e, t in (1, 2].
template <typename T, int V, int SPLIT>
__global__ void __launch_bounds__(kThreads)
    scale_kernel(const T* M, int64_t ld, int64_t stride, int64_t rows, int64_t cols, const float* part_f,
                 const double* part_d, int parts, float eps, int sx, __half* X, int64_t ld_x, int64_t stride_x,
                 int64_t lo, float* t, int* done, int* status) {
  __shared__ float scale;
  __shared__ float red[kThreads / 32];
  const int b = blockIdx.y;
  float s = 0.f;
  for (int p = threadIdx.x; p < parts; p += kThreads) s += part_f[(int64_t)b * parts + p];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool first = blockIdx.x == 0;
    if (first) done[b] = 0;
    if (first && b == 0)
      for (int i = 0; i < kDoneExtra; ++i) done[gridDim.y + i] = 0;
    for (int w = 1; w < kThreads / 32; ++w) s += red[w];
    int e = 0;
    float f = 0.f;  // norm = f 2^e, f in [0.5, 1)
    bool finite = true;
    if (s == 0.f || (s > 1e-30f && s < 1e30f)) {
      f = frexpf(fmaxf(sqrtf(s), eps), &e);
    } else {  // beyond fp32's range, or not finite
      double d = 0.0;
      for (int p = 0; p < parts; ++p) d += part_d[(int64_t)b * parts + p];
      d = sqrt(d);
      finite = d <= 1.7e308;
      if (finite) f = (float)frexp(d > (double)eps ? d : (double)eps, &e);
    }
    if (!finite) {  // NaN or inf: so is the result
      scale = 1.f;
      if (first) {
        t[b] = NAN;
        if (status) atomicOr(status, SOAP_STATUS_NONFINITE);
      }
    } else {
      const int q = min(sx - e, 120);  // a norm near fp32's smallest: t takes what fp32's range leaves
      scale = ldexpf(1.f, q);
      if (first) t[b] = ldexpf(1.f / f, sx - e - q);
    }
  }
  __syncthreads();
  const float k = scale;
  const T* m = M + (int64_t)b * stride;
  __half* x = X + (int64_t)b * stride_x;
  const int64_t packs = (cols + V - 1) / V;
  const int64_t total = rows * packs, step = (int64_t)gridDim.x * kThreads;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += step) {
    const int64_t r = i / packs, c = (i - r * packs) * V;
    const Pack<T, V> p = *reinterpret_cast<const Pack<T, V>*>(m + r * ld + c);
    Pack<__half, V> h, l;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float v = to_f32(p.v[e]) * k;
      h.v[e] = __float2half_rn(v);
      l.v[e] = __float2half_rn(v - __half2float(h.v[e]));
    }
    *reinterpret_cast<Pack<__half, V>*>(x + r * ld_x + c) = h;
    if (SPLIT == 2) *reinterpret_cast<Pack<__half, V>*>(x + lo + r * ld_x + c) = l;
  }
}

struct Plan {
  int64_t rows, cols, batch;
  int r, k;       // the smaller side (the Gram matrix's) and the larger
  bool tall;      // rows > cols
  bool split;
  int cluster;  // CTAs per matrix of the kernel for small sides; 0: run_steps
  int ld_x, ld_s;
  int parts;    // partial sums of squares per matrix
  int64_t x_elems, s_elems;  // per buffer, planes included
  size_t part_off, t_off, done_off, x_off[2], s_off, b_off, bytes;
};

int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

Plan make_plan(int64_t batch, int64_t rows, int64_t cols, int32_t type) {
  Plan p{};
  p.rows = rows;
  p.cols = cols;
  p.batch = batch;
  p.tall = rows > cols;
  p.r = (int)std::min(rows, cols);
  p.k = (int)std::max(rows, cols);
  p.split = type != SOAP_BF16;
  p.cluster = small_cluster((int)rows, (int)cols, (int)batch, p.split);
  if (p.cluster > 0) {
    p.bytes = 256;
    return p;
  }
  p.parts = (int)std::min<int64_t>(std::max<int64_t>(1, kMaxParts / batch), (rows + 7) / 8);
  p.ld_x = (int)up(cols, 8);
  p.ld_s = (int)up(p.r, 8);
  const int64_t planes = batch * (p.split ? 2 : 1);
  p.x_elems = planes * rows * p.ld_x;
  p.s_elems = planes * p.r * p.ld_s;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += up((int64_t)bytes, 256);
    return at;
  };
  p.part_off = take((size_t)batch * p.parts * (sizeof(double) + sizeof(float)));
  p.t_off = take((size_t)batch * sizeof(float));
  p.done_off = take((size_t)(batch + kDoneExtra) * sizeof(int));
  p.x_off[0] = take((size_t)p.x_elems * 2);
  p.x_off[1] = take((size_t)p.x_elems * 2);
  p.s_off = take((size_t)p.s_elems * 2);
  p.b_off = take((size_t)p.s_elems * 2);
  p.bytes = off;
  return p;
}

bool bad_sizes(int64_t batch, int64_t rows, int64_t cols, int32_t type) {
  if (batch < 1 || batch > 65535 || rows < 1 || cols < 1 || rows > 65536 || cols > 65536) return true;
  if (rows * cols > (int64_t(1) << 31) - 1) return true;
  return type < SOAP_F32 || type > SOAP_F16;
}

// The power of two that scales values of magnitude up to `bound` to below 2^15.
int scale_exp(double bound) {
  if (!(bound > 1e-30)) bound = 1e-30;
  if (!(bound < 1e30)) bound = 1e30;
  int e;
  std::frexp(bound, &e);  // bound <= 2^e
  return 15 - e;
}

// max |b s + c s^2| for 0 <= s <= u
double poly_bound(double b, double c, double u) {
  double m = std::fabs(u * (b + c * u));
  if (c != 0.0) {
    const double s = -b / (2 * c);
    if (s > 0 && s < u) m = std::max(m, std::fabs(s * (b + c * s)));
  }
  return m;
}

// max |x (a + b x^2 + c x^4)| for 0 <= x <= u
double step_bound(double a, double b, double c, double u) {
  auto f = [&](double s) { return s > 0 ? std::fabs(std::sqrt(s) * (a + s * (b + c * s))) : 0.0; };
  const double top = u * u;
  double m = f(top);
  const double d = 9 * b * b - 20 * a * c;  // a + 3 b s + 5 c s^2 = 0
  if (c != 0.0) {
    if (d >= 0)
      for (double sign : {-1.0, 1.0}) {
        const double s = (-3 * b + sign * std::sqrt(d)) / (10 * c);
        if (s > 0 && s < top) m = std::max(m, f(s));
      }
  } else if (b != 0.0) {
    const double s = -a / (3 * b);
    if (s > 0 && s < top) m = std::max(m, f(s));
  }
  return m;
}

template <typename T, int V>
cudaError_t prepare(const Plan& p, const T* M, int64_t ld, int64_t stride, float eps, int sx, const Steps& q,
                    float* part_f, double* part_d, float* t, cudaStream_t s) {
  const double n = (double)p.batch * p.rows * p.cols;
  const int64_t want = std::max<int64_t>(1, kMaxParts / p.batch);
  const int parts = p.parts;
  {
    ProfScope prof(kFamElementwise, 2.0 * n, n * sizeof(T), s);
    norm_kernel<T, V><<<dim3(parts, (unsigned)p.batch), kThreads, 0, s>>>(M, ld, stride, p.rows, p.cols, part_f,
                                                                          part_d);
  }
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ProfScope prof(kFamElementwise, n, n * (sizeof(T) + (p.split ? 4 : 2)), s);
  const int64_t packs = p.rows * ((p.cols + V - 1) / V);
  const dim3 grid((unsigned)std::min<int64_t>(want, (packs + kThreads - 1) / kThreads), (unsigned)p.batch);
  const int64_t sx_elems = p.rows * q.ld_x, lo = sx_elems * p.batch;
  if (p.split)
    scale_kernel<T, V, 2><<<grid, kThreads, 0, s>>>(M, ld, stride, p.rows, p.cols, part_f, part_d, parts, eps, sx,
                                                    q.x[0], q.ld_x, sx_elems, lo, t, q.done, q.status);
  else
    scale_kernel<T, V, 1><<<grid, kThreads, 0, s>>>(M, ld, stride, p.rows, p.cols, part_f, part_d, parts, eps, sx,
                                                    q.x[0], q.ld_x, sx_elems, lo, t, q.done, q.status);
  return cudaGetLastError();
}

template <typename T>
cudaError_t prepare_t(const Plan& p, const void* M, int64_t ld, int64_t stride, float eps, int sx, const Steps& q,
                      float* part_f, double* part_d, float* t, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = reinterpret_cast<uintptr_t>(M) % 16 == 0 && ld % V == 0 && (p.batch == 1 || stride % V == 0) &&
                   p.cols % V == 0;
  const T* m = static_cast<const T*>(M);
  return vec ? prepare<T, V>(p, m, ld, stride, eps, sx, q, part_f, part_d, t, s)
             : prepare<T, 1>(p, m, ld, stride, eps, sx, q, part_f, part_d, t, s);
}

cudaError_t run(const Plan& p, const void* M, int64_t ld, int64_t stride, int32_t type, const float* coeffs, int steps,
                float eps, void* out, int64_t ld_out, int64_t stride_out, uint8_t* ws, int* status, cudaStream_t s) {
  Steps q{};
  q.rows = (int)p.rows;
  q.cols = (int)p.cols;
  q.batch = (int)p.batch;
  q.steps = steps;
  q.split = p.split;
  for (int i = 0; i < 2; ++i) q.x[i] = reinterpret_cast<__half*>(ws + p.x_off[i]);
  q.s = reinterpret_cast<__half*>(ws + p.s_off);
  q.b = reinterpret_cast<__half*>(ws + p.b_off);
  q.ld_x = p.ld_x;
  q.ld_s = p.ld_s;
  float* t = reinterpret_cast<float*>(ws + p.t_off);
  q.t = t;
  q.done = reinterpret_cast<int*>(ws + p.done_off);
  q.out = out;
  q.out_type = type;
  q.ld_out = ld_out;
  q.stride_out = stride_out;
  q.status = status;
  const WaitLimit limit = wait_limit();
  q.wait_ns = limit.ns;
  q.hold = limit.hold;
  double u = 1.0;  // bound of the singular values
  int sx = scale_exp(2.0);
  const int sx0 = sx;
  for (int i = 0; i < steps; ++i) {
    const double a = coeffs ? coeffs[3 * i] : 15.0 / 8, b = coeffs ? coeffs[3 * i + 1] : -10.0 / 8,
                 c = coeffs ? coeffs[3 * i + 2] : 3.0 / 8;
    const int ss = scale_exp(2 * u * u), sb = scale_exp(2 * poly_bound(b, c, u * u));
    u = step_bound(a, b, c, u);
    const int sn = i + 1 == steps && p.cluster == 0 ? 0 : scale_exp(2 * u);
    // S 2^ss = 2^(ss - 2 sx) (X 2^sx) (X 2^sx)^T, B 2^sb = c 2^(sb - 2 ss) (S 2^ss)^2 + b 2^(sb - ss) (S 2^ss),
    // X' 2^sn = 2^(sn - sb - sx) (B 2^sb) (X 2^sx) + a 2^(sn - sx) (X 2^sx)
    q.coef[i] = {(float)std::ldexp(1.0, ss - 2 * sx), (float)std::ldexp(c, sb - 2 * ss), (float)std::ldexp(b, sb - ss),
                 (float)std::ldexp(1.0, sn - sb - sx), (float)std::ldexp(a, sn - sx)};
    sx = sn;
  }
  q.out_exp = sx;
  if (p.cluster > 0) return run_small(q, p.cluster, M, ld, stride, eps, sx0, s);
  double* part_d = reinterpret_cast<double*>(ws + p.part_off);
  float* part_f = reinterpret_cast<float*>(part_d + p.batch * p.parts);
  cudaError_t e;
  if (type == SOAP_F32)
    e = prepare_t<float>(p, M, ld, stride, eps, sx0, q, part_f, part_d, t, s);
  else if (type == SOAP_BF16)
    e = prepare_t<__nv_bfloat16>(p, M, ld, stride, eps, sx0, q, part_f, part_d, t, s);
  else
    e = prepare_t<__half>(p, M, ld, stride, eps, sx0, q, part_f, part_d, t, s);
  return e == cudaSuccess ? run_steps(q, s) : e;
}

bool bad_operand(const void* p, int64_t ld, int64_t stride, int64_t batch, int64_t rows, int64_t cols, int32_t type) {
  if (!p || reinterpret_cast<uintptr_t>(p) % dtype_size(type) || ld < cols) return true;
  return batch > 1 && stride < (rows - 1) * ld + cols;
}

}  // namespace
}  // namespace ortho
}  // namespace soap

using namespace soap;

extern "C" {

size_t muon_orthogonalize_workspace_bytes(int32_t batch, int64_t rows, int64_t cols, int32_t type) {
  if (ortho::bad_sizes(batch, rows, cols, type)) return 0;
  return ortho::make_plan(batch, rows, cols, type).bytes;
}

soap_status_t muon_orthogonalize(int32_t batch, int64_t rows, int64_t cols, const void* M, int64_t ld, int64_t stride,
                                 int32_t type, const float* coeffs, int32_t ns_steps, float eps, void* out,
                                 int64_t ld_out, int64_t stride_out, void* workspace, size_t workspace_bytes,
                                 int32_t* status, soap_stream_t stream) {
  if (ortho::bad_sizes(batch, rows, cols, type)) return SOAP_ERR_INVALID_ARG;
  if (ns_steps < 1 || ns_steps > ortho::kMaxSteps || !(eps > 0.f) || !std::isfinite(eps)) return SOAP_ERR_INVALID_ARG;
  if (coeffs)
    for (int i = 0; i < 3 * ns_steps; ++i)
      if (!std::isfinite(coeffs[i])) return SOAP_ERR_INVALID_ARG;
  if (ortho::bad_operand(M, ld, stride, batch, rows, cols, type) ||
      ortho::bad_operand(out, ld_out, stride_out, batch, rows, cols, type))
    return SOAP_ERR_INVALID_ARG;
  if (status && reinterpret_cast<uintptr_t>(status) % 4) return SOAP_ERR_INVALID_ARG;
  const ortho::Plan p = ortho::make_plan(batch, rows, cols, type);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || workspace_bytes < p.bytes)
    return SOAP_ERR_INVALID_ARG;
  const cudaError_t e = ortho::run(p, M, ld, stride, type, coeffs, ns_steps, eps, out, ld_out, stride_out,
                                   static_cast<uint8_t*>(workspace), status, (cudaStream_t)stream);
  return e == cudaSuccess ? SOAP_OK : e == cudaErrorInvalidValue ? SOAP_ERR_INVALID_ARG : SOAP_ERR_CUDA;
}

}  // extern "C"
