// The gated feed-forward block and its backward pass (include/layer.h, layer_ffn_*).
//
//   g = x Wg,  u = x Wu,  h = act(g) u,  y = h Wd
//   dh = dy Wd^T,  dg = dh u act'(g),  du = dh act(g),  dx = dg Wg^T + du Wu^T,
//   dWg = x^T dg,  dWu = x^T du,  dWd = h^T dy        (per group of rows)
//
// A launch per product, 64 x 64 tiles on the fp32 pipe: the same for every type, order and size.
#include <algorithm>
#include <cstdint>

#include "../../include/layer.h"
#include "profile.h"
#include "soap_internal.h"
#include "types.h"

namespace soap {
namespace {

constexpr int kMaxGroups = 1024, kMaxSide = 65536;
constexpr int64_t kMaxRows = INT32_MAX - 65536;

// One factor pair of a product: A (m, k) at m * am + k * ak, B (k, n) at k * bk + n * bn, elements between groups.
struct Factors {
  const void *a, *b;
  int64_t am, ak, a_group, bk, bn, b_group;
};

enum Out { kGatedOut, kGradOut, kPlain };

struct Product {
  const int* bounds;  // the groups' sanitised offsets
  int rows_are;       // 0: A's rows and the results' are the group's rows; 1: k runs over the group's rows
  int M, N, K;
  Factors f[2];
  int pairs;          // of factors whose products are added (kGatedOut: g from the first, u from the second)
  int act;
  void* out;          // (m, n) at m * om + n * on + group * o_group
  int64_t om, on, o_group;
  void *h, *dg, *du;  // [rows][N]
  float* pre;         // [rows][2][N]
  int64_t width;
};

__device__ __forceinline__ void activation(int act, float g, float& a, float& da) {
  if (act == LAYER_SILU) {
    const float s = 1.f / (1.f + expf(-g));
    a = g * s;
    da = s * (1.f + g * (1.f - s));
  } else {
    const float p = 0.5f * (1.f + erff(g * 0.70710678118654752f));
    a = g * p;
    da = p + g * 0.3989422804014327f * expf(-0.5f * g * g);
  }
}

template <typename T, int OUT>
__global__ void __launch_bounds__(256) product_kernel(const __grid_constant__ Product p) {
  constexpr int BM = 64, BN = 64, BK = 16, NP = OUT == kGatedOut ? 2 : 1;
  __shared__ float sa[BK][BM + 1], sb[NP][BK][BN + 1];
  const int group = blockIdx.z, r0 = p.bounds[group], r1 = p.bounds[group + 1];
  const int M = p.rows_are ? p.M : r1 - r0, K = p.rows_are ? r1 - r0 : p.K;
  const int m0 = blockIdx.y * BM, n0 = blockIdx.x * BN;
  if (m0 >= M) return;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float acc[NP][4][4] = {};
  for (int seg = 0; seg < (OUT == kGatedOut ? 1 : p.pairs); ++seg) {
    const Factors& f = p.f[seg];
    const T* A = static_cast<const T*>(f.a) + group * f.a_group + (int64_t)r0 * (p.rows_are ? f.ak : f.am);
    for (int k0 = 0; k0 < K; k0 += BK) {
      for (int i = threadIdx.x; i < BM * BK; i += 256) {
        const bool along = f.ak == 1;
        const int m = along ? i / BK : i % BM, k = along ? i % BK : i / BM;
        sa[k][m] = m0 + m < M && k0 + k < K ? to_f32(A[(int64_t)(m0 + m) * f.am + (int64_t)(k0 + k) * f.ak]) : 0.f;
      }
#pragma unroll
      for (int q = 0; q < NP; ++q) {
        const Factors& fb = p.f[seg + q];
        const T* B = static_cast<const T*>(fb.b) + group * fb.b_group + (p.rows_are ? (int64_t)r0 * fb.bk : 0);
        for (int i = threadIdx.x; i < BN * BK; i += 256) {
          const bool along = fb.bk == 1;
          const int n = along ? i / BK : i % BN, k = along ? i % BK : i / BN;
          sb[q][k][n] = n0 + n < p.N && k0 + k < K ? to_f32(B[(int64_t)(k0 + k) * fb.bk + (int64_t)(n0 + n) * fb.bn]) : 0.f;
        }
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < BK; ++k)
#pragma unroll
        for (int q = 0; q < NP; ++q)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[q][i][j] = fmaf(sa[k][ty + 16 * i], sb[q][k][tx + 16 * j], acc[q][i][j]);
      __syncthreads();
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
      if (m >= M || n >= p.N) continue;
      const int64_t row = (int64_t)r0 + m, at = row * p.width + n;
      float a, da;
      if constexpr (OUT == kGatedOut) {
        activation(p.act, acc[0][i][j], a, da);
        static_cast<T*>(p.h)[at] = from_f32<T>(a * acc[1][i][j]);
        if (p.pre) {
          p.pre[row * 2 * p.width + n] = acc[0][i][j];
          p.pre[(row * 2 + 1) * p.width + n] = acc[1][i][j];
        }
      } else if constexpr (OUT == kGradOut) {
        const float g = p.pre[row * 2 * p.width + n], u = p.pre[(row * 2 + 1) * p.width + n], dh = acc[0][i][j];
        activation(p.act, g, a, da);
        static_cast<T*>(p.h)[at] = from_f32<T>(a * u);
        static_cast<T*>(p.dg)[at] = from_f32<T>(dh * u * da);
        static_cast<T*>(p.du)[at] = from_f32<T>(dh * a);
      } else {
        static_cast<T*>(p.out)[(p.rows_are ? (int64_t)m : row) * p.om + (int64_t)n * p.on + group * p.o_group] =
            from_f32<T>(acc[0][i][j]);
      }
    }
}

// bounds[g]: the largest of offsets[0 .. g], within 0 .. rows.
__global__ void __launch_bounds__(1024) bounds_kernel(const int* offsets, int groups, int rows, int* bounds, int* status) {
  __shared__ int top[2][kMaxGroups + 1];
  bool off = false;
  for (int i = threadIdx.x; i <= groups; i += 1024) {
    const int v = offsets ? offsets[i] : i == 0 ? 0 : rows;
    off |= v < 0 || v > rows || (offsets && i > 0 && v < offsets[i - 1]);
    top[0][i] = min(max(v, 0), rows);
  }
  if (off && status) atomicOr(status, kStatusRange);
  int at = 0;
  for (int d = 1; d <= groups; d *= 2, at ^= 1) {
    __syncthreads();
    for (int i = threadIdx.x; i <= groups; i += 1024) top[at ^ 1][i] = max(top[at][i], i >= d ? top[at][i - d] : 0);
  }
  __syncthreads();
  for (int i = threadIdx.x; i <= groups; i += 1024) bounds[i] = top[at][i];
}

// Rows of no group become 0.
template <typename T>
__global__ void __launch_bounds__(256) outside_kernel(const int* bounds, int groups, int64_t rows, T* y, int64_t ld, int width) {
  const int first = bounds[0], last = bounds[groups];
  for (int64_t r = blockIdx.x; r < first + (rows - last); r += gridDim.x) {
    T* row = y + (r < first ? r : r - first + last) * ld;
    for (int c = threadIdx.x; c < width; c += 256) row[c] = from_f32<T>(0.f);
  }
}

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

bool bad_ptr(const void* p, size_t size) { return p && reinterpret_cast<uintptr_t>(p) % size; }

bool bad_matrix(const layer_matrix_t* m, int64_t rows, int64_t cols, int groups, size_t size) {
  if (!m || !m->data || bad_ptr(m->data, size)) return true;
  const int64_t along = m->columns ? rows : cols, across = m->columns ? cols : rows;
  return m->ld < along || (groups > 1 && m->stride < (across - 1) * m->ld + along);
}

bool bad_sizes(int64_t rows, int64_t hidden, int64_t width, int32_t groups, int32_t type) {
  return rows < 0 || rows > kMaxRows || hidden < 1 || hidden > kMaxSide || width < 1 || width > kMaxSide || groups < 1 ||
         groups > kMaxGroups || type < SOAP_F32 || type > SOAP_F16;
}

// What a call has in hand.
struct Call {
  int64_t rows;
  int hidden, width, groups;
  const int32_t* offsets;
  int type, act;
  const layer_matrix_t *gate, *up, *down;
  int* status;
  uint8_t* ws;
};

bool bad_call(const Call& c, size_t ws_bytes, bool backward) {
  const size_t size = dtype_size(c.type);
  return (!c.offsets && c.groups != 1) || bad_ptr(c.offsets, 4) || bad_ptr(c.status, 4) ||
         (c.act != LAYER_SILU && c.act != LAYER_GELU) || bad_matrix(c.gate, c.hidden, c.width, c.groups, size) ||
         bad_matrix(c.up, c.hidden, c.width, c.groups, size) || bad_matrix(c.down, c.width, c.hidden, c.groups, size) ||
         !c.gate->columns != !c.up->columns || !c.ws || bad_ptr(c.ws, 256) ||
         ws_bytes < layer_ffn_workspace_bytes(c.rows, c.hidden, c.width, c.groups, c.type, 1, backward);
}

// (i, j) of a matrix at i * r + j * c
struct Steps {
  int64_t r, c;
};
Steps steps_of(const layer_matrix_t& m) { return m.columns ? Steps{1, m.ld} : Steps{m.ld, 1}; }

template <typename T, int OUT>
cudaError_t launch(const Product& p, int64_t rows, int groups, cudaStream_t s) {
  const int64_t m = p.rows_are ? p.M : rows;
  if (m == 0) return cudaSuccess;
  // (a grid is at most 65535 high: tall ones in pieces would need a row offset; the tiled kernel has none)
  if ((m + 63) / 64 > 65535) return cudaErrorInvalidValue;
  product_kernel<T, OUT><<<dim3((p.N + 63) / 64, (unsigned)((m + 63) / 64), groups), 256, 0, s>>>(p);
  return cudaGetLastError();
}

template <typename T>
cudaError_t forward(const Call& c, const void* x, int64_t ld_x, void* y, int64_t ld_y, float* pre, cudaStream_t s) {
  int* bounds = reinterpret_cast<int*>(c.ws);
  T* h = reinterpret_cast<T*>(c.ws + up256((kMaxGroups + 1) * 4));
  bounds_kernel<<<1, 1024, 0, s>>>(c.offsets, c.groups, (int)c.rows, bounds, c.status);
  if (c.offsets) outside_kernel<T><<<256, 256, 0, s>>>(bounds, c.groups, c.rows, static_cast<T*>(y), ld_y, c.hidden);
  Product p{};
  p.bounds = bounds;
  p.N = c.width;
  p.K = c.hidden;
  const layer_matrix_t* w[2] = {c.gate, c.up};
  for (int i = 0; i < 2; ++i) p.f[i] = {x, w[i]->data, ld_x, 1, 0, steps_of(*w[i]).r, steps_of(*w[i]).c, w[i]->stride};
  p.act = c.act;
  p.h = h;
  p.pre = pre;
  p.width = c.width;
  cudaError_t e = launch<T, kGatedOut>(p, c.rows, c.groups, s);
  if (e != cudaSuccess) return e;
  p.N = c.hidden;
  p.K = c.width;
  p.f[0] = {h, c.down->data, c.width, 1, 0, steps_of(*c.down).r, steps_of(*c.down).c, c.down->stride};
  p.pairs = 1;
  p.out = y;
  p.om = ld_y;
  p.on = 1;
  return launch<T, kPlain>(p, c.rows, c.groups, s);
}

template <typename T>
cudaError_t backward(const Call& c, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const float* pre, void* dx,
                     int64_t ld_dx, const layer_matrix_t* const (&grads)[3], cudaStream_t s) {
  int* bounds = reinterpret_cast<int*>(c.ws);
  T* h = reinterpret_cast<T*>(c.ws + up256((kMaxGroups + 1) * 4));
  const size_t n = up256((size_t)c.rows * c.width * sizeof(T)) / sizeof(T);
  T *dg = h + n, *du = dg + n;
  bounds_kernel<<<1, 1024, 0, s>>>(c.offsets, c.groups, (int)c.rows, bounds, c.status);
  if (c.offsets) outside_kernel<T><<<256, 256, 0, s>>>(bounds, c.groups, c.rows, static_cast<T*>(dx), ld_dx, c.hidden);
  Product p{};
  p.bounds = bounds;
  p.N = c.width;
  p.K = c.hidden;
  p.f[0] = {dy, c.down->data, ld_dy, 1, 0, steps_of(*c.down).c, steps_of(*c.down).r, c.down->stride};
  p.pairs = 1;
  p.act = c.act;
  p.h = h;
  p.dg = dg;
  p.du = du;
  p.pre = const_cast<float*>(pre);
  p.width = c.width;
  cudaError_t e = launch<T, kGradOut>(p, c.rows, c.groups, s);
  if (e != cudaSuccess) return e;
  p.N = c.hidden;
  p.K = c.width;
  const layer_matrix_t* w[2] = {c.gate, c.up};
  for (int i = 0; i < 2; ++i)
    p.f[i] = {i ? du : dg, w[i]->data, c.width, 1, 0, steps_of(*w[i]).c, steps_of(*w[i]).r, w[i]->stride};
  p.pairs = 2;
  p.out = dx;
  p.om = ld_dx;
  p.on = 1;
  e = launch<T, kPlain>(p, c.rows, c.groups, s);
  const void* left[3] = {x, x, h};
  const void* right[3] = {dg, du, dy};
  for (int i = 0; i < 3 && e == cudaSuccess && grads[0]; ++i) {
    p.rows_are = 1;
    p.M = i < 2 ? c.hidden : c.width;
    p.N = i < 2 ? c.width : c.hidden;
    p.pairs = 1;
    p.f[0] = {left[i], right[i], 1, i < 2 ? ld_x : (int64_t)c.width, 0, i < 2 ? (int64_t)c.width : ld_dy, 1, 0};
    p.out = grads[i]->data;
    p.om = steps_of(*grads[i]).r;
    p.on = steps_of(*grads[i]).c;
    p.o_group = grads[i]->stride;
    e = launch<T, kPlain>(p, c.rows, c.groups, s);
  }
  return e;
}

}  // namespace
}  // namespace soap

using namespace soap;

extern "C" {

size_t layer_ffn_pre_elems(int64_t rows, int64_t width, int32_t groups) {
  if (bad_sizes(rows, 1, width, groups, SOAP_F32)) return 0;
  return (size_t)rows * 2 * width;
}

size_t layer_ffn_workspace_bytes(int64_t rows, int64_t hidden, int64_t width, int32_t groups, int32_t type,
                                 int32_t aligned, int32_t backward) {
  if (bad_sizes(rows, hidden, width, groups, type)) return 0;
  return up256((kMaxGroups + 1) * 4) + (backward ? 3 : 1) * up256((size_t)rows * width * dtype_size(type));
}

soap_status_t layer_ffn_forward(int64_t rows, int64_t hidden, int64_t width, int32_t groups,
                                const int32_t* offsets, const void* x, int64_t ld_x, int32_t type,
                                const layer_matrix_t* gate, const layer_matrix_t* up, const layer_matrix_t* down,
                                int32_t act, void* y, int64_t ld_y, float* pre, int32_t* status, void* workspace,
                                size_t workspace_bytes, soap_stream_t stream) {
  if (bad_sizes(rows, hidden, width, groups, type)) return SOAP_ERR_INVALID_ARG;
  const Call c{rows, (int)hidden, (int)width, groups, offsets, type, act, gate, up, down, status,
               static_cast<uint8_t*>(workspace)};
  const size_t size = dtype_size(type);
  if (bad_call(c, workspace_bytes, false) || bad_ptr(pre, 16)) return SOAP_ERR_INVALID_ARG;
  if (rows > 0 && (!x || bad_ptr(x, size) || ld_x < hidden || !y || bad_ptr(y, size) || ld_y < hidden))
    return SOAP_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  ProfScope prof(kFamGemmTc, 6.0 * rows * hidden * width, 3.0 * groups * hidden * width * size, s);
  const cudaError_t e = type == SOAP_F32    ? forward<float>(c, x, ld_x, y, ld_y, pre, s)
                        : type == SOAP_BF16 ? forward<__nv_bfloat16>(c, x, ld_x, y, ld_y, pre, s)
                                            : forward<__half>(c, x, ld_x, y, ld_y, pre, s);
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

soap_status_t layer_ffn_backward(int64_t rows, int64_t hidden, int64_t width, int32_t groups,
                                 const int32_t* offsets, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x,
                                 int32_t type, const layer_matrix_t* gate, const layer_matrix_t* up,
                                 const layer_matrix_t* down, int32_t act, const float* pre, void* dx, int64_t ld_dx,
                                 const layer_matrix_t* d_gate, const layer_matrix_t* d_up,
                                 const layer_matrix_t* d_down, int32_t* status, void* workspace,
                                 size_t workspace_bytes, soap_stream_t stream) {
  if (bad_sizes(rows, hidden, width, groups, type)) return SOAP_ERR_INVALID_ARG;
  const Call c{rows, (int)hidden, (int)width, groups, offsets, type, act, gate, up, down, status,
               static_cast<uint8_t*>(workspace)};
  const size_t size = dtype_size(type);
  if (bad_call(c, workspace_bytes, true) || bad_ptr(pre, 16)) return SOAP_ERR_INVALID_ARG;
  if (rows > 0 && (!x || bad_ptr(x, size) || ld_x < hidden || !dy || bad_ptr(dy, size) || ld_dy < hidden || !dx ||
                   bad_ptr(dx, size) || ld_dx < hidden || !pre))
    return SOAP_ERR_INVALID_ARG;
  const layer_matrix_t* grads[3] = {d_gate, d_up, d_down};
  if (!d_gate != !d_up || !d_gate != !d_down) return SOAP_ERR_INVALID_ARG;
  if (d_gate)
    for (int i = 0; i < 3; ++i) {
      const layer_matrix_t* w = i == 0 ? gate : i == 1 ? up : down;
      if (bad_matrix(grads[i], i < 2 ? hidden : width, i < 2 ? width : hidden, groups, size) ||
          !grads[i]->columns != !w->columns)
        return SOAP_ERR_INVALID_ARG;
    }
  cudaStream_t s = (cudaStream_t)stream;
  ProfScope prof(kFamGemmTc, 12.0 * rows * hidden * width, 3.0 * groups * hidden * width * size, s);
  const cudaError_t e =
      type == SOAP_F32    ? backward<float>(c, dy, ld_dy, x, ld_x, pre, dx, ld_dx, grads, s)
      : type == SOAP_BF16 ? backward<__nv_bfloat16>(c, dy, ld_dy, x, ld_x, pre, dx, ld_dx, grads, s)
                          : backward<__half>(c, dy, ld_dy, x, ld_x, pre, dx, ld_dx, grads, s);
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

}  // extern "C"
