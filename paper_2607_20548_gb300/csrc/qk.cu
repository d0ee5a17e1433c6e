// Norms of queries and keys for each head with the rotation by position in the same pass, and the
// backward pass (include/layer.h, layer_qk_*).
//
//   r = 1 / sqrt(mean(x^2) + eps),  n = x r,  m = n w,  (a, b) -> (a c - b s, b c + a s)
//   dm: dy turned back,  g = dm w,  dx = r (g - n mean(g n)),  dw = sum dm n
//
// Bound by memory: x is read and y written once (backward: x and dy read, dx written once). A pair of the
// rotation stays in one lane, so that turning it exchanges nothing: a lane holds 8 pairs of a head, as units
// of V neighbouring first and V neighbouring second elements (V: up to 16 bytes, as far as the parts' sizes
// and alignments allow), and 1 to 32 lanes a head. All of a lane's heads are of one token, whose cosines and
// sines it fetches once; heads that are independent of one another are asked for together. The mean of g n is
// r times that of g x, so that a head's two sums cross its lanes in one exchange.
#include <algorithm>
#include <atomic>
#include <cstdint>

#include "../../include/layer.h"
#include "profile.h"
#include "soap_internal.h"
#include "types.h"

namespace soap {
namespace {

constexpr int kPairs = 8;       // per lane
constexpr int kWarps = 8;       // per CTA
constexpr int kMaxDim = 512, kMaxHeads = 32768;
constexpr int64_t kMaxTokens = INT32_MAX - 65536;

struct Heads {
  void* p;
  int64_t batch, token, head;  // strides
};

struct Qk {
  uint32_t tokens, length;
  int heads[2];  // q, k
  int dim, rotary;
  Heads x[2], out[2], dy[2];  // forward: x to out; backward: dy and x to out (dx)
  const void* w[2];
  float eps;
  const float *cos, *sin;
  int64_t places;
  const void* positions;
  int positions_64;
  int* status;
  int lanes;        // per head
  int steps;        // of 32 / lanes heads in a chunk
  int chunks[2];    // forward: of q's and k's heads together, in [0]
  float* partial;   // backward: [CTAs][dim], q's CTAs first, or nullptr
  uint32_t ctas_q;
};

__device__ __forceinline__ int64_t place_of(const Heads& h, const Qk& a, uint32_t token, int head) {
  const uint32_t b = token / a.length, s = token - b * a.length;
  return (int64_t)b * h.batch + (int64_t)s * h.token + (int64_t)head * h.head;
}

template <int V>
__device__ __forceinline__ void load_f32(const float* p, float* v) {
#pragma unroll
  for (int i = 0; i < V; i += V < 4 ? V : 4) {
    const Pack<float, (V < 4 ? V : 4)> q = *reinterpret_cast<const Pack<float, (V < 4 ? V : 4)>*>(p + i);
#pragma unroll
    for (int e = 0; e < (V < 4 ? V : 4); ++e) v[i + e] = q.v[e];
  }
}
template <typename W, int V>
__device__ __forceinline__ void load_w(const W* p, float* v) {
  if constexpr (sizeof(W) == 4) {
    load_f32<V>(p, v);
  } else {
    const Pack<W, V> q = *reinterpret_cast<const Pack<W, V>*>(p);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = to_f32(q.v[e]);
  }
}

// A lane's part of a head: units lane, lane + lanes, ...; unit u has V first elements at first(u), V second ones
// at second(u). Half-split pairs: (j, j + rotary / 2); what is not rotated goes as neighbouring blocks.
template <int V, bool INTER>
struct Units {
  int dim, rotary;
  __device__ __forceinline__ bool has(int u) const { return u * 2 * V < dim; }
  __device__ __forceinline__ bool turns(int u) const { return u * 2 * V < rotary; }
  __device__ __forceinline__ int first(int u) const { return !INTER && turns(u) ? u * V : 2 * u * V; }
  __device__ __forceinline__ int second(int u) const { return !INTER && turns(u) ? rotary / 2 + u * V : 2 * u * V + V; }
};

template <typename T, int V>
struct Raw {
  Pack<T, V> a[kPairs / V], b[kPairs / V];
};

template <typename T, int V, bool INTER>
__device__ __forceinline__ void fetch(Raw<T, V>& r, const T* p, const Units<V, INTER>& un, int lane, int lanes) {
#pragma unroll
  for (int i = 0; i < kPairs / V; ++i) {
    const int u = i * lanes + lane;
    if (p && un.has(u)) {
      r.a[i] = *reinterpret_cast<const Pack<T, V>*>(p + un.first(u));
      r.b[i] = *reinterpret_cast<const Pack<T, V>*>(p + un.second(u));
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) r.a[i].v[e] = r.b[i].v[e] = from_f32<T>(0.f);
    }
  }
}

// The pair j of unit i: elements 2 j and 2 j + 1 of the unit's 2 V, or element j of its halves.
template <bool INTER, typename T, int V>
__device__ __forceinline__ float2 pair_of(const Raw<T, V>& r, int i, int j) {
  if (!INTER) return make_float2(to_f32(r.a[i].v[j]), to_f32(r.b[i].v[j]));
  const int e = 2 * j;
  return make_float2(to_f32(e < V ? r.a[i].v[e % V] : r.b[i].v[e % V]),
                     to_f32(e + 1 < V ? r.a[i].v[(e + 1) % V] : r.b[i].v[(e + 1) % V]));
}
template <bool INTER, typename T, int V>
__device__ __forceinline__ void set_pair(Raw<T, V>& r, int i, int j, float2 v) {
  const T x = from_f32<T>(v.x), y = from_f32<T>(v.y);
  if (!INTER) {
    r.a[i].v[j] = x;
    r.b[i].v[j] = y;
    return;
  }
  const int e = 2 * j;
  (e < V ? r.a[i].v[e % V] : r.b[i].v[e % V]) = x;
  (e + 1 < V ? r.a[i].v[(e + 1) % V] : r.b[i].v[(e + 1) % V]) = y;
}

template <typename T, int V, bool INTER>
__device__ __forceinline__ void store(T* p, const Raw<T, V>& r, const Units<V, INTER>& un, int lane, int lanes) {
#pragma unroll
  for (int i = 0; i < kPairs / V; ++i) {
    const int u = i * lanes + lane;
    if (un.has(u)) {
      *reinterpret_cast<Pack<T, V>*>(p + un.first(u)) = r.a[i];
      *reinterpret_cast<Pack<T, V>*>(p + un.second(u)) = r.b[i];
    }
  }
}

// A lane's cosines and sines (1 and 0 where nothing turns), and whether the token's position is in range.
template <int V, bool INTER>
__device__ __forceinline__ bool angles(const Qk& a, uint32_t token, const Units<V, INTER>& un, int lane, float (&c)[kPairs],
                                       float (&s)[kPairs]) {
  int64_t at = 0;
  bool ok = true;
  if (a.rotary > 0) {
    at = !a.positions ? token % a.length
         : a.positions_64 ? static_cast<const int64_t*>(a.positions)[token]
                          : static_cast<const int32_t*>(a.positions)[token];
    ok = at >= 0 && at < a.places;
  }
#pragma unroll
  for (int i = 0; i < kPairs / V; ++i) {
    const int u = i * a.lanes + lane;
    if (ok && un.turns(u)) {
      const int64_t j = at * (a.rotary / 2) + u * V;
      load_f32<V>(a.cos + j, c + i * V);
      load_f32<V>(a.sin + j, s + i * V);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) c[i * V + e] = 1.f, s[i * V + e] = 0.f;
    }
  }
  return ok;
}

// The weights of a lane's pairs.
template <typename W, int V, bool INTER>
__device__ __forceinline__ void weights(const void* w, const Units<V, INTER>& un, int lane, int lanes, float2 (&v)[kPairs]) {
#pragma unroll
  for (int i = 0; i < kPairs / V; ++i) {
    const int u = i * lanes + lane;
    float x[V], y[V];
    if (w && un.has(u)) {
      load_w<W, V>(static_cast<const W*>(w) + un.first(u), x);
      load_w<W, V>(static_cast<const W*>(w) + un.second(u), y);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = y[e] = 1.f;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (!INTER) v[i * V + j] = make_float2(x[j], y[j]);
      else
        v[i * V + j] = make_float2(2 * j < V ? x[(2 * j) % V] : y[(2 * j) % V],
                                   2 * j + 1 < V ? x[(2 * j + 1) % V] : y[(2 * j + 1) % V]);
    }
  }
}

__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A warp for a token's chunk of UN steps at most, 32 / lanes heads each, of q's and then k's heads.
template <typename T, typename W, int V, bool INTER, int UN>
__global__ void __launch_bounds__(32 * kWarps) qk_fwd_kernel(const __grid_constant__ Qk a) {
  const uint32_t token = blockIdx.x * kWarps + threadIdx.y;
  if (token >= a.tokens) return;  // whole warps
  const int lanes = a.lanes, lane = threadIdx.x & (lanes - 1), at = threadIdx.x / lanes, per = 32 / lanes;
  const Units<V, INTER> un{a.dim, a.rotary};
  const int all = a.heads[0] + a.heads[1], h0 = blockIdx.y * a.steps * per + at;
  Raw<T, V> x[UN];
#pragma unroll
  for (int s = 0; s < UN; ++s) {
    const int h = h0 + s * per, k = h >= a.heads[0];
    const T* p = nullptr;
    if (s < a.steps && h < all)
      p = static_cast<const T*>(a.x[k].p) + place_of(a.x[k], a, token, k ? h - a.heads[0] : h);
    fetch(x[s], p, un, lane, lanes);
  }
  float c[kPairs], sn[kPairs];
  const bool ok = angles(a, token, un, lane, c, sn);
  if (!ok && threadIdx.x == 0 && a.status) atomicOr(a.status, kStatusRange);
#pragma unroll
  for (int s = 0; s < UN; ++s) {
    if (s >= a.steps) break;
    const int h = h0 + s * per, k = h >= a.heads[0];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const float2 v = pair_of<INTER>(x[s], i / V, i % V);
      sum = fmaf(v.x, v.x, fmaf(v.y, v.y, sum));
    }
    sum = lanes_sum(sum, lanes);
    if (h >= all) continue;  // (the exchange above takes all lanes)
    const float r = ok ? 1.f / sqrtf(sum / (float)a.dim + a.eps) : NAN;
    float2 w[kPairs];
    weights<W>(a.w[k], un, lane, lanes, w);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const float2 v = pair_of<INTER>(x[s], i / V, i % V);
      const float m0 = v.x * r * w[i].x, m1 = v.y * r * w[i].y;
      set_pair<INTER>(x[s], i / V, i % V, make_float2(m0 * c[i] - m1 * sn[i], m1 * c[i] + m0 * sn[i]));
    }
    store(static_cast<T*>(a.out[k].p) + place_of(a.out[k], a, token, k ? h - a.heads[0] : h), x[s], un, lane, lanes);
  }
}

// The backward pass: persistent CTAs, the first ctas_q of them for q's heads, the others for k's; a warp takes every
// (its CTAs x kWarps)-th chunk and keeps its lanes' part of dweight in registers.
template <typename T, typename W, int V, bool INTER, int UN>
__global__ void __launch_bounds__(32 * kWarps) qk_bwd_kernel(const __grid_constant__ Qk a) {
  extern __shared__ float sums[];  // [kWarps][dim]
  const int k = blockIdx.x >= a.ctas_q;
  const uint32_t cta = blockIdx.x - (k ? a.ctas_q : 0), ctas = k ? gridDim.x - a.ctas_q : a.ctas_q;
  const int lanes = a.lanes, lane = threadIdx.x & (lanes - 1), at = threadIdx.x / lanes, per = 32 / lanes;
  const Units<V, INTER> un{a.dim, a.rotary};
  const int all = a.heads[k];
  const uint32_t chunks = a.chunks[k];
  float2 w[kPairs], dw[kPairs];
  weights<W>(a.w[k], un, lane, lanes, w);
#pragma unroll
  for (int i = 0; i < kPairs; ++i) dw[i] = make_float2(0.f, 0.f);
  const uint32_t step = ctas * kWarps, first = cta * kWarps + threadIdx.y;
  const uint32_t dt = step / chunks, dc = step % chunks;
  uint32_t chunk = first % chunks;
  // (a token index some steps further on stays below 2^32: step is at most kWarps times a few CTAs per SM)
  for (uint32_t token = first / chunks; token < a.tokens;) {
    const int h0 = chunk * a.steps * per + at;
    Raw<T, V> x[UN], dy[UN];
#pragma unroll
    for (int s = 0; s < UN; ++s) {
      const int h = h0 + s * per;
      const bool live = s < a.steps && h < all;
      fetch(x[s], live ? static_cast<const T*>(a.x[k].p) + place_of(a.x[k], a, token, h) : nullptr, un, lane, lanes);
      fetch(dy[s], live ? static_cast<const T*>(a.dy[k].p) + place_of(a.dy[k], a, token, h) : nullptr, un, lane, lanes);
    }
    float c[kPairs], sn[kPairs];
    const bool ok = angles(a, token, un, lane, c, sn);
    if (!ok && threadIdx.x == 0 && a.status) atomicOr(a.status, kStatusRange);
#pragma unroll
    for (int s = 0; s < UN; ++s) {
      if (s >= a.steps) break;
      const int h = h0 + s * per;
      float2 dm[kPairs];
      float xx = 0.f, gx = 0.f;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float2 v = pair_of<INTER>(x[s], i / V, i % V), d = pair_of<INTER>(dy[s], i / V, i % V);
        dm[i] = make_float2(d.x * c[i] + d.y * sn[i], d.y * c[i] - d.x * sn[i]);
        xx = fmaf(v.x, v.x, fmaf(v.y, v.y, xx));
        gx = fmaf(dm[i].x * w[i].x, v.x, fmaf(dm[i].y * w[i].y, v.y, gx));
      }
      xx = lanes_sum(xx, lanes);
      gx = lanes_sum(gx, lanes);
      if (h >= all) continue;
      const float r = ok ? 1.f / sqrtf(xx / (float)a.dim + a.eps) : NAN;
      const float mean = r * (gx / (float)a.dim);
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float2 v = pair_of<INTER>(x[s], i / V, i % V);
        const float n0 = v.x * r, n1 = v.y * r;
        dw[i].x = fmaf(dm[i].x, n0, dw[i].x);
        dw[i].y = fmaf(dm[i].y, n1, dw[i].y);
        set_pair<INTER>(x[s], i / V, i % V,
                        make_float2(r * (dm[i].x * w[i].x - n0 * mean), r * (dm[i].y * w[i].y - n1 * mean)));
      }
      store(static_cast<T*>(a.out[k].p) + place_of(a.out[k], a, token, h), x[s], un, lane, lanes);
    }
    token += dt;
    chunk += dc;
    if (chunk >= chunks) {
      chunk -= chunks;
      ++token;
    }
  }
  if (!a.partial) return;
  // the warp's heads, then the CTA's warps, always in the same order
#pragma unroll
  for (int i = 0; i < kPairs; ++i)
    for (int o = lanes; o < 32; o <<= 1) {
      dw[i].x += __shfl_xor_sync(0xffffffffu, dw[i].x, o);
      dw[i].y += __shfl_xor_sync(0xffffffffu, dw[i].y, o);
    }
  if (at == 0) {
    float* row = sums + threadIdx.y * a.dim;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const int u = (i / V) * lanes + lane, j = i % V;
      if (un.has(u)) {
        row[INTER ? un.first(u) + 2 * j : un.first(u) + j] = dw[i].x;
        row[INTER ? un.first(u) + 2 * j + 1 : un.second(u) + j] = dw[i].y;
      }
    }
  }
  __syncthreads();
  for (int j = threadIdx.y * 32 + threadIdx.x; j < a.dim; j += 32 * kWarps) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) t += sums[i * a.dim + j];
    a.partial[(int64_t)blockIdx.x * a.dim + j] = t;
  }
}

// dweight[j] = the sum of the CTAs' parts, for 32 columns of q's or k's; a warp adds up every 16th CTA's.
constexpr int kSumWarps = 16;
__global__ void __launch_bounds__(32 * kSumWarps)
    qk_sum_kernel(const float* partial, uint32_t ctas_q, uint32_t ctas, int dim, float* dq, float* dk) {
  __shared__ float part[kSumWarps][32];
  const int k = blockIdx.y, j = blockIdx.x * 32 + threadIdx.x;
  const uint32_t from = k ? ctas_q : 0, to = k ? ctas : ctas_q;
  float t = 0.f;
  if (j < dim)
    for (uint32_t i = from + threadIdx.y; i < to; i += kSumWarps) t += partial[(int64_t)i * dim + j];
  part[threadIdx.y][threadIdx.x] = t;
  __syncthreads();
  float* const out = k ? dk : dq;
  if (threadIdx.y == 0 && j < dim && out) {
    t = 0.f;
#pragma unroll
    for (int i = 0; i < kSumWarps; ++i) t += part[i][threadIdx.x];
    out[j] = t;
  }
}

// ---- host ----

bool odd_ptr(const void* p, size_t size) { return p && reinterpret_cast<uintptr_t>(p) % size; }

// Whether a unit of V elements of `size` bytes lies on its own boundary in every head.
bool units_fit(const Heads& h, int V, size_t size, bool live) {
  if (!live) return true;
  const uint64_t all = (uint64_t)h.batch | (uint64_t)h.token | (uint64_t)h.head;
  return reinterpret_cast<uintptr_t>(h.p) % std::min<size_t>(16, V * size) == 0 && all % V == 0;
}

int unit_size(const Qk& a, size_t size, size_t w_size, bool backward) {
  for (int V = (int)(16 / size); V > 1; V /= 2) {
    bool fit = a.dim / 2 % V == 0 && a.rotary / 2 % V == 0;
    for (int k = 0; k < 2; ++k) {
      const bool live = a.heads[k] > 0;
      fit = fit && units_fit(a.x[k], V, size, live) && units_fit(a.out[k], V, size, live) &&
            (!backward || units_fit(a.dy[k], V, size, live)) &&
            reinterpret_cast<uintptr_t>(a.w[k]) % std::min<size_t>(16, V * w_size) == 0;
    }
    fit = fit && (reinterpret_cast<uintptr_t>(a.cos) | reinterpret_cast<uintptr_t>(a.sin)) %
                         std::min<size_t>(16, V * sizeof(float)) == 0;
    if (fit) return V;
  }
  return 1;
}

template <typename F>
cudaError_t with_unit(int V, F&& f) {
  if (V == 8) return f(std::integral_constant<int, 8>());
  if (V == 4) return f(std::integral_constant<int, 4>());
  if (V == 2) return f(std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 1>());
}

int sm_count() {
  static std::atomic<int> of[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  int n = dev < 64 ? of[dev].load(std::memory_order_relaxed) : 0;
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev < 64) of[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

constexpr int kBwdCtas = 4 * 160;  // at most, of q's and k's heads together; per SM as many as fit

// The lanes of a head, and chunks of heads of `un` steps at most, of about the same size.
void plan(Qk& a, int un, int heads, int& chunks) {
  const int per = 32 / a.lanes, steps = (heads + per - 1) / per;
  chunks = (steps + un - 1) / un;
}

template <typename T, typename W, int V, bool INTER>
cudaError_t fwd_t(Qk a, cudaStream_t s) {
  constexpr int UN = sizeof(T) == 2 ? 4 : 2;
  const int units = a.dim / 2 / V, per_lane = kPairs / V;
  for (a.lanes = 1; a.lanes * per_lane < units;) a.lanes *= 2;
  const int heads = a.heads[0] + a.heads[1], per = 32 / a.lanes, steps = (heads + per - 1) / per;
  plan(a, UN, heads, a.chunks[0]);
  a.steps = (steps + a.chunks[0] - 1) / a.chunks[0];
  const dim3 grid((a.tokens + kWarps - 1) / kWarps, a.chunks[0]);
  qk_fwd_kernel<T, W, V, INTER, UN><<<grid, dim3(32, kWarps), 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T, typename W, int V, bool INTER>
cudaError_t bwd_t(Qk a, float* dq, float* dk, cudaStream_t s) {
  constexpr int UN = sizeof(T) == 2 ? 2 : 1;
  const int units = a.dim / 2 / V, per_lane = kPairs / V;
  for (a.lanes = 1; a.lanes * per_lane < units;) a.lanes *= 2;
  a.steps = UN;
  const size_t smem = (size_t)kWarps * a.dim * sizeof(float);
  static std::atomic<int> per_sm{0};  // of this kernel, with the most shared memory it takes
  int fit = per_sm.load(std::memory_order_relaxed);
  if (fit == 0) {
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, qk_bwd_kernel<T, W, V, INTER, UN>,
                                                                        32 * kWarps, kWarps * kMaxDim * sizeof(float));
    if (e != cudaSuccess) return e;
    fit = std::max(1, std::min(4, fit));
    per_sm.store(fit, std::memory_order_relaxed);
  }
  const int sms = sm_count();
  if (sms < 1) return cudaErrorInvalidDevice;
  int64_t want[2];
  for (int k = 0; k < 2; ++k) {
    plan(a, UN, a.heads[k], a.chunks[k]);
    want[k] = ((int64_t)a.tokens * a.chunks[k] + kWarps - 1) / kWarps;
  }
  const int64_t most = std::min(kBwdCtas, sms * fit);
  uint32_t ctas[2] = {(uint32_t)std::min(want[0], most), (uint32_t)std::min(want[1], most)};
  if (want[0] + want[1] > most) {  // shares by their chunks
    for (int k = 0; k < 2; ++k)
      ctas[k] = (uint32_t)std::min<int64_t>(want[k], std::max<int64_t>(want[k] > 0, most * want[k] / (want[0] + want[1])));
  }
  a.ctas_q = ctas[0];
  qk_bwd_kernel<T, W, V, INTER, UN><<<ctas[0] + ctas[1], dim3(32, kWarps), a.partial ? smem : 0, s>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess && a.partial) {
    qk_sum_kernel<<<dim3((a.dim + 31) / 32, 2), dim3(32, kSumWarps), 0, s>>>(a.partial, ctas[0], ctas[0] + ctas[1], a.dim,
                                                                             dq, dk);
    e = cudaGetLastError();
  }
  return e;
}

template <typename F>
cudaError_t with_types(int32_t xt, int32_t wt, F&& f) {
  if (xt == SOAP_F32) return f(float(), float());
  if (xt == SOAP_BF16)
    return wt == SOAP_F32 ? f(__nv_bfloat16(), float()) : f(__nv_bfloat16(), __nv_bfloat16());
  return wt == SOAP_F32 ? f(__half(), float()) : f(__half(), __half());
}

// Operands' strides are not negative; results' are those of heads, tokens and sequences that lie apart.
bool bad_heads(const layer_heads_t* h, const Qk& a, int k, int64_t batch, size_t size, bool result) {
  if (a.heads[k] == 0 || a.tokens == 0) return false;
  if (!h || !h->data || odd_ptr(h->data, size)) return true;
  if (h->batch_stride < 0 || h->token_stride < 0 || h->head_stride < 0) return true;
  if (!result) return false;
  return (a.heads[k] > 1 && h->head_stride < a.dim) || (a.length > 1 && h->token_stride < a.dim) ||
         (batch > 1 && h->batch_stride < a.dim);
}

Heads heads_of(const layer_heads_t* h, const Qk& a, int k, int64_t batch) {
  if (a.heads[k] == 0 || !h) return Heads{};
  // (strides that nothing multiplies do not count)
  return Heads{h->data, batch > 1 ? h->batch_stride : 0, a.length > 1 ? h->token_stride : 0,
               a.heads[k] > 1 ? h->head_stride : 0};
}

// Checks what both passes have in common; false: refused.
bool common(Qk& a, int64_t batch, int64_t length, int32_t heads, int32_t kv_heads, int32_t dim, int32_t rotary,
            const layer_heads_t* q, const layer_heads_t* k, int32_t type, const void* q_weight, const void* k_weight,
            int32_t w_type, float eps, const float* cos, const float* sin, int64_t places, const void* positions,
            int32_t positions_64, int32_t* status) {
  if (batch < 0 || length < 0 || batch > kMaxTokens || length > kMaxTokens || batch * length > kMaxTokens) return false;
  if (heads < 0 || kv_heads < 0 || heads > kMaxHeads || kv_heads > kMaxHeads) return false;
  if (dim < 2 || dim > kMaxDim || dim % 2 || rotary < 0 || rotary > dim || rotary % 2) return false;
  if (type < SOAP_F32 || type > SOAP_F16 || (w_type != SOAP_F32 && w_type != type) || !(eps >= 0.f)) return false;
  if (odd_ptr(q_weight, dtype_size(w_type)) || odd_ptr(k_weight, dtype_size(w_type)) || odd_ptr(status, 4)) return false;
  a.tokens = (uint32_t)(batch * length);
  a.length = (uint32_t)std::max<int64_t>(length, 1);
  a.heads[0] = heads;
  a.heads[1] = kv_heads;
  a.dim = dim;
  a.rotary = rotary;
  if (rotary > 0) {
    if (odd_ptr(cos, 4) || odd_ptr(sin, 4) || odd_ptr(positions, positions_64 ? 8 : 4)) return false;
    if (places < 0 || (a.tokens > 0 && (!cos || !sin))) return false;
    a.cos = cos;
    a.sin = sin;
    a.places = places;
    a.positions = positions;
    a.positions_64 = positions_64;
  }
  const size_t size = dtype_size(type);
  if (bad_heads(q, a, 0, batch, size, false) || bad_heads(k, a, 1, batch, size, false)) return false;
  a.x[0] = heads_of(q, a, 0, batch);
  a.x[1] = heads_of(k, a, 1, batch);
  a.w[0] = q_weight;
  a.w[1] = k_weight;
  a.eps = eps;
  a.status = status;
  return true;
}

}  // namespace
}  // namespace soap

using namespace soap;

extern "C" {

soap_status_t layer_qk_forward(int64_t batch, int64_t length, int32_t heads, int32_t kv_heads, int32_t dim,
                               int32_t rotary, int32_t interleaved, const layer_heads_t* q, const layer_heads_t* k,
                               int32_t type, const void* q_weight, const void* k_weight, int32_t w_type, float eps,
                               const float* cos, const float* sin, int64_t places, const void* positions,
                               int32_t positions_64, const layer_heads_t* q_out, const layer_heads_t* k_out,
                               int32_t* status, soap_stream_t stream) {
  Qk a{};
  if (!common(a, batch, length, heads, kv_heads, dim, rotary, q, k, type, q_weight, k_weight, w_type, eps, cos, sin,
              places, positions, positions_64, status))
    return SOAP_ERR_INVALID_ARG;
  const size_t size = dtype_size(type);
  if (bad_heads(q_out, a, 0, batch, size, true) || bad_heads(k_out, a, 1, batch, size, true)) return SOAP_ERR_INVALID_ARG;
  if (a.tokens == 0 || heads + kv_heads == 0) return SOAP_OK;
  a.out[0] = heads_of(q_out, a, 0, batch);
  a.out[1] = heads_of(k_out, a, 1, batch);
  cudaStream_t s = (cudaStream_t)stream;
  const double n = (double)a.tokens * (heads + kv_heads) * dim;
  ProfScope prof(kFamElementwise, 8.0 * n, 2.0 * n * size, s);
  const cudaError_t e = with_types(type, w_type, [&](auto t, auto w) {
    using T = decltype(t);
    using W = decltype(w);
    return with_unit(unit_size(a, size, sizeof(W), false), [&](auto v) {
      constexpr int V = decltype(v)::value;
      if constexpr (V * sizeof(T) > 16) return cudaErrorInvalidValue;
      else return interleaved ? fwd_t<T, W, V, true>(a, s) : fwd_t<T, W, V, false>(a, s);
    });
  });
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

size_t layer_qk_workspace_bytes(int64_t batch, int64_t length, int32_t heads, int32_t kv_heads, int32_t dim) {
  if (batch < 0 || length < 0 || batch > kMaxTokens || length > kMaxTokens || batch * length > kMaxTokens) return 0;
  if (heads < 0 || kv_heads < 0 || heads > kMaxHeads || kv_heads > kMaxHeads || dim < 2 || dim > kMaxDim || dim % 2) return 0;
  // no more CTAs than there are heads, a warp's one at least
  const int64_t most = batch * length * (heads + (int64_t)kv_heads) + 2;
  return (size_t)std::min<int64_t>(kBwdCtas + 2, most) * dim * sizeof(float);
}

soap_status_t layer_qk_backward(int64_t batch, int64_t length, int32_t heads, int32_t kv_heads, int32_t dim,
                                int32_t rotary, int32_t interleaved, const layer_heads_t* dq,
                                const layer_heads_t* dk, const layer_heads_t* q, const layer_heads_t* k,
                                int32_t type, const void* q_weight, const void* k_weight, int32_t w_type, float eps,
                                const float* cos, const float* sin, int64_t places, const void* positions,
                                int32_t positions_64, const layer_heads_t* dx_q, const layer_heads_t* dx_k,
                                float* d_qweight, float* d_kweight, int32_t* status, void* workspace,
                                size_t workspace_bytes, soap_stream_t stream) {
  Qk a{};
  if (!common(a, batch, length, heads, kv_heads, dim, rotary, q, k, type, q_weight, k_weight, w_type, eps, cos, sin,
              places, positions, positions_64, status))
    return SOAP_ERR_INVALID_ARG;
  const size_t size = dtype_size(type);
  if (bad_heads(dq, a, 0, batch, size, false) || bad_heads(dk, a, 1, batch, size, false) ||
      bad_heads(dx_q, a, 0, batch, size, true) || bad_heads(dx_k, a, 1, batch, size, true))
    return SOAP_ERR_INVALID_ARG;
  if (!d_qweight != !d_kweight || odd_ptr(d_qweight, 4) || odd_ptr(d_kweight, 4)) return SOAP_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  if (a.tokens == 0 || heads + kv_heads == 0) {
    cudaError_t e = cudaSuccess;
    if (d_qweight) e = cudaMemsetAsync(d_qweight, 0, (size_t)dim * 4, s);
    if (e == cudaSuccess && d_kweight) e = cudaMemsetAsync(d_kweight, 0, (size_t)dim * 4, s);
    return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
  }
  if (d_qweight) {
    if (!workspace || odd_ptr(workspace, 16) ||
        workspace_bytes < layer_qk_workspace_bytes(batch, length, heads, kv_heads, dim))
      return SOAP_ERR_INVALID_ARG;
    a.partial = static_cast<float*>(workspace);
  }
  a.dy[0] = heads_of(dq, a, 0, batch);
  a.dy[1] = heads_of(dk, a, 1, batch);
  a.out[0] = heads_of(dx_q, a, 0, batch);
  a.out[1] = heads_of(dx_k, a, 1, batch);
  const double n = (double)a.tokens * (heads + kv_heads) * dim;
  ProfScope prof(kFamElementwise, 18.0 * n, 3.0 * n * size, s);
  const cudaError_t e = with_types(type, w_type, [&](auto t, auto w) {
    using T = decltype(t);
    using W = decltype(w);
    return with_unit(unit_size(a, size, sizeof(W), true), [&](auto v) {
      constexpr int V = decltype(v)::value;
      if constexpr (V * sizeof(T) > 16) return cudaErrorInvalidValue;
      else
        return interleaved ? bwd_t<T, W, V, true>(a, d_qweight, d_kweight, s)
                           : bwd_t<T, W, V, false>(a, d_qweight, d_kweight, s);
    });
  });
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

}  // extern "C"
