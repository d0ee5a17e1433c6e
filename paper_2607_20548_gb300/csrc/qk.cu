// Norms of queries and keys for each head with the rotation by position in the same pass, and the
// backward pass (include/layer.h, layer_qk_*).
//
//   r = 1 / sqrt(mean(x^2) + eps),  n = x r,  m = n w,  (a, b) -> (a c - b s, b c + a s)
//   dm: dy turned back,  g = dm w,  dx = r (g - n mean(g n)),  dw = sum dm n
//
// Bound by memory: x is read and y written once (backward: x and dy read, dx written once). Heads whose rows are whole
// 16-byte units come in by TMA, tiles of tokens and heads into a ring in shared memory; results leave from registers.
// Others, and calls of a few tokens, are read by the lanes that work on them. A pair of the rotation stays in one lane,
// so that turning it exchanges nothing: a lane holds 8 pairs of a head, as units of V neighbouring first and V
// neighbouring second elements (V: 16 bytes where the parts' sizes and alignments allow, else 2 or 1), and 1 to 32
// lanes a head. The mean of g n is r times that of g x, so that a head's two sums cross its lanes together. Arithmetic
// goes two elements at a time: with one, and with the angles, the tile's place and the rest worked out for every head
// in place of every four (backward two), instructions set the time (65536 tokens x 32 heads of 128 fp16, forward: 324 us,
// now 172 = 6.3 TB/s; 131072 x 20 bf16, both passes 1769, now 571 = 5.9 TB/s).
#include <algorithm>
#include <atomic>
#include <cstdint>

#include "../../include/layer.h"
#include "pair.h"
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
  uint32_t tokens, length, period;  // (period: the sequences' own length, where several count as one)
  int heads[2];  // q, k
  int dim, rotary;
  Heads x[2], out[2], dy[2];  // forward: x to out; backward: dy and x to out (dx)
  const void* w[2];
  float eps, inv_dim;
  const float *cos, *sin;
  int64_t places;
  const void* positions;
  int positions_64;
  int* status;
  int lanes;        // per head
  int steps;        // of 32 / lanes heads in a chunk
  int chunks[2];    // forward: of q's and k's heads together, in [0]
  // tiles: heads and tokens in one, tiles along the heads, heads between a lane's; tiles in all; slots of the ring and their bytes
  int tile_heads[2], tile_tokens[2], tile_chunks[2], tile_apart[2];
  uint32_t along[2];  // tiles along a sequence, 0: there is one sequence
  uint32_t tiles[2];
  int slots, slot_bytes;
  uint64_t wait_ns;
  const int* hold;
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

// A lane's 8 pairs: the first and the second elements, two by two, for the instructions that take two fp32 values.
struct Eight {
  float2 a[kPairs / 2], b[kPairs / 2];
};

// Pairs of unit i: elements 2 j and 2 j + 1 of the unit's 2 V, or element j of its halves.
template <bool INTER, typename T, int V>
__device__ __forceinline__ Eight unpack(const Raw<T, V>& r) {
  Eight o;
#pragma unroll
  for (int q = 0; q < kPairs / 2; ++q) {
    if constexpr (V == 1) {
      o.a[q] = make_float2(to_f32(r.a[2 * q].v[0]), to_f32(r.a[2 * q + 1].v[0]));
      o.b[q] = make_float2(to_f32(r.b[2 * q].v[0]), to_f32(r.b[2 * q + 1].v[0]));
    } else {
      const int i = 2 * q / V, j = 2 * q % V, e = 2 * j;
      if constexpr (!INTER) {
        o.a[q] = to_pair(r.a[i].v + j);
        o.b[q] = to_pair(r.b[i].v + j);
      } else {
        const float2 x = to_pair(e < V ? r.a[i].v + e : r.b[i].v + (e - V));
        const float2 y = to_pair(e + 2 < V ? r.a[i].v + e + 2 : r.b[i].v + (e + 2 - V));
        o.a[q] = make_float2(x.x, y.x);
        o.b[q] = make_float2(x.y, y.y);
      }
    }
  }
  return o;
}
template <bool INTER, typename T, int V>
__device__ __forceinline__ void pack(const Eight& o, Raw<T, V>& r) {
#pragma unroll
  for (int q = 0; q < kPairs / 2; ++q) {
    if constexpr (V == 1) {
      r.a[2 * q].v[0] = from_f32<T>(o.a[q].x), r.a[2 * q + 1].v[0] = from_f32<T>(o.a[q].y);
      r.b[2 * q].v[0] = from_f32<T>(o.b[q].x), r.b[2 * q + 1].v[0] = from_f32<T>(o.b[q].y);
    } else {
      const int i = 2 * q / V, j = 2 * q % V, e = 2 * j;
      if constexpr (!INTER) {
        from_pair(o.a[q], r.a[i].v + j);
        from_pair(o.b[q], r.b[i].v + j);
      } else {
        from_pair(make_float2(o.a[q].x, o.b[q].x), e < V ? r.a[i].v + e : r.b[i].v + (e - V));
        from_pair(make_float2(o.a[q].y, o.b[q].y), e + 2 < V ? r.a[i].v + e + 2 : r.b[i].v + (e + 2 - V));
      }
    }
  }
}
__device__ __forceinline__ float dot(const Eight& x, const Eight& y) {
  float2 t = mul2(x.a[0], y.a[0]), u = mul2(x.b[0], y.b[0]);
#pragma unroll
  for (int q = 1; q < kPairs / 2; ++q) {
    t = fma2(x.a[q], y.a[q], t);
    u = fma2(x.b[q], y.b[q], u);
  }
  t = add2(t, u);
  return t.x + t.y;
}
__device__ __forceinline__ Eight times(const Eight& x, const Eight& y) {
  Eight o;
#pragma unroll
  for (int q = 0; q < kPairs / 2; ++q) o.a[q] = mul2(x.a[q], y.a[q]), o.b[q] = mul2(x.b[q], y.b[q]);
  return o;
}
__device__ __forceinline__ Eight times(const Eight& x, float r) {
  Eight o;
#pragma unroll
  for (int q = 0; q < kPairs / 2; ++q) o.a[q] = mul2(x.a[q], pair(r)), o.b[q] = mul2(x.b[q], pair(r));
  return o;
}
__device__ __forceinline__ Eight times_one(float r) {
  Eight o;
#pragma unroll
  for (int q = 0; q < kPairs / 2; ++q) o.a[q] = o.b[q] = pair(r);
  return o;
}
__device__ __forceinline__ Eight fma8(const Eight& x, const Eight& y, const Eight& z) {
  Eight o;
#pragma unroll
  for (int q = 0; q < kPairs / 2; ++q) o.a[q] = fma2(x.a[q], y.a[q], z.a[q]), o.b[q] = fma2(x.b[q], y.b[q], z.b[q]);
  return o;
}

// The angles of a lane's pairs: cosines, sines.
struct Angles {
  float2 c[kPairs / 2], s[kPairs / 2];
};
// Each pair (a, b) -> (a c - b s, b c + a s), or back.
template <bool BACK>
__device__ __forceinline__ Eight turn(const Eight& m, const Angles& t) {
  Eight o;
#pragma unroll
  for (int q = 0; q < kPairs / 2; ++q) {
    const float2 less = make_float2(-t.s[q].x, -t.s[q].y);
    o.a[q] = fma2(m.b[q], BACK ? t.s[q] : less, mul2(m.a[q], t.c[q]));
    o.b[q] = fma2(m.a[q], BACK ? less : t.s[q], mul2(m.b[q], t.c[q]));
  }
  return o;
}
// What is turned by v's angle, from c and s of V neighbouring pairs.
template <int V>
__device__ __forceinline__ void load_angles(Angles& t, int i, const float* cos, const float* sin, bool turns) {
  float c[V], s[V];
  if (turns) {
    load_f32<V>(cos, c);
    load_f32<V>(sin, s);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) c[e] = 1.f, s[e] = 0.f;
  }
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int p = i * V + e;
    if (p % 2)
      t.c[p / 2].y = c[e], t.s[p / 2].y = s[e];
    else
      t.c[p / 2].x = c[e], t.s[p / 2].x = s[e];
  }
}

// The forward pass of a head in x, whose sum of squares is xx, in place; the backward pass, which adds to dw too.
template <bool INTER, typename T, int V>
__device__ __forceinline__ void forward(Raw<T, V>& x, float r, const Eight& w, const Angles& t) {
  pack<INTER>(turn<false>(times(times(unpack<INTER>(x), r), w), t), x);
}
template <bool INTER, typename T, int V>
__device__ __forceinline__ void backward(Raw<T, V>& x, const Eight& dm, float r, float mean, const Eight& w, Eight& dw) {
  const Eight n = times(unpack<INTER>(x), r);
  dw = fma8(dm, n, dw);
  pack<INTER>(fma8(n, times_one(-r * mean), times(times(dm, w), r)), x);
}

// The same from shared memory, where there is always something to read.
template <typename T, int V, bool INTER>
__device__ __forceinline__ void take(Raw<T, V>& r, const T* p, const Units<V, INTER>& un, int lane, int lanes) {
#pragma unroll
  for (int i = 0; i < kPairs / V; ++i) {
    const int u = i * lanes + lane;
    if (un.has(u)) {
      r.a[i] = *reinterpret_cast<const Pack<T, V>*>(p + un.first(u));
      r.b[i] = *reinterpret_cast<const Pack<T, V>*>(p + un.second(u));
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) r.a[i].v[e] = r.b[i].v[e] = from_f32<T>(0.f);
    }
  }
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
__device__ __forceinline__ bool angles(const Qk& a, uint32_t token, const Units<V, INTER>& un, int lane, Angles& t) {
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
    const int64_t j = at * (a.rotary / 2) + u * V;
    load_angles<V>(t, i, a.cos + j, a.sin + j, ok && un.turns(u));
  }
  return ok;
}

// The weights of a lane's pairs.
template <typename W, int V, bool INTER>
__device__ __forceinline__ void weights(const void* w, const Units<V, INTER>& un, int lane, int lanes, Eight& v) {
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
      const int p = i * V + j;
      const float first = !INTER ? x[j] : 2 * j < V ? x[(2 * j) % V] : y[(2 * j) % V];
      const float second = !INTER ? y[j] : 2 * j + 1 < V ? x[(2 * j + 1) % V] : y[(2 * j + 1) % V];
      if (p % 2)
        v.a[p / 2].y = first, v.b[p / 2].y = second;
      else
        v.a[p / 2].x = first, v.b[p / 2].x = second;
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
  Angles t;
  const bool ok = angles(a, token, un, lane, t);
  if (!ok && threadIdx.x == 0 && a.status) atomicOr(a.status, kStatusRange);
#pragma unroll
  for (int s = 0; s < UN; ++s) {
    if (s >= a.steps) break;
    const int h = h0 + s * per, k = h >= a.heads[0];
    const Eight v = unpack<INTER>(x[s]);
    const float sum = lanes_sum(dot(v, v), lanes);
    if (h >= all) continue;  // (the exchange above takes all lanes)
    const float r = ok ? rsqrtf(fmaf(sum, a.inv_dim, a.eps)) : NAN;
    Eight w;
    weights<W>(a.w[k], un, lane, lanes, w);
    forward<INTER>(x[s], r, w, t);
    store(static_cast<T*>(a.out[k].p) + place_of(a.out[k], a, token, k ? h - a.heads[0] : h), x[s], un, lane, lanes);
  }
}

// A CTA's part of dweight: the sums over a warp's heads, then over the CTA's warps, always in the same order.
template <int V, bool INTER>
__device__ __forceinline__ void put_sums(const Eight& dw, float* row, const Units<V, INTER>& un, int lane, int lanes,
                                         bool first) {
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    float x = i % 2 ? dw.a[i / 2].y : dw.a[i / 2].x, y = i % 2 ? dw.b[i / 2].y : dw.b[i / 2].x;
    for (int o = lanes; o < 32; o <<= 1) {
      x += __shfl_xor_sync(0xffffffffu, x, o);
      y += __shfl_xor_sync(0xffffffffu, y, o);
    }
    const int u = (i / V) * lanes + lane, j = i % V;
    if (first && un.has(u)) {
      row[INTER ? un.first(u) + 2 * j : un.first(u) + j] = x;
      row[INTER ? un.first(u) + 2 * j + 1 : un.second(u) + j] = y;
    }
  }
}
__device__ __forceinline__ void add_sums(const float* sums, const Qk& a, int thread, int threads) {
  for (int j = thread; j < a.dim; j += threads) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) t += sums[i * a.dim + j];
    a.partial[(int64_t)blockIdx.x * a.dim + j] = t;
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
  Eight w, dw = times_one(0.f);
  weights<W>(a.w[k], un, lane, lanes, w);
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
    Angles t;
    const bool ok = angles(a, token, un, lane, t);
    if (!ok && threadIdx.x == 0 && a.status) atomicOr(a.status, kStatusRange);
#pragma unroll
    for (int s = 0; s < UN; ++s) {
      if (s >= a.steps) break;
      const int h = h0 + s * per;
      const Eight v = unpack<INTER>(x[s]), dm = turn<true>(unpack<INTER>(dy[s]), t);
      const float xx = lanes_sum(dot(v, v), lanes), gx = lanes_sum(dot(times(dm, w), v), lanes);
      if (h >= all) continue;
      const float r = ok ? rsqrtf(fmaf(xx, a.inv_dim, a.eps)) : NAN;
      backward<INTER>(x[s], dm, r, r * (gx * a.inv_dim), w, dw);
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
  put_sums<V, INTER>(dw, sums + threadIdx.y * a.dim, un, lane, lanes, at == 0);
  __syncthreads();
  add_sums(sums, a, threadIdx.y * 32 + threadIdx.x, 32 * kWarps);
}

// ---- heads in tiles ----

struct QkMaps {
  CUtensorMap x[2], dy[2];  // of q, of k: (element, head, token, sequence)
};

constexpr int kRingBytes = 98304;  // two CTAs per SM
constexpr int kMaxSlots = 12;

__device__ __forceinline__ void load_heads(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int h, int t, int b) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(tc::smem_u32(bar)), "r"(0), "r"(h), "r"(t), "r"(b)
      : "memory");
}
// Where tile i of q's (k = 0) or k's heads is.
struct Tile {
  int h0;
  uint32_t b, t0;  // sequence, first token in it
};
__device__ __forceinline__ Tile tile_at(const Qk& a, int k, uint32_t i) {
  const uint32_t chunks = a.tile_chunks[k];
  uint32_t row = i, b = 0;
  if (chunks > 1) row = i / chunks;
  const int h0 = (int)(i - row * chunks) * a.tile_heads[k];
  if (a.along[k] > 0) {  // several sequences
    b = row / a.along[k];
    row -= b * a.along[k];
  }
  return Tile{h0, b, row * a.tile_tokens[k]};
}

// Persistent CTAs, the first ctas_q of them for q's heads, the others for k's, each with every (its CTAs)-th tile. The
// angles of a lane's token in the next tile are on their way to its registers while it works on this one, from the L1
// for all heads of a token but the first, and the position in the tile after that. (Rows of angles brought into the
// ring by one warp, by bulk copies or 16 bytes a lane, took that warp 100 ns a token.)
template <typename T, typename W, int V, bool INTER, bool BACK>
__global__ void __launch_bounds__(32 * kWarps, 2)
    qk_tile_kernel(const __grid_constant__ QkMaps maps, const __grid_constant__ Qk a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kMaxSlots], empty[kMaxSlots];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~uintptr_t(127));
  const int k = blockIdx.x >= a.ctas_q;
  const uint32_t cta = blockIdx.x - (k ? a.ctas_q : 0), ctas = k ? gridDim.x - a.ctas_q : a.ctas_q;
  const int lane32 = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int HB = a.tile_heads[k], TB = a.tile_tokens[k];
  // a slot: x's tile, backward dy's
  const int tile_bytes = HB * TB * a.dim * (int)sizeof(T), dy_at = (tile_bytes + 127) & ~127;
  auto request = [&](uint32_t i, int s) {
    const Tile t = tile_at(a, k, i);
    uint8_t* const slot = smem + s * a.slot_bytes;
    tc::expect_tx(&full[s], (BACK ? 2 : 1) * tile_bytes);
    load_heads(tc::smem_u32(slot), &maps.x[k], &full[s], t.h0, t.t0, t.b);
    if (BACK) load_heads(tc::smem_u32(slot + dy_at), &maps.dy[k], &full[s], t.h0, t.t0, t.b);
  };
  if (threadIdx.x == 0) {
    for (int s = 0; s < a.slots; ++s) {
      tc::mbar_init(&full[s], 1);
      tc::mbar_init(&empty[s], kWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    // (a flag that nothing sets: nothing is asked for, and the waits run out)
    const bool held = a.hold && !tc::flag_wait(a.hold, a.wait_ns);
    for (int s = 0; s < a.slots && !held; ++s)
      if (cta + s * ctas < a.tiles[k]) request(cta + s * ctas, s);
  }
  // a lane has heads in_tile, in_tile + apart, ... of a token in the tile
  const int lanes = a.lanes, lane = lane32 & (lanes - 1), group = threadIdx.x / lanes, apart = a.tile_apart[k];
  const Units<V, INTER> un{a.dim, a.rotary};
  const int in_tile = group % apart, token_in_tile = group / apart;
  const bool real = token_in_tile < TB;
  // (a lane without a head of the tile's reads another one's, and stores nothing)
  const int from = (real ? token_in_tile * HB + in_tile : 0) * a.dim;
  const Heads& o = a.out[k];
  T* const out = static_cast<T*>(o.p) + (int64_t)in_tile * o.head + (int64_t)token_in_tile * o.token;
  const int64_t out_apart = (int64_t)apart * o.head;
  // the position of this lane's token in tile i; -1: there is none
  auto position = [&](uint32_t i) -> int64_t {
    if (a.rotary == 0 || !real || i >= a.tiles[k]) return -1;
    const Tile t = tile_at(a, k, i);
    const uint32_t in = t.t0 + token_in_tile, token = t.b * a.length + in;
    if (in >= a.length) return -1;
    if (!a.positions) return token % a.period;
    return a.positions_64 ? static_cast<const int64_t*>(a.positions)[token] : static_cast<const int32_t*>(a.positions)[token];
  };
  auto angles_of = [&](Angles& t, int64_t at) {
    const bool in = at >= 0 && at < a.places;
    const int64_t first = (in ? at : 0) * (a.rotary / 2);
#pragma unroll
    for (int j = 0; j < kPairs / V; ++j) {
      const int u = j * lanes + lane;
      load_angles<V>(t, j, a.cos + first + u * V, a.sin + first + u * V, in && un.turns(u));
    }
    return in || a.rotary == 0;
  };
  Eight w, dw = times_one(0.f);
  weights<W>(a.w[k], un, lane, lanes, w);
  // (backward there are no registers for two tiles' angles: they come for this tile, the position is there before)
  Angles turns;
  bool in_table = true;
  int64_t next_at = position(cta);
  if (!BACK) {
    in_table = angles_of(turns, next_at);
    next_at = position(cta + ctas);
  }
  __syncthreads();
  int s = 0;
  uint32_t parity = 0;
  bool ok = true;
  for (uint32_t i = cta; i < a.tiles[k]; i += ctas) {
    const uint8_t* const slot = smem + s * a.slot_bytes;
    Angles next;
    bool next_in = true;
    if (BACK) {
      in_table = angles_of(turns, next_at);
      next_at = position(i + ctas);
    } else {
      next_in = angles_of(next, next_at);
      next_at = position(i + 2 * ctas);
    }
    // after a wait that ran out: nothing more is waited for, all results become NaN
    if (ok && !tc::mbar_wait(&full[s], parity, 2 * a.wait_ns)) {
      ok = false;
      if (a.status) atomicOr(a.status, kStatusTimeout);
    }
    ok = __all_sync(0xffffffffu, ok);
    const Tile t = tile_at(a, k, i);
    const int heads = min(HB, a.heads[k] - t.h0);  // of this tile
    const bool there = real && t.t0 + token_in_tile < a.length, good = ok && in_table;
    if (there && ok && !in_table && a.status) atomicOr(a.status, kStatusRange);
    T* to = out + (int64_t)t.b * o.batch + (int64_t)t.t0 * o.token + (int64_t)t.h0 * o.head;
    const T* at = reinterpret_cast<const T*>(slot) + from;
    for (int h = in_tile; h - in_tile < heads; h += apart, to += out_apart, at += apart * a.dim) {
      Raw<T, V> x, dy;
      const bool live = there && h < heads;
      const T* const own = h < HB ? at : at - apart * a.dim;
      take(x, own, un, lane, lanes);
      if (BACK) take(dy, reinterpret_cast<const T*>(reinterpret_cast<const uint8_t*>(own) + dy_at), un, lane, lanes);
      const Eight v = unpack<INTER>(x);
      const float r = rsqrtf(fmaf(lanes_sum(dot(v, v), lanes), a.inv_dim, a.eps));
      if constexpr (BACK) {
        const Eight dm = turn<true>(unpack<INTER>(dy), turns);
        const float gx = lanes_sum(dot(times(dm, w), v), lanes);
        if (live) {  // (the exchanges above take all lanes)
          const float rr = good ? r : NAN;
          backward<INTER>(x, dm, rr, rr * (gx * a.inv_dim), w, dw);
          store(to, x, un, lane, lanes);
        }
      } else if (live) {
        forward<INTER>(x, good ? r : NAN, w, turns);
        store(to, x, un, lane, lanes);
      }
    }
    __syncwarp();
    if (lane32 == 0) {
      asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(tc::smem_u32(&empty[s])) : "memory");
      if (warp == (s & (kWarps - 1)) && ok && i != cta) {  // the slot before this one is free, or soon: what comes next there
        const int before = s > 0 ? s - 1 : a.slots - 1;
        const uint64_t far = (uint64_t)i + (uint64_t)(a.slots - 1) * ctas;
        if (far < a.tiles[k]) {
          if (tc::mbar_wait(&empty[before], s > 0 ? parity : parity ^ 1, 2 * a.wait_ns)) request((uint32_t)far, before);
        }
      }
    }
    if (++s == a.slots) {
      s = 0;
      parity ^= 1;
    }
    if (!BACK) {
      turns = next;
      in_table = next_in;
    }
  }
  if (!ok) {  // copies in flight land before the shared memory goes away: far above a copy's time
    const uint64_t t0 = tc::globaltimer();
    while (tc::globaltimer() - t0 < 10000000ull) {
    }
  }
  if (!BACK || !a.partial) return;
  __syncthreads();  // nothing of the ring is used any more
  float* const sums = reinterpret_cast<float*>(smem);
  put_sums<V, INTER>(dw, sums + warp * a.dim, un, lane, lanes, lane32 < lanes);
  __syncthreads();
  add_sums(sums, a, threadIdx.x, blockDim.x);
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
  for (int V = (int)(16 / size); V > 1; V = V > 2 ? 2 : 1) {  // (8 or 4, 2, 1)
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
  if (V == 4) return f(std::integral_constant<int, 4>());  // (fp32)
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

void share_ctas(Qk& a, const int64_t (&want)[2], int64_t most, uint32_t (&ctas)[2]) {
  for (int k = 0; k < 2; ++k) ctas[k] = (uint32_t)std::min(want[k], most);
  if (want[0] + want[1] > most) {  // shares by their work
    for (int k = 0; k < 2; ++k)
      ctas[k] = (uint32_t)std::min<int64_t>(want[k], std::max<int64_t>(want[k] > 0, most * want[k] / (want[0] + want[1])));
  }
  a.ctas_q = ctas[0];
}

cudaError_t sum_parts(const Qk& a, const uint32_t (&ctas)[2], float* dq, float* dk, cudaStream_t s) {
  if (!a.partial) return cudaSuccess;
  qk_sum_kernel<<<dim3((a.dim + 31) / 32, 2), dim3(32, kSumWarps), 0, s>>>(a.partial, ctas[0], ctas[0] + ctas[1], a.dim, dq, dk);
  return cudaGetLastError();
}

bool heads_map(CUtensorMap* map, const Heads& h, const Qk& a, int k, uint32_t batch, CUtensorMapDataType type, size_t size) {
  auto fn = tc::encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)a.dim, (cuuint64_t)a.heads[k], a.length, batch};
  // (a step that is never taken: any)
  auto step = [&](int64_t n, int64_t stride) { return (cuuint64_t)(n > 1 ? stride * (int64_t)size : 16); };
  const cuuint64_t strides[3] = {step(a.heads[k], h.head), step(a.length, h.token), step(batch, h.batch)};
  const cuuint32_t box[4] = {(cuuint32_t)a.dim, (cuuint32_t)a.tile_heads[k], (cuuint32_t)a.tile_tokens[k], 1};
  const cuuint32_t steps[4] = {1, 1, 1, 1};
  return fn(map, type, 4, h.p, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles of heads, where they can be copied as such and there is enough to do; done: whether that was so. Below two tiles
// for every SM the lanes' own loads are as quick.
template <typename T, typename W, int V, bool INTER, bool BACK>
cudaError_t tiles_t(Qk a, float* dq, float* dk, cudaStream_t s, bool& done) {
  done = false;
  if (a.dim > 256 || a.dim * sizeof(T) % 16) return cudaSuccess;
  for (int k = 0; k < 2; ++k)
    if (a.heads[k] > 0 && !(units_fit(a.x[k], 16 / sizeof(T), sizeof(T), true) &&
                            (!BACK || units_fit(a.dy[k], 16 / sizeof(T), sizeof(T), true))))
      return cudaSuccess;
  uint32_t batch = a.tokens / a.length;
  // sequences that lie one behind the other are one
  a.period = a.length;
  bool one = true;
  for (int k = 0; k < 2 && batch > 1; ++k)
    for (const Heads* h : {&a.x[k], &a.out[k], &a.dy[k]})
      one = one && (!h->p || h->batch == (int64_t)a.length * h->token);
  if (one) {
    a.length = a.tokens;
    batch = 1;
  }
  const int per_lane = kPairs / V;
  for (a.lanes = 1; a.lanes * per_lane < a.dim / 2 / V;) a.lanes *= 2;
  const int rows = kWarps * 32 / a.lanes, several = sizeof(T) == 4 ? 1 : BACK ? 2 : 4;
  int64_t want[2];
  int bytes = 0;
  for (int k = 0; k < 2; ++k) {
    want[k] = a.tiles[k] = 0;
    if (a.heads[k] == 0) continue;
    for (const Heads* h : {&a.x[k], &a.dy[k]})
      if (h->p && ((a.heads[k] > 1 && h->head < a.dim) || (a.length > 1 && h->token < 1) || (batch > 1 && h->batch < 1)))
        return cudaSuccess;
    // (a lane takes up to `several` heads of its token: what a tile costs beside its heads is shared by them)
    a.tile_heads[k] = std::min({a.heads[k], rows * several, 256});
    a.tile_apart[k] = (a.tile_heads[k] + several - 1) / several;
    a.tile_tokens[k] = std::min(256, rows / a.tile_apart[k]);
    a.tile_chunks[k] = (a.heads[k] + a.tile_heads[k] - 1) / a.tile_heads[k];
    a.along[k] = batch > 1 ? (a.length + a.tile_tokens[k] - 1) / a.tile_tokens[k] : 0;
    const int64_t n = (int64_t)batch * ((a.length + a.tile_tokens[k] - 1) / a.tile_tokens[k]) * a.tile_chunks[k];
    if (n > UINT32_MAX / 2 || (int64_t)a.tile_tokens[k] > 8 * (int64_t)a.length) return cudaSuccess;
    want[k] = a.tiles[k] = (uint32_t)n;
    const int tile = (a.tile_heads[k] * a.tile_tokens[k] * a.dim * (int)sizeof(T) + 127) & ~127;
    bytes = std::max(bytes, (BACK ? 2 : 1) * tile);
  }
  const int sms = sm_count();
  if (sms < 1) return cudaErrorInvalidDevice;
  if (want[0] + want[1] < 2 * sms) return cudaSuccess;
  a.slot_bytes = (bytes + 127) & ~127;
  a.slots = std::min(kMaxSlots, kRingBytes / a.slot_bytes);
  if (a.slots < 2) return cudaSuccess;
  const CUtensorMapDataType type = sizeof(T) == 4                          ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : std::is_same<T, __nv_bfloat16>::value ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                                           : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  QkMaps maps{};
  for (int k = 0; k < 2; ++k)
    if (a.heads[k] > 0 && (!heads_map(&maps.x[k], a.x[k], a, k, batch, type, sizeof(T)) ||
                           (BACK && !heads_map(&maps.dy[k], a.dy[k], a, k, batch, type, sizeof(T)))))
      return cudaSuccess;  // (steps beyond what a map holds)
  const WaitLimit limit = wait_limit();
  a.wait_ns = limit.ns;
  a.hold = limit.hold;
  auto kernel = qk_tile_kernel<T, W, V, INTER, BACK>;
  constexpr int smem = kRingBytes + 128;
  static std::atomic<bool> set[64];  // the kernel's shared-memory attribute, per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev >= 64 || !set[dev].load(std::memory_order_relaxed))) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess && dev < 64) set[dev].store(true, std::memory_order_relaxed);
  }
  if (e != cudaSuccess) return e;
  uint32_t ctas[2];
  share_ctas(a, want, 2 * sms, ctas);
  kernel<<<ctas[0] + ctas[1], 32 * kWarps, smem, s>>>(maps, a);
  e = cudaGetLastError();
  if (e == cudaSuccess) e = sum_parts(a, ctas, dq, dk, s);
  done = true;
  return e;
}

template <typename T, typename W, int V, bool INTER>
cudaError_t fwd_t(Qk a, cudaStream_t s) {
  bool done;
  const cudaError_t e = tiles_t<T, W, V, INTER, false>(a, nullptr, nullptr, s, done);
  if (done || e != cudaSuccess) return e;
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
  bool done;
  const cudaError_t tiled = tiles_t<T, W, V, INTER, true>(a, dq, dk, s, done);
  if (done || tiled != cudaSuccess) return tiled;
  constexpr int UN = sizeof(T) == 2 ? 2 : 1;
  const int units = a.dim / 2 / V, per_lane = kPairs / V;
  for (a.lanes = 1; a.lanes * per_lane < units;) a.lanes *= 2;
  a.steps = UN;
  const size_t smem = (size_t)kWarps * a.dim * sizeof(float);
  static std::atomic<int> per_sm[64];  // of this kernel, with the most shared memory it takes, per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  int fit = dev < 64 ? per_sm[dev].load(std::memory_order_relaxed) : 0;
  if (fit == 0) {
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, qk_bwd_kernel<T, W, V, INTER, UN>, 32 * kWarps,
                                                      kWarps * kMaxDim * sizeof(float));
    if (e != cudaSuccess) return e;
    fit = std::max(1, std::min(4, fit));
    if (dev < 64) per_sm[dev].store(fit, std::memory_order_relaxed);
  }
  const int sms = sm_count();
  if (sms < 1) return cudaErrorInvalidDevice;
  int64_t want[2];
  for (int k = 0; k < 2; ++k) {
    plan(a, UN, a.heads[k], a.chunks[k]);
    want[k] = ((int64_t)a.tokens * a.chunks[k] + kWarps - 1) / kWarps;
  }
  const int64_t most = std::min(kBwdCtas, sms * fit);
  uint32_t ctas[2];
  share_ctas(a, want, most, ctas);
  qk_bwd_kernel<T, W, V, INTER, UN><<<ctas[0] + ctas[1], dim3(32, kWarps), a.partial ? smem : 0, s>>>(a);
  e = cudaGetLastError();
  return e == cudaSuccess ? sum_parts(a, ctas, dq, dk, s) : e;
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
    if (places < 0 || places > INT32_MAX || (a.tokens > 0 && (!cos || !sin))) return false;
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
  a.inv_dim = 1.f / (float)dim;
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
      if constexpr (V > 2 && V * sizeof(T) != 16) return cudaErrorInvalidValue;
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
      if constexpr (V > 2 && V * sizeof(T) != 16) return cudaErrorInvalidValue;
      else
        return interleaved ? bwd_t<T, W, V, true>(a, d_qweight, d_kweight, s)
                           : bwd_t<T, W, V, false>(a, d_qweight, d_kweight, s);
    });
  });
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

}  // extern "C"
