// What the feed-forward block's two kernels share on the device.
#pragma once

#include "../../include/layer.h"
#include "ffn.h"
#include "types.h"

namespace soap {
namespace ffn {

template <int TYPE>
struct Element;
template <>
struct Element<SOAP_F32> {
  using T = float;
};
template <>
struct Element<SOAP_BF16> {
  using T = __nv_bfloat16;
};
template <>
struct Element<SOAP_F16> {
  using T = __half;
};

// The plan's numbers that every unit takes.
struct Head {
  int total, first[3], tiles[2], splits[2], parts;
};
// The largest i < n with prefix[i] <= q; all lanes of a warp take part (one round of loads for up to 32 groups, two
// beyond: a binary search's dependent ones took longer than a small unit).
__device__ __forceinline__ int group_of(const int* prefix, int n, int q) {
  const int lane = threadIdx.x & 31, step = up_div(n, 32);
  int i = lane * step;
  const unsigned coarse = __ballot_sync(0xffffffffu, i < n && prefix[i] <= q);
  const int first = (31 - __clz(coarse)) * step;
  if (step == 1) return first;
  i = first + lane;
  return first + 31 - __clz(__ballot_sync(0xffffffffu, lane < step && i < n && prefix[i] <= q));
}

// Tile i of nm x nn in groups of 8 row tiles, row tile fastest, so that tiles in flight share operands in L2.
__device__ __forceinline__ void tile_place(int i, int nm, int nn, int& m, int& n) {
  const int of8 = 8 * nn, gr = i / of8, in = i - gr * of8, rows = min(8, nm - gr * 8);
  n = in / rows;
  m = gr * 8 + in - n * rows;
}

// act(g) and its derivative. 16-bit results: the hardware's exponential and quotient (2^-21 of the result).
template <int TYPE, int ACT>
__device__ __forceinline__ void activation(float g, float& a, float& da) {
  if (ACT == LAYER_SILU) {
    const float s = TYPE == SOAP_F32 ? 1.f / (1.f + expf(-g)) : __fdividef(1.f, 1.f + __expf(-g));
    a = g * s;
    da = s * fmaf(g, 1.f - s, 1.f);
  } else {
    const float p = 0.5f * (1.f + erff(g * 0.70710678118654752f));
    const float e = TYPE == SOAP_F32 ? expf(-0.5f * g * g) : __expf(-0.5f * g * g);
    a = g * p;
    da = fmaf(g * 0.3989422804014327f, e, p);
  }
}
// A block's rows: v = act(v) w; or, from g, u and v = dh: g = dg, u = h, v = du. One of two straight pieces of code (a
// choice per element has the instructions of both fetched: 8 us of a small call's 55).
template <int TYPE, int ACT>
__device__ __forceinline__ void gate(float (&v)[32], const float (&w)[32]) {
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    float a, da;
    activation<TYPE, ACT>(v[j], a, da);
    v[j] = a * w[j];
  }
}
template <int TYPE, int ACT>
__device__ __forceinline__ void gate_back(float (&g)[32], float (&u)[32], float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    float a, da;
    activation<TYPE, ACT>(g[j], a, da);
    g[j] = v[j] * u[j] * da;
    u[j] *= a;
    v[j] *= a;
  }
}

// 32 elements of this lane's row to or from a block in which the rows' 16-byte pieces lie side by side (at p: this
// lane's first).
__device__ __forceinline__ void put_lines(float4* p, const float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) p[32 * j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
}
__device__ __forceinline__ void get_lines(const float4* p, float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float4 x = p[32 * j];
    v[4 * j] = x.x, v[4 * j + 1] = x.y, v[4 * j + 2] = x.z, v[4 * j + 3] = x.w;
  }
}
// (what other CTAs have stored meanwhile: past this SM's L1)
__device__ __forceinline__ void get_lines_l2(const float4* p, float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float4 x = __ldcg(p + 32 * j);
    v[4 * j] = x.x, v[4 * j + 1] = x.y, v[4 * j + 2] = x.z, v[4 * j + 3] = x.w;
  }
}

}  // namespace ffn
}  // namespace soap
