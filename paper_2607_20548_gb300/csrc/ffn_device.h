// What the feed-forward block's two kernels share on the device.
#pragma once

#include <climits>

#include "../../include/layer.h"
#include "ffn.h"
#include "pair.h"
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
// Parts along K of a tile of `slices` slices (0: none), where there may be `most` for the pairs' sake: a part of p
// costs its slices' time, 0.3 us for each of their products of planes, and adding up p parts 5 us and about as much as a slice for each, so that
// short sums stay whole, and the best p for others is about the root of those products' number.
__device__ __forceinline__ int parts_of(int slices, int most, int products) {
  if (slices == 0) return 0;
  const int whole = max(1, up_div(slices, kMaxSlices)), cost = slices * products;
  return cost < kMinParted ? whole : max(whole, min(most, min(slices, (int)sqrtf((float)cost))));
}

// The list of `tiles` row tiles, and of `parts` parts along the rows for each tile of the weights' gradients.
__device__ __forceinline__ Head head_of(const Args& a, int tiles, int parts) {
  Head h;
  int at = 0;
  for (int p = 0; p < 2; ++p) {
    const int n = tiles * up_div(p == 0 ? a.width : a.hidden, a.col_tile[p]);
    h.first[p] = at;
    h.tiles[p] = n;
    h.splits[p] = n > 0 ? parts_of(a.slices[p], a.pool / n, a.products) : 1;
    if (p == 0 && a.h) h.splits[p] = 1;  // (few rows: g and u meet in the tile)
    at += n * h.splits[p];
  }
  h.first[2] = at;
  h.parts = parts;
  h.total = at + parts * (a.each[0] + a.each[1] + a.each[2]);
  return h;
}
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

// What a scout's lanes hold of up to 64 groups, lane and lane + 32 of each, so that a unit's place takes no loads (a
// chain of five, 4 us with the memory busy, when the units of 8 slices took 2.3). Dense: one group of all rows.
struct Groups {
  bool held;      // else there are more, and units look in memory
  bool all_done;  // the first phase is stored: nothing more is waited for
  int tiles[2], length[2], start[2], blocks[2], parts[2], part_count[2], slots[2];

  __device__ __forceinline__ void load(const Args& a) {
    const Plan& l = *a.plan;
    const int lane = threadIdx.x & 31;
    all_done = false;
    held = a.groups <= 64;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int g = lane + 32 * h;
      const bool in = held && g < a.groups;
      tiles[h] = in ? l.row_tiles[g] : INT_MAX;
      start[h] = in ? l.bounds[g] : 0;
      length[h] = in ? l.bounds[g + 1] - l.bounds[g] : 0;
      blocks[h] = in ? l.blocks[g] : 0;
      parts[h] = in ? l.parts[g] : INT_MAX;
      part_count[h] = in ? l.parts[g + 1] - l.parts[g] : 0;
      slots[h] = in ? l.slots[g] : 0;
    }
  }
  // The last group whose count before it is at most q.
  __device__ __forceinline__ static int find(const int (&before)[2], int q) {
    const unsigned lo = __ballot_sync(0xffffffffu, before[0] <= q), hi = __ballot_sync(0xffffffffu, before[1] <= q);
    return hi ? 63 - __clz(hi) : 31 - __clz(lo);
  }
  __device__ __forceinline__ static int of(const int (&v)[2], int g) {
    const int lo = __shfl_sync(0xffffffffu, v[0], g & 31), hi = __shfl_sync(0xffffffffu, v[1], g & 31);
    return g < 32 ? lo : hi;
  }
  // Whether all groups' rows of the first phase are stored, `stored` blocks for each tile of them.
  __device__ __forceinline__ bool done(const Args& a) {
    if (all_done || !held) return all_done;
    const int lane = threadIdx.x & 31;
    bool ok = true;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (length[h] > 0) ok = ok && tc::load_acquire(a.done_group + lane + 32 * h) >= a.stored * up_div(length[h], a.row_tile);
    __syncwarp();
    return all_done = __all_sync(0xffffffffu, ok);
  }
};

// Tile i of nm x nn in groups of 8 row tiles, row tile fastest, so that tiles in flight share operands in L2.
__device__ __forceinline__ void tile_place(int i, int nm, int nn, int& m, int& n) {
  const int of8 = 8 * nn, gr = i / of8, in = i - gr * of8, rows = min(8, nm - gr * 8);
  n = in / rows;
  m = gr * 8 + in - n * rows;
}

// Phi(g), from e = e^(-g^2 / 2): Phi(-|g|) is e t P(t) with t = 1 / (1 + 0.35 |g|), where P of degree 8 is fitted to
// e^(g^2 / 2) Phi(-|g|) / t on |g| <= 14.5 (least squares of the relative error, reweighted until its peaks were even:
// 2^-24.9; 2^-21.5 with all fp32 roundings). So small values of Phi are right to a few steps of themselves, where 1 + erf
// cancels (at -5 steps of a tenth, below -5.5 nothing), and the exponential serves the derivative too.
__device__ __forceinline__ float2 normal_cdf(float2 g, float2 e) {
  constexpr float kFit[9] = {0.139621302485466f,    0.1398635357618332f,   0.11982118338346481f,
                             0.10555292665958405f,  -0.02321339212357998f, 0.15932124853134155f,
                             -0.25584039092063904f, 0.1440316140651703f,   -0.029158029705286026f};
  const float2 d = fma2(make_float2(fabsf(g.x), fabsf(g.y)), pair(0.35f), pair(1.f));
  const float2 t = make_float2(__fdividef(1.f, d.x), __fdividef(1.f, d.y));
  float2 s = pair(kFit[8]);
#pragma unroll
  for (int i = 7; i >= 0; --i) s = fma2(s, t, pair(kFit[i]));
  const float2 q = mul2(mul2(s, t), e), r = add2(pair(1.f), make_float2(-q.x, -q.y));
  return make_float2(g.x < 0.f ? q.x : r.x, g.y < 0.f ? q.y : r.y);
}

// act(g) and its derivative for two elements at a time, with the hardware's exponential (relative error 2^-22 + |g|
// 2^-24) and quotient.
template <int ACT>
__device__ __forceinline__ void activation(float2 g, float2& a, float2& da) {
  const float2 one = pair(1.f);
  if (ACT == LAYER_SILU) {
    const float2 e = add2(make_float2(__expf(-g.x), __expf(-g.y)), one);
    const float2 s = make_float2(__fdividef(1.f, e.x), __fdividef(1.f, e.y));
    a = mul2(g, s);
    da = fma2(a, add2(one, make_float2(-s.x, -s.y)), s);  // s (1 + g (1 - s))
  } else {
    const float2 h = mul2(mul2(g, g), pair(-0.5f)), e = make_float2(__expf(h.x), __expf(h.y)), p = normal_cdf(g, e);
    a = mul2(g, p);
    da = fma2(mul2(g, pair(0.3989422804014327f)), e, p);
  }
}
// A block's rows: v = act(v) w; or, from g, u and v = dh: g = dg, u = h, v = du. One of two straight pieces of code (a
// choice per element has the instructions of both fetched: 8 us of a small call's 55), two elements at a time: the
// instructions of 32 x 32 elements set an epilogue's pace (backward 0.75 us a block of a warp with one at a time).
template <int ACT, int N>
__device__ __forceinline__ void gate(float (&v)[N], const float (&w)[N]) {
#pragma unroll
  for (int j = 0; j < N; j += 2) {
    float2 a, da;
    activation<ACT>(make_float2(v[j], v[j + 1]), a, da);
    a = mul2(a, make_float2(w[j], w[j + 1]));
    v[j] = a.x, v[j + 1] = a.y;
  }
}
template <int ACT>
__device__ __forceinline__ void gate_back(float (&g)[32], float (&u)[32], float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 32; j += 2) {
    const float2 uj = make_float2(u[j], u[j + 1]), vj = make_float2(v[j], v[j + 1]);
    float2 a, da;
    activation<ACT>(make_float2(g[j], g[j + 1]), a, da);
    const float2 dg = mul2(mul2(vj, uj), da), h = mul2(uj, a), du = mul2(vj, a);
    g[j] = dg.x, g[j + 1] = dg.y;
    u[j] = h.x, u[j + 1] = h.y;
    v[j] = du.x, v[j + 1] = du.y;
  }
}

// What the rounding of x to a type has left (nothing of what is not finite there).
template <typename T>
__device__ __forceinline__ float rest_of(float x, T rounded) {
  const float r = to_f32(rounded);
  return fabsf(r) < INFINITY ? x - r : 0.f;
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
