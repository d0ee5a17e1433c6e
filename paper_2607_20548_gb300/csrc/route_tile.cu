// Routing of many tokens (include/layer.h): two lanes per token.
//
// A warp brings 16 rows of logits into shared memory and two lanes go through a row, 16 bytes at a time in
// turn; rows lie an odd number of 16-byte units apart, so that neither the lanes' walks along their
// rows nor the sums down the columns meet in a bank. The k largest are kept sorted: four logits are sorted
// and merged in at a time, and the two lanes' lists at the end. A 16-bit logit's key holds its index; fp32
// values go without theirs, and a second look at the row marks what reaches the k-th value, whose places
// follow from the list. Probabilities are summed down the columns with a lane per 32-bit word, the sums
// staying in registers over all of a warp's tiles.
//
// What bounds it is instructions and their latency, not memory: with k = 6 and 500009 x 127 fp32 logits,
// 138 us forward (2.0 TB/s) and 134 backward (4.1 TB/s; rows of 128, which move 16 bytes at a time: 122
// and 99). Before, in that order: a thread per token and 32 rows per warp, so that shared memory held half
// the warps, 203 and 145; logits inserted one by one, and the copies' conditions worked out per row, 240
// and 174; a group of lanes per token (route.cu), most of its instructions exchanges, 312 and 241.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "route.h"
#include "soap_internal.h"

namespace soap {
namespace route {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kRows = 16;                  // a warp's tile: two lanes per row
constexpr int kTokens = kWarps * kRows;      // a CTA's at a time
constexpr int kRowBits = (1 << kRows) - 1;
constexpr int kStride = kRows + 1;         // of the choices' lists
constexpr int kMaxList = 8;               // places of a thread's list
constexpr int kMaxWords = 6 * 32;         // 32-bit words of a row
constexpr int kSmemPerSm = 228 * 1024;

int row_bytes(int experts, int32_t type) { return experts * (int)dtype_size(type); }
__host__ __device__ __forceinline__ int pitch_of(int bytes) { return 16 * (((bytes + 15) / 16) | 1); }

__device__ __forceinline__ void wait_copies() {
  asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  if constexpr (N == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// f(address in the tile, address in the matrix) for the units of UNIT bytes of each row in `rows` (a bit per
// row): row by row, a lane per unit, MOST units per lane at most. What a lane does in a row is the same in
// all rows, so that the conditions stay in predicates (worked out per row, they took a third of a
// backward pass's instructions).
template <int UNIT, int MOST, typename F>
__device__ __forceinline__ void each_unit(uint32_t tile, int pitch, uint8_t* base, int64_t ld_bytes, uint32_t rows,
                                          int units, int lane, F&& f) {
  uint32_t t = tile + lane * UNIT;
  uint8_t* g = base + lane * UNIT;
  bool some[MOST];
#pragma unroll
  for (int b = 0; b < MOST; ++b) some[b] = lane + 32 * b < units;
  auto row = [&] {
#pragma unroll
    for (int b = 0; b < MOST; ++b)
      if (some[b]) f(t + 32 * UNIT * b, g + 32 * UNIT * b);
    t += pitch;
    g += ld_bytes;
  };
  if (rows == kRowBits) {
#pragma unroll 4
    for (int r = 0; r < kRows; ++r) row();
  } else {
    for (int r = 0; r < kRows; ++r) {
      if (rows >> r & 1) {
        row();
      } else {
        t += pitch;
        g += ld_bytes;
      }
    }
  }
}

// Rows of a matrix into a tile. mode: bytes that may move at once (16, 4 or 2).
template <typename T, int NW>
__device__ __forceinline__ void load_rows(uint8_t* tile, int pitch, const T* base, int64_t ld, uint32_t rows,
                                          int experts, int mode, int lane) {
  uint8_t* src = const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(base));
  const uint32_t dst = static_cast<uint32_t>(__cvta_generic_to_shared(tile));
  const int bytes = experts * (int)sizeof(T);
  const int64_t ldb = ld * (int64_t)sizeof(T);
  if (mode == 16)
    each_unit<16, (NW + 3) / 4>(dst, pitch, src, ldb, rows, bytes / 16, lane,
                                [](uint32_t t, const uint8_t* g) { copy_async<16>(t, g); });
  else if (mode == 4)
    each_unit<4, NW>(dst, pitch, src, ldb, rows, bytes / 4, lane,
                     [](uint32_t t, const uint8_t* g) { copy_async<4>(t, g); });
  else if constexpr (sizeof(T) == 2)
    each_unit<2, 2 * NW>(dst, pitch, src, ldb, rows, bytes / 2, lane, [](uint32_t t, const uint8_t* g) {
      asm volatile("st.shared.u16 [%0], %1;" ::"r"(t), "h"(*reinterpret_cast<const uint16_t*>(g)) : "memory");
    });
  wait_copies();
  __syncwarp();
}
template <typename T, int NW>
__device__ __forceinline__ void store_rows(uint8_t* tile, int pitch, T* base, int64_t ld, uint32_t rows, int experts,
                                           int mode, int lane) {
  __syncwarp();
  uint8_t* dst = reinterpret_cast<uint8_t*>(base);
  const uint32_t src = static_cast<uint32_t>(__cvta_generic_to_shared(tile));
  const int bytes = experts * (int)sizeof(T);
  const int64_t ldb = ld * (int64_t)sizeof(T);
  if (mode == 16)
    each_unit<16, (NW + 3) / 4>(src, pitch, dst, ldb, rows, bytes / 16, lane, [](uint32_t t, uint8_t* g) {
      uint4 v;
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                   : "r"(t)
                   : "memory");
      *reinterpret_cast<uint4*>(g) = v;
    });
  else if (mode == 4)
    each_unit<4, NW>(src, pitch, dst, ldb, rows, bytes / 4, lane, [](uint32_t t, uint8_t* g) {
      uint32_t v;
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(t) : "memory");
      *reinterpret_cast<uint32_t*>(g) = v;
    });
  else if constexpr (sizeof(T) == 2)
    each_unit<2, 2 * NW>(src, pitch, dst, ldb, rows, bytes / 2, lane, [](uint32_t t, uint8_t* g) {
      uint16_t v;
      asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(t) : "memory");
      *reinterpret_cast<uint16_t*>(g) = v;
    });
  __syncwarp();
}

// f(j, values) for a row's 16-byte units that are whole, then g(j, value) for the elements left: every other
// unit, the first lane of a row from the first one; the elements left are the second's.
template <typename T, typename F, typename G>
__device__ __forceinline__ void walk(const uint8_t* row, int half, int experts, F&& f, G&& g) {
  constexpr int V = 16 / sizeof(T);
  for (int j = half * V; j + V <= experts; j += 2 * V) {
    const Pack<T, V> p = *reinterpret_cast<const Pack<T, V>*>(row + j * sizeof(T));
    float v[V];
#pragma unroll
    for (int q = 0; q < V; q += 2) {
      const float2 x = to_pair(p.v + q);
      v[q] = x.x;
      v[q + 1] = x.y;
    }
    f(j, v);
  }
  if (half)
    for (int j = experts / V * V; j < experts; ++j) g(j, to_f32(reinterpret_cast<const T*>(row)[j]));
}
// The same on fp32 values in place: f(four values, j) and g(one, j).
template <typename F, typename G>
__device__ __forceinline__ void each_four(uint8_t* row, int half, int experts, F&& f, G&& g) {
  for (int j = half * 4; j + 4 <= experts; j += 8) f(*reinterpret_cast<float4*>(row + j * 4), j);
  if (half)
    for (int j = experts / 4 * 4; j < experts; ++j) g(reinterpret_cast<float*>(row)[j], j);
}

// The sum over a row's two lanes.
__device__ __forceinline__ float both(float v) { return v + __shfl_xor_sync(0xffffffffu, v, kRows); }

struct Tile {
  int64_t t0;       // the tile's first token
  bool here, live;  // this lane's token exists / is not masked
  uint32_t rows;    // the rows to read, a bit each
};
__device__ __forceinline__ Tile tile_at(int64_t i, int64_t tokens, const uint8_t* mask, int r) {
  Tile t;
  t.t0 = i * kRows;
  t.here = t.t0 + r < tokens;
  t.live = t.here && (!mask || mask[t.t0 + r] != 0);
  // a tile with a live row is read whole: to leave single rows out costs more than it saves
  t.rows = __any_sync(0xffffffffu, t.live) ? __ballot_sync(0xffffffffu, t.here) & kRowBits : 0u;
  return t;
}

__device__ __forceinline__ void exchange(float& a, float& b) {
  const float hi = fmaxf(a, b);
  b = fminf(a, b);
  a = hi;
}
__device__ __forceinline__ void exchange(uint32_t& a, uint32_t& b) {
  const uint32_t hi = max(a, b);
  b = min(a, b);
  a = hi;
}
// One more value into a falling list of the K largest.
template <int K, typename L>
__device__ __forceinline__ void insert(L (&list)[K], L x) {
#pragma unroll
  for (int q = 0; q < K; ++q) exchange(list[q], x);
}
// list[i] and other[K - 1 - i], the larger of each pair: the K largest of two falling lists (other may be
// shorter), falling and then rising, which a bitonic merge puts in order (as if larger values filled the
// places up to a power of two).
template <int K, int N, typename L>
__device__ __forceinline__ void merge(L (&list)[K], const L (&other)[N]) {
#pragma unroll
  for (int i = 0; i < K; ++i)
    if (K - 1 - i < N) {
      if constexpr (std::is_same_v<L, float>)
        list[i] = fmaxf(list[i], other[K - 1 - i]);
      else
        list[i] = max(list[i], other[K - 1 - i]);
    }
  constexpr int P = K <= 2 ? 2 : K <= 4 ? 4 : 8, O = P - K;
#pragma unroll
  for (int h = P / 2; h > 0; h /= 2)
#pragma unroll
    for (int i = O; i < P; ++i)
      if ((i & h) == 0 && i + h < P) exchange(list[i - O], list[i + h - O]);
}
// Four more values: 28 minima and maxima for K = 6 (one by one: 48), and most of them do not wait for one
// another.
template <int K, typename L>
__device__ __forceinline__ void insert4(L (&list)[K], L a, L b, L c, L d) {
  exchange(a, b);
  exchange(c, d);
  exchange(a, c);
  exchange(b, d);
  exchange(b, c);
  const L four[4] = {a, b, c, d};
  merge<K, 4, L>(list, four);
}

template <typename T, int K, int NW>
__global__ void __launch_bounds__(kThreads, 3)
    tile_fwd_kernel(const Forward a, const Totals out, const int mode) {
  constexpr bool kPacked = sizeof(T) == 2;
  constexpr int V = 16 / sizeof(T), W = 4 / sizeof(T);  // elements per unit and per word
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float red[kWarps + 1];
  const int lane = threadIdx.x % 32, r = lane % kRows, half = lane / kRows, warp = threadIdx.x / 32;
  const int experts = a.experts, k = a.k;
  const int pitch = pitch_of(experts * (int)sizeof(T));
  uint8_t* tile = smem + warp * kRows * pitch;
  float2* stat = reinterpret_cast<float2*>(smem + kWarps * kRows * pitch) + warp * kRows;
  // the tile's choices, choice q of row r at q * kStride + r
  int32_t* idx = reinterpret_cast<int32_t*>(smem + kWarps * kRows * (pitch + 8)) + warp * kStride * k;
  float* gate = reinterpret_cast<float*>(idx + kWarps * kStride * k);
  int* counts = reinterpret_cast<int*>(smem + kWarps * (kRows * (pitch + 8) + kStride * 8 * k));
  for (int c = threadIdx.x; c <= experts; c += kThreads) counts[c] = 0;
  __syncthreads();
  uint8_t* row = tile + r * pitch;
  float acc[NW * W];
#pragma unroll
  for (int i = 0; i < NW * W; ++i) acc[i] = 0.f;
  int seen = 0;
  const int64_t tiles = (a.tokens + kRows - 1) / kRows;
  for (int64_t i = (int64_t)blockIdx.x * kWarps + warp; i < tiles; i += (int64_t)gridDim.x * kWarps) {
    const Tile t = tile_at(i, a.tokens, a.mask, r);
    load_rows<T, NW>(tile, pitch, static_cast<const T*>(a.logits) + t.t0 * a.ld, a.ld, t.rows, experts, mode, lane);
    const int mine = t.live ? experts : 0;  // elements of the row
    // the K largest, in falling order: keys with indices, or values
    using L = std::conditional_t<kPacked, uint32_t, float>;
    L list[K];
#pragma unroll
    for (int q = 0; q < K; ++q) list[q] = kPacked ? (L)0 : (L)-INFINITY;
    auto key = [](int j, float v) -> L {
      if constexpr (kPacked)
        return pack_key(order_key(v), j);
      else
        return v;
    };
    walk<T>(row, half, mine,
            [&](int j, const float (&v)[V]) {
#pragma unroll
              for (int q = 0; q < V; q += 4)
                insert4<K, L>(list, key(j + q, v[q]), key(j + q + 1, v[q + 1]), key(j + q + 2, v[q + 2]),
                              key(j + q + 3, v[q + 3]));
            },
            [&](int j, float v) { insert<K, L>(list, key(j, v)); });
    L others[K];
#pragma unroll
    for (int q = 0; q < K; ++q) others[q] = __shfl_xor_sync(0xffffffffu, list[q], kRows);
    merge<K, K, L>(list, others);
    const float most = kPacked ? key_value(unpack_key((uint32_t)list[0])) : (float)list[0];
    bool bad = kPacked ? ((uint32_t)list[0] & ~kLow) >= kKeyInf : most == INFINITY;
    bool counted = (kPacked ? (uint32_t)list[0] > (kKeyNegInf | kLow) : most > -INFINITY) && !bad;
    // fp32: what reaches the k-th value, a bit per logit, before the row is written over
    uint32_t marked[NW];
    if constexpr (!kPacked) {
      float least = list[0];
#pragma unroll
      for (int q = 1; q < K; ++q)
        if (q < k) least = list[q];
#pragma unroll
      for (int b = 0; b < NW; ++b) {
        uint32_t m = 0;
        each_four(row + 128 * b, half, min(32, mine - 32 * b),
                  [&](const float4& v, int j) {
                    const uint32_t four = (v.x >= least ? 1u : 0u) | (v.y >= least ? 2u : 0u) |
                                          (v.z >= least ? 4u : 0u) | (v.w >= least ? 8u : 0u);
                    m |= four << j;
                  },
                  [&](float v, int j) { m |= (v >= least ? 1u : 0u) << j; });
        marked[b] = m | __shfl_xor_sync(0xffffffffu, m, kRows);
      }
    }
    // fp32: the choices' indices, by their place in the list
    if constexpr (!kPacked) {
      uint32_t used = 0;
      int base = 0;
      uint32_t m = marked[0];
      for (int q = half; q < k; q += 2) idx[q * kStride + r] = -1;
      __syncwarp();
      while (true) {
        // on to the row's next marked logit (its two lanes do the same)
#pragma unroll
        for (int b = 1; b < NW; ++b)
          if (m == 0 && base < 32 * b) {
            m = marked[b];
            base = 32 * b;
          }
        if (!__any_sync(0xffffffffu, m != 0)) break;
        if (m != 0) {
          const int j = __ffs(m) - 1;
          m &= m - 1;
          const float v = reinterpret_cast<const float*>(row)[base + j];
          int place = 0;
#pragma unroll
          for (int q = 0; q < K; ++q) place += list[q] > v;
          place += __ffs(~(used >> place)) - 1;  // after the equal ones before it
          if (place < k && v > -INFINITY) {
            used |= 1u << place;
            if (half == 0) idx[place * kStride + r] = base + j;
          }
        }
      }
    }
    // the row's exponentials and their sum (fp32: written over the logits)
    __syncwarp();
    float sum = 0.f;
    if constexpr (kPacked) {
      walk<T>(row, half, mine,
              [&](int, const float (&v)[V]) {
#pragma unroll
                for (int q = 0; q < V; ++q) sum += exp_neg(v[q] - most);
              },
              [&](int, float v) { sum += exp_neg(v - most); });
    } else {
      const float shift = counted ? most : INFINITY;  // e^-inf for rows that do not count
      each_four(row, half, experts,
                [&](float4& p, int) {
                  const float4 v = make_float4(exp_neg(p.x - shift), exp_neg(p.y - shift), exp_neg(p.z - shift),
                                               exp_neg(p.w - shift));
                  sum += (v.x + v.y) + (v.z + v.w);
                  p = v;
                },
                [&](float& p, int) {
                  p = exp_neg(p - shift);
                  sum += p;
                });
    }
    sum = both(sum);
    bool found = false;
    if (t.live && (bad || (counted && sum != sum))) {  // +inf, or a NaN, which no comparison sees
      bad = found = true;
      counted = false;
    }
    // a row of nothing but NaN and -inf has no largest value
    const bool empty = t.live && !counted && !bad;
    if (__any_sync(0xffffffffu, empty)) {
      float s = 0.f;
      if constexpr (kPacked)
        walk<T>(row, half, empty ? experts : 0, [&](int, const float (&v)[V]) {
#pragma unroll
          for (int q = 0; q < V; ++q) s += v[q];
        }, [&](int, float v) { s += v; });
      else
        s = sum;
      s = both(s);
      if (empty && s != s) bad = found = true;
    }
    if (found && half == 0 && a.status) atomicOr(a.status, SOAP_STATUS_NONFINITE);
    seen += half == 0 && (counted || bad);
    const float inv = bad ? NAN : counted ? 1.f / sum : 0.f;
    if (half == 0) stat[r] = make_float2(most, inv);
    if (half == 0 && a.stats && t.here) a.stats[t.t0 + r] = bad ? make_float2(NAN, NAN) : make_float2(most, inv);
    // the gates, from the list
    float mine_g[K], total = 0.f;
#pragma unroll
    for (int q = 0; q < K; ++q) {
      bool some;
      float v;
      if constexpr (kPacked) {
        some = counted && q < k && list[q] > (kKeyNegInf | kLow);
        v = key_value(unpack_key(list[q]));
      } else {
        some = counted && q < k && list[q] > -INFINITY;
        v = list[q];
      }
      mine_g[q] = some ? exp_neg(v - most) : 0.f;
      total += mine_g[q];
      if (q < k && q % 2 == half) {  // the row's lanes take turns
        int at = -1;
        if (some) at = kPacked ? packed_index((uint32_t)list[q]) : idx[q * kStride + r];
        if (at >= 0) atomicAdd(&counts[at], 1);
        idx[q * kStride + r] = at;
      }
    }
    const float scale = bad ? NAN : a.normalize ? (total > 0.f ? 1.f / total : 0.f) : inv;
#pragma unroll
    for (int q = 0; q < K; ++q)
      if (q < k && q % 2 == half) gate[q * kStride + r] = mine_g[q] * scale;
    __syncwarp();
    const int n = (int)min((int64_t)kRows, a.tokens - t.t0) * k;
    {
      int l = lane / k, q = lane - l * k;
      const int dl = 32 / k, dq = 32 - dl * k;
      for (int i2 = lane; i2 < n; i2 += 32) {
        a.indices[t.t0 * k + i2] = idx[q * kStride + l];
        a.gates[t.t0 * k + i2] = gate[q * kStride + l];
        l += dl;
        q += dq;
        if (q >= k) {
          q -= k;
          ++l;
        }
      }
    }
    // sums of probabilities down the columns: a lane per word (rows that do not count hold anything)
    auto add_row = [&](int at) {
      const float2 st = stat[at];
#pragma unroll
      for (int b = 0; b < NW; ++b) {
        const int c = 32 * b + lane;
        if (c * W < experts) {
          if constexpr (kPacked) {
            const float2 v = to_pair(reinterpret_cast<const T*>(tile + at * pitch) + 2 * c);
            acc[2 * b] = fmaf(exp_neg(v.x - st.x), st.y, acc[2 * b]);
            acc[2 * b + 1] = fmaf(exp_neg(v.y - st.x), st.y, acc[2 * b + 1]);
          } else {
            acc[b] = fmaf(reinterpret_cast<const float*>(tile + at * pitch)[c], st.y, acc[b]);
          }
        }
      }
    };
    const uint32_t count_rows = __ballot_sync(0xffffffffu, counted || bad);
    for (int r4 = 0; r4 < kRows; r4 += 4) {
      if ((count_rows >> r4 & 15u) == 15u) {
#pragma unroll
        for (int q = 0; q < 4; ++q) add_row(r4 + q);
      } else {
        for (int q = r4; q < r4 + 4; ++q)
          if (count_rows >> q & 1u) add_row(q);
      }
    }
    __syncwarp();  // the tile may be loaded again
  }
  seen = __reduce_add_sync(0xffffffffu, seen);
  if (lane == 0 && seen) atomicAdd(&counts[experts], seen);
  __syncthreads();  // the tiles are done with: their place takes the warps' column sums
  float* shared = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int i = 0; i < NW * W; ++i) {
    const int c = (32 * (i / W) + lane) * W + i % W;
    if (c < experts) shared[warp * experts + c] = acc[i];
  }
  finish_columns<kWarps>(shared, counts, red, experts, k, a.part_p, a.part_c, out);
}

template <typename T, int NW>
__global__ void __launch_bounds__(kThreads, 3)
    tile_bwd_kernel(const Backward a, const int mode_in, const int mode_out) {
  constexpr int V = 16 / sizeof(T);
  extern __shared__ __align__(16) uint8_t smem[];
  const int lane = threadIdx.x % 32, r = lane % kRows, half = lane / kRows, warp = threadIdx.x / 32;
  const int experts = a.experts, k = a.k;
  const int pitch = pitch_of(experts * (int)sizeof(T));
  float* up = reinterpret_cast<float*>(smem);  // the balance loss's gradient of the probabilities
  const int up_bytes = (experts * 4 + 15) / 16 * 16;
  uint8_t* tile = smem + up_bytes + warp * kRows * pitch;
  // the tile's choices and their gates' gradients, choice q of row r at q * kStride + r; choice q is the
  // business of the row's lane q % 2
  int32_t* idx = reinterpret_cast<int32_t*>(smem + up_bytes + kWarps * kRows * pitch) + warp * kStride * k;
  float* dg = reinterpret_cast<float*>(idx + kWarps * kStride * k);
  const int n_live = *a.live;
  const float per = n_live > 0 ? a.scale / (float)n_live / (float)n_live : 0.f;
  for (int c = threadIdx.x; c < experts; c += kThreads) up[c] = per * (float)a.counts[c];
  __syncthreads();
  uint8_t* row = tile + r * pitch;
  const int64_t tiles = (a.tokens + kRows - 1) / kRows;
  for (int64_t i = (int64_t)blockIdx.x * kWarps + warp; i < tiles; i += (int64_t)gridDim.x * kWarps) {
    const Tile t = tile_at(i, a.tokens, a.mask, r);
    if (a.dgates) {
      const int n = (int)min((int64_t)kRows, a.tokens - t.t0) * k;
      int l = lane / k, q = lane - l * k;
      const int dl = 32 / k, dq = 32 - dl * k;
      for (int i2 = lane; i2 < n; i2 += 32) {
        idx[q * kStride + l] = a.indices[t.t0 * k + i2];
        dg[q * kStride + l] = a.dgates[t.t0 * k + i2];
        l += dl;
        q += dq;
        if (q >= k) {
          q -= k;
          ++l;
        }
      }
    }
    const float2 st = t.live ? a.stats[t.t0 + r] : make_float2(0.f, 0.f);
    load_rows<T, NW>(tile, pitch, static_cast<const T*>(a.logits) + t.t0 * a.ld, a.ld, t.rows, experts, mode_in, lane);
    const bool counted = st.y > 0.f;
    const int mine = counted ? experts : 0;
    // the gates' gradient at the chosen probabilities, kept as what reaches p
    float dot = 0.f;
    if (a.dgates) {
      float s = 0.f;
      for (int q = half; q < k; q += 2) {
        const int at = t.live ? idx[q * kStride + r] : -1;
        if (at < 0 || at >= experts) continue;
        const float p = exp_neg(to_f32(reinterpret_cast<const T*>(row)[at]) - st.x) * st.y;
        s += p;
        dot = fmaf(dg[q * kStride + r], p, dot);
      }
      if (a.normalize) {
        // gate_r = p_r / s: d p_r = (d gate_r - sum_j d gate_j gate_j) / s, whose sum with the p_r is zero
        s = both(s);
        const float mean = both(dot) / s, inv = 1.f / s;
        for (int q = half; q < k; q += 2) dg[q * kStride + r] = (dg[q * kStride + r] - mean) * inv;
        dot = 0.f;
      }
    }
    __syncwarp();  // the chosen logits have been read
    float d4[4] = {0.f, 0.f, 0.f, 0.f};
    if constexpr (sizeof(T) == 4) {  // the probabilities stay in the row
      each_four(row, half, mine,
                [&](float4& p, int j) {
                  const float4 u = *reinterpret_cast<const float4*>(up + j);
                  const float4 v = make_float4(exp_neg(p.x - st.x) * st.y, exp_neg(p.y - st.x) * st.y,
                                               exp_neg(p.z - st.x) * st.y, exp_neg(p.w - st.x) * st.y);
                  d4[0] = fmaf(v.x, u.x, d4[0]);
                  d4[1] = fmaf(v.y, u.y, d4[1]);
                  d4[2] = fmaf(v.z, u.z, d4[2]);
                  d4[3] = fmaf(v.w, u.w, d4[3]);
                  p = v;
                },
                [&](float& p, int j) {
                  p = exp_neg(p - st.x) * st.y;
                  d4[0] = fmaf(p, up[j], d4[0]);
                });
    } else {
      walk<T>(row, half, mine,
              [&](int j, const float (&v)[V]) {
#pragma unroll
                for (int q = 0; q < V; ++q) d4[q % 4] = fmaf(exp_neg(v[q] - st.x), up[j + q], d4[q % 4]);
              },
              [&](int j, float v) { d4[0] = fmaf(exp_neg(v - st.x), up[j], d4[0]); });
    }
    float sum = (d4[0] + d4[1]) + (d4[2] + d4[3]);
    if (sizeof(T) == 2) sum *= st.y;
    dot = both(dot + sum);
    __syncwarp();  // fp32: the row's other lane has written its probabilities (a shuffle orders no memory)
    // the chosen logits' own gradients, before the row is written over
    if (a.dgates)
      for (int q = half; q < k; q += 2) {
        const int at = counted ? idx[q * kStride + r] : -1;
        if (at < 0 || at >= experts) {
          idx[q * kStride + r] = -1;
          continue;
        }
        const float x = to_f32(reinterpret_cast<const T*>(row)[at]);
        const float p = sizeof(T) == 4 ? x : exp_neg(x - st.x) * st.y;
        dg[q * kStride + r] = p * (up[at] + dg[q * kStride + r] - dot);
      }
    __syncwarp();
    if (counted) {
      if constexpr (sizeof(T) == 4) {
        each_four(row, half, experts,
                  [&](float4& p, int j) {
                    const float4 u = *reinterpret_cast<const float4*>(up + j);
                    p = make_float4(p.x * (u.x - dot), p.y * (u.y - dot), p.z * (u.z - dot), p.w * (u.w - dot));
                  },
                  [&](float& p, int j) { p *= up[j] - dot; });
      } else {
        for (int j = half * V; j + V <= experts; j += 2 * V) {
          Pack<T, V> p = *reinterpret_cast<const Pack<T, V>*>(row + j * sizeof(T));
#pragma unroll
          for (int q = 0; q < V; q += 2) {
            const float2 v = to_pair(p.v + q), u = *reinterpret_cast<const float2*>(up + j + q);
            from_pair(make_float2(exp_neg(v.x - st.x) * st.y * (u.x - dot), exp_neg(v.y - st.x) * st.y * (u.y - dot)),
                      p.v + q);
          }
          *reinterpret_cast<Pack<T, V>*>(row + j * sizeof(T)) = p;
        }
        if (half)
          for (int j = experts / V * V; j < experts; ++j) {
            T* p = reinterpret_cast<T*>(row) + j;
            *p = from_f32<T>(exp_neg(to_f32(*p) - st.x) * st.y * (up[j] - dot));
          }
      }
    } else {  // zeros, or NaN for a row that holds a NaN or +inf
      const T fill = from_f32<T>(t.live && st.y != st.y ? NAN : 0.f);
      for (int j = half; j < experts; j += 2) reinterpret_cast<T*>(row)[j] = fill;
    }
    __syncwarp();
    if (a.dgates)
      for (int q = half; q < k; q += 2) {
        const int at = idx[q * kStride + r];
        if (counted && at >= 0) reinterpret_cast<T*>(row)[at] = from_f32<T>(dg[q * kStride + r]);
      }
    const uint32_t all = __ballot_sync(0xffffffffu, t.here) & kRowBits;
    store_rows<T, NW>(tile, pitch, static_cast<T*>(a.dlogits) + t.t0 * a.ld_d, a.ld_d, all, experts, mode_out, lane);
  }
}

// ---- launches ------------------------------------------------------------------------------

size_t fwd_smem(int experts, int k, int32_t type) {
  return (size_t)kWarps * (kRows * (pitch_of(row_bytes(experts, type)) + 8) + kStride * 8 * k) + (experts + 1) * 4;
}
size_t bwd_smem(int experts, int k, int32_t type) {
  return (experts * 4 + 15) / 16 * 16 +
         (size_t)kWarps * (kRows * pitch_of(row_bytes(experts, type)) + kStride * 8 * k);
}

// Bytes that rows may move at once.
int mode_of(const void* p, int64_t ld, int experts, int32_t type) {
  const uintptr_t bytes = reinterpret_cast<uintptr_t>(p) | (uintptr_t)((ld | experts) * dtype_size(type));
  return bytes % 16 == 0 ? 16 : bytes % 4 == 0 ? 4 : 2;
}

int per_sm(size_t smem) { return std::max(1, std::min(3, (int)(kSmemPerSm / (smem + 1024 + 64)))); }

template <typename K>
cudaError_t allow_smem(K kernel, std::atomic<uint64_t>& set) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t(1) << dev : 0;
  if (bit && (set.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
  if (e == cudaSuccess) set.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

template <typename T, int K, int NW>
cudaError_t launch_fwd(const Forward& f, const Totals& out, int ctas, size_t smem, int mode, cudaStream_t s) {
  static std::atomic<uint64_t> set{0};
  const auto kernel = tile_fwd_kernel<T, K, NW>;
  const cudaError_t e = allow_smem(kernel, set);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = kTileCluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, f, out, mode);
}

template <typename T, int K>
cudaError_t fwd_words(const Forward& f, const Totals& out, int ctas, size_t smem, int mode, cudaStream_t s) {
  const int words = (f.experts * (int)sizeof(T) + 3) / 4;
  if (words <= 32) return launch_fwd<T, K, 1>(f, out, ctas, smem, mode, s);
  if (words <= 64) return launch_fwd<T, K, 2>(f, out, ctas, smem, mode, s);
  if (words <= 128) return launch_fwd<T, K, 4>(f, out, ctas, smem, mode, s);
  return launch_fwd<T, K, 6>(f, out, ctas, smem, mode, s);
}

template <typename T>
cudaError_t fwd_list(const Forward& f, const Totals& out, int ctas, size_t smem, int mode, cudaStream_t s) {
  if (f.k <= 2) return fwd_words<T, 2>(f, out, ctas, smem, mode, s);
  if (f.k <= 4) return fwd_words<T, 4>(f, out, ctas, smem, mode, s);
  if (f.k <= 6) return fwd_words<T, 6>(f, out, ctas, smem, mode, s);
  return fwd_words<T, 8>(f, out, ctas, smem, mode, s);
}

template <typename T, int NW>
cudaError_t launch_bwd(const Backward& b, int32_t type, cudaStream_t s) {
  static std::atomic<uint64_t> set{0};
  const auto kernel = tile_bwd_kernel<T, NW>;
  const cudaError_t e = allow_smem(kernel, set);
  if (e != cudaSuccess) return e;
  const size_t smem = bwd_smem(b.experts, b.k, type);
  const int64_t want = (b.tokens + kTokens - 1) / kTokens;
  const int ctas = (int)std::min<int64_t>(want, 152 * per_sm(smem));
  kernel<<<ctas, kThreads, smem, s>>>(b, mode_of(b.logits, b.ld, b.experts, type),
                                      mode_of(b.dlogits, b.ld_d, b.experts, type));
  return cudaGetLastError();
}
template <typename T>
cudaError_t bwd_words(const Backward& b, int32_t type, cudaStream_t s) {
  const int words = (b.experts * (int)sizeof(T) + 3) / 4;
  if (words <= 32) return launch_bwd<T, 1>(b, type, s);
  if (words <= 64) return launch_bwd<T, 2>(b, type, s);
  if (words <= 128) return launch_bwd<T, 4>(b, type, s);
  return launch_bwd<T, 6>(b, type, s);
}

}  // namespace

bool tile_fits(int64_t tokens, int experts, int k, int32_t type) {
  return tokens >= kFewTokens && k <= kMaxList && row_bytes(experts, type) <= kMaxWords * 4;
}

int tile_forward_ctas(int64_t tokens, int experts, int k, int32_t type) {
  const int64_t want = (tokens + kTokens - 1) / kTokens;
  const int most = std::min(kTileCluster * kMaxParts, 152 * per_sm(fwd_smem(experts, k, type)));
  return (int)std::min<int64_t>(most / kTileCluster, (want + kTileCluster - 1) / kTileCluster) * kTileCluster;
}

cudaError_t tile_forward(const Forward& f, const Totals& out, int32_t type, cudaStream_t s) {
  const int ctas = tile_forward_ctas(f.tokens, f.experts, f.k, type);
  const size_t smem = fwd_smem(f.experts, f.k, type);
  const int mode = mode_of(f.logits, f.ld, f.experts, type);
  if (type == SOAP_F32) return fwd_list<float>(f, out, ctas, smem, mode, s);
  if (type == SOAP_BF16) return fwd_list<__nv_bfloat16>(f, out, ctas, smem, mode, s);
  return fwd_list<__half>(f, out, ctas, smem, mode, s);
}

cudaError_t tile_backward(const Backward& b, int32_t type, cudaStream_t s) {
  if (type == SOAP_F32) return bwd_words<float>(b, type, s);
  if (type == SOAP_BF16) return bwd_words<__nv_bfloat16>(b, type, s);
  return bwd_words<__half>(b, type, s);
}

}  // namespace route
}  // namespace soap
