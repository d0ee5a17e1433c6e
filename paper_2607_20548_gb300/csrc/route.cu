// A mixture-of-experts router's decision and its gradient (include/layer.h).
//
//   p = softmax(z); the k largest (z, lower index first); gates; counts_e; P_e = sum_t p_te
//   loss = coef E / (k n) sum_e counts_e P_e / n
//   dz_e = p_e (u_e - sum_j p_j u_j),  u = coef dloss E / (k n^2) counts + (d gates -> p)
//
// A group of G lanes (8, 16 or 32) takes a token; a lane holds NE of its logits in registers, V
// consecutive ones per access, and has asked for its next token's while it works on one. The choice
// runs on 32-bit keys in the logits' order: each lane keeps its keys sorted (or, many, scans them),
// and k times the group's largest head is found and popped by its owner. A 16-bit logit's key holds
// its index below its value, so that keys differ; of equal fp32 keys the lowest index is looked for
// only when two lanes hold the largest one. Instructions bound it (measured: 440 per token of 127 fp32
// logits with k = 6, backward 224; 30000 x 512 fp32, k = 8: 94 us, backward 46), so what each exchange
// does is kept to a minimum and the gates are computed once per choice, by the lane that writes it. Calls
// with enough tokens to fill the GPU, k of up to 8 and rows of up to 768 bytes (192 fp32 logits, 384 of 16
// bits) go to route_tile.cu, at a third of that; few tokens need the lanes, and wider rows and larger k stay
// here for want of a tile kernel.
//
// Column sums of p stay in registers over all of a warp's tokens, counts in shared memory. A cluster
// adds its CTAs' sums through distributed shared memory in a fixed order; one cluster finishes by
// itself (few tokens: one launch), several leave a partial row each that a second kernel adds.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/layer.h"
#include "profile.h"
#include "route.h"

namespace soap {
namespace {

using namespace route;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxExperts = 1024;
constexpr int kMaxCtas = 608;  // four per SM
constexpr int kMaxK = 32;

template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <int G>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  if constexpr (G == 32) {
    return __reduce_max_sync(0xffffffffu, v);
  } else {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  }
}

// a before b in the sorted list: (key, index) pairs as they stand in one lane.
template <bool PACKED>
__device__ __forceinline__ void order(uint32_t& a, int& ia, uint32_t& b, int& ib) {
  if (PACKED) {
    const uint32_t hi = max(a, b);
    b = min(a, b);
    a = hi;
  } else {
    const bool up = b > a;  // equal keys stay as they are, by rising index
    const uint32_t hi = up ? b : a;
    b = up ? a : b;
    a = hi;
    const int i = up ? ib : ia;
    ib = up ? ia : ib;
    ia = i;
  }
}

// A group's part of a row: element i of a lane is logit at(lane, i). The number of experts is a
// multiple of V; whether V logits move as one access depends on the rows' alignment, which lane
// holds which does not, so that the same logits give the same bits wherever they lie.
template <typename T, int G, int NE, int V>
struct Row {
  Pack<T, V> p[NE / V];
  static __device__ __forceinline__ int at(int lane, int i) { return ((i / V) * G + lane) * V + i % V; }
  __device__ __forceinline__ void load(const T* row, int experts, int lane, bool vec) {
#pragma unroll
    for (int i = 0; i < NE; i += V)
      if (at(lane, i) < experts) {
        if (V == 1 || vec) {
          p[i / V] = *reinterpret_cast<const Pack<T, V>*>(row + at(lane, i));
        } else {
#pragma unroll
          for (int q = 0; q < V; ++q) p[i / V].v[q] = row[at(lane, i + q)];
        }
      }
  }
  __device__ __forceinline__ void values(bool live, int experts, int lane, float (&z)[NE]) const {
#pragma unroll
    for (int i = 0; i < NE; ++i) z[i] = live && at(lane, i) < experts ? to_f32(p[i / V].v[i % V]) : -INFINITY;
  }
};

template <typename T, int G, int NE, int V>
__global__ void __launch_bounds__(kThreads)
    route_fwd_kernel(const Forward a, const Totals out, const bool vec) {
  constexpr bool kPacked = sizeof(T) == 2;
  constexpr bool kSorted = NE <= 8;
  constexpr int kRec = kMaxK / G;
  using R = Row<T, G, NE, V>;
  const T* const logits = static_cast<const T*>(a.logits);
  const int64_t ld = a.ld, tokens = a.tokens;
  const uint8_t* const mask = a.mask;
  const int experts = a.experts, k = a.k;
  extern __shared__ float shared[];       // [warps][experts] column sums (the first row: the CTA's) ...
  int* counts = reinterpret_cast<int*>(shared + kWarps * experts);  // ... [experts + 1]: choices, tokens counted
  __shared__ float red[kWarps + 1];
  __shared__ int won[kPacked ? 1 : kThreads / G][kPacked ? 1 : kMaxK];  // a group's choices
  const int lane = threadIdx.x % G, warp = threadIdx.x / 32;
  for (int c = threadIdx.x; c <= experts; c += kThreads) counts[c] = 0;
  __syncthreads();
  float acc[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) acc[i] = 0.f;
  int seen = 0;
  const int64_t groups = (int64_t)gridDim.x * (kThreads / G);
  int64_t t = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  R row;
  bool live = t < tokens && (!mask || mask[t] != 0);
  if (live) row.load(logits + t * ld, experts, lane, vec);
  // a warp's tokens are consecutive: all its groups stay while its first one has a token
  for (int64_t first = t - (threadIdx.x % 32) / G; first < tokens; first += groups, t += groups) {
    float z[NE], e[NE];
    row.values(live, experts, lane, z);
    live = t + groups < tokens && (!mask || mask[t + groups] != 0);
    if (live) row.load(logits + (t + groups) * ld, experts, lane, vec);  // the next token's
    uint32_t key[NE];
    int idx[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      key[i] = order_key(z[i]);
      idx[i] = R::at(lane, i);
      if (kPacked) key[i] = pack_key(key[i], idx[i]);
    }
    auto head_of = [&](uint32_t& head, int& head_idx) {
      head = key[0];
      head_idx = idx[0];
      if (!kSorted) {
#pragma unroll
        for (int i = 1; i < NE; ++i) {
          if (!kPacked && key[i] > head) head_idx = idx[i];
          head = max(head, key[i]);
        }
      }
    };
    if (kSorted) {
      if (kPacked && NE == 8) {  // 19 exchanges
        constexpr int net[19][2] = {{0, 2}, {1, 3}, {4, 6}, {5, 7}, {0, 4}, {1, 5}, {2, 6}, {3, 7}, {0, 1}, {2, 3},
                                    {4, 5}, {6, 7}, {2, 4}, {3, 5}, {1, 4}, {3, 6}, {1, 2}, {3, 4}, {5, 6}};
#pragma unroll
        for (int x = 0; x < 19; ++x)
          order<kPacked>(key[net[x][0] % NE], idx[net[x][0] % NE], key[net[x][1] % NE], idx[net[x][1] % NE]);
      } else {
#pragma unroll
        for (int i = 1; i < NE; ++i)
#pragma unroll
          for (int j = i; j > 0; --j) order<kPacked>(key[j - 1], idx[j - 1], key[j], idx[j]);
      }
    }
    uint32_t head;
    int head_idx;
    head_of(head, head_idx);
    uint32_t top = group_max<G>(head);  // the largest key left
    const bool bad = (kPacked ? top & ~kLow : top) >= kKeyInf;
    const bool counted = top > kKeyNegInf && !bad;
    const float most = key_value(kPacked ? unpack_key(top) : top);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      e[i] = counted ? exp_neg(z[i] - most) : 0.f;
      sum += e[i];
    }
    sum = group_sum<G>(sum);
    const float inv = 1.f / sum;
    if (counted)
#pragma unroll
      for (int i = 0; i < NE; ++i) acc[i] = fmaf(e[i], inv, acc[i]);
    if (bad) {
#pragma unroll
      for (int i = 0; i < NE; ++i) acc[i] = NAN;
      if (a.status && lane == 0) atomicOr(a.status, SOAP_STATUS_NONFINITE);
    }
    seen += counted || bad;
    if (a.stats && lane == 0 && t < tokens)
      a.stats[t] = bad ? make_float2(NAN, NAN) : make_float2(most, counted ? inv : 0.f);
    // k times the largest key; what it is stays with lane r of the group
    uint32_t my_key[kRec];
#pragma unroll
    for (int j = 0; j < kRec; ++j) {
      my_key[j] = 0u;
      for (int r = 0; r < G && j * G + r < k; ++r) {
        if (j + r > 0) top = group_max<G>(head);
        if (lane == r) my_key[j] = top;
        bool mine = head == top;
        if (!kPacked) {
          // of equal keys in several lanes, the one of the lowest index
          const uint32_t who =
              __ballot_sync(0xffffffffu, mine) >> ((threadIdx.x % 32) / G * G) & (0xffffffffu >> (32 - G));
          if (__any_sync(0xffffffffu, (who & (who - 1)) != 0)) {
            const uint32_t low = ~group_max<G>(mine ? ~(uint32_t)head_idx : 0u);
            mine = mine && (uint32_t)head_idx == low;
          }
          if (mine) won[threadIdx.x / G][j * G + r] = head_idx;
        }
        if (mine) {
          if (kSorted) {
#pragma unroll
            for (int i = 1; i < NE; ++i) {
              key[i - 1] = key[i];
              if (!kPacked) idx[i - 1] = idx[i];
            }
            key[NE - 1] = 0u;
          } else {
#pragma unroll
            for (int i = 0; i < NE; ++i)
              if (kPacked ? key[i] == top : idx[i] == head_idx) key[i] = 0u;
          }
        }
        head_of(head, head_idx);
      }
    }
    if (!kPacked) __syncwarp();
    int my_idx[kRec];
    float my_gate[kRec], total = 0.f;
#pragma unroll
    for (int j = 0; j < kRec; ++j) {
      const bool some = counted && my_key[j] > (kPacked ? kKeyNegInf | kLow : kKeyNegInf);
      my_idx[j] = !some ? -1 : kPacked ? packed_index(my_key[j]) : won[threadIdx.x / G][j * G + lane];
      my_gate[j] = some ? exp_neg(key_value(kPacked ? unpack_key(my_key[j]) : my_key[j]) - most) * inv : 0.f;
      total += my_gate[j];
      if (some) atomicAdd(&counts[my_idx[j]], 1);
    }
    if (a.normalize) {
      total = group_sum<G>(total);
      if (total > 0.f)
#pragma unroll
        for (int j = 0; j < kRec; ++j) my_gate[j] /= total;
    }
    if (t < tokens)
#pragma unroll
      for (int j = 0; j < kRec; ++j)
        if (j * G + lane < k) {
          a.indices[t * k + j * G + lane] = my_idx[j];
          a.gates[t * k + j * G + lane] = bad ? NAN : my_gate[j];
        }
    if (!kPacked) __syncwarp();  // the choices have been read
  }
  // column sums: the groups of a warp by shuffles, the warps in order
  if (lane == 0 && seen) atomicAdd(&counts[experts], seen);
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    float v = acc[i];
#pragma unroll
    for (int o = G; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    const int c = R::at(lane, i);
    if (threadIdx.x % 32 < G && c < experts) shared[warp * experts + c] = v;
  }
  finish_columns<kWarps>(shared, counts, red, experts, k, a.part_p, a.part_c, out);
}

// Adds the clusters' partial rows in a fixed order; the loss. One CTA of 1024 threads: a warp takes 32
// columns of every few-th row.
__global__ void __launch_bounds__(1024)
    route_sum_kernel(const float* part_p, const int* part_c, int parts, int experts, int k, Totals out) {
  __shared__ float sum_p[32][32];
  __shared__ int sum_c[32][32];
  __shared__ float red[32];
  __shared__ int total;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  asm volatile("griddepcontrol.wait;" ::: "memory");  // launched ahead: it starts as the last CTAs of the kernel before exit
  const int blocks = (experts + 31) / 32, ways = 32 / blocks;  // at most 32 blocks of columns
  const int block = warp % blocks, way = warp / blocks, c = block * 32 + lane;
  float v = 0.f;
  int cnt = 0;
  if (way < ways && c < experts) {
#pragma unroll 8
    for (int p = way; p < parts; p += ways) {
      v += part_p[(int64_t)p * experts + c];
      cnt += part_c[(int64_t)p * (experts + 1) + c];
    }
  }
  sum_p[warp][lane] = v;
  sum_c[warp][lane] = cnt;
  if (warp == 31) {
    int n = 0;
    for (int p = lane; p < parts; p += 32) n += part_c[(int64_t)p * (experts + 1) + experts];
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) total = n;
  }
  __syncthreads();
  const int n = total;
  float dot = 0.f;
  if (way == 0 && c < experts) {
    float s = 0.f;
    cnt = 0;
    for (int w = 0; w < ways; ++w) {
      s += sum_p[w * blocks + block][lane];
      cnt += sum_c[w * blocks + block][lane];
    }
    const float mean = n > 0 ? s / (float)n : 0.f;
    out.counts[c] = cnt;
    if (out.mean_probs) out.mean_probs[c] = mean;
    dot = (float)cnt * mean;
  }
  dot = block_sum(dot, red);
  if (threadIdx.x == 0) {
    *out.live = n;
    *out.loss = loss_of(dot, n, experts, k, out.coef);
  }
}

template <typename T, int G, int NE, int V>
__global__ void __launch_bounds__(kThreads)
    route_bwd_kernel(const Backward a, const bool vec) {
  constexpr int kRec = kMaxK / G;
  using R = Row<T, G, NE, V>;
  const T* const logits = static_cast<const T*>(a.logits);
  T* const dlogits = static_cast<T*>(a.dlogits);
  const int64_t ld = a.ld, ld_d = a.ld_d, tokens = a.tokens;
  const uint8_t* const mask = a.mask;
  const int32_t *const indices = a.indices, *const counts = a.counts;
  const float* const dgates = a.dgates;
  const int experts = a.experts, k = a.k;
  const int lane = threadIdx.x % G;
  const int64_t groups = (int64_t)gridDim.x * (kThreads / G);
  int64_t t = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  R row;
  bool live = t < tokens && (!mask || mask[t] != 0);
  if (live) row.load(logits + t * ld, experts, lane, vec);
  const int n = *a.live;
  const float per = n > 0 ? a.scale / (float)n / (float)n : 0.f;
  float up[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const int c = R::at(lane, i);
    up[i] = c < experts ? per * (float)counts[c] : 0.f;
  }
  for (int64_t first = t - (threadIdx.x % 32) / G; first < tokens; first += groups, t += groups) {
    const bool here = live;
    float z[NE];
    row.values(here, experts, lane, z);
    const float2 st = here ? a.stats[t] : make_float2(0.f, 0.f);  // the largest logit, 1 / sum of e^(z - largest)
    const bool bad = st.y != st.y;
    // the gates' gradient at the chosen logits: lane r holds choices r, r + G, ...
    int at[kRec];
    float d[kRec], pc[kRec], s = 0.f, dot = 0.f;
#pragma unroll
    for (int j = 0; j < kRec; ++j) {
      at[j] = -1;
      d[j] = pc[j] = 0.f;
      const int r = j * G + lane;
      if (dgates && here && r < k) {
        const int c = indices[t * k + r];
        if (c >= 0 && c < experts) {
          at[j] = c;
          d[j] = dgates[t * k + r];
          pc[j] = exp_neg(to_f32(logits[t * ld + c]) - st.x) * st.y;
          s += pc[j];
          dot = fmaf(d[j], pc[j], dot);
        }
      }
    }
    live = t + groups < tokens && (!mask || mask[t + groups] != 0);
    if (live) row.load(logits + (t + groups) * ld, experts, lane, vec);  // the next token's
    if (dgates && a.normalize) {
      // gate_r = p_r / s: d p_r = (d gate_r - sum_j d gate_j gate_j) / s, whose sum with the p_r is zero
      s = group_sum<G>(s);
      dot = group_sum<G>(dot) / s;
#pragma unroll
      for (int j = 0; j < kRec; ++j)
        if (at[j] >= 0) d[j] = (d[j] - dot) / s;
      dot = 0.f;
    }
    float p[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      p[i] = st.y > 0.f ? exp_neg(z[i] - st.x) * st.y : 0.f;
      dot = fmaf(p[i], up[i], dot);
    }
    dot = group_sum<G>(dot);
    if (t < tokens) {
      T* out = dlogits + t * ld_d;
#pragma unroll
      for (int i = 0; i < NE; i += V) {
        if (R::at(lane, i) >= experts) continue;
        Pack<T, V> o;
#pragma unroll
        for (int q = 0; q < V; ++q) o.v[q] = from_f32<T>(bad ? NAN : p[i + q] * (up[i + q] - dot));
        if (V == 1 || vec) {
          *reinterpret_cast<Pack<T, V>*>(out + R::at(lane, i)) = o;
        } else {
#pragma unroll
          for (int q = 0; q < V; ++q) out[R::at(lane, i + q)] = o.v[q];
        }
      }
    }
    if (dgates) {  // the chosen ones again, with the gates' part (ordered after the row's stores)
      __syncwarp();
#pragma unroll
      for (int j = 0; j < kRec; ++j)
        if (at[j] >= 0)
          dlogits[t * ld_d + at[j]] = from_f32<T>(pc[j] * (per * (float)counts[at[j]] + d[j] - dot));
    }
  }
}

// ---- launches ------------------------------------------------------------------------------

// f(group size, registers per lane): a lane holds up to 8 logits before the group grows (fp32, whose
// exchanges move an index too: up to 4), and up to 32 in the end.
template <typename T, typename F>
cudaError_t with_shape(int experts, F&& f) {
  using std::integral_constant;
  using I8 = integral_constant<int, 8>;
  using I16 = integral_constant<int, 16>;
  using I32 = integral_constant<int, 32>;
  if (experts <= 8) return f(I8(), integral_constant<int, 1>());
  if (experts <= 16) return f(I8(), integral_constant<int, 2>());
  if (experts <= 32) return f(I8(), integral_constant<int, 4>());
  if constexpr (sizeof(T) == 2) {
    if (experts <= 64) return f(I8(), I8());
    if (experts <= 128) return f(I16(), I8());
  } else {
    if (experts <= 64) return f(I16(), integral_constant<int, 4>());
    if (experts <= 128) return f(I32(), integral_constant<int, 4>());
  }
  if (experts <= 256) return f(I32(), I8());
  if (experts <= 512) return f(I32(), I16());
  return f(I32(), I32());
}

template <typename F>
cudaError_t with_type(int32_t type, F&& f) {
  if (type == SOAP_F32) return f(float());
  return type == SOAP_BF16 ? f(__nv_bfloat16()) : f(__half());
}

// Tokens per CTA and pass, at least (fp32's groups).
int tokens_per_cta(int experts) { return kThreads / (experts <= 32 ? 8 : experts <= 64 ? 16 : 32); }

// CTAs: for few tokens one cluster that finishes alone, of up to 8 CTAs, else whole clusters, up to four
// CTAs per SM.
int ctas_for(int64_t tokens, int experts, int* cluster) {
  const int64_t want = std::max<int64_t>(1, (tokens + tokens_per_cta(experts) - 1) / tokens_per_cta(experts));
  int c = 1;
  while (c < kCluster && c < want) c *= 2;
  *cluster = c;
  if (want <= 4 * kCluster) return c;
  return (int)std::min<int64_t>(kMaxCtas, (want + kCluster - 1) / kCluster * kCluster);
}

// f(T(), group size, registers per lane, logits per access, whether the rows allow such accesses).
template <int TENSORS, typename F>
cudaError_t with_row(int32_t type, int experts, const void* a, int64_t ld_a, const void* b, int64_t ld_b, F&& f) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    return with_shape<T>(experts, [&](auto g, auto ne) {
      constexpr int NE = decltype(ne)::value, V = std::min<int>(NE, 16 / sizeof(T));
      if (V == 1 || experts % V) return f(t, g, ne, std::integral_constant<int, 1>(), true);
      uintptr_t bytes = reinterpret_cast<uintptr_t>(a) | ld_a * sizeof(T);
      if (TENSORS == 2) bytes |= reinterpret_cast<uintptr_t>(b) | ld_b * sizeof(T);
      return f(t, g, ne, std::integral_constant<int, V>(), bytes % (V * sizeof(T)) == 0);
    });
  });
}

bool bad_ptr(const void* p, size_t size) { return !p || reinterpret_cast<uintptr_t>(p) % size; }

bool bad_route(int64_t tokens, int32_t experts, int32_t k, const void* logits, int64_t ld, int32_t type, float coef) {
  if (tokens < 0 || tokens > INT32_MAX || experts < 1 || experts > kMaxExperts) return true;
  if (k < 1 || k > experts || k > 32 || type < SOAP_F32 || type > SOAP_F16 || !std::isfinite(coef)) return true;
  return tokens > 0 && (bad_ptr(logits, dtype_size(type)) || ld < experts);
}

}  // namespace
}  // namespace soap

using namespace soap;

extern "C" {

size_t layer_route_workspace_bytes(int64_t tokens, int32_t experts) {
  if (tokens < 0 || tokens > INT32_MAX || experts < 1 || experts > kMaxExperts) return 0;
  int cluster;
  const size_t parts = tokens >= kFewTokens ? kMaxParts : ctas_for(tokens, experts, &cluster) / cluster;
  return parts * (2 * (size_t)experts + 1) * 4;
}

soap_status_t layer_route_forward(int64_t tokens, int32_t experts, int32_t k, const void* logits, int64_t ld,
                                  int32_t type, const uint8_t* mask, int32_t normalize, float coef,
                                  int32_t* indices, float* gates, float* stats, int32_t* counts,
                                  int32_t* live, float* mean_probs, float* loss, int32_t* status, void* workspace,
                                  size_t workspace_bytes, soap_stream_t stream) {
  if (bad_route(tokens, experts, k, logits, ld, type, coef)) return SOAP_ERR_INVALID_ARG;
  if (tokens > 0 && (bad_ptr(indices, 4) || bad_ptr(gates, 4))) return SOAP_ERR_INVALID_ARG;
  if (bad_ptr(counts, 4) || bad_ptr(live, 4) || bad_ptr(loss, 4) || (mean_probs && bad_ptr(mean_probs, 4)) ||
      (stats && bad_ptr(stats, 8)) ||
      (status && bad_ptr(status, 4)) || bad_ptr(workspace, 16) ||
      workspace_bytes < layer_route_workspace_bytes(tokens, experts))
    return SOAP_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  const bool tiles = tile_fits(tokens, experts, k, type);
  int cluster = kTileCluster;
  const int ctas = tiles ? tile_forward_ctas(tokens, experts, k, type) : ctas_for(tokens, experts, &cluster);
  const int parts = ctas / cluster;
  float* part_p = static_cast<float*>(workspace);
  int* part_c = reinterpret_cast<int*>(part_p + (size_t)parts * experts);
  const Totals out{counts, live, mean_probs, loss, coef};
  const Forward f{logits, ld, mask, tokens, experts, k, normalize, indices, gates, reinterpret_cast<float2*>(stats),
                  part_p, part_c, status};
  const double n = (double)tokens * experts;
  ProfScope prof(kFamElementwise, 6.0 * n, n * dtype_size(type) + 8.0 * tokens * k, s);
  cudaLaunchAttribute attr;
  cudaLaunchConfig_t cfg{};
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  cudaError_t e;
  if (tiles) {
    e = tile_forward(f, out, type, s);
  } else {
    cfg.blockDim = dim3(kThreads);
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.dynamicSmemBytes = (size_t)((kWarps + 1) * experts + 1) * 4;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = cluster;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    e = with_row<1>(type, experts, logits, ld, nullptr, 0, [&](auto t, auto g, auto ne, auto v, bool vec) {
      using T = decltype(t);
      return cudaLaunchKernelEx(&cfg, route_fwd_kernel<T, decltype(g)::value, decltype(ne)::value, decltype(v)::value>,
                                f, out, vec);
    });
  }
  if (e == cudaSuccess && parts > 1) {
    cfg.gridDim = dim3(1);
    cfg.blockDim = dim3(1024);
    cfg.dynamicSmemBytes = 0;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    e = cudaLaunchKernelEx(&cfg, route_sum_kernel, (const float*)part_p, (const int*)part_c, parts, (int)experts,
                           (int)k, out);
  }
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

soap_status_t layer_route_backward(int64_t tokens, int32_t experts, int32_t k, const void* logits, int64_t ld,
                                   int32_t type, const uint8_t* mask, int32_t normalize, float coef, float dloss,
                                   const int32_t* indices, const float* stats, const int32_t* counts,
                                   const int32_t* live, const float* dgates, void* dlogits, int64_t ld_d,
                                   soap_stream_t stream) {
  if (bad_route(tokens, experts, k, logits, ld, type, coef) || !std::isfinite(dloss)) return SOAP_ERR_INVALID_ARG;
  if (tokens == 0) return SOAP_OK;
  if (bad_ptr(stats, 8) || bad_ptr(counts, 4) || bad_ptr(live, 4) || bad_ptr(dlogits, dtype_size(type)) ||
      ld_d < experts || (dgates && (bad_ptr(dgates, 4) || bad_ptr(indices, 4))))
    return SOAP_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  const double n = (double)tokens * experts;
  const Backward b{logits, ld, mask, tokens, experts, k, normalize, (float)((double)coef * dloss * experts / k),
                   indices, reinterpret_cast<const float2*>(stats), counts, live, dgates, dlogits, ld_d};
  ProfScope prof(kFamElementwise, 6.0 * n, 2.0 * n * dtype_size(type) + 12.0 * tokens * k, s);
  cudaError_t e;
  if (tile_fits(tokens, experts, k, type)) {
    e = tile_backward(b, type, s);
  } else {
    const int64_t want = (tokens + tokens_per_cta(experts) - 1) / tokens_per_cta(experts);
    const int ctas = (int)std::min<int64_t>(kMaxCtas, want);
    e = with_row<2>(type, experts, logits, ld, dlogits, ld_d, [&](auto t, auto g, auto ne, auto v, bool vec) {
      using T = decltype(t);
      route_bwd_kernel<T, decltype(g)::value, decltype(ne)::value, decltype(v)::value>
          <<<ctas, kThreads, 0, s>>>(b, vec);
      return cudaGetLastError();
    });
  }
  return e == cudaSuccess ? SOAP_OK : SOAP_ERR_CUDA;
}

}  // extern "C"
