// Orthogonalisation of matrices with a small side (muon_orthogonalize): a cluster per matrix, everything
// on chip, one launch.
//
// X (r x k, r <= 128; a tall matrix is brought in transposed) stays in shared memory as fp16 (split: hi
// and lo planes), its columns dealt to the cluster's CTAs. A step forms each CTA's part of S = X X^T,
// adds the parts through distributed shared memory (each CTA some of the elements, in a fixed order,
// written to all), forms B = b S + c S^2 in every CTA and X' = a X + B X on its own columns, in place.
//
// These products are too small for the 5th-generation tensor cores to pay: a 256-wide accumulation of
// K = 2048 takes 128 dependent instructions of 140 cycles there, 10 us, and its result comes back through
// tensor memory. Warp-level mma (16 x 8 x 16, fp32 accumulators in registers) does the step's few million
// products in a microsecond or two. 2048 x 64 takes 6 us a step, of which 2.5 are S, B and X' themselves and
// 2.5 the exchange and its barriers (in cycles: S 1300, exchange 4800, B 1400, X' 2100); as tiles of
// steps_kernel, with a signal between the phases, 20. With r near 128 the mma's rate bounds it (8000 x 100:
// 24 us a step, more than half of them X').
#include <algorithm>
#include <atomic>
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
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 16;  // 8 is what every GPU takes, 16 this one
constexpr int kMaxSmem = 224 * 1024;
// Most K elements per accumulator run of split operands. The mma's accumulator truncates as the tensor memory's
// does, 2^-25 of a sum per 16 products: over the 3136 elements that a CTA has of 16 x 50000, S came out 1.5e-5
// too small and the result 7.6e-6 too large; 5.4e-7 in runs of 256 that are added in fp32 (4 % of that case's
// time, 1 to 2 % of others').
constexpr int kRun = 256;

struct Layout {
  int r, k, tall;
  int rp;        // r rounded up to a multiple of 16
  int kc, kcp;   // columns of a CTA, rounded up to a multiple of 16
  int x_pitch, s_pitch, p_pitch;  // elements between rows of X, of S and B, of the partial sums
};

__host__ __device__ inline size_t x_bytes(const Layout& l, int split) { return (size_t)split * l.rp * l.x_pitch * 2; }
__host__ __device__ inline size_t s_bytes(const Layout& l, int split) { return (size_t)split * l.rp * l.s_pitch * 2; }
// B and the partial sums share their place: the sums have been read when B is written.
__host__ __device__ inline size_t b_bytes(const Layout& l, int split) {
  const size_t b = s_bytes(l, split), p = (size_t)l.rp * l.p_pitch * 4;
  return b > p ? b : p;
}

Layout make_layout(int rows, int cols, int cluster) {
  Layout l{};
  l.r = std::min(rows, cols);
  l.k = std::max(rows, cols);
  l.tall = rows > cols;
  l.rp = (l.r + 15) / 16 * 16;
  l.kc = (l.k + cluster - 1) / cluster;
  l.kc = (l.kc + 15) / 16 * 16;
  l.kcp = l.kc;
  l.x_pitch = l.kcp + 8;  // rows an odd number of 16-byte units apart: ldmatrix without conflicts
  l.s_pitch = l.rp + 8;
  l.p_pitch = l.rp + 4;
  return l;
}

size_t smem_bytes(const Layout& l, int split) { return x_bytes(l, split) + s_bytes(l, split) + b_bytes(l, split) + 16; }

__device__ __forceinline__ uint32_t smem_at(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// Four 8 x 8 matrices of 16-bit elements, a row's address per lane.
__device__ __forceinline__ void ldmatrix(uint32_t (&f)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(f[0]), "=r"(f[1]), "=r"(f[2]), "=r"(f[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldmatrix_t(uint32_t (&f)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(f[0]), "=r"(f[1]), "=r"(f[2]), "=r"(f[3])
               : "r"(at)
               : "memory");
}
// c += a (16 x 16) b (16 x 8)
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer(uint32_t at, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(rank));
  return r;
}
__device__ __forceinline__ float4 peer_load4(uint32_t at) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(at)
               : "memory");
  return v;
}
__device__ __forceinline__ float peer_load(uint32_t at) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void peer_store2(uint32_t at, uint32_t x, uint32_t y) {
  asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(x), "r"(y) : "memory");
}

__device__ __forceinline__ uint32_t half2_bits(float x, float y) {
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 bits_half2(uint32_t b) { return __half22float2(*reinterpret_cast<const __half2*>(&b)); }

// A raw element in X's place until the norm is known: 16-bit types in the hi plane, an fp32's halves in the
// two planes.
__device__ __forceinline__ void put_raw(__half* hi, __half*, __nv_bfloat16 v) { *reinterpret_cast<__nv_bfloat16*>(hi) = v; }
__device__ __forceinline__ void put_raw(__half* hi, __half*, __half v) { *hi = v; }
__device__ __forceinline__ void put_raw(__half* hi, __half* lo, float v) {
  const uint32_t u = __float_as_uint(v);
  *reinterpret_cast<uint16_t*>(hi) = (uint16_t)(u >> 16);
  *reinterpret_cast<uint16_t*>(lo) = (uint16_t)u;
}
__device__ __forceinline__ float get_raw(const __half* hi, const __half*, __nv_bfloat16) {
  return to_f32(*reinterpret_cast<const __nv_bfloat16*>(hi));
}
__device__ __forceinline__ float get_raw(const __half* hi, const __half*, __half) { return to_f32(*hi); }
__device__ __forceinline__ float get_raw(const __half* hi, const __half* lo, float) {
  return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(hi) << 16 | *reinterpret_cast<const uint16_t*>(lo));
}

// f(element i, j of X's slice, address of V consecutive elements of the matrix): in the matrix's order, V
// elements along its rows per call; the same calls by the same threads every time.
template <int V, typename T, typename F>
__device__ __forceinline__ void each_pack(const Layout& l, T* M, int64_t ld, int c0, int columns, F&& f) {
  if (columns <= 0) return;
  const int rows = l.tall ? columns : l.r, width = l.tall ? l.r : columns;
  T* m = M + (l.tall ? (int64_t)c0 * ld : c0);
  const int packs = (width + V - 1) / V;
  int row = threadIdx.x / packs, p = threadIdx.x - row * packs;
  const int drow = kThreads / packs, dp = kThreads - drow * packs;
#pragma unroll 4
  for (; row < rows;) {
    f(row, p * V, m + (int64_t)row * ld + p * V);
    row += drow;
    p += dp;
    if (p >= packs) {
      p -= packs;
      ++row;
    }
  }
}

template <typename T, int SPLIT, int RT, int V>
__global__ void __launch_bounds__(kThreads)
    small_kernel(const __grid_constant__ Steps a, const Layout l, const T* M, int64_t ld, int64_t stride, float eps,
                 int sx) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float red[kWarps][2];
  __shared__ float mine[2];  // this CTA's sum of squares and largest magnitude
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint32_t rank = cluster_rank(), size = cluster_size();
  const int b = blockIdx.x / size;
  __half* const X = reinterpret_cast<__half*>(smem);
  __half* const S = reinterpret_cast<__half*>(smem + x_bytes(l, SPLIT));
  __half* const B = reinterpret_cast<__half*>(smem + x_bytes(l, SPLIT) + s_bytes(l, SPLIT));
  float* const part = reinterpret_cast<float*>(B);
  const int x_plane = l.rp * l.x_pitch, s_plane = l.rp * l.s_pitch;
  const int c0 = rank * l.kc, columns = max(0, min(l.kc, l.k - c0));

  // zeros around the slice
  for (int i = threadIdx.x; i < (int)(x_bytes(l, SPLIT) / 16); i += kThreads)
    reinterpret_cast<uint4*>(X)[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
  // place of element e of the pack at (row, c) of the slice as the matrix has it
  auto place = [&](int row, int c) { return l.tall ? c * l.x_pitch + row : row * l.x_pitch + c; };
  const int width = l.tall ? l.r : columns;
  float sum = 0.f, most = 0.f;
  each_pack<V>(l, M + (int64_t)b * stride, ld, c0, columns, [&](int row, int c, const T* p) {
    Pack<T, V> v = *reinterpret_cast<const Pack<T, V>*>(p);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      __half* x = X + place(row, c + e);
      put_raw(x, x + x_plane, v.v[e]);
      const float f = to_f32(v.v[e]);
      sum = fmaf(f, f, sum);
      most = fmaxf(most, fabsf(f));
    }
  });
  auto reduce = [&](float s, float m, float& all_s, float& all_m) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    }
    if (lane == 0) {
      red[warp][0] = s;
      red[warp][1] = m;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < kWarps; ++w) {
        s += red[w][0];
        m = fmaxf(m, red[w][1]);
      }
      mine[0] = s;
      mine[1] = m;
    }
    cluster_sync();
    all_s = all_m = 0.f;
    for (uint32_t q = 0; q < size; ++q) {
      all_s += peer_load(peer(smem_at(&mine[0]), q));
      all_m = fmaxf(all_m, peer_load(peer(smem_at(&mine[1]), q)));
    }
  };
  float all, top;
  reduce(sum, most, all, top);
  int back = 0;  // squares were taken of elements times 2^back
  if (top > 0.f && top < INFINITY && !(top > 0x1p-40f && top < 0x1p50f)) {  // beyond the range of fp32 squares
    int e;
    frexpf(top, &e);
    back = -e;
    cluster_sync();  // the others have read `mine`
    sum = 0.f;
    const T* unused = nullptr;
    each_pack<V>(l, unused, 0, 0, columns, [&](int row, int c, const T*) {
#pragma unroll
      for (int q = 0; q < V; ++q)
        if (c + q < width) {
          const __half* x = X + place(row, c + q);
          const float f = ldexpf(get_raw(x, x + x_plane, T()), back);
          sum = fmaf(f, f, sum);
        }
    });
    reduce(sum, 0.f, all, most);
  }
  // 1 / max(norm, eps) = t 2^-e
  const bool bad = !(all < INFINITY) || !(top < INFINITY);
  int e = 0;
  float t = 1.f;
  if (!bad) {
    int en, ee;
    const float fn = frexpf(sqrtf(all), &en), fe = frexpf(eps, &ee);
    en -= back;
    const bool norm = all > 0.f && (en > ee || (en == ee && fn > fe));
    e = norm ? en : ee;
    t = 1.f / (norm ? fn : fe);
  } else if (a.status && rank == 0 && threadIdx.x == 0) {
    atomicOr(a.status, SOAP_STATUS_NONFINITE);
  }
  const int q1 = min(sx - e, 120);  // a norm near fp32's smallest: t takes what fp32's range leaves
  const float scale = bad ? NAN : ldexpf(1.f, q1);
  t = ldexpf(t, sx - e - q1);
  {
    const T* unused = nullptr;
    each_pack<V>(l, unused, 0, 0, columns, [&](int row, int c, const T*) {
#pragma unroll
      for (int q = 0; q < V; ++q)
        if (c + q < width) {
          __half* x = X + place(row, c + q);
          const float f = get_raw(x, x + x_plane, T()) * scale;
          const __half h = __float2half_rn(f);
          *x = h;
          if (SPLIT == 2) x[x_plane] = __float2half_rn(f - __half2float(h));
        }
    });
  }
  __syncthreads();

  // ldmatrix addresses: A (16 rows from i, 16 elements from k) and B as rows of n: the lane's row and column
  const int a_row = lane % 16, a_col = lane / 16 * 8;
  const int b_row = lane / 16 * 8 + lane % 8, b_col = lane / 8 % 2 * 8;
  const uint32_t x_at = smem_at(X), s_at = smem_at(S), b_at = smem_at(B);
  const int c_row = lane / 4, c_col = lane % 4 * 2;  // the lane's place in a result: (row, col), (row + 8, col)
  const int mt = l.rp / 16;

  // rows i0 .. + 15 and n0 .. + 31 of P Q^T over K elements, P and Q with rows `pitch` apart
  auto product = [&](float (&acc)[4][4], uint32_t p_at, uint32_t plane, int pitch, int i0, int n0, int K) {
    float small[4][4], runs[4][4];
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[n][q] = small[n][q] = runs[n][q] = 0.f;
    const uint32_t pa = p_at + ((i0 + a_row) * pitch + a_col) * 2;
    const uint32_t pb0 = p_at + ((n0 + b_row) * pitch + b_col) * 2, pb1 = pb0 + 16 * pitch * 2;
    const bool second = n0 + 16 < l.rp;
    for (int k = 0; k < K; k += 16) {
      uint32_t fa[4], fb[2][4], la[4], lb[2][4];
      ldmatrix(fa, pa + k * 2);
      ldmatrix(fb[0], pb0 + k * 2);
      if (second) ldmatrix(fb[1], pb1 + k * 2);
      if (SPLIT == 2) {
        ldmatrix(la, pa + plane + k * 2);
        ldmatrix(lb[0], pb0 + plane + k * 2);
        if (second) ldmatrix(lb[1], pb1 + plane + k * 2);
      }
#pragma unroll
      for (int n = 0; n < 4; ++n)
        if (n < 2 || second) {
          mma(acc[n], fa, fb[n / 2][n % 2 * 2], fb[n / 2][n % 2 * 2 + 1]);
          if (SPLIT == 2) {
            mma(small[n], la, fb[n / 2][n % 2 * 2], fb[n / 2][n % 2 * 2 + 1]);
            mma(small[n], fa, lb[n / 2][n % 2 * 2], lb[n / 2][n % 2 * 2 + 1]);
          }
        }
      if (SPLIT == 2 && (k + 16) % kRun == 0)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            runs[n][q] += acc[n][q];
            acc[n][q] = 0.f;
          }
    }
    if (SPLIT == 2)
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[n][q] += runs[n][q] + small[n][q];
  };
  const int nt = (l.rp + 31) / 32;
  // f(i0, n0, whether to write the mirror image too) for this warp's 16 x 32 tiles of a symmetric matrix. With
  // more tiles than warps, those on and below the diagonal's 32 x 32 blocks (of r = 100: 16 of 28), which
  // saves mma's: what bounds such sizes.
  auto each_tile = [&](auto&& f) {
    if constexpr (RT == 8) {
      int i = 0;
      for (int m = 0; m < mt; ++m)
        for (int n = 0; n <= m / 2; ++n, ++i)
          if (i % kWarps == warp) f(16 * m, 32 * n, m / 2 > n);
    } else {
      for (int i = warp; i < mt * nt; i += kWarps) f(i / nt * 16, i % nt * 32, false);
    }
  };
  // lanes per four elements of S, so that all of the cluster's threads have some of its parts to add (by one
  // thread each, S of 64 x 64 occupies a quarter of a cluster of 16); a warp's are whole
  int share = 1;
  while (share < (int)size && 2 * share * l.rp * (l.rp / 4) <= (int)size * kThreads) share *= 2;
  const int first_quad = (rank * kThreads + threadIdx.x) / share;

  for (int step = 0; step < a.steps; ++step) {
    const StepCoef& c = a.coef[step];
    const float ft = step == 0 ? t : 1.f;
    // this CTA's part of X X^T
    each_tile([&](int i0, int n0, bool mirror) {
      float acc[4][4];
      product(acc, x_at, x_plane * 2, l.x_pitch, i0, n0, l.kcp);
#pragma unroll
      for (int n = 0; n < 4; ++n)
        if (n0 + n * 8 < l.rp) {
          float* p = part + (i0 + c_row) * l.p_pitch + n0 + n * 8 + c_col;
          *reinterpret_cast<float2*>(p) = make_float2(acc[n][0], acc[n][1]);
          *reinterpret_cast<float2*>(p + 8 * l.p_pitch) = make_float2(acc[n][2], acc[n][3]);
          if (mirror) {
            float* t = part + (n0 + n * 8 + c_col) * l.p_pitch + i0 + c_row;
            t[0] = acc[n][0];
            t[l.p_pitch] = acc[n][1];
            t[8] = acc[n][2];
            t[l.p_pitch + 8] = acc[n][3];
          }
        }
    });
    cluster_sync();
    {  // S: four elements at a time by `share` lanes, each some of the cluster's parts, in order, and then to
       // some of its CTAs
      const int quads = l.rp / 4;
      const float alpha = c.s_alpha * ft * ft;
      for (int i = first_quad; i < l.rp * quads; i += size * kThreads / share) {
        const int row = i / quads, col = (i - row * quads) * 4;
        const uint32_t at = smem_at(part + row * l.p_pitch + col);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (uint32_t q = lane % share; q < size; q += share) {
          const float4 x = peer_load4(peer(at, q));
          v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
        }
        for (int o = 1; o < share; o *= 2) {
          v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
          v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
          v.z += __shfl_xor_sync(0xffffffffu, v.z, o);
          v.w += __shfl_xor_sync(0xffffffffu, v.w, o);
        }
        v = make_float4(v.x * alpha, v.y * alpha, v.z * alpha, v.w * alpha);
        const uint32_t h0 = half2_bits(v.x, v.y), h1 = half2_bits(v.z, v.w);
        const uint32_t to = s_at + (row * l.s_pitch + col) * 2;
        uint32_t l0 = 0, l1 = 0;
        if (SPLIT == 2) {
          const float2 f0 = bits_half2(h0), f1 = bits_half2(h1);
          l0 = half2_bits(v.x - f0.x, v.y - f0.y);
          l1 = half2_bits(v.z - f1.x, v.w - f1.y);
        }
        for (uint32_t q = lane % share; q < size; q += share) {
          peer_store2(peer(to, q), h0, h1);
          if (SPLIT == 2) peer_store2(peer(to + s_plane * 2, q), l0, l1);
        }
      }
    }
    cluster_sync();
    // B = b S + c S S
    each_tile([&](int i0, int n0, bool mirror) {
      float acc[4][4];
      product(acc, s_at, s_plane * 2, l.s_pitch, i0, n0, l.rp);
#pragma unroll
      for (int n = 0; n < 4; ++n)
        if (n0 + n * 8 < l.rp)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int at = (i0 + c_row + 8 * h) * l.s_pitch + n0 + n * 8 + c_col;
            float2 s = bits_half2(*reinterpret_cast<const uint32_t*>(S + at));
            if (SPLIT == 2) {
              const float2 lo = bits_half2(*reinterpret_cast<const uint32_t*>(S + s_plane + at));
              s = make_float2(s.x + lo.x, s.y + lo.y);
            }
            const float x = fmaf(c.b_beta, s.x, c.b_alpha * acc[n][2 * h]);
            const float y = fmaf(c.b_beta, s.y, c.b_alpha * acc[n][2 * h + 1]);
            const uint32_t hi = half2_bits(x, y);
            *reinterpret_cast<uint32_t*>(B + at) = hi;
            uint32_t lo = 0;
            if (SPLIT == 2) {
              const float2 f = bits_half2(hi);
              lo = half2_bits(x - f.x, y - f.y);
              *reinterpret_cast<uint32_t*>(B + s_plane + at) = lo;
            }
            if (mirror) {
              uint16_t* t = reinterpret_cast<uint16_t*>(B) + (n0 + n * 8 + c_col) * l.s_pitch + i0 + c_row + 8 * h;
              t[0] = (uint16_t)hi;
              t[l.s_pitch] = (uint16_t)(hi >> 16);
              if (SPLIT == 2) {
                t[s_plane] = (uint16_t)lo;
                t[s_plane + l.s_pitch] = (uint16_t)(lo >> 16);
              }
            }
          }
    });
    __syncthreads();
    // X' = a X + B X: a warp takes 16 columns at a time, all rows, and writes them over X
    for (int n0 = warp * 16; n0 < l.kcp; n0 += kWarps * 16) {
      float acc[RT][2][4];
#pragma unroll
      for (int m = 0; m < RT; ++m)
#pragma unroll
        for (int q = 0; q < 8; ++q) acc[m][q / 4][q % 4] = 0.f;
      for (int k = 0; k < l.rp; k += 16) {
        uint32_t fx[4], lx[4];
        const uint32_t at = x_at + ((k + a_row) * l.x_pitch + n0 + a_col) * 2;
        ldmatrix_t(fx, at);
        if (SPLIT == 2) ldmatrix_t(lx, at + x_plane * 2);
#pragma unroll
        for (int m = 0; m < RT; ++m)
          if (m < mt) {
            uint32_t fb[4], lb[4];
            const uint32_t bt = b_at + ((16 * m + a_row) * l.s_pitch + k + a_col) * 2;
            ldmatrix(fb, bt);
            if (SPLIT == 2) {
              ldmatrix(lb, bt + s_plane * 2);
              mma(acc[m][0], lb, fx[0], fx[1]);
              mma(acc[m][1], lb, fx[2], fx[3]);
              mma(acc[m][0], fb, lx[0], lx[1]);
              mma(acc[m][1], fb, lx[2], lx[3]);
            }
            mma(acc[m][0], fb, fx[0], fx[1]);
            mma(acc[m][1], fb, fx[2], fx[3]);
          }
      }
      __syncwarp();  // every lane's reads of these columns come before their writes
      const float alpha = c.x_alpha * ft, beta = c.x_beta * ft;
#pragma unroll
      for (int m = 0; m < RT; ++m)
        if (m < mt)
#pragma unroll
          for (int q = 0; q < 4; ++q) {  // (n, h)
            uint32_t* x = reinterpret_cast<uint32_t*>(X + (16 * m + c_row + 8 * (q % 2)) * l.x_pitch + n0 + q / 2 * 8 +
                                                      c_col);
            uint32_t* xl = reinterpret_cast<uint32_t*>(reinterpret_cast<__half*>(x) + x_plane);
            float2 v = bits_half2(*x);
            if (SPLIT == 2) {
              const float2 lo = bits_half2(*xl);
              v = make_float2(v.x + lo.x, v.y + lo.y);
            }
            v.x = fmaf(beta, v.x, alpha * acc[m][q / 2][2 * (q % 2)]);
            v.y = fmaf(beta, v.y, alpha * acc[m][q / 2][2 * (q % 2) + 1]);
            const uint32_t hi = half2_bits(v.x, v.y);
            *x = hi;
            if (SPLIT == 2) {
              const float2 f = bits_half2(hi);
              *xl = half2_bits(v.x - f.x, v.y - f.y);
            }
          }
    }
    __syncthreads();
  }

  T* const out = static_cast<T*>(a.out) + (int64_t)b * a.stride_out;
  const float last = ldexpf(1.f, -a.out_exp);
  each_pack<V>(l, out, a.ld_out, c0, columns, [&](int row, int c, T* p) {
    Pack<T, V> v;
#pragma unroll
    for (int q = 0; q < V; ++q) {
      const __half* x = X + place(row, c + q);
      float f = __half2float(*x);
      if (SPLIT == 2) f += __half2float(x[x_plane]);
      v.v[q] = from_f32<T>(f * last);
    }
    *reinterpret_cast<Pack<T, V>*>(p) = v;
  });
}

template <typename T, int SPLIT, int RT, int V>
cudaError_t launch(const Steps& p, const Layout& l, int cluster, const void* M, int64_t ld, int64_t stride, float eps,
                   int sx, cudaStream_t s) {
  static std::atomic<uint64_t> attr_set{0};  // one bit per device that has the shared-memory attribute
  const auto kernel = small_kernel<T, SPLIT, RT, V>;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t(1) << dev : 0;
  if (bit == 0 || !(attr_set.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    attr_set.fetch_or(bit, std::memory_order_relaxed);
  }
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(p.batch * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem_bytes(l, SPLIT);
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p, l, static_cast<const T*>(M), ld, stride, eps, sx);
}

template <typename T, int SPLIT>
cudaError_t launch_t(const Steps& p, const Layout& l, int cluster, const void* M, int64_t ld, int64_t stride, float eps,
                     int sx, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const bool many = p.batch > 1;
  const uintptr_t bits = reinterpret_cast<uintptr_t>(M) | reinterpret_cast<uintptr_t>(p.out) |
                         (uintptr_t)(ld | p.ld_out | (many ? stride | p.stride_out : 0)) * sizeof(T);
  const bool vec = bits % 16 == 0 && p.cols % V == 0 && (l.tall || l.kc % V == 0);
  if (l.rp <= 32)
    return vec ? launch<T, SPLIT, 2, V>(p, l, cluster, M, ld, stride, eps, sx, s)
               : launch<T, SPLIT, 2, 1>(p, l, cluster, M, ld, stride, eps, sx, s);
  if (l.rp <= 64)
    return vec ? launch<T, SPLIT, 4, V>(p, l, cluster, M, ld, stride, eps, sx, s)
               : launch<T, SPLIT, 4, 1>(p, l, cluster, M, ld, stride, eps, sx, s);
  return vec ? launch<T, SPLIT, 8, V>(p, l, cluster, M, ld, stride, eps, sx, s)
             : launch<T, SPLIT, 8, 1>(p, l, cluster, M, ld, stride, eps, sx, s);
}

}  // namespace

// By the time of a step, in us, as measured on both sides (in brackets): here 6 for the exchange and
// 1 / 0.9e6 per product of an SM (2048 x 64: 6; 64 of 128 x 1000 with 4 CTAs each, two rounds: 36), CTAs
// of an SM sharing it; in steps_kernel 0.07 per 16 elements of a tile's K, at least 3.7 a tile (its
// epilogue), the three phases one after the other plus 6, and all tiles over the pairs, half as much again
// for the waits between phases (2048 x 64: 20; 64 of 128 x 1000: 35; 20 of 5000 x 100: 96). Split operands
// take three products for one.
int small_cluster(int rows, int cols, int batch, bool split) {
  if (std::min(rows, cols) > 128) return 0;
  const double mult = split ? 3 : 1, r = std::min(rows, cols), k = std::max(rows, cols);
  const double least = split ? 9 : 3.7, phase_s = std::max(least, k / 16 * 0.07 * mult),
               phase_b = std::max(least, r / 16 * 0.07 * mult);
  const double nx = std::ceil(k / 256);
  double best = phase_s + 2 * phase_b + 6 + 1.5 * batch * (phase_s + phase_b * (1 + nx)) / 76;
  int cluster = 0;
  for (int c = 1; c <= kMaxCluster; c *= 2) {
    const Layout l = make_layout(rows, cols, c);
    const size_t smem = smem_bytes(l, split ? 2 : 1);
    if (smem > (size_t)kMaxSmem || (c > 1 && l.kc * (c - 1) >= l.k)) continue;  // too large, or a CTA without columns
    const int per_sm = std::min<int>(2, kMaxSmem / (int)(smem + 1024));
    const double at_once = std::floor(152.0 / c) * per_sm, rounds = std::ceil(batch / at_once);
    const double shared = std::min<double>(per_sm, std::ceil((double)batch * c / 152));
    const double us = rounds * (6 + mult * shared * (2.0 * l.rp * l.rp * l.kc + (double)l.rp * l.rp * l.rp) / 0.9e6);
    if (us < best) {
      best = us;
      cluster = c;
    }
  }
  return cluster;
}

cudaError_t run_small(const Steps& p, int cluster, const void* M, int64_t ld, int64_t stride, float eps, int sx,
                      cudaStream_t s) {
  const Layout l = make_layout(p.rows, p.cols, cluster);
  const double r = l.r, k = l.k, b = p.batch;
  ProfScope prof(kFamGemmTc, b * p.steps * (r * r * k + r * r * r + 2.0 * r * r * k),
                 2.0 * b * r * k * dtype_size(p.out_type), s);
  if (p.out_type == SOAP_F32) return launch_t<float, 2>(p, l, cluster, M, ld, stride, eps, sx, s);
  if (p.out_type == SOAP_BF16) return launch_t<__nv_bfloat16, 1>(p, l, cluster, M, ld, stride, eps, sx, s);
  return launch_t<__half, 2>(p, l, cluster, M, ld, stride, eps, sx, s);
}

}  // namespace ortho
}  // namespace soap
