// The products of the stand-alone orthogonalisation (muon_orthogonalize), on the 5th-generation
// tensor cores: out = t^p (alpha A B^T + beta C), fp16 operands (kind::f16), fp32 accumulation.
//
// Operands may be stored along either dimension: a row-major matrix serves as A or B with K along
// its rows (K-major) or down its columns (MN-major), so X X^T, X^T X, B X and X B all read X as it
// lies and no transposed copy exists. Split operands (x = hi + lo, 22 bits) take three products,
// hi hi + hi lo + lo hi, into the same accumulator from one load of the four tiles.
//
// A CTA pair (cta_group::2) computes tiles of 256 x 256 or 256 x 128, each CTA holding 128 rows of
// A and half of B's rows, or a single CTA tiles of 128 x 128. Warp 0 issues TMA loads of
// 64-element K slices into a ring, warp 1 (of the pair's first CTA) the MMAs into one of two TMEM
// accumulators, four warps drain the other one: tensor memory -> registers -> alpha/beta -> shared
// memory -> coalesced stores. A symmetric result computes its tiles on and below the diagonal and
// stores each twice, the second time transposed. Every mbarrier wait is bounded; one that runs out
// sets SOAP_STATUS_TIMEOUT and the CTA drains its copies, frees its tensor memory and returns.
//
// The accumulator truncates: measured, a sum loses 2^-25 of itself per 16 products. With 11-bit
// operands that is nothing; split ones keep the small products in an accumulator of their own and
// take K in runs of 512, whose sums the epilogue warps add in fp32 registers.
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <mutex>

#include "ortho.h"
#include "profile.h"
#include "soap_internal.h"
#include "tc_ptx.h"
#include "types.h"

namespace soap {
namespace ortho {
namespace {

using namespace tc;

constexpr int BK = 64;
constexpr int kBox = 64 * 64 * 2;        // one TMA box: 64 rows of 128 bytes
constexpr int kRing = 192 * 1024;        // bytes of the operand ring
constexpr int kAcc = 2;                  // TMEM accumulators
constexpr int kRunBlocks = 8;            // K slices per accumulator run of split operands
constexpr int kEpiWarps = 4;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kStagePitch16 = 80, kStagePitch32 = 144;  // staged 32-element rows, free of bank conflicts
constexpr int kStaging = 2 * 32 * kStagePitch16;        // per epilogue warp: hi and lo, or fp32
constexpr int kSmem = 1024 + kRing + kEpiWarps * kStaging + 256;
constexpr uint64_t kWaitNs = 2000000000ull;

struct Args {
  int M, N, K, batch, symmetric;
  float alpha, beta;
  const __half* cin;
  int64_t cin_ld, cin_stride, cin_lo;
  const float* t;
  int t_pow;
  __half* out;
  int64_t ld, stride, lo;
  void* user;
  int user_type, user_vec;
  int64_t user_ld, user_stride;
  int* status;
};

__device__ __forceinline__ void expect_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}

// The address of this CTA's shared-memory object in the pair's first CTA.
__device__ __forceinline__ uint32_t in_leader(const void* p) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(p)));
  return r;
}

// `bar` is a shared::cluster address: in a pair both CTAs' copies count on the first one's barrier.
template <int CG>
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  if (CG == 2)
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
}

// ROWS x 64 elements of an operand at (row m0, k0) as boxes of 64: rows of 64 K elements each
// (K-major), or 64 K rows of 64 columns (MN-major).
template <int MAJOR, int ROWS, int CG>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int m0, int k0, int z) {
#pragma unroll
  for (int i = 0; i < ROWS / 64; ++i)
    if (MAJOR == kRowsK)
      tma_box<CG>(dst + i * kBox, map, bar, k0, m0 + i * 64, z);
    else
      tma_box<CG>(dst + i * kBox, map, bar, m0 + i * 64, k0, z);
}

// Descriptor of the 16 K elements at step kk of such a tile. K-major: 32 bytes further along the
// swizzled rows, 8-row groups 1024 B apart. MN-major: 16 rows further down, 8-row K groups 1024 B
// apart, the next 64 columns one box away.
template <int MAJOR>
__device__ __forceinline__ uint64_t tile_desc(uint32_t base, int kk) {
  const uint32_t addr = base + (MAJOR == kRowsK ? kk * 32 : kk * 16 * 128);
  uint64_t d = 0;
  d |= static_cast<uint64_t>((addr & 0x3FFFF) >> 4);
  d |= static_cast<uint64_t>((MAJOR == kRowsK ? 16 : kBox) >> 4) << 16;  // leading byte offset
  d |= static_cast<uint64_t>(1024 >> 4) << 32;                           // stride byte offset
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;  // 128-byte swizzle
  return d;
}

// kind::f16: D = f32, A = B = f16; bits 15 and 16 mark MN-major operands.
__host__ __device__ constexpr uint32_t idesc_f16(int m, int n, int a_mn, int b_mn) {
  return (1u << 4) | (static_cast<uint32_t>(a_mn) << 15) | (static_cast<uint32_t>(b_mn) << 16) |
         (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}

template <int CG>
__device__ __forceinline__ void umma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if (CG == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate));
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate));
}

// Arrives on `bar` (in a pair: on both CTAs' barriers at that place) when the MMAs so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint64_t* bar) {
  if (CG == 2)
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
            smem_u32(bar)),
        "h"((uint16_t)3)
        : "memory");
  else
    umma_commit(bar);
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

// Tile t of the launch -> (m0, n0, matrix). Full results go in groups of 8 row tiles (row tile
// fastest), so that tiles in flight share operands in L2; symmetric ones row by row of the triangle
// (R tiles across for each square on the diagonal).
template <int TM, int TN>
__device__ __forceinline__ void tile_at(int t, int symmetric, int ntm, int ntn, int& m0, int& n0, int& b) {
  constexpr int R = TM / TN;
  if (symmetric) {
    const int per = R * (ntm * (ntm + 1) / 2);
    b = t / per;
    const int w = t - b * per, r = w / R;
    int i = (int)((sqrtf(8.f * (float)r + 1.f) - 1.f) * 0.5f);
    while (i * (i + 1) / 2 > r) --i;
    while ((i + 1) * (i + 2) / 2 <= r) ++i;
    m0 = i * TM;
    n0 = ((r - i * (i + 1) / 2) * R + w % R) * TN;
    return;
  }
  const int per = ntm * ntn;
  b = t / per;
  const int r = t - b * per;
  const int g = r / (8 * ntn), w = r - g * 8 * ntn;
  const int rows = min(8, ntm - g * 8);
  m0 = (g * 8 + w % rows) * TM;
  n0 = (w / rows) * TN;
}

// 16 bytes of staged row j (part c of 4) to a 32-column block of an internal matrix.
__device__ __forceinline__ void copy_block16(const uint8_t* stage, __half* dst, int64_t ld, int rows, int cols,
                                             int lane) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int j = u * 8 + lane / 4, c = lane % 4;
    if (j < rows && c * 8 < cols)
      *reinterpret_cast<uint4*>(dst + (int64_t)j * ld + c * 8) =
          *reinterpret_cast<const uint4*>(stage + j * kStagePitch16 + c * 16);
  }
}

template <typename T>
__device__ __forceinline__ void store_user(uint8_t* stage, const float (&o)[32], T* dst, int64_t ld, int rows,
                                           int cols, bool vec, int lane) {
  constexpr int pitch = sizeof(T) == 4 ? kStagePitch32 : kStagePitch16;
  constexpr int V = 16 / sizeof(T);
#pragma unroll
  for (int u = 0; u < 32 / V; ++u) {
    Pack<T, V> p;
#pragma unroll
    for (int e = 0; e < V; ++e) p.v[e] = from_f32<T>(o[u * V + e]);
    *reinterpret_cast<Pack<T, V>*>(stage + lane * pitch + u * 16) = p;
  }
  __syncwarp();
  if (vec) {
    constexpr int L = 32 / V;  // lanes per row
#pragma unroll
    for (int u = 0; u < L; ++u) {
      const int j = u * (32 / L) + lane / L, c = lane % L;
      if (j < rows && c * V < cols)
        *reinterpret_cast<Pack<T, V>*>(dst + (int64_t)j * ld + c * V) =
            *reinterpret_cast<const Pack<T, V>*>(stage + j * pitch + c * 16);
    }
  } else {
    for (int j = 0; j < rows; ++j)
      if (lane < cols) dst[(int64_t)j * ld + lane] = *reinterpret_cast<const T*>(stage + j * pitch + lane * sizeof(T));
  }
  __syncwarp();
}

template <int SPLIT>
struct Cin {
  uint4 h[4], l[4];
};

// This lane's 32 elements of C at `src` (the lane's row, `cols` columns left).
template <int SPLIT>
__device__ __forceinline__ void load_cin(Cin<SPLIT>& c, const __half* src, int64_t lo, int cols) {
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (u * 8 < cols) {
      c.h[u] = *reinterpret_cast<const uint4*>(src + u * 8);
      if (SPLIT == 2) c.l[u] = *reinterpret_cast<const uint4*>(src + lo + u * 8);
    }
}

template <int SPLIT>
__device__ __forceinline__ void add_cin(const Cin<SPLIT>& c, float beta, int cols, float (&o)[32]) {
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (u * 8 < cols) {
      const __half* h = reinterpret_cast<const __half*>(&c.h[u]);
      const __half* l = reinterpret_cast<const __half*>(&c.l[u]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float x = __half2float(h[e]);
        if (SPLIT == 2) x += __half2float(l[e]);
        o[u * 8 + e] = fmaf(beta, x, o[u * 8 + e]);
      }
    }
}

// A warp's 32 x 32 block of the result (row r0 + lane in o): to the caller's matrix, or to an
// internal one, there also to the mirror position.
template <int SPLIT>
__device__ __forceinline__ void store_block(const Args& g, uint8_t* stage, float (&o)[32], int b, int r0, int c0,
                                            int rows, int cols, bool mirror, int lane) {
  if (g.user) {
    const int64_t at = (int64_t)b * g.user_stride + (int64_t)r0 * g.user_ld + c0;
    if (g.user_type == SOAP_F32)
      store_user(stage, o, static_cast<float*>(g.user) + at, g.user_ld, rows, cols, g.user_vec, lane);
    else if (g.user_type == SOAP_BF16)
      store_user(stage, o, static_cast<__nv_bfloat16*>(g.user) + at, g.user_ld, rows, cols, g.user_vec, lane);
    else
      store_user(stage, o, static_cast<__half*>(g.user) + at, g.user_ld, rows, cols, g.user_vec, lane);
    return;
  }
  __half* out = g.out + (int64_t)b * g.stride;
#pragma unroll
  for (int h = 0; h < SPLIT; ++h) {
    uint8_t* st = stage + h * 32 * kStagePitch16;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      Pack<__half, 8> p;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p.v[e] = __float2half_rn(o[u * 8 + e]);
        o[u * 8 + e] -= __half2float(p.v[e]);
      }
      *reinterpret_cast<Pack<__half, 8>*>(st + lane * kStagePitch16 + u * 16) = p;
    }
  }
  __syncwarp();
#pragma unroll
  for (int h = 0; h < SPLIT; ++h)
    copy_block16(stage + h * 32 * kStagePitch16, out + h * g.lo + (int64_t)r0 * g.ld + c0, g.ld, rows, cols, lane);
  if (mirror) {  // read a staged row per lane, write it as a column
#pragma unroll
    for (int h = 0; h < SPLIT; ++h) {
      uint8_t* st = stage + h * 32 * kStagePitch16;
      Pack<__half, 8> p[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) p[u] = *reinterpret_cast<const Pack<__half, 8>*>(st + lane * kStagePitch16 + u * 16);
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 32; ++j)
        *reinterpret_cast<__half*>(st + j * kStagePitch16 + lane * 2) = p[j / 8].v[j % 8];
    }
    __syncwarp();
#pragma unroll
    for (int h = 0; h < SPLIT; ++h)
      copy_block16(stage + h * 32 * kStagePitch16, out + h * g.lo + (int64_t)c0 * g.ld + r0, g.ld, cols, rows, lane);
  }
  __syncwarp();
}

template <int AM, int BMJ, int SPLIT, int CG, int BN>
__global__ void __launch_bounds__(kThreads, 1)
    product_kernel(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb, const Args g) {
  constexpr int TM = 128 * CG;                   // rows of a tile; 128 of them in each CTA
  constexpr int NB = BN / CG;                    // rows of B in each CTA
  constexpr int kTileA = 128 * BK * 2, kTileB = NB * BK * 2;
  constexpr int kStage = SPLIT * (kTileA + kTileB);  // A (hi, lo), B (hi, lo)
  constexpr int kStages = kRing / kStage;
  constexpr int kCols = kAcc * SPLIT * BN;       // tensor memory: accumulators of the hi (and lo) products
  static_assert(kCols <= 512 && (kCols & (kCols - 1)) == 0, "tensor memory columns");
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* staging = smem + kRing;
  uint64_t* full = reinterpret_cast<uint64_t*>(staging + kEpiWarps * kStaging);
  uint64_t* empty = full + kStages;
  uint64_t* acc_full = empty + kStages;
  uint64_t* acc_empty = acc_full + kAcc;
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(acc_empty + kAcc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_at + 1);
  volatile int* consumed = abort_flag + 1;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = CG == 2 ? (int)(blockIdx.x & 1) : 0;  // in the pair
  const int first = blockIdx.x / CG, step = gridDim.x / CG;
  const int kblocks = (g.K + BK - 1) / BK;
  const int run = SPLIT == 2 ? kRunBlocks : kblocks;  // K slices per accumulator
  const int ntm = (g.M + TM - 1) / TM, ntn = (g.N + BN - 1) / BN;
  const int ntiles = (g.symmetric ? TM / BN * (ntm * (ntm + 1) / 2) : ntm * ntn) * g.batch;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < kAcc; ++a) {
      mbar_init(&acc_full[a], 1);
      mbar_init(&acc_empty[a], CG * kEpiWarps);
    }
    *abort_flag = 0;
    *consumed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&ta)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tb)) : "memory");
  }
  if (warp == 1) {
    if (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_at)),
                   "r"(kCols));
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_at)),
                   "r"(kCols));
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync();  // both CTAs' barriers are ready
  tc_fence_after();
  const uint32_t tmem = *tmem_at;
  // what is above overlaps the end of the launch before; its results are read and its operands
  // written over only from here on
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  if (warp == 0) {
    if (lane == 0) {
      int it = 0;
      for (int t = first; t < ntiles && !*abort_flag; t += step) {
        int m0, n0, b;
        tile_at<TM, BN>(t, g.symmetric, ntm, ntn, m0, n0, b);
        for (int kb = 0; kb < kblocks; ++kb, ++it) {
          const int s = it % kStages;
          if (!mbar_wait(&empty[s], ((it / kStages) & 1) ^ 1, kWaitNs) || *abort_flag) {
            *abort_flag = 1;
            break;
          }
          if (rank == 0) expect_tx(&full[s], CG * kStage);
          const uint32_t bar = CG == 2 ? in_leader(&full[s]) : smem_u32(&full[s]);
          const uint32_t st = smem_u32(smem + s * kStage);
#pragma unroll
          for (int h = 0; h < SPLIT; ++h) {
            load_tile<AM, 128, CG>(st + h * kTileA, &ta, bar, m0 + rank * 128, kb * BK, b + h * g.batch);
            load_tile<BMJ, NB, CG>(st + SPLIT * kTileA + h * kTileB, &tb, bar, n0 + rank * NB, kb * BK,
                                   b + h * g.batch);
          }
        }
      }
      // every slice consumed, and its release arrived here, before this CTA's barriers go away
      for (int i = max(0, it - kStages); i < it && !*abort_flag; ++i)
        if (!mbar_wait(&empty[i % kStages], (i / kStages) & 1, kWaitNs)) *abort_flag = 1;
      if (*abort_flag) {
        // copies in flight land before the shared memory goes away: those of the slices not yet
        // consumed, whose barriers only the pair's first CTA holds, within a bound far above a copy's time
        if (rank == 0)
          for (int i = *consumed; i < it; ++i) mbar_wait(&full[i % kStages], (i / kStages) & 1, 10000000ull);
        const uint64_t t0 = globaltimer();
        while (globaltimer() - t0 < 10000000ull) {
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc = idesc_f16(TM, BN, AM, BMJ);
      int it = 0, n = 0;
      for (int t = first; t < ntiles && !*abort_flag; t += step) {
        for (int k0 = 0; k0 < kblocks && !*abort_flag; k0 += run, ++n) {
          const int a = n % kAcc;
          if (n >= kAcc && !mbar_wait(&acc_empty[a], ((n / kAcc) & 1) ^ 1, kWaitNs)) {
            *abort_flag = 1;
            break;
          }
          tc_fence_after();
          const uint32_t d = tmem + static_cast<uint32_t>(a * SPLIT * BN);
          const int k1 = min(kblocks, k0 + run);
          for (int kb = k0; kb < k1; ++kb, ++it) {
            const int s = it % kStages;
            if (!mbar_wait(&full[s], (it / kStages) & 1, kWaitNs) || *abort_flag) {
              *abort_flag = 1;
              break;
            }
            *consumed = it + 1;
            tc_fence_after();
            const uint32_t as = smem_u32(smem + s * kStage), bs = as + SPLIT * kTileA;
#pragma unroll
            for (int kk = 0; kk < BK / 16; ++kk) {
              const uint32_t more = kb > k0 || kk > 0;
              umma_f16<CG>(d, tile_desc<AM>(as, kk), tile_desc<BMJ>(bs, kk), idesc, more);
              if (SPLIT == 2) {
                umma_f16<CG>(d + BN, tile_desc<AM>(as + kTileA, kk), tile_desc<BMJ>(bs, kk), idesc, more);
                umma_f16<CG>(d + BN, tile_desc<AM>(as, kk), tile_desc<BMJ>(bs + kTileB, kk), idesc, 1);
              }
            }
            commit<CG>(&empty[s]);
          }
          if (!*abort_flag) commit<CG>(&acc_full[a]);
        }
      }
    }
  } else {
    const int q = warp & 3;  // accumulator lanes 32 q .. 32 q + 31
    uint8_t* stage = staging + (warp - 2) * kStaging;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(32 * q) << 16);
    int n = 0;
    auto wait_acc = [&](int a) {
      const bool ok = mbar_wait(&acc_full[a], (n / kAcc) & 1, kWaitNs) && !*abort_flag;
      if (!ok) {
        if (lane == 0 && g.status) atomicOr(g.status, kStatusTimeout);
        *abort_flag = 1;
      }
      tc_fence_after();
      return __all_sync(0xffffffffu, ok);
    };
    auto release_acc = [&](int a) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        const uint32_t bar = CG == 2 ? in_leader(&acc_empty[a]) : smem_u32(&acc_empty[a]);
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
      }
    };
    for (int t = first; t < ntiles; t += step) {
      int m0, n0, b;
      tile_at<TM, BN>(t, g.symmetric, ntm, ntn, m0, n0, b);
      const int r0 = m0 + rank * 128 + 32 * q, r = r0 + lane;
      const int rows = min(32, g.M - r0);
      const bool mirror = g.symmetric && n0 + BN <= m0;
      float f = 1.f;
      if (g.t_pow > 0) {
        f = g.t[b];
        if (g.t_pow > 1) f *= f;
      }
      const float alpha = g.alpha * f, beta = g.beta * f;
      const bool has_c = g.cin && r < g.M;
      const __half* src = g.cin + (int64_t)b * g.cin_stride + (int64_t)r * g.cin_ld + n0;
      if constexpr (SPLIT == 1) {
        const int a = n % kAcc;
        Cin<1> c_now, c_next;
        if (has_c) load_cin<1>(c_now, src, 0, g.N - n0);
        if (!wait_acc(a)) break;
        for (int c = 0; c < BN / 32; ++c) {
          const int cols = min(32, g.N - n0 - 32 * c);
          if (cols <= 0) break;
          if (has_c && c + 1 < BN / 32) load_cin<1>(c_next, src + 32 * (c + 1), 0, g.N - n0 - 32 * (c + 1));
          float o[32];
          __syncwarp();
          tmem_ld32(lanes + static_cast<uint32_t>(a * BN + 32 * c), o);
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] *= alpha;
          if (has_c) add_cin<1>(c_now, beta, cols, o);
          if (rows > 0) store_block<1>(g, stage, o, b, r0, n0 + 32 * c, rows, cols, mirror, lane);
          c_now = c_next;
        }
        release_acc(a);
        ++n;
      } else {
        float sum[BN / 32][32];
        bool ok = true;
        for (int k0 = 0; k0 < kblocks; k0 += run, ++n) {
          const int a = n % kAcc;
          if (!(ok = wait_acc(a))) break;
#pragma unroll
          for (int c = 0; c < BN / 32; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float o[32];
              tmem_ld32(lanes + static_cast<uint32_t>((a * 2 + (h ^ 1)) * BN + 32 * c), o);
#pragma unroll
              for (int j = 0; j < 32; ++j) sum[c][j] = k0 == 0 && h == 0 ? o[j] : sum[c][j] + o[j];
            }
          release_acc(a);
        }
        if (!ok) break;
#pragma unroll
        for (int c = 0; c < BN / 32; ++c) {
          const int cols = min(32, g.N - n0 - 32 * c);
          if (cols > 0 && rows > 0) {
            Cin<2> cin;
            if (has_c) load_cin<2>(cin, src + 32 * c, g.cin_lo, cols);
#pragma unroll
            for (int j = 0; j < 32; ++j) sum[c][j] *= alpha;
            if (has_c) add_cin<2>(cin, beta, cols, sum[c]);
            __syncwarp();
            store_block<2>(g, stage, sum[c], b, r0, n0 + 32 * c, rows, cols, mirror, lane);
          }
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync();  // neither CTA leaves while the other may still reach its shared memory
  if (warp == 1) {
    tc_fence_after();
    if (CG == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols));
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols));
  }
}

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  });
  return fn;
}

template <int AM, int BMJ, int SPLIT, int CG, int BN>
cudaError_t launch(const Mat& a, const Mat& b, const Args& g, int64_t tiles, int dev, int sms, cudaStream_t s) {
  static std::atomic<uint64_t> attr_set{0};  // one bit per device that has the shared-memory attribute
  const auto kernel = product_kernel<AM, BMJ, SPLIT, CG, BN>;
  const uint64_t bit = (dev >= 0 && dev < 64) ? uint64_t(1) << dev : 0;
  if (bit == 0 || !(attr_set.load(std::memory_order_relaxed) & bit)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    attr_set.fetch_or(bit, std::memory_order_relaxed);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(CG * std::min<int64_t>(tiles, sms / CG)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CG;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, a.map, b.map, g);
}

int64_t tile_count(const Args& g, int tm, int tn) {
  const int64_t ntm = (g.M + tm - 1) / tm, ntn = (g.N + tn - 1) / tn;
  return (g.symmetric ? tm / tn * (ntm * (ntm + 1) / 2) : ntm * ntn) * g.batch;
}

// Tile shape by the time of its waves: a 256 x 256 pair tile takes 128 cycles per 16 K elements at
// the tensor cores' rate, a 256 x 128 one 64 and somewhat more for its operand traffic, a single
// CTA's 128 x 128 tile 64 and half as much again.
template <int AM, int BMJ, int SPLIT>
cudaError_t launch_best(const Mat& a, const Mat& b, const Args& g, cudaStream_t s) {
  int dev = 0, sms = 152;
  if (cudaGetDevice(&dev) != cudaSuccess) dev = 0;
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const int64_t t256 = tile_count(g, 256, 256), t128 = tile_count(g, 256, 128), t1 = tile_count(g, 128, 128);
  if (std::max(t1, t128) > (int64_t(1) << 30)) return cudaErrorInvalidValue;
  const int64_t pairs = std::max(1, sms / 2);
  const int64_t c256 = (t256 + pairs - 1) / pairs * 128, c128 = (t128 + pairs - 1) / pairs * 75;
  const int64_t c1 = (t1 + sms - 1) / sms * 100;
  if (SPLIT == 1 && c256 <= c128 && c256 <= c1) return launch<AM, BMJ, SPLIT, 2, SPLIT == 1 ? 256 : 128>(a, b, g, t256, dev, sms, s);
  if (c128 <= c1) return launch<AM, BMJ, SPLIT, 2, 128>(a, b, g, t128, dev, sms, s);
  return launch<AM, BMJ, SPLIT, 1, 128>(a, b, g, t1, dev, sms, s);
}

}  // namespace

bool make_map(Mat& m, int planes) {
  auto fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows, (cuuint64_t)planes};
  cuuint64_t strides[2] = {(cuuint64_t)m.ld * 2, (cuuint64_t)m.stride * 2};
  cuuint32_t box[3] = {64, 64, 1};
  cuuint32_t es[3] = {1, 1, 1};
  return fn(&m.map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, m.p, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t product(const Product& p, const Mat& a, const Mat& b, cudaStream_t s) {
  Args g{};
  g.M = p.M;
  g.N = p.N;
  g.K = p.K;
  g.batch = p.batch;
  g.symmetric = p.symmetric;
  g.alpha = p.alpha;
  g.beta = p.beta;
  if (p.cin) {
    g.cin = p.cin->p;
    g.cin_ld = p.cin->ld;
    g.cin_stride = p.cin->stride;
    g.cin_lo = p.cin->stride * p.batch;
  }
  g.t = p.t;
  g.t_pow = p.t_pow;
  if (p.out) {
    g.out = p.out->p;
    g.ld = p.out->ld;
    g.stride = p.out->stride;
    g.lo = p.out->stride * p.batch;
  } else {
    const size_t size = dtype_size(p.user_type);
    g.user = p.user;
    g.user_type = p.user_type;
    g.user_ld = p.user_ld;
    g.user_stride = p.user_stride;
    g.user_vec = reinterpret_cast<uintptr_t>(p.user) % 16 == 0 && (p.user_ld * size) % 16 == 0 &&
                 (p.batch == 1 || (p.user_stride * size) % 16 == 0) && (p.N * size) % 16 == 0;
  }
  g.status = p.status;
  const double half = p.symmetric ? 0.5 : 1.0;
  const double mn = (double)p.M * p.N * p.batch;
  ProfScope prof(kFamGemmTc, 2.0 * half * mn * p.K,
                 2.0 * (p.split ? 2 : 1) * ((double)(p.M + (p.symmetric ? 0 : p.N)) * p.K * p.batch + mn), s);
  if (p.a_major == kRowsK && p.b_major == kRowsK)
    return p.split ? launch_best<kRowsK, kRowsK, 2>(a, b, g, s) : launch_best<kRowsK, kRowsK, 1>(a, b, g, s);
  if (p.a_major == kRowsK)
    return p.split ? launch_best<kRowsK, kRowsM, 2>(a, b, g, s) : launch_best<kRowsK, kRowsM, 1>(a, b, g, s);
  if (p.b_major == kRowsM)
    return p.split ? launch_best<kRowsM, kRowsM, 2>(a, b, g, s) : launch_best<kRowsM, kRowsM, 1>(a, b, g, s);
  return cudaErrorInvalidValue;
}

}  // namespace ortho
}  // namespace soap
