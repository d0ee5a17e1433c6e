// The Newton-Schulz steps of the stand-alone orthogonalisation (muon_orthogonalize) on the
// 5th-generation tensor cores: per step S = X X^T, B = b S + c S^2, X' = a X + B X (X^T X and X B
// for tall matrices) on fp16 operands (kind::f16) with fp32 accumulation, all steps of all matrices
// in one launch.
//
// Operands are read as they lie: a row-major matrix serves as A or B with K along its rows
// (K-major) or down its columns (MN-major), so no transposed copy exists. S and B are symmetric:
// only their 256 x 256 tiles on and below the diagonal are computed and stored, and an operand tile
// above the diagonal is read from the one below it, the other way round.
//
// Split operands (x = hi + lo, 22 bits) take three products, hi hi, lo hi and hi lo, from one load
// of the four tiles. The accumulator truncates: measured, a sum loses 2^-25 of itself per 16
// products. With 11-bit operands that is nothing; split ones keep the small products in an
// accumulator of their own and take K in runs of at most 768, whose sums the epilogue adds in fp32.
//
// Schedule. Persistent CTA pairs (cta_group::2, a pair's 256 x 256 tile has 128 rows in each CTA)
// walk one list of tiles in turn: for each step all S tiles, then all B tiles, then all X' tiles. A
// tile waits until its matrix's tiles of the phase before are stored, which a counter per matrix
// tells; such a wait always points to tiles earlier in the list, so with all pairs resident (a
// cooperative launch) it ends. Against a launch per product (measured at 64 matrices of 768 x 2048:
// 337 us a step) this has no partly filled last wave per product and no launch latency.
//
// In a CTA, warp 0 issues TMA loads of 64-element K slices into a ring, warp 1 (of the pair's first
// CTA) the MMAs, and eight epilogue warps drain the accumulator, 32 x 64 elements at a time: C comes
// in and the result leaves by TMA through shared memory, and a tile is reported stored while the
// next one's C is on its way (plain stores and a fence per tile took 7 us of a tile's epilogue, more
// than the MMAs of a tile with K = 768). An MMA that adds to the accumulator of the one before it
// takes 140 cycles however narrow (measured), so tiles are 256 wide; the issuing thread has little
// time beside it, so its loops are compiled for each pair of operand orders (with orders chosen at
// run time a slice took 790 cycles in place of 540). Every
// wait is bounded; one that runs out sets SOAP_STATUS_TIMEOUT and the CTA drains its copies, frees
// its tensor memory and returns.
#include <cuda.h>
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
constexpr int kBox = 64 * 64 * 2;      // one TMA box: 64 rows of 128 bytes
constexpr int kTile = 2 * kBox;        // a CTA's 128 x 64 elements of an operand
constexpr int kRunBlocks = 12;         // most K slices per accumulator run of split operands
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kBlock = 32 * 128;       // a staged block: 32 rows of 128 bytes
constexpr int kPerTile = 2 * kEpiWarps;       // what a tile adds to its matrix's counter
constexpr uint64_t kWaitNs = 2000000000ull;

template <int SPLIT>
struct Config {
  static constexpr int kStage = SPLIT * 2 * kTile;  // A (hi, lo), B (hi, lo)
  static constexpr int kStages = SPLIT == 2 ? 3 : 5;
  static constexpr int kAcc = SPLIT == 2 ? 1 : 2;   // accumulators of 256 columns (split: and one of lo products)
  static constexpr int kBufs = SPLIT == 2 ? 1 : 2;  // staged blocks per epilogue warp
  static constexpr int kStaging = kBufs * kBlock;
  static constexpr int kSmem = 1024 + kStages * kStage + kEpiWarps * kStaging + 512;
};

struct Maps {
  CUtensorMap x[2], s, b;      // boxes of 64 x 64: operands
  CUtensorMap ex[2], es, eb;   // boxes of 64 columns x 32 rows: C and results
};

// Tiles of the list. Groups of `group` matrices go through all steps one after the other.
struct Layout {
  int r, k, tall, group;
  int ns, nx, nxm, nxn;  // tiles of S (and B), of X', row and column tiles of X'
  int total;
};

struct Tile {
  int step, phase, b;     // phase 0: S, 1: B, 2: X'
  int m0, n0, M, N, K;
  int need;               // the matrix's counter before this tile may start
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

// Both CTAs' copies count on the barrier of the pair's first one (`bar`, a shared::cluster address).
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}

// 128 x 64 elements of an operand at (row m0, k0) as boxes of 64: rows of 64 K elements each
// (K-major), or 64 K rows of 64 columns (MN-major).
template <int MN>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int m0, int k0, int z) {
  tma_box(dst, map, bar, MN ? m0 : k0, MN ? k0 : m0, z);
  tma_box(dst + kBox, map, bar, MN ? m0 + 64 : k0, MN ? k0 : m0 + 64, z);
}

// Descriptor of the 16 K elements at step kk of such a tile. K-major: 32 bytes further along the
// swizzled rows, 8-row groups 1024 B apart. MN-major: 16 rows further down, 8-row K groups 1024 B
// apart, the next 64 columns one box away.
template <int MN>
__device__ __forceinline__ uint64_t tile_desc(uint32_t base, int kk) {
  const uint32_t addr = base + (MN ? kk * 16 * 128 : kk * 32);
  uint64_t d = 0;
  d |= static_cast<uint64_t>((addr & 0x3FFFF) >> 4);
  d |= static_cast<uint64_t>((MN ? kBox : 16) >> 4) << 16;  // leading byte offset
  d |= static_cast<uint64_t>(1024 >> 4) << 32;              // stride byte offset
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;  // 128-byte swizzle
  return d;
}

// kind::f16, M = N = 256: D = f32, A = B = f16; bits 15 and 16 mark MN-major operands.
__host__ __device__ constexpr uint32_t idesc_f16(int a_mn, int b_mn) {
  return (1u << 4) | (static_cast<uint32_t>(a_mn) << 15) | (static_cast<uint32_t>(b_mn) << 16) | ((256u >> 3) << 17) |
         ((256u >> 4) << 24);
}

__device__ __forceinline__ void umma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate));
}

// Arrives on both CTAs' barriers at `bar`'s place when the MMAs so far are done.
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
          smem_u32(bar)),
      "h"((uint16_t)3)
      : "memory");
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&v)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

__device__ __forceinline__ int load_acquire(const int* p) {
  int v;
  asm volatile("ld.acquire.gpu.global.b32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}

// Bounded wait for a matrix's counter.
__device__ __forceinline__ bool wait_done(const int* done, int need) {
  if (load_acquire(done) >= need) return true;
  const uint64_t t0 = globaltimer();
  for (;;) {
    for (int i = 0; i < 64; ++i)
      if (load_acquire(done) >= need) return true;
    if (globaltimer() - t0 > kWaitNs) return false;
  }
}

// Step and phase of list entry p; i: its place among its group's tiles of that phase.
__device__ __forceinline__ void phase_at(uint32_t p, const Layout& l, const Steps& a, int& group, int& step, int& phase,
                                         uint32_t& i) {
  const uint32_t per = 2 * l.ns + l.nx;  // of a matrix in a step
  uint32_t n = a.batch, w = p;
  group = 0;
  if (l.group < a.batch) {
    const uint32_t per_group = l.group * a.steps * per;
    group = p / per_group;
    w = p - group * per_group;
    n = min(l.group, a.batch - group * l.group);  // the group's matrices
  }
  step = w / (n * per);
  i = w - step * n * per;
  const uint32_t ns = n * l.ns;
  phase = i >= 2 * ns ? 2 : i >= ns ? 1 : 0;
  i -= phase * ns;
}

__device__ __forceinline__ Tile tile_at(uint32_t p, const Layout& l, const Steps& a) {
  Tile t;
  int g;
  uint32_t i;
  phase_at(p, l, a, g, t.step, t.phase, i);
  t.need = (t.step * (2 * l.ns + l.nx) + t.phase * l.ns) * kPerTile;
  const uint32_t each = t.phase == 2 ? l.nx : l.ns;
  const uint32_t b = i / each;
  i -= b * each;
  t.b = b + g * l.group;
  if (t.phase < 2) {  // row by row of the triangle
    t.M = t.N = l.r;
    t.K = t.phase == 0 ? l.k : l.r;
    uint32_t row = (uint32_t)((sqrtf(8.f * (float)i + 1.f) - 1.f) * 0.5f);
    while (row * (row + 1) / 2 > i) --row;
    while ((row + 1) * (row + 2) / 2 <= i) ++row;
    t.m0 = row * 256;
    t.n0 = (i - row * (row + 1) / 2) * 256;
  } else {  // in groups of 8 row tiles, row tile fastest, so that tiles in flight share operands in L2
    t.M = a.rows;
    t.N = a.cols;
    t.K = l.r;
    const uint32_t of8 = 8 * l.nxn;
    const uint32_t gr = i / of8, in = i - gr * of8;
    const uint32_t rows = min(8, l.nxm - (int)gr * 8);
    const uint32_t col = in / rows;
    t.m0 = (gr * 8 + in - col * rows) * 256;
    t.n0 = col * 256;
  }
  return t;
}

// Where along K (in slices) the operands' order changes. An operand that is a row tile of a
// symmetric matrix is K-major up to the end of its diagonal tile and MN-major, from the mirrored
// tiles, beyond it. a, b: slices before the change of A and B.
__device__ __forceinline__ void order_change(const Tile& t, int tall, int kblocks, int& a, int& b) {
  const int ia = min(kblocks, (t.m0 / 256 + 1) * 4), ib = min(kblocks, (t.n0 / 256 + 1) * 4);
  if (t.phase == 0) {  // X X^T along the rows; X^T X down the columns
    a = b = tall ? 0 : kblocks;
  } else if (t.phase == 1) {  // S S
    a = ia;
    b = ib;
  } else {  // B X, X down its columns; tall: X B
    a = tall ? kblocks : ia;
    b = tall ? ib : 0;
  }
}

// Place of row j's 16-byte chunk c in a staged block of rows of 64 bytes (16-bit elements) or 128
// (fp32): permuted so that neither rows nor columns of chunks meet in a bank.
__device__ __forceinline__ int at16(int j, int c) { return j * 64 + ((c ^ ((j >> 1) & 3)) * 16); }
__device__ __forceinline__ int at32(int j, int c) { return j * 128 + ((c ^ (j & 7)) * 16); }

// A 64-column x 32-row block between global memory and a staging buffer (128-byte swizzle).
__device__ __forceinline__ void fetch_block(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z) {
  expect_tx(bar, kBlock);
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ void send_block(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(src), "r"(x), "r"(y), "r"(z)
               : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// The sent blocks' buffers have been read / the blocks are in global memory.
__device__ __forceinline__ void sent_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void sent_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// This thread's plain accesses to shared memory come before later TMA accesses to it.
__device__ __forceinline__ void before_tma() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// v += beta * this lane's row of a staged block, columns 32 h .. 32 h + 31.
__device__ __forceinline__ void add_row(const uint8_t* stage, int h, float beta, float (&v)[32], int lane) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const uint4 w = *reinterpret_cast<const uint4*>(stage + at32(lane, 4 * h + u));
    const __half2* q = reinterpret_cast<const __half2*>(&w);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = __half22float2(q[e]);
      v[u * 8 + 2 * e] = fmaf(beta, f.x, v[u * 8 + 2 * e]);
      v[u * 8 + 2 * e + 1] = fmaf(beta, f.y, v[u * 8 + 2 * e + 1]);
    }
  }
}

// Rounds v to fp16 into this lane's row of a staged block; with REST, v keeps what the rounding left.
template <bool REST>
__device__ __forceinline__ void put_row(uint8_t* stage, int h, float (&v)[32], int lane) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    uint4 w;
    __half2* q = reinterpret_cast<__half2*>(&w);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      q[e] = __floats2half2_rn(v[u * 8 + 2 * e], v[u * 8 + 2 * e + 1]);
      if (REST) {
        const float2 f = __half22float2(q[e]);
        v[u * 8 + 2 * e] -= f.x;
        v[u * 8 + 2 * e + 1] -= f.y;
      }
    }
    *reinterpret_cast<uint4*>(stage + at32(lane, 4 * h + u)) = w;
  }
}

// A 32 x 32 block (this lane's row in v) to the caller's matrix, through the staging buffer.
template <typename T>
__device__ __forceinline__ void store_user(uint8_t* stage, const float (&v)[32], T* dst, int64_t ld, int rows,
                                           int cols, bool vec, int lane) {
  auto place = [](int j, int c) { return sizeof(T) == 4 ? at32(j, c) : at16(j, c); };
  constexpr int V = 16 / sizeof(T), L = 32 / V;  // elements per access, accesses per row
#pragma unroll
  for (int u = 0; u < L; ++u) {
    Pack<T, V> p;
#pragma unroll
    for (int e = 0; e < V; ++e) p.v[e] = from_f32<T>(v[u * V + e]);
    *reinterpret_cast<Pack<T, V>*>(stage + place(lane, u)) = p;
  }
  __syncwarp();
  if (vec) {
#pragma unroll
    for (int u = 0; u < L; ++u) {
      const int j = u * (32 / L) + lane / L, c = lane % L;
      if (j < rows && c * V < cols)
        *reinterpret_cast<Pack<T, V>*>(dst + (int64_t)j * ld + c * V) =
            *reinterpret_cast<const Pack<T, V>*>(stage + place(j, c));
    }
  } else {
    for (int j = 0; j < rows; ++j)
      if (lane < cols)
        dst[(int64_t)j * ld + lane] =
            *reinterpret_cast<const T*>(stage + place(j, lane / V) + (lane % V) * sizeof(T));
  }
  __syncwarp();
}

__device__ __forceinline__ void store_user_any(uint8_t* stage, const float (&v)[32], const Steps& a, bool vec, int b,
                                               int r0, int c0, int rows, int cols, int lane) {
  const int64_t at = (int64_t)b * a.stride_out + (int64_t)r0 * a.ld_out + c0;
  if (a.out_type == SOAP_F32)
    store_user(stage, v, static_cast<float*>(a.out) + at, a.ld_out, rows, cols, vec, lane);
  else if (a.out_type == SOAP_BF16)
    store_user(stage, v, static_cast<__nv_bfloat16*>(a.out) + at, a.ld_out, rows, cols, vec, lane);
  else
    store_user(stage, v, static_cast<__half*>(a.out) + at, a.ld_out, rows, cols, vec, lane);
}

// A thread's place in the ring: the slot and the parity it waits for.
struct Ring {
  int s = 0;
  uint32_t parity = 0;
  bool ok = true;
};

// K slices kb .. to - 1 of a tile into the ring: rows am of A's map and bn of B's.
template <int SPLIT, int A_MN, int B_MN>
__device__ __forceinline__ void load_slices(Ring& st, int kb, int to, const CUtensorMap* ma, const CUtensorMap* mb,
                                            int am, int bn, int b, int batch, uint32_t ring, uint64_t* full,
                                            uint64_t* empty, uint32_t leader_full, int rank) {
  using C = Config<SPLIT>;
  for (; kb < to; ++kb) {
    if (!(st.ok = mbar_wait(&empty[st.s], st.parity, kWaitNs))) return;
    if (rank == 0) expect_tx(&full[st.s], 2 * C::kStage);
    const uint32_t at = ring + st.s * C::kStage, bar = leader_full + st.s * 8;
#pragma unroll
    for (int h = 0; h < SPLIT; ++h) {
      load_tile<A_MN>(at + h * kTile, ma, bar, am, kb * BK, b + h * batch);
      load_tile<B_MN>(at + (SPLIT + h) * kTile, mb, bar, bn, kb * BK, b + h * batch);
    }
    if (++st.s == C::kStages) {
      st.s = 0;
      st.parity ^= 1;
    }
  }
}

// `count` K slices from the ring into the accumulator at d (split: the small products at d + 256).
template <int SPLIT, int A_MN, int B_MN>
__device__ __forceinline__ void issue_slices(Ring& st, int count, uint32_t& more, uint32_t ring, uint64_t* full,
                                             uint64_t* empty, uint32_t d) {
  using C = Config<SPLIT>;
  constexpr uint32_t idesc = idesc_f16(A_MN, B_MN);
  for (; count > 0; --count) {
    if (!(st.ok = mbar_wait(&full[st.s], st.parity, kWaitNs))) return;
    tc_fence_after();
    const uint32_t as = ring + st.s * C::kStage, bs = as + SPLIT * kTile;
#pragma unroll
    for (int kk = 0; kk < BK / 16; ++kk) {
      umma_f16(d, tile_desc<A_MN>(as, kk), tile_desc<B_MN>(bs, kk), idesc, more);
      if (SPLIT == 2) {
        umma_f16(d + 256, tile_desc<A_MN>(as + kTile, kk), tile_desc<B_MN>(bs, kk), idesc, more);
        umma_f16(d + 256, tile_desc<A_MN>(as, kk), tile_desc<B_MN>(bs + kTile, kk), idesc, 1);
      }
      more = 1;
    }
    commit_pair(&empty[st.s]);
    if (++st.s == C::kStages) {
      st.s = 0;
      st.parity ^= 1;
    }
  }
}

template <int SPLIT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    steps_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Steps a, const Layout l, const int out_vec) {
  using C = Config<SPLIT>;
  constexpr int kStages = C::kStages, kAcc = C::kAcc;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* staging = smem + kStages * C::kStage;
  uint64_t* full = reinterpret_cast<uint64_t*>(staging + kEpiWarps * C::kStaging);
  uint64_t* empty = full + kStages;
  uint64_t* acc_full = empty + kStages;
  uint64_t* acc_empty = acc_full + kAcc;
  uint64_t* cin_full = acc_empty + kAcc;
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(cin_full + kEpiWarps * C::kBufs);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_at + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)(blockIdx.x & 1);  // in the pair
  const int first = blockIdx.x / 2, stride = gridDim.x / 2;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int i = 0; i < kAcc; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], 2 * kEpiWarps);
    }
    for (int i = 0; i < kEpiWarps * C::kBufs; ++i) mbar_init(&cin_full[i], 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_at)), "r"(512));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // both CTAs' barriers are ready
  tc_fence_after();
  const uint32_t tmem = *tmem_at;

  if (warp == 0) {
    if (lane == 0) {
      Ring st;
      st.parity = 1;  // of a slot's release
      int used = 0;   // slots filled so far (up to kStages)
      const uint32_t ring = smem_u32(smem), bars = in_leader(full);
      for (int p = first; p < l.total && st.ok && !*abort_flag; p += stride) {
        const Tile t = tile_at(p, l, a);
        const int kblocks = (t.K + BK - 1) / BK;
        int a_change, b_change;
        order_change(t, l.tall, kblocks, a_change, b_change);
        const CUtensorMap* x = &maps.x[t.step & 1];
        const CUtensorMap* ma = t.phase == 0 ? x : t.phase == 1 ? &maps.s : l.tall ? x : &maps.b;
        const CUtensorMap* mb = t.phase == 0 ? x : t.phase == 1 ? &maps.s : l.tall ? &maps.b : x;
        if (!(st.ok = wait_done(a.done + t.b, t.need))) break;
        asm volatile("fence.proxy.async;" ::: "memory");  // what other CTAs stored, before copies of it
        const int am = t.m0 + rank * 128, bn = t.n0 + rank * 128;
        used = min(used + kblocks, kStages);
        for (int kb = 0; kb < kblocks && st.ok;) {  // stretches of slices of one order
          const bool a_mn = kb >= a_change, b_mn = kb >= b_change;
          const int to = min(a_mn ? kblocks : a_change, b_mn ? kblocks : b_change);
          if (a_mn && b_mn)
            load_slices<SPLIT, 1, 1>(st, kb, to, ma, mb, am, bn, t.b, a.batch, ring, full, empty, bars, rank);
          else if (a_mn)
            load_slices<SPLIT, 1, 0>(st, kb, to, ma, mb, am, bn, t.b, a.batch, ring, full, empty, bars, rank);
          else if (b_mn)
            load_slices<SPLIT, 0, 1>(st, kb, to, ma, mb, am, bn, t.b, a.batch, ring, full, empty, bars, rank);
          else
            load_slices<SPLIT, 0, 0>(st, kb, to, ma, mb, am, bn, t.b, a.batch, ring, full, empty, bars, rank);
          kb = to;
        }
      }
      // every slice consumed, and its release arrived here, before this CTA's barriers go away
      for (int i = 0; i < kStages && st.ok && !*abort_flag; ++i) {
        if (used == kStages || st.s - 1 - i >= 0) {
          const int slot = (st.s - 1 - i + kStages) % kStages;
          st.ok = mbar_wait(&empty[slot], slot < st.s ? st.parity ^ 1 : st.parity, kWaitNs);
        }
      }
      if (!st.ok || *abort_flag) {
        *abort_flag = 1;
        if (a.status) atomicOr(a.status, kStatusTimeout);
        // copies in flight land before the shared memory goes away: far above a copy's time
        const uint64_t t0 = globaltimer();
        while (globaltimer() - t0 < 10000000ull) {
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      Ring st;
      int n = 0;
      const uint32_t ring = smem_u32(smem);
      for (int p = first; p < l.total && st.ok && !*abort_flag; p += stride) {
        const Tile t = tile_at(p, l, a);
        const int kblocks = (t.K + BK - 1) / BK;
        int a_change, b_change;
        order_change(t, l.tall, kblocks, a_change, b_change);
        const int runs = SPLIT == 2 ? (kblocks + kRunBlocks - 1) / kRunBlocks : 1;
        for (int run = 0; run < runs && st.ok; ++run, ++n) {
          const int ac = n % kAcc;
          if (n >= kAcc && !(st.ok = mbar_wait(&acc_empty[ac], ((n / kAcc) & 1) ^ 1, kWaitNs))) break;
          tc_fence_after();
          const uint32_t d = tmem + static_cast<uint32_t>(ac * 256);
          const int k1 = SPLIT == 2 ? kblocks * (run + 1) / runs : kblocks;
          int kb = SPLIT == 2 ? kblocks * run / runs : 0;
          uint32_t more = 0;
          while (kb < k1 && st.ok) {  // stretches of slices of one order
            const bool a_mn = kb >= a_change, b_mn = kb >= b_change;
            const int to = min(k1, min(a_mn ? k1 : a_change, b_mn ? k1 : b_change));
            if (a_mn && b_mn)
              issue_slices<SPLIT, 1, 1>(st, to - kb, more, ring, full, empty, d);
            else if (a_mn)
              issue_slices<SPLIT, 1, 0>(st, to - kb, more, ring, full, empty, d);
            else if (b_mn)
              issue_slices<SPLIT, 0, 1>(st, to - kb, more, ring, full, empty, d);
            else
              issue_slices<SPLIT, 0, 0>(st, to - kb, more, ring, full, empty, d);
            kb = to;
          }
          if (st.ok) commit_pair(&acc_full[ac]);
        }
      }
      if (!st.ok) *abort_flag = 1;
    }
  } else {
    const int q = warp & 3;            // accumulator lanes 32 q .. 32 q + 31
    const int half = (warp - 2) / 4;   // columns 128 half .. 128 half + 127
    uint8_t* stage = staging + (warp - 2) * C::kStaging;
    const uint32_t stage_at = smem_u32(stage);
    uint64_t* cin_bar = cin_full + (warp - 2) * C::kBufs;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(32 * q) << 16) + 128 * half;
    int n = 0;
    uint32_t cin_parity[2] = {0, 0};
    int* unreported = nullptr;  // counter of the matrix whose tile this warp has sent but not reported
    auto wait_acc = [&](int ac) {
      const bool ok = mbar_wait(&acc_full[ac], (n / kAcc) & 1, kWaitNs) && !*abort_flag;
      tc_fence_after();
      return __all_sync(0xffffffffu, ok);
    };
    auto release_acc = [&](int ac) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0)
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_leader(&acc_empty[ac]))
                     : "memory");
    };
    auto report = [&]() {
      if (unreported && lane == 0) {
        sent_done();
        asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(unreported) : "memory");
      }
      unreported = nullptr;
    };
    bool ok = true;
    for (int p = first; p < l.total && ok; p += stride) {
      const Tile t = tile_at(p, l, a);
      const int r0 = t.m0 + rank * 128 + 32 * q, n0 = t.n0 + 128 * half;
      const int rows = min(32, t.M - r0);
      // this warp's 32 x 64 blocks: none below the last row, and to the last column
      const int blocks = rows > 0 && n0 < t.N ? min(2, (t.N - n0 + 63) / 64) : 0;
      const bool last = t.phase == 2 && t.step + 1 == a.steps;
      const StepCoef& c = a.coef[t.step];
      float alpha = t.phase == 0 ? c.s_alpha : t.phase == 1 ? c.b_alpha : c.x_alpha;
      float beta = t.phase == 1 ? c.b_beta : c.x_beta;
      if (t.step == 0 && t.phase != 1) {
        const float f = a.t[t.b];
        alpha *= t.phase == 0 ? f * f : f;
        beta *= f;
      }
      const bool has_c = t.phase > 0 && blocks > 0;
      const CUtensorMap* cin = t.phase == 1 ? &maps.es : &maps.ex[t.step & 1];
      const CUtensorMap* out = t.phase == 0 ? &maps.es : t.phase == 1 ? &maps.eb : &maps.ex[(t.step & 1) ^ 1];
      // C is what other CTAs stored; what this tile writes over has been read. A tile that has to wait
      // may wait for this warp's own last one: that is reported first.
      int* done = a.done + t.b;
      if (lane == 0) ok = load_acquire(done) >= t.need;
      if (!__shfl_sync(0xffffffffu, ok, 0)) {
        report();
        if (lane == 0) ok = wait_done(done, t.need);
        if (!(ok = __shfl_sync(0xffffffffu, ok, 0))) break;
      }
      ok = true;
      auto fetch = [&](int i, int h) {  // block i's part h of C into buffer i % kBufs
        if (lane == 0)
          fetch_block(stage_at + (i % C::kBufs) * kBlock, cin, &cin_bar[i % C::kBufs], n0 + 64 * i, r0,
                      t.b + h * a.batch);
      };
      auto fetched = [&](int i) {
        const int k = i % C::kBufs;
        ok = mbar_wait(&cin_bar[k], cin_parity[k], kWaitNs);
        cin_parity[k] ^= 1;
        ok = __all_sync(0xffffffffu, ok);
      };
      auto send = [&](int i, int h) {
        before_tma();
        __syncwarp();
        if (lane == 0) send_block(out, stage_at + (i % C::kBufs) * kBlock, n0 + 64 * i, r0, t.b + h * a.batch);
      };
      auto to_user = [&](uint8_t* st, int i, int h, const float (&v)[32]) {
        const int c0 = n0 + 64 * i + 32 * h;
        if (c0 < t.N) store_user_any(st, v, a, out_vec, t.b, r0, c0, rows, min(32, t.N - c0), lane);
      };
      if (has_c) {
        asm volatile("fence.proxy.async;" ::: "memory");
        if (SPLIT == 1)
          for (int i = 0; i < blocks; ++i) fetch(i, 0);
        else
          fetch(0, 1);
      }
      report();
      if constexpr (SPLIT == 1) {
        const int ac = n % kAcc;
        if (!(ok = wait_acc(ac))) break;
        if (blocks == 0) release_acc(ac);
        for (int i = 0; i < blocks && ok; ++i) {
          uint8_t* st = stage + i * kBlock;
          float v[2][32];
          tmem_ld32(lanes + static_cast<uint32_t>(ac * 256 + 64 * i), v[0]);
          tmem_ld32(lanes + static_cast<uint32_t>(ac * 256 + 64 * i + 32), v[1]);
          if (i + 1 == blocks) release_acc(ac);
          if (has_c) fetched(i);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[h][j] *= alpha;
            if (has_c) add_row(st, h, beta, v[h], lane);
          }
          if (last) {
            __syncwarp();
            to_user(st, i, 0, v[0]);
            to_user(st, i, 1, v[1]);
            before_tma();
          } else {
            put_row<false>(st, 0, v[0], lane);
            put_row<false>(st, 1, v[1], lane);
            send(i, 0);
          }
        }
        ++n;
      } else {
        float sum[4][32];
        const int kblocks = (t.K + BK - 1) / BK;
        const int runs = (kblocks + kRunBlocks - 1) / kRunBlocks;
        for (int i = 0; i < runs; ++i, ++n) {
          if (!(ok = wait_acc(0))) break;
#pragma unroll
          for (int b = 0; b < 8; ++b)
            if (b / 4 < blocks) {
              float hi[16], small[16];
              tmem_ld16(lanes + 16 * b, hi);
              tmem_ld16(lanes + 256 + 16 * b, small);
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                float& x = sum[b / 2][(b & 1) * 16 + j];
                x = i == 0 ? small[j] + hi[j] : x + (small[j] + hi[j]);
              }
            }
          release_acc(0);
        }
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (i < blocks && ok) {
            float(&v0)[32] = sum[2 * i];
            float(&v1)[32] = sum[2 * i + 1];
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              v0[j] *= alpha;
              v1[j] *= alpha;
            }
            if (has_c) {  // the small part first
              if (i > 0) fetch(i, 1);
              fetched(i);
              add_row(stage, 0, beta, v0, lane);
              add_row(stage, 1, beta, v1, lane);
              before_tma();
              __syncwarp();
              fetch(i, 0);
              fetched(i);
              add_row(stage, 0, beta, v0, lane);
              add_row(stage, 1, beta, v1, lane);
            }
            if (last) {
              __syncwarp();
              to_user(stage, i, 0, v0);
              to_user(stage, i, 1, v1);
              before_tma();
            } else {
              put_row<true>(stage, 0, v0, lane);
              put_row<true>(stage, 1, v1, lane);
              send(i, 0);
              if (lane == 0) sent_read();
              __syncwarp();
              put_row<false>(stage, 0, v0, lane);
              put_row<false>(stage, 1, v1, lane);
              send(i, 1);
              if (lane == 0) sent_read();
            }
            __syncwarp();
          }
      }
      if (lane == 0) sent_read();
      __syncwarp();
      unreported = done;
    }
    report();
    if (!ok) {
      *abort_flag = 1;
      if (lane == 0 && a.status) atomicOr(a.status, kStatusTimeout);
      // loads of C in flight land before the shared memory goes away: far above a copy's time
      const uint64_t t0 = globaltimer();
      while (globaltimer() - t0 < 10000000ull) {
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync();  // neither CTA leaves while the other may still reach its shared memory
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
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

// Boxes of 64 columns x box_rows, 128-byte swizzle.
bool make_map(CUtensorMap* map, __half* p, int rows, int cols, int ld, int planes, int box_rows) {
  auto fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)rows * ld * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
  cuuint32_t es[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, p, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int SPLIT>
cudaError_t launch(const Maps& maps, const Steps& p, const Layout& l, int out_vec, cudaStream_t s) {
  // per device: the most pairs that are resident at once, found (with the kernel's shared-memory
  // attribute set) on the first launch there
  static std::atomic<int> pairs_of[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(2);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Config<SPLIT>::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeCooperative;
  attr[1].val.cooperative = 1;
  cfg.attrs = attr;
  int pairs = dev >= 0 && dev < 64 ? pairs_of[dev].load(std::memory_order_relaxed) : 0;
  if (pairs == 0) {
    e = cudaFuncSetAttribute(steps_kernel<SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Config<SPLIT>::kSmem);
    if (e != cudaSuccess) return e;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&pairs, steps_kernel<SPLIT>, &cfg);
    if (e != cudaSuccess) return e;
    if (pairs < 1) return cudaErrorLaunchOutOfResources;
    if (dev >= 0 && dev < 64) pairs_of[dev].store(pairs, std::memory_order_relaxed);
  }
  // no more pairs than the longest phase has tiles
  const int64_t most = (int64_t)l.group * std::max(l.ns, l.nx);
  cfg.gridDim = dim3((unsigned)(2 * std::min<int64_t>(pairs, most)));
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, steps_kernel<SPLIT>, maps, p, l, out_vec);
}

}  // namespace

cudaError_t run_steps(const Steps& p, cudaStream_t s) {
  Layout l{};
  l.r = std::min(p.rows, p.cols);
  l.k = std::max(p.rows, p.cols);
  l.tall = p.rows > p.cols;
  const int n = (l.r + 255) / 256;
  l.ns = n * (n + 1) / 2;
  l.nxm = (p.rows + 255) / 256;
  l.nxn = (p.cols + 255) / 256;
  l.nx = l.nxm * l.nxn;
  l.group = p.batch;
  const int64_t per = 2 * (int64_t)l.ns + l.nx;
  if (per * p.batch * p.steps > INT32_MAX / kPerTile) l.group = 1;
  if (per * l.group * p.steps > INT32_MAX / kPerTile) return cudaErrorInvalidValue;
  if (per * p.batch * p.steps > INT32_MAX - 1024) return cudaErrorInvalidValue;
  l.total = (int)(per * p.batch * p.steps);

  const int planes = p.batch * (p.split ? 2 : 1);
  Maps maps;
  for (int i = 0; i < 2; ++i)
    if (!make_map(&maps.x[i], p.x[i], p.rows, p.cols, p.ld_x, planes, 64) ||
        !make_map(&maps.ex[i], p.x[i], p.rows, p.cols, p.ld_x, planes, 32))
      return cudaErrorInvalidValue;
  if (!make_map(&maps.s, p.s, l.r, l.r, p.ld_s, planes, 64) || !make_map(&maps.es, p.s, l.r, l.r, p.ld_s, planes, 32) ||
      !make_map(&maps.b, p.b, l.r, l.r, p.ld_s, planes, 64) || !make_map(&maps.eb, p.b, l.r, l.r, p.ld_s, planes, 32))
    return cudaErrorInvalidValue;
  const size_t size = dtype_size(p.out_type);
  const int out_vec = reinterpret_cast<uintptr_t>(p.out) % 16 == 0 && (p.ld_out * size) % 16 == 0 &&
                      (p.batch == 1 || (p.stride_out * size) % 16 == 0) && (p.cols * size) % 16 == 0;
  const double r = l.r, k = l.k, b = p.batch;
  ProfScope prof(kFamGemmTc, b * p.steps * (r * r * k + r * r * r + 2.0 * r * r * k),
                 b * (p.rows * (double)p.cols) * (2.0 * (p.split ? 2 : 1) + size), s);
  return p.split ? launch<2>(maps, p, l, out_vec, s) : launch<1>(maps, p, l, out_vec, s);
}

}  // namespace ortho
}  // namespace soap
