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
// accumulator of their own and take K in runs of at most 1024, whose sums the epilogue adds in fp32.
//
// Schedule. Persistent CTA pairs (cta_group::2, a pair's 256 x 256 tile has 128 rows in each CTA) take
// tiles from one list, each its next one when it begins the one before: for each step all S tiles, then
// all B tiles, then all X' tiles. (Every 76th tile for a pair, fixed in advance, takes 5% longer with 3
// matrices of 2048 x 8192, where S tiles take four times as long as others, and 13% with 5 of 777 x 1365.) A
// tile waits until its matrix's tiles of the phase before are stored, which a counter per matrix tells;
// such a wait always points to tiles earlier in the list, which are taken, so with all pairs resident (a
// cooperative launch) it ends. Against a launch per product (337 us a step at 64 matrices of 768 x 2048, here
// 237 in a row of calls under the power limit) this has no partly filled last wave per product and no launch
// latency.
//
// In a CTA, one warp takes tiles and waits for their inputs, two issue TMA loads of A's and B's 64-element K
// slices into a ring (on the diagonal of S and B, A's alone: both operands are the same rows), one (of the
// pair's first CTA) the MMAs, and eight drain the accumulator, 32 x 64 elements at a time: C comes in and
// the result leaves by TMA through shared memory, and a tile is reported stored while the next one's C is
// on its way (plain stores and a fence per tile took 7 us of a tile's epilogue, more than the MMAs of a
// tile with K = 768). An MMA that adds to the accumulator of the one before it takes 140 cycles however
// narrow (measured), so tiles are 256 wide; the issuing thread has little time beside it, so its loops are
// compiled for each pair of operand orders (with orders chosen at run time a slice took 790 cycles in place
// of 540). Every wait is bounded (soap_wait_limit); one that runs out sets SOAP_STATUS_TIMEOUT and the CTA
// drains its copies, frees its tensor memory and returns; the last CTA then makes all results NaN.
//
// What bounds it: at 8192 x 8192 the tensor cores (1.83 PFLOP/s, 0.95 of what a library product of that size
// reaches); with K of 768 to 2048 the operands' way from L2 (1.3 to 1.6 PFLOP/s: with both loading threads
// ahead and the ring full, the MMAs wait a quarter of the time for data); with a few matrices of a few tiles
// the chain of phases, each the time of a tile and of handing it on (fp16 1365 x 777: 84 us a step).
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
constexpr int kRunBlocks = 16;         // most K slices per accumulator run of split operands
constexpr int kEpiWarps = 8;
constexpr int kLoadB = 2 + kEpiWarps, kScout = kLoadB + 1;  // warps
constexpr int kThreads = 32 * (kScout + 1);
constexpr int kBlock = 32 * 128;       // a staged block: 32 rows of 128 bytes
constexpr int kPerTile = 2 * kEpiWarps;       // what a tile adds to its matrix's counter
constexpr int kTaken = 16;

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
  CUtensorMap xk[2], sk, bk;   // boxes of 64 columns x 128 rows: K-major operands
  CUtensorMap x[2], s, b;      // boxes of 64 x 64: MN-major operands
  CUtensorMap ex[2], es, eb;   // boxes of 64 columns x 32 rows: C and results
};

// The list.
struct Layout {
  int r, k, tall;
  int ns, nx, nxm, nxn;  // tiles of S (and B), of X', row and column tiles of X'
  int total;
};

struct Tile {
  int step, phase, b;     // phase 0: S, 1: B, 2: X'
  int m0, n0, M, N, K;
  int need;               // the matrix's counter before this tile may start
  // S and B on the diagonal: both operands are the same rows, which are loaded once
  __device__ __forceinline__ bool same() const { return phase < 2 && m0 == n0; }
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

// 128 x 64 elements of an operand at (row m0, k0): 128 rows of 64 K elements (K-major), or two boxes of
// 64 K rows of 64 columns (MN-major).
template <int MN>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int m0, int k0, int z) {
  tma_box(dst, map, bar, MN ? m0 : k0, MN ? k0 : m0, z);
  if (MN) tma_box(dst + kBox, map, bar, m0 + 64, k0, z);
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

// Columns taddr .. taddr + 63, and 16 columns at each of two places, of this lane's accumulator row.
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, float (&v)[32], float (&w)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
      "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, %34, %35, %36, %37, %38, %39, %40, %41, "
      "%42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, "
      "%62, %63}, [%64];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
        "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]),
        "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]),
        "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]),
        "=f"(v[29]), "=f"(v[30]), "=f"(v[31]), "=f"(w[0]), "=f"(w[1]), "=f"(w[2]), "=f"(w[3]), "=f"(w[4]),
        "=f"(w[5]), "=f"(w[6]), "=f"(w[7]), "=f"(w[8]), "=f"(w[9]), "=f"(w[10]), "=f"(w[11]), "=f"(w[12]),
        "=f"(w[13]), "=f"(w[14]), "=f"(w[15]), "=f"(w[16]), "=f"(w[17]), "=f"(w[18]), "=f"(w[19]),
        "=f"(w[20]), "=f"(w[21]), "=f"(w[22]), "=f"(w[23]), "=f"(w[24]), "=f"(w[25]), "=f"(w[26]),
        "=f"(w[27]), "=f"(w[28]), "=f"(w[29]), "=f"(w[30]), "=f"(w[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld16x2(uint32_t t0, uint32_t t1, float (&v)[16], float (&w)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%32];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%33];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
        "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]),
        "=f"(v[15]), "=f"(w[0]), "=f"(w[1]), "=f"(w[2]), "=f"(w[3]), "=f"(w[4]), "=f"(w[5]), "=f"(w[6]),
        "=f"(w[7]), "=f"(w[8]), "=f"(w[9]), "=f"(w[10]), "=f"(w[11]), "=f"(w[12]), "=f"(w[13]), "=f"(w[14]),
        "=f"(w[15])
      : "r"(t0), "r"(t1)
      : "memory");
}

__device__ __forceinline__ int load_acquire(const int* p) {
  int v;
  asm volatile("ld.acquire.gpu.global.b32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}

// Bounded wait for a matrix's counter.
__device__ __forceinline__ bool wait_done(const int* done, int need, uint64_t limit_ns) {
  if (load_acquire(done) >= need) return true;
  const uint64_t t0 = globaltimer();
  for (;;) {
    for (int i = 0; i < 64; ++i)
      if (load_acquire(done) >= need) return true;
    if (globaltimer() - t0 > limit_ns) return false;
  }
}

// Counts between a CTA's warps: of the tiles whose inputs are there, and of those whose loads have begun.
__device__ __forceinline__ void set_ready(uint32_t at, int n) {
  asm volatile("st.release.cta.shared::cta.b32 [%0], %1;" ::"r"(at), "r"(n) : "memory");
}
__device__ __forceinline__ int get_ready(uint32_t at) {
  int n;
  asm volatile("ld.acquire.cta.shared::cta.b32 %0, [%1];" : "=r"(n) : "r"(at) : "memory");
  return n;
}
__device__ __forceinline__ bool wait_ready(uint32_t at, int n, uint64_t limit_ns) {
  const uint64_t t0 = globaltimer();
  for (;;) {
    for (int i = 0; i < 64; ++i)
      if (get_ready(at) >= n) return true;
    if (globaltimer() - t0 > limit_ns) return false;
  }
}
// The same across the pair and for most of a tile's time: with pauses, since a loop of loads takes issue
// slots and power from the others.
__device__ __forceinline__ bool wait_given(uint32_t at, int n, uint64_t limit_ns) {
  const uint64_t t0 = globaltimer();
  for (;;) {
    int v;
    asm volatile("ld.acquire.cluster.shared::cta.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    if (v >= n) return true;
    if (globaltimer() - t0 > limit_ns) return false;
    __nanosleep(100);
  }
}

__device__ __forceinline__ Tile tile_at(uint32_t p, const Layout& l, const Steps& a) {
  Tile t;
  const uint32_t per = 2 * l.ns + l.nx, ns = a.batch * l.ns;  // of a matrix in a step; of all in phase 0
  t.step = p / (a.batch * per);
  uint32_t i = p - t.step * a.batch * per;
  t.phase = i >= 2 * ns ? 2 : i >= ns ? 1 : 0;
  i -= t.phase * ns;
  const uint32_t each = t.phase == 2 ? l.nx : l.ns;
  t.b = i / each;
  i -= t.b * each;
  t.need = (t.step * per + t.phase * l.ns) * kPerTile;
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
// The buffers of all sent blocks but the last N have been read / those blocks are in global memory.
template <int N>
__device__ __forceinline__ void sent_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void sent_done() {
  asm volatile("cp.async.bulk.wait_group %0;" ::"n"(N) : "memory");
}
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

// K slices kb .. to - 1 of an operand's 128 rows from `row` on into the ring at `ring`, the operand's place in
// the first slot. bytes, if not 0: what this thread tells the barrier that a slot takes, all operands in both
// CTAs. is_b: the second operand's thread, whose arrival the barrier counts in either CTA, also where it has
// nothing to load (skip): otherwise nothing would hold the others back to one that falls behind over a run of
// diagonal tiles, and two rounds of the ring behind it takes another round's parity for its own.
template <int SPLIT, int MN>
__device__ __forceinline__ void load_slices(Ring& st, int kb, int to, const CUtensorMap* map, int row, int b,
                                            int batch, uint32_t ring, uint64_t* full, uint64_t* empty,
                                            uint32_t leader_full, uint32_t bytes, bool is_b, bool skip, uint64_t limit_ns) {
  using C = Config<SPLIT>;
  for (; kb < to; ++kb) {
    if (!(st.ok = mbar_wait(&empty[st.s], st.parity, limit_ns))) return;
    if (bytes) expect_tx(&full[st.s], bytes);
    const uint32_t at = ring + st.s * C::kStage, bar = leader_full + st.s * 8;
#pragma unroll
    for (int h = 0; h < SPLIT; ++h)
      if (!skip) load_tile<MN>(at + h * kTile, map, bar, row, kb * BK, b + h * batch);
    if (is_b) asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
    if (++st.s == C::kStages) {
      st.s = 0;
      st.parity ^= 1;
    }
  }
}

// `count` K slices from the ring into the accumulator at d (split: the small products at d + 256).
template <int SPLIT, int A_MN, int B_MN>
__device__ __forceinline__ void issue_slices(Ring& st, int count, uint32_t& more, uint32_t b_at, uint32_t ring,
                                             uint64_t* full, uint64_t* empty, uint32_t d, uint64_t limit_ns) {
  using C = Config<SPLIT>;
  constexpr uint32_t idesc = idesc_f16(A_MN, B_MN);
  for (; count > 0; --count) {
    if (!(st.ok = mbar_wait(&full[st.s], st.parity, limit_ns))) return;
    tc_fence_after();
    const uint32_t as = ring + st.s * C::kStage, bs = as + b_at;
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

// An epilogue warp's part of a tile: up to two blocks of 32 rows x 64 columns from (r0, n0).
struct Work {
  Tile t;
  int r0, n0, blocks;
  bool has_c, last;    // the result takes C; it goes to the caller's matrix
  float alpha, beta;
  const CUtensorMap *cin, *out;
};

__device__ __forceinline__ Work work_at(const Tile& t, const Steps& a, const Maps& maps, int row, int col) {
  Work w;
  w.t = t;
  w.r0 = t.m0 + row;
  w.n0 = t.n0 + col;
  // none below the last row, and to the last column
  w.blocks = w.r0 < t.M && w.n0 < t.N ? min(2, (t.N - w.n0 + 63) / 64) : 0;
  w.has_c = t.phase > 0 && w.blocks > 0;
  w.last = t.phase == 2 && t.step + 1 == a.steps;
  const StepCoef& c = a.coef[t.step];
  w.alpha = t.phase == 0 ? c.s_alpha : t.phase == 1 ? c.b_alpha : c.x_alpha;
  w.beta = t.phase == 1 ? c.b_beta : c.x_beta;
  if (t.step == 0 && t.phase != 1) {
    const float f = a.t[t.b];
    w.alpha *= t.phase == 0 ? f * f : f;
    w.beta *= f;
  }
  w.cin = t.phase == 1 ? &maps.es : &maps.ex[t.step & 1];
  w.out = t.phase == 0 ? &maps.es : t.phase == 1 ? &maps.eb : &maps.ex[(t.step & 1) ^ 1];
  return w;
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
  const uint32_t ready_at = smem_u32(tmem_at + 2), begun_at = ready_at + 4, given_at = ready_at + 8;
  // the list's places that this pair has taken, tile m's at m % kTaken (all roles of a pair are within the
  // ring's slots and the accumulators of each other: every slot takes both CTAs' loading threads), -1 at the end
  volatile int* taken = reinterpret_cast<volatile int*>(tmem_at + 5);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)(blockIdx.x & 1);  // in the pair
  const uint64_t lim = a.wait_ns;          // bound of every wait (for another role of the pair: twice)

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 3);  // the pair's first CTA's first loading thread, both CTAs' second ones
      mbar_init(&empty[s], 1);
    }
    for (int i = 0; i < kAcc; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], 2 * kEpiWarps);
    }
    for (int i = 0; i < kEpiWarps * C::kBufs; ++i) mbar_init(&cin_full[i], 1);
    *abort_flag = 0;
    set_ready(ready_at, 0);
    set_ready(begun_at, 0);
    set_ready(given_at, 0);
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

  if (warp == kScout) {
    // the pair's first CTA takes a tile as its loads of the one before begin, and tells the second; each then
    // waits for the tile's inputs
    if (lane == 0) {
      bool ok = rank != 0 || !a.hold || flag_wait(a.hold, lim);  // a flag that nothing sets: every role's wait runs out
      for (int m = 0; ok && !*abort_flag; ++m) {
        int p;
        if (rank == 0) {
          if (!(ok = wait_given(begun_at, m, 2 * lim))) break;
          p = atomicAdd(a.done + a.batch, 1);
          if (p >= l.total) p = -1;
          uint32_t peer;
          asm("mapa.shared::cluster.u32 %0, %1, 1;" : "=r"(peer) : "r"(smem_u32(tmem_at)));
          asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(peer + 20 + 4 * (m % kTaken)), "r"(p) : "memory");
          asm volatile("st.release.cluster.shared::cluster.b32 [%0], %1;" ::"r"(peer + 16), "r"(m + 1) : "memory");
          taken[m % kTaken] = p;
        } else {
          if (!(ok = wait_given(given_at, m + 1, 2 * lim))) break;
          p = taken[m % kTaken];
        }
        if (p >= 0) {
          const Tile t = tile_at(p, l, a);
          if (!(ok = wait_done(a.done + t.b, t.need, lim))) break;
          asm volatile("fence.proxy.async;" ::: "memory");  // what other CTAs stored, before copies of it
        }
        set_ready(ready_at, m + 1);
        if (p < 0) break;
      }
      if (!ok) {
        *abort_flag = 1;
        if (a.status) atomicOr(a.status, kStatusTimeout);
      }
    }
  } else if (warp == 0 || warp == kLoadB) {
    if (lane == 0) {
      const bool is_b = warp == kLoadB;
      Ring st;
      st.parity = 1;  // of a slot's release
      int used = 0;   // slots filled so far (up to kStages)
      const uint32_t ring = smem_u32(smem) + (is_b ? SPLIT * kTile : 0), bars = in_leader(full);
      for (int m = 0; !*abort_flag; ++m) {
        if (!(st.ok = wait_ready(ready_at, m + 1, 2 * lim))) break;
        const int p = taken[m % kTaken];
        if (p < 0) break;
        if (!is_b) set_ready(begun_at, m + 1);
        const Tile t = tile_at(p, l, a);
        const int kblocks = (t.K + BK - 1) / BK;
        int a_change, b_change;
        order_change(t, l.tall, kblocks, a_change, b_change);
        const int change = is_b ? b_change : a_change;
        const bool of_x = t.phase == 0 || (t.phase == 2 && is_b == !l.tall);
        const CUtensorMap* mk = of_x ? &maps.xk[t.step & 1] : t.phase == 1 ? &maps.sk : &maps.bk;
        const CUtensorMap* mn = of_x ? &maps.x[t.step & 1] : t.phase == 1 ? &maps.s : &maps.b;
        const int row = (is_b ? t.n0 : t.m0) + rank * 128;
        const uint32_t bytes = rank != 0 || is_b ? 0 : (t.same() ? 1 : 2) * Config<SPLIT>::kStage;
        const bool skip = is_b && t.same();
        used = min(used + kblocks, kStages);
        if (change > 0)
          load_slices<SPLIT, 0>(st, 0, change, mk, row, t.b, a.batch, ring, full, empty, bars, bytes, is_b, skip, lim);
        if (st.ok && change < kblocks)
          load_slices<SPLIT, 1>(st, change, kblocks, mn, row, t.b, a.batch, ring, full, empty, bars, bytes, is_b, skip, lim);
        if (!st.ok) break;
      }
      // every slice consumed, and its release arrived here, before this CTA's barriers go away
      for (int i = 0; i < kStages && st.ok && !*abort_flag; ++i) {
        if (used == kStages || st.s - 1 - i >= 0) {
          const int slot = (st.s - 1 - i + kStages) % kStages;
          st.ok = mbar_wait(&empty[slot], slot < st.s ? st.parity ^ 1 : st.parity, lim);
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
      for (int m = 0; st.ok && !*abort_flag; ++m) {
        if (!(st.ok = wait_ready(ready_at, m + 1, 2 * lim))) break;
        const int p = taken[m % kTaken];
        if (p < 0) break;
        const Tile t = tile_at(p, l, a);
        const int kblocks = (t.K + BK - 1) / BK;
        int a_change, b_change;
        order_change(t, l.tall, kblocks, a_change, b_change);
        const uint32_t b_at = t.same() ? 0 : SPLIT * kTile;
        const int runs = SPLIT == 2 ? (kblocks + kRunBlocks - 1) / kRunBlocks : 1;
        for (int run = 0; run < runs && st.ok; ++run, ++n) {
          const int ac = n % kAcc;
          if (n >= kAcc && !(st.ok = mbar_wait(&acc_empty[ac], ((n / kAcc) & 1) ^ 1, lim))) break;
          tc_fence_after();
          const uint32_t d = tmem + static_cast<uint32_t>(ac * 256);
          const int k1 = SPLIT == 2 ? kblocks * (run + 1) / runs : kblocks;
          int kb = SPLIT == 2 ? kblocks * run / runs : 0;
          uint32_t more = 0;
          while (kb < k1 && st.ok) {  // stretches of slices of one order
            const bool a_mn = kb >= a_change, b_mn = kb >= b_change;
            const int to = min(k1, min(a_mn ? k1 : a_change, b_mn ? k1 : b_change));
            if (a_mn && b_mn)
              issue_slices<SPLIT, 1, 1>(st, to - kb, more, b_at, ring, full, empty, d, lim);
            else if (a_mn)
              issue_slices<SPLIT, 1, 0>(st, to - kb, more, b_at, ring, full, empty, d, lim);
            else if (b_mn)
              issue_slices<SPLIT, 0, 1>(st, to - kb, more, b_at, ring, full, empty, d, lim);
            else
              issue_slices<SPLIT, 0, 0>(st, to - kb, more, b_at, ring, full, empty, d, lim);
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
    int k = 0;                  // blocks so far: block k uses buffer k % kBufs
    uint32_t cin_parity = 0;    // one bit per buffer
    int* unreported = nullptr;  // counter of the matrix whose tile this warp has sent but not reported
    bool ok = true;
    auto wait_acc = [&](int ac) {
      ok = mbar_wait(&acc_full[ac], (n / kAcc) & 1, lim) && !*abort_flag;
      tc_fence_after();
      return ok = __all_sync(0xffffffffu, ok);
    };
    auto release_acc = [&](int ac) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0)
        asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_leader(&acc_empty[ac])) : "memory");
    };
    // Reports the last tile; `newer` blocks of the present one have been sent since.
    auto report = [&](auto newer) {
      if (unreported && lane == 0) {
        sent_done<decltype(newer)::value>();
        asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(unreported) : "memory");
      }
      unreported = nullptr;
    };
    auto fetch = [&](const Work& w, int i, int h, int buf) {  // w's block i, part h of C
      if (lane == 0)
        fetch_block(stage_at + buf * kBlock, w.cin, &cin_bar[buf], w.n0 + 64 * i, w.r0, w.t.b + h * a.batch);
    };
    auto fetched = [&](int buf) {
      ok = mbar_wait(&cin_bar[buf], (cin_parity >> buf) & 1, lim);
      cin_parity ^= 1u << buf;
      return ok = __all_sync(0xffffffffu, ok);
    };
    auto send = [&](const Work& w, int i, int h, int buf) {
      before_tma();
      __syncwarp();
      if (lane == 0) send_block(w.out, stage_at + buf * kBlock, w.n0 + 64 * i, w.r0, w.t.b + h * a.batch);
    };
    auto to_user = [&](const Work& w, uint8_t* st, int i, int h, const float (&v)[32]) {
      const int c0 = w.n0 + 64 * i + 32 * h;
      if (c0 < w.t.N)
        store_user_any(st, v, a, out_vec, w.t.b, w.r0, c0, min(32, w.t.M - w.r0), min(32, w.t.N - c0), lane);
    };
    const int wr = rank * 128 + 32 * q, wc = 128 * half;  // this warp's place in a tile
    Work w{}, next{};
    bool known = false;  // w is the next tile, and the first block of its C is on its way if it takes any
    for (int m = 0;; ++m) {
      if (!known) {
        // a tile that has to wait may wait for this warp's own last one: that is reported first
        int there = lane == 0 ? get_ready(ready_at) : 0;
        if (__shfl_sync(0xffffffffu, there, 0) <= m) {
          report(std::integral_constant<int, 0>());
          if (lane == 0) ok = wait_ready(ready_at, m + 1, 2 * lim);
          if (!(ok = __shfl_sync(0xffffffffu, ok, 0))) break;
        }
        __syncwarp();
        const int p = taken[m % kTaken];
        if (p < 0) break;
        w = work_at(tile_at(p, l, a), a, maps, wr, wc);
        if (w.has_c) {
          if (lane == 0) sent_read<0>();
          fetch(w, 0, SPLIT - 1, k % C::kBufs);
        }
      }
      known = false;
      const float alpha = w.alpha, beta = w.beta;
      if constexpr (SPLIT == 1) {
        const int ac = n % kAcc;
        if (!wait_acc(ac)) break;
        if (w.blocks == 0) release_acc(ac);
        for (int i = 0; i < w.blocks; ++i, ++k) {
          const int buf = k & 1;
          uint8_t* st = stage + buf * kBlock;
          float v[2][32];
          tmem_ld64(lanes + static_cast<uint32_t>(ac * 256 + 64 * i), v[0], v[1]);
          if (i + 1 == w.blocks) release_acc(ac);
          // the next block's C, into the buffer of the block before
          if (i + 1 < w.blocks) {
            if (w.has_c) {
              if (lane == 0) sent_read<0>();
              fetch(w, i + 1, 0, buf ^ 1);
            }
          } else {
            const int there = lane == 0 ? get_ready(ready_at) : 0;
            if (__shfl_sync(0xffffffffu, there, 0) > m + 1) {
              __syncwarp();
              const int p = taken[(m + 1) % kTaken];
              if (p >= 0) {
                known = true;
                next = work_at(tile_at(p, l, a), a, maps, wr, wc);
                if (next.has_c) {
                  if (lane == 0) sent_read<0>();
                  fetch(next, 0, 0, buf ^ 1);
                }
              }
            }
          }
          if (w.has_c) {
            if (!fetched(buf)) break;
          } else {
            if (lane == 0) sent_read<1>();
            __syncwarp();
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[h][j] *= alpha;
            if (w.has_c) add_row(st, h, beta, v[h], lane);
          }
          if (w.last) {
            __syncwarp();
            to_user(w, st, i, 0, v[0]);
            to_user(w, st, i, 1, v[1]);
            before_tma();
            __syncwarp();
          } else {
            put_row<false>(st, 0, v[0], lane);
            put_row<false>(st, 1, v[1], lane);
            send(w, i, 0, buf);
            if (i == 0) report(std::integral_constant<int, 1>());
          }
        }
        if (!ok) break;
        ++n;
        report(std::integral_constant<int, 0>());  // where this tile sent nothing
      } else {
        report(std::integral_constant<int, 0>());
        float sum[4][32];
        const int kblocks = (w.t.K + BK - 1) / BK;
        const int runs = (kblocks + kRunBlocks - 1) / kRunBlocks;
        for (int i = 0; i < runs; ++i, ++n) {
          if (!wait_acc(0)) break;
#pragma unroll
          for (int b = 0; b < 8; ++b)
            if (b / 4 < w.blocks) {
              float hi[16], small[16];
              tmem_ld16x2(lanes + 16 * b, lanes + 256 + 16 * b, hi, small);
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
          if (i < w.blocks && ok) {
            float(&v0)[32] = sum[2 * i];
            float(&v1)[32] = sum[2 * i + 1];
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              v0[j] *= alpha;
              v1[j] *= alpha;
            }
            if (w.has_c) {  // the small part first
              if (i > 0) fetch(w, i, 1, 0);
              if (!fetched(0)) break;
              add_row(stage, 0, beta, v0, lane);
              add_row(stage, 1, beta, v1, lane);
              before_tma();
              __syncwarp();
              fetch(w, i, 0, 0);
              if (!fetched(0)) break;
              add_row(stage, 0, beta, v0, lane);
              add_row(stage, 1, beta, v1, lane);
            }
            if (w.last) {
              __syncwarp();
              to_user(w, stage, i, 0, v0);
              to_user(w, stage, i, 1, v1);
              before_tma();
            } else {
              put_row<true>(stage, 0, v0, lane);
              put_row<true>(stage, 1, v1, lane);
              send(w, i, 0, 0);
              if (lane == 0) sent_read<0>();
              __syncwarp();
              put_row<false>(stage, 0, v0, lane);
              put_row<false>(stage, 1, v1, lane);
              send(w, i, 1, 0);
              if (lane == 0) sent_read<0>();
            }
            __syncwarp();
          }
        if (!ok) break;
      }
      unreported = a.done + w.t.b;
      if (known) w = next;
    }
    if (ok) report(std::integral_constant<int, 0>());
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

  // Where a wait gave up, the last CTA makes all results NaN, so that none is taken for an answer.
  if (threadIdx.x == 0) {
    int* const through = a.done + a.batch + 1;
    if (*abort_flag) atomicOr(through + 1, 1);
    __threadfence();  // this CTA's results (and its word) come before its count
    const bool last = atomicAdd(through, 1) == (int)gridDim.x - 1;
    __threadfence();
    *abort_flag = last && atomicOr(through + 1, 0) != 0;
  }
  __syncthreads();
  if (*abort_flag)
    for (int b = 0; b < a.batch; ++b)
      for (int r = warp; r < a.rows; r += kThreads / 32)
        for (int c = lane; c < a.cols; c += 32) {
          const int64_t at = (int64_t)b * a.stride_out + (int64_t)r * a.ld_out + c;
          if (a.out_type == SOAP_F32)
            static_cast<float*>(a.out)[at] = NAN;
          else if (a.out_type == SOAP_BF16)
            static_cast<__nv_bfloat16*>(a.out)[at] = from_f32<__nv_bfloat16>(NAN);
          else
            static_cast<__half*>(a.out)[at] = from_f32<__half>(NAN);
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
  const int64_t most = (int64_t)p.batch * std::max(l.ns, l.nx);
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
  const int64_t per = 2 * (int64_t)l.ns + l.nx;
  if (per * p.steps > INT32_MAX / kPerTile || per * p.batch * p.steps > INT32_MAX - 1024)
    return cudaErrorInvalidValue;
  l.total = (int)(per * p.batch * p.steps);

  const int planes = p.batch * (p.split ? 2 : 1);
  Maps maps;
  for (int i = 0; i < 2; ++i)
    if (!make_map(&maps.x[i], p.x[i], p.rows, p.cols, p.ld_x, planes, 64) ||
        !make_map(&maps.xk[i], p.x[i], p.rows, p.cols, p.ld_x, planes, 128) ||
        !make_map(&maps.ex[i], p.x[i], p.rows, p.cols, p.ld_x, planes, 32))
      return cudaErrorInvalidValue;
  if (!make_map(&maps.sk, p.s, l.r, l.r, p.ld_s, planes, 128) ||
      !make_map(&maps.bk, p.b, l.r, l.r, p.ld_s, planes, 128) ||
      !make_map(&maps.s, p.s, l.r, l.r, p.ld_s, planes, 64) ||
      !make_map(&maps.b, p.b, l.r, l.r, p.ld_s, planes, 64) ||
      !make_map(&maps.es, p.s, l.r, l.r, p.ld_s, planes, 32) ||
      !make_map(&maps.eb, p.b, l.r, l.r, p.ld_s, planes, 32))
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
