// What the kernels on pairs of CTAs (cta_group::2, a 256 x 256 tile with 128 rows in each CTA) share: TMA copies of
// operand tiles into a ring, matrix descriptors of both orders, bounded waits between the roles, blocks of
// 32 rows on their way through shared memory to global memory.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>

#include <cstdint>
#include <mutex>

#include "tc_ptx.h"
#include "types.h"

namespace soap {
namespace tc {

constexpr int BK = 64;
constexpr int kBox = 64 * 64 * 2;      // one TMA box: 64 rows of 128 bytes
constexpr int kTile = 2 * kBox;        // a CTA's 128 x 64 elements of an operand

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

// Place of row j's 16-byte chunk c in a staged block of rows of 64 bytes (16-bit elements) or 128
// (fp32): permuted so that neither rows nor columns of chunks meet in a bank.
__device__ __forceinline__ int at16(int j, int c) { return j * 64 + ((c ^ ((j >> 1) & 3)) * 16); }
__device__ __forceinline__ int at32(int j, int c) { return j * 128 + ((c ^ (j & 7)) * 16); }

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

// 16 columns of this lane's accumulator row, at one place or two.
__device__ __forceinline__ void tmem_ld16(uint32_t t, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(t)
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

// A thread's place in the ring: the slot and the parity it waits for.
struct Ring {
  int s = 0;
  uint32_t parity = 0;
  bool ok = true;
};

inline PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
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

}  // namespace tc
}  // namespace soap
