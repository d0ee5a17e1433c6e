// What layer norm's forward and backward kernels share: how the rows come in, sums over a row's
// threads, and the choice of a row's threads. Included by layer_norm.cu and layer_norm_bwd.cu.
//
// Bound by memory: x is read and y written once (backward: x and dy read, dx written once). A
// group of threads holds a row in registers, so that the variance is a second pass over registers
// (not E[x^2] - mu^2, which cancels) and nothing is read twice. CTAs are persistent: each thread
// keeps its columns' weights (backward: and their gradients' sums) in registers over all its rows
// (read again for every row, fp32 weights are four times the traffic of a bf16 x through L1: 345 us
// at 32768 x 8192), and rows come in ahead by bulk copies into a ring in shared memory (asynchronous
// 16-byte copies by every thread stopped at 2.7 TB/s of reads). A bulk copy moves whole 16-byte units:
// of rows that begin or end inside one, the neighbour's part comes along, except before the first row and
// after the last. Narrow rows, a warp's each, are short of work per copy: they come, a row ahead, into
// registers (60000 x 100 bf16: 16 us forward, 20 backward; by bulk copies 20 and 26). Pairs of elements go
// through the fp32 pipe together.
#pragma once

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>

#include "../../include/layer.h"
#include "profile.h"
#include "soap_internal.h"
#include "tc_ptx.h"
#include "types.h"

namespace soap {
namespace {

constexpr int kMaxThreads = 512;  // of the kernels for rows too wide to be held
// A CTA's threads by the elements of a row that each holds: few registers, twice the threads.
constexpr int threads_for(int elems) { return elems <= 8 ? 1024 : 512; }
constexpr int kMaxGroups = 16;    // row groups of a CTA
constexpr int64_t kMaxRows = INT32_MAX - 65536;  // a row index some steps further on stays an int

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// One barrier among a row group's threads (blockDim.x of them, more than a warp).
__device__ __forceinline__ void group_barrier() {
  asm volatile("bar.sync %0, %1;" ::"r"((int)threadIdx.y + 1), "r"((int)blockDim.x) : "memory");
}

// What a row group's warps exchange: two values per warp, in two halves used in turn, so that one
// barrier per exchange is enough (a half is written again only after the barrier of the exchange
// between).
struct Exchange {
  float2* buf;  // [2][blockDim.y][blockDim.x / 32]
  int half = 0;
  // Afterwards lane l holds warp l's values ((0, 0) from the last warp on).
  __device__ __forceinline__ float2 all(float x, float y) {
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    float2* p = buf + (half * blockDim.y + threadIdx.y) * warps;
    half ^= 1;
    if (lane == 0) p[threadIdx.x >> 5] = make_float2(x, y);
    group_barrier();
    return lane < warps ? p[lane] : make_float2(0.f, 0.f);
  }
};

// The rows of N matrices (x; or x and dy) for a row group, up to DEPTH rows ahead, NV packs of V elements
// per thread and row.
template <typename T, int V, int NV, int N, int DEPTH, bool FULL, bool RING>
struct Rows {
  static constexpr bool kWhole = V * sizeof(T) == 16;  // rows are whole 16-byte units
  const T* base[N];
  int64_t ld[N];
  int rows, step, width;
  uint8_t* ring;    // the group's: ring_bytes
  uint64_t* full;   // the group's barriers, one per stage
  int* status;
  WaitLimit wait;   // soap_wait_limit's settings
  int s = 0;
  // kDead: a wait of this thread's ran out. What it gets is invalid (a sum that it takes part in has to become
  // NaN, and with it the row's results), and it neither waits nor asks for more.
  uint32_t parity = 0;
  static constexpr uint32_t kDead = 2;
  __device__ __forceinline__ bool dead() const { return RING && parity >= kDead; }
  Pack<T, V> ahead[RING ? 1 : N][RING ? 1 : NV];

  // Of a group of `threads`: a row, and the parts of its neighbours that come along.
  static __host__ __device__ constexpr int slot_bytes(int threads) {
    return threads * NV * V * (int)sizeof(T) + (kWhole ? 0 : 32);
  }
  static __host__ __device__ constexpr int ring_bytes(int threads) {
    return RING ? DEPTH * N * slot_bytes(threads) : 0;
  }

  __device__ __forceinline__ uint8_t* slot(int stage, int n) const {
    return ring + (stage * N + n) * slot_bytes(blockDim.x);
  }
  static __device__ __forceinline__ void copy(uint8_t* dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
            tc::smem_u32(dst)),
        "l"(src), "r"(bytes), "r"(bar)
        : "memory");
  }
  // One thread asks for a row into a stage.
  __device__ __forceinline__ void request(int row, int stage) {
    if (row >= rows) return;
    const uint32_t bar = tc::smem_u32(full + stage);
    if constexpr (kWhole) {
      const uint32_t bytes = (uint32_t)width * sizeof(T);
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(N * bytes) : "memory");
#pragma unroll
      for (int m = 0; m < N; ++m) copy(slot(stage, m), base[m] + (int64_t)row * ld[m], bytes, bar);
    } else {
      uintptr_t lo[N], hi[N];
      uint32_t bytes = 0;
#pragma unroll
      for (int m = 0; m < N; ++m) {
        const uintptr_t begin = reinterpret_cast<uintptr_t>(base[m] + (int64_t)row * ld[m]);
        const uintptr_t end = begin + (uintptr_t)width * sizeof(T);
        lo[m] = begin & ~uintptr_t(15);
        hi[m] = (end + 15) & ~uintptr_t(15);
        // nothing from before the first row or after the last (rows here are longer than a unit)
        if (row == 0 || row == rows - 1) {
          uint8_t* const dst = slot(stage, m);
          const uintptr_t at = lo[m];
          if (row == 0 && lo[m] < begin) lo[m] += 16;
          if (row == rows - 1 && hi[m] > end) hi[m] -= 16;
          if (hi[m] < lo[m]) hi[m] = lo[m];
          for (uintptr_t a = begin; a < end; a += sizeof(T))
            if (a < lo[m] || a >= hi[m]) {
              *reinterpret_cast<T*>(dst + (a - at)) = *reinterpret_cast<const T*>(a);
            } else {
              a = hi[m] - sizeof(T);
            }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // before later copies to the place
        }
        bytes += (uint32_t)(hi[m] - lo[m]);
      }
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
#pragma unroll
      for (int m = 0; m < N; ++m) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(base[m] + (int64_t)row * ld[m]) & ~uintptr_t(15);
        if (hi[m] > lo[m])
          copy(slot(stage, m) + (lo[m] - at), reinterpret_cast<const void*>(lo[m]), (uint32_t)(hi[m] - lo[m]), bar);
      }
    }
  }
  // A row into registers, zero beyond its end.
  __device__ __forceinline__ void load(int row) {
#pragma unroll
    for (int m = 0; m < N; ++m)
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * V;
        if (row < rows && c < width) {
          ahead[m][i] = *reinterpret_cast<const Pack<T, V>*>(base[m] + (int64_t)row * ld[m] + c);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) ahead[m][i].v[e] = from_f32<T>(0.f);
        }
      }
  }
  // Before the first row: called by all threads of the CTA.
  __device__ __forceinline__ void start(int row) {
    if constexpr (!RING) {
      load(row);
      return;
    }
    if (threadIdx.x == 0) {
      for (int q = 0; q < DEPTH; ++q) tc::mbar_init(full + q, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      // (a flag that nothing sets: no row comes, and the group's waits run out)
      const bool held = wait.hold && !tc::flag_wait(wait.hold, wait.ns);
      for (int q = 0; q < DEPTH && !held; ++q) request(row + q * step, q);
    }
    __syncthreads();
  }
  // The row, zero beyond its end.
  __device__ __forceinline__ void get(int row, Pack<T, V> (&p)[N][NV]) {
    if constexpr (!RING) {
#pragma unroll
      for (int m = 0; m < N; ++m)
#pragma unroll
        for (int i = 0; i < NV; ++i) p[m][i] = ahead[m][i];
      load(row + step);
      return;
    }
    if (!dead() && !tc::mbar_wait(full + s, parity, wait.ns)) {
      parity |= kDead;
      if (status) atomicOr(status, SOAP_STATUS_TIMEOUT);
    }
#pragma unroll
    for (int m = 0; m < N; ++m) {
      const uint8_t* from = slot(s, m);
      if constexpr (!kWhole) from += reinterpret_cast<uintptr_t>(base[m] + (int64_t)row * ld[m]) & 15;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = i * blockDim.x + threadIdx.x;
        if (FULL || c * V < width) {
          p[m][i] = reinterpret_cast<const Pack<T, V>*>(from)[c];
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) p[m][i].v[e] = from_f32<T>(0.f);
        }
      }
    }
  }
  // After a point that all of the group's threads have reached since get(): the slots are free.
  __device__ __forceinline__ void refill(int row) {
    if constexpr (!RING) return;
    if (threadIdx.x == 0 && !dead()) request(row + DEPTH * step, s);  // (no second copy into a slot that never filled)
    if (++s == DEPTH) {
      s = 0;
      parity ^= 1;
    }
  }
  // After the last row.
  __device__ __forceinline__ void finish() const {
    if constexpr (!RING) return;
    if (dead()) {  // copies in flight land before the shared memory goes away: far above a copy's time
      const uint64_t t0 = tc::globaltimer();
      while (tc::globaltimer() - t0 < 10000000ull) {
      }
    }
  }
};

// Elements 2 k and 2 k + 1 of a thread's packs as fp32.
template <typename T, int V, int NV>
__device__ __forceinline__ float2 values(const Pack<T, V> (&p)[NV], int k) {
  if constexpr (V == 1)
    return make_float2(to_f32(p[2 * k].v[0]), to_f32(p[2 * k + 1].v[0]));
  else
    return to_pair(p[2 * k / V].v + 2 * k % V);
}

// A row's results in pack i (V == 1: packs i and i + 1), rounded once.
template <typename T, int V, bool FULL>
__device__ __forceinline__ void put(T* row, int width, int i, const float2* v) {
#pragma unroll
  for (int j = 0; j < (V == 1 ? 2 : 1); ++j) {
    const int c = ((i + j) * blockDim.x + threadIdx.x) * V;
    if (!FULL && c >= width) break;
    Pack<T, V> o;
    if constexpr (V == 1) {
      o.v[0] = from_f32<T>(j ? v[0].y : v[0].x);
    } else {
#pragma unroll
      for (int e = 0; e < V; e += 2) from_pair(v[e / 2], o.v + e);
    }
    *reinterpret_cast<Pack<T, V>*>(row + c) = o;
  }
}

// A thread's columns of a vector as fp32 pairs (`none` beyond the width, or everywhere without one).
template <typename W, int V, int NV>
__device__ __forceinline__ void columns(const W* w, float none, int width, float2 (&v)[NV * V / 2]) {
#pragma unroll
  for (int k = 0; k < NV * V; ++k) {
    const int c = ((k / V) * blockDim.x + threadIdx.x) * V + k % V;
    const float x = w && c < width ? to_f32(w[c]) : none;
    if (k % 2)
      v[k / 2].y = x;
    else
      v[k / 2].x = x;
  }
}

// Sum over a one-row CTA's threads, for the kernels that do not hold a row.
template <int N>
__device__ __forceinline__ void block_sum(float (&v)[N], float* buf) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
  __syncthreads();
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) buf[(threadIdx.x >> 5) * N + i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.f;
  for (int j = 0; j < (int)blockDim.x / 32; ++j)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += buf[j * N + i];
}

// ---- launch choice -------------------------------------------------------------------------

constexpr int kSms = 152;
constexpr int kParts = 2 * kSms;  // most CTAs, and partial rows

struct NormShape {
  int nv, tx;  // accesses per thread and row, threads per row
};

// Threads for a row of `width` elements in accesses of v: a warp where 16 elements per thread are
// enough, else the fewest that give a thread no more than `elems` elements, or more up to `most` where
// the row needs it. nv = 0: too wide for that.
NormShape norm_shape(int64_t width, int v, int elems, int most) {
  const int64_t packs = (width + v - 1) / v;
  for (int nv = v == 1 ? 2 : 1; nv * v <= 16; nv *= 2)
    if (packs <= 32 * nv) return {nv, 32};
  for (int e = elems; e <= most; e *= 2)
    for (int tx = 64; tx <= threads_for(e); tx *= 2)
      if (packs * v <= (int64_t)tx * e) return {e / v, tx};
  return {0, 0};
}

// With few rows per SM a row's own time counts: 8 elements per thread and many threads. With many, rows
// side by side in an SM hide each other's chains of sums: more elements per thread, so that more rows
// fit (forward, 32768 x 8192 bf16: 258 us with 8, 260 with 16, 200 with 32; backward, whose columns'
// sums take registers too, 495, 472 and spills).
bool many_rows(int64_t rows) { return rows >= 16 * kSms; }

int norm_threads(const NormShape& n, int v) { return n.tx >= 128 ? threads_for(n.nv * v) : 512; }

// Rows per CTA: full CTAs, unless the rows would then not reach every SM.
int norm_groups(int64_t rows, const NormShape& n, int v) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(norm_threads(n, v) / n.tx, (rows + kSms - 1) / kSms));
}

// CTAs: two per SM where one does not fill it.
int norm_ctas(int64_t rows, const NormShape& n, int v, int ty) {
  const int most = n.tx * ty <= 512 && n.nv * v <= 8 ? kParts : kSms;
  return (int)std::min<int64_t>(most, (rows + ty - 1) / ty);
}

template <typename F>
cudaError_t with_nv(int nv, F&& f) {
  switch (nv) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 4: return f(std::integral_constant<int, 4>());
    case 8: return f(std::integral_constant<int, 8>());
    case 16: return f(std::integral_constant<int, 16>());
    default: return f(std::integral_constant<int, 32>());
  }
}

// f(elements per access) for rows whose addresses and lengths in bytes, ORed, are `bytes`: 16 bytes, else
// 8, else 4, else an element.
template <typename T, typename F>
cudaError_t with_access(uintptr_t bytes, F&& f) {
  if (bytes % 16 == 0) return f(std::integral_constant<int, 16 / sizeof(T)>());
  if (bytes % 8 == 0) return f(std::integral_constant<int, 8 / sizeof(T)>());
  if (sizeof(T) == 2 && bytes % 4 == 0) return f(std::integral_constant<int, sizeof(T) == 2 ? 2 : 1>());
  return f(std::integral_constant<int, 1>());
}

// f(whether the row has exactly the group's elements, whether rows come through shared memory): the first
// told apart for the widest accesses. Through registers go a warp's rows of up to 8 elements per thread (with
// 16, 20000 x 511 fp32 takes 27 us forward and 45 backward, through shared memory 25 and 33); more threads
// per row have 8 elements each at least.
template <int V, int E, typename F>
cudaError_t with_full(bool full, int tx, F&& f) {
  if constexpr (E >= 8)
    if (E > 8 || tx > 32) {
      if (V >= 4 && full) return f(std::integral_constant<bool, (V >= 4)>(), std::true_type());
      return f(std::false_type(), std::true_type());
    }
  if constexpr (E <= 8) return f(std::false_type(), std::false_type());
  return cudaErrorInvalidValue;
}

uintptr_t address(const void* p) { return reinterpret_cast<uintptr_t>(p); }

// One bit per device on which the kernel has its shared-memory attribute.
template <typename K>
cudaError_t allow_smem(K kernel, int bytes, std::atomic<uint64_t>& set) {
  if (bytes <= 48 * 1024 - 4096) return cudaSuccess;  // beside the static part
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t(1) << dev : 0;
  if (bit && (set.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
  if (e == cudaSuccess) set.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// f(T(), W()) for an activation and a weight type.
template <typename F>
cudaError_t with_types(int32_t xt, int32_t wt, F&& f) {
  if (xt == SOAP_F32) return f(float(), float());
  if (xt == SOAP_BF16)
    return wt == SOAP_F32 ? f(__nv_bfloat16(), float()) : f(__nv_bfloat16(), __nv_bfloat16());
  return wt == SOAP_F32 ? f(__half(), float()) : f(__half(), __half());
}

bool bad_ptr(const void* p, size_t size) { return p && reinterpret_cast<uintptr_t>(p) % size; }

bool bad_norm(int64_t rows, int64_t width, int32_t xt, const void* w, const void* b, int32_t wt) {
  if (rows < 0 || width < 1 || rows > kMaxRows || width > INT32_MAX) return true;
  if (xt < SOAP_F32 || xt > SOAP_F16 || (wt != SOAP_F32 && wt != xt)) return true;
  return bad_ptr(w, dtype_size(wt)) || bad_ptr(b, dtype_size(wt));
}

bool bad_rows(const void* p, int64_t ld, int64_t rows, int64_t width, int32_t t) {
  return rows > 0 && (!p || bad_ptr(p, dtype_size(t)) || ld < width);
}

}  // namespace
}  // namespace soap
