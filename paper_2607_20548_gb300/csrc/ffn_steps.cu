// The products of the gated feed-forward block on the 5th-generation tensor cores: all of a call's in one launch,
//   forward   g, u = x Wg, x Wu -> h = act(g) u;  y = h Wd
//   backward  dh = dy Wd^T -> dg, du, h;  dx = dg Wg^T + du Wu^T;  dWg, dWu = x^T dg, x^T du;  dWd = h^T dy
// for every group of rows, with fp32 accumulation.
//
// Operands are read as they lie, with K along their rows (K-major) or down their columns (MN-major), so that no
// transposed copy exists. 16-bit operands go to the tensor cores as they are. An fp32 operand comes as three bf16
// planes that hold its 24 bits, and the six products of planes whose terms reach 2^-24 are added, small ones first:
// the accumulator cuts (a sum loses 2^-25 of itself per 16 products, measured), so that K goes in runs of 256, whose
// sums the epilogue adds up, rounding to nearest, in the other half of the tensor memory (in registers, 128 a thread,
// the compiler spilled them: 5 groups of 2048 x 768, 2000 rows, both passes 595 us in place of 453).
//
// Schedule. Persistent CTA pairs (cta_group::2: a pair's 256 x 256 tile has 128 rows in each CTA) take units from one
// list, each its next one when it begins the one before: a phase's tiles, or parts of them along K where the tiles are
// fewer than the pairs (the part that is stored last adds up all of them, always in the same order). Tiles of the
// first phase are 256 rows by 128 columns of both g and u, one CTA of the pair loading Wg's, the other Wu's, so that
// both values of an element meet in one thread. A unit waits until what it reads of the phase before is stored, which
// counters per row tile and per group tell; such waits point to earlier units, which are taken by CTAs that run, so
// that they end.
//
// In a CTA, one warp takes units and waits for their inputs, two issue TMA loads of the factors' 64-element K slices
// into a ring, one (of the pair's first CTA) the MMAs, and eight drain the accumulator in blocks of 32 x 32, which leave
// by TMA through shared memory. g and u are kept for the backward pass in fp32, in blocks of 32 x 32 with the rows
// side by side, so that a warp writes and reads them in whole lines without shared memory. Every wait is bounded
// (soap_wait_limit); one that runs out sets SOAP_STATUS_TIMEOUT, the CTA drains its copies, frees its tensor memory and
// returns, and the last CTA then makes all results NaN.
#include <algorithm>
#include <atomic>

#include "../../include/layer.h"
#include "ffn.h"
#include "ffn_device.h"
#include "pair.h"
#include "profile.h"
#include "soap_internal.h"

namespace soap {
namespace ffn {
namespace {

using namespace tc;

enum Kind { kEnd = -1, kGated, kGrad, kOut, kWeight };

constexpr int kEpiWarps = 8;
constexpr int kLoadB = 2, kScout = 3, kFirstEpi = 4;  // warps
constexpr int kThreads = 32 * (kFirstEpi + kEpiWarps);
// registers of a launch's 168 per thread as the roles' warps share them: 4 x 72 + 8 x 216 = 12 x 168
constexpr int kFewRegisters = 72, kManyRegisters = 216;
constexpr int kStages = 6, kStage = 2 * kTile;
constexpr int kStaging = 4096;      // per epilogue warp: 2 blocks of 32 x 32 of 16 bits, 1 of fp32 (two of it and a stage
                                    // of the ring less: 2% longer)
constexpr int kPerTile = 2 * kEpiWarps;  // what a tile adds to its counters
// units that the roles of a pair may be apart, and more: 2 + 6 + 2 + 1 (every unit takes at least one of the ring's
// slots, of which each takes both CTAs' loading threads, and one of two accumulators)
constexpr int kKept = 16;
constexpr int kShort = 16;          // slices of a unit that is short
constexpr int kRun = 4;             // slices in a run of fp32 operands

struct Unit {
  int kind, group, prod;
  int m0, n0, M, N;  // of the result (a row phase: rows of the group)
  int start;         // the group's first row
  int s0, s1;        // slices
  int splits, part, slot, tile;  // parts along K; this one, its place among the partial sums, and its tile's
  int tiles;                     // places between two parts' sums
  int row_tile, block;           // among all groups'
  int need;                      // the group's row tiles
};
constexpr int kSmem = 1024 + kStages * kStage + kEpiWarps * kStaging + kKept * (int)sizeof(Unit) + 256;
static_assert(kSmem <= 232448, "shared memory");

// kind::f16, M = 256: D = f32, A and B bf16 or f16; bits 15 and 16 mark MN-major operands.
__host__ __device__ constexpr uint32_t idesc_16(bool bf16, int a_mn, int b_mn, int n) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (static_cast<uint32_t>(a_mn) << 15) |
         (static_cast<uint32_t>(b_mn) << 16) | (static_cast<uint32_t>(n >> 3) << 17) | ((256u >> 4) << 24);
}

// 32 columns at each of two places of this lane's accumulator row.
__device__ __forceinline__ void tmem_ld32x2(uint32_t t0, uint32_t t1, float (&v)[32], float (&w)[32]) {
  uint32_t r[64];
#define SOAP_LD32(o, at)                                                                                              \
  asm volatile(                                                                                                       \
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "                                                                       \
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "                                       \
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"                       \
      : "=r"(r[o]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]),    \
        "=r"(r[o + 7]), "=r"(r[o + 8]), "=r"(r[o + 9]), "=r"(r[o + 10]), "=r"(r[o + 11]), "=r"(r[o + 12]),             \
        "=r"(r[o + 13]), "=r"(r[o + 14]), "=r"(r[o + 15]), "=r"(r[o + 16]), "=r"(r[o + 17]), "=r"(r[o + 18]),          \
        "=r"(r[o + 19]), "=r"(r[o + 20]), "=r"(r[o + 21]), "=r"(r[o + 22]), "=r"(r[o + 23]), "=r"(r[o + 24]),          \
        "=r"(r[o + 25]), "=r"(r[o + 26]), "=r"(r[o + 27]), "=r"(r[o + 28]), "=r"(r[o + 29]), "=r"(r[o + 30]),          \
        "=r"(r[o + 31])                                                                                               \
      : "r"(at))
  SOAP_LD32(0, t0);
  SOAP_LD32(32, t1);
#undef SOAP_LD32
  // (the values pass through the wait, so that nothing reads them before it)
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 64; ++i) asm volatile("" : "+r"(r[i]));
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    v[i] = __uint_as_float(r[i]);
    w[i] = __uint_as_float(r[32 + i]);
  }
}

__device__ __forceinline__ void tmem_st16(uint32_t t, const float (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};\n\t"
      "tcgen05.wait::st.sync.aligned;" ::"f"(v[0]),
      "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]),
      "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "r"(t)
      : "memory");
}

__device__ __forceinline__ Unit unit_at(int p, const Args& a, const Head& h, const Groups& c) {
  const Plan& l = *a.plan;
  const bool dense = a.clips == nullptr;  // then all prefixes are 0 and everything there is
  Unit u{};
  const int phase = p >= h.first[2] ? 2 : p >= h.first[1] ? 1 : 0;
  int i = p - (phase == 2 ? h.first[2] : phase == 1 ? h.first[1] : 0);
  if (phase < 2) {
    u.slot = i;
    const int tiles = phase == 0 ? h.tiles[0] : h.tiles[1], wide = phase == 0 ? a.col_tile[0] : a.col_tile[1];
    u.N = phase == 0 ? a.width : a.hidden;
    u.kind = phase == 1 ? kOut : a.backward ? kGrad : kGated;
    u.splits = phase == 0 ? h.splits[0] : h.splits[1];
    u.tiles = tiles;
    u.part = i / tiles;
    i -= u.part * tiles;
    u.tile = i;
    const int nn = up_div(u.N, wide);
    int nm = up_div(a.rows, 256);
    u.M = a.rows;
    if (!dense) {
      if (c.held) {
        u.group = Groups::find(c.tiles, i / nn);
        u.row_tile = Groups::of(c.tiles, u.group);
        u.start = Groups::of(c.start, u.group);
        u.M = Groups::of(c.length, u.group);
        u.block = Groups::of(c.blocks, u.group);
      } else {
        u.group = group_of(l.row_tiles, a.groups, i / nn);
        u.row_tile = l.row_tiles[u.group];
        u.start = l.bounds[u.group];
        u.M = l.bounds[u.group + 1] - u.start;
        u.block = l.blocks[u.group];
      }
      nm = up_div(u.M, 256);
      i -= u.row_tile * nn;
    }
    int m, n;
    tile_place(i, nm, nn, m, n);
    u.need = nm;
    u.m0 = m * 256;
    u.n0 = n * wide;
    u.row_tile += m;
    u.block += m * 8;
    const int slices = a.slices[phase];
    u.s0 = (int)((int64_t)slices * u.part / u.splits);
    u.s1 = (int)((int64_t)slices * (u.part + 1) / u.splits);
  } else {
    const int each = a.each[0] + a.each[1] + a.each[2], q = i / each;
    u.kind = kWeight;
    u.tiles = each;
    int rows = a.rows, slots = 0;
    u.splits = h.parts;
    u.part = q;
    if (!dense) {
      if (c.held) {
        u.group = Groups::find(c.parts, q);
        u.part = q - Groups::of(c.parts, u.group);
        u.splits = Groups::of(c.part_count, u.group);
        slots = Groups::of(c.slots, u.group);
        u.start = Groups::of(c.start, u.group);
        rows = Groups::of(c.length, u.group);
      } else {
        u.group = group_of(l.parts, a.groups, q);
        u.part = q - l.parts[u.group];
        u.splits = l.parts[u.group + 1] - l.parts[u.group];
        slots = l.slots[u.group];
        u.start = l.bounds[u.group];
        rows = l.bounds[u.group + 1] - u.start;
      }
    }
    u.need = up_div(rows, 256);
    i -= q * each;
    u.tile = slots * each + i;
    u.slot = u.tile + u.part * each;
    u.prod = i >= a.each[0] + a.each[1] ? 2 : i >= a.each[0] ? 1 : 0;
    i -= u.prod == 2 ? a.each[0] + a.each[1] : u.prod == 1 ? a.each[0] : 0;
    u.M = a.wrows[u.prod];
    u.N = a.wcols[u.prod];
    int m, n;
    tile_place(i, up_div(u.M, 256), up_div(u.N, a.col_tile[2]), m, n);
    u.m0 = m * 256;
    u.n0 = n * a.col_tile[2];
    const int slices = up_div(rows, BK) << a.plane_bits;
    u.s0 = (int)((int64_t)slices * u.part / u.splits);
    u.s1 = (int)((int64_t)slices * (u.part + 1) / u.splits);
  }
  return u;
}

// Products of planes (of A's, of B's) that an fp32 product is made of, small ones first.
constexpr int kTerms = 6;
__device__ __forceinline__ int term_a(int t) { return (0x201100 >> (4 * (5 - t))) & 0xf; }
__device__ __forceinline__ int term_b(int t) { return (0x021010 >> (4 * (5 - t))) & 0xf; }

// The slices of a unit in the order in which all roles take them.
template <int TYPE>
struct Order {
  static constexpr bool kSplit = TYPE == SOAP_F32;
  static constexpr int kTermsOf = kSplit ? kTerms : 1;
  __device__ __forceinline__ static int end_of_run(int from, int s1) { return kSplit ? min(s1, from + kRun) : s1; }
};

// One factor's slices of a unit into the ring.
struct Loader {
  Ring st;
  uint32_t ring, bars;
  uint64_t *full, *empty;
  uint64_t lim;
};

template <int MN>
__device__ __forceinline__ void load_run(Loader& l, int from, int to, int kblocks, int k_at, const CUtensorMap* m0,
                                         const CUtensorMap* m1, int row, int z, uint32_t bytes, int bits, int planes, bool half) {
  for (; from < to; ++from) {
    // (slices of both planes one after the other, so that the other factor's second load comes from L2)
    const int kb = from >> bits;
    Ring& st = l.st;
    if (!(st.ok = mbar_wait(&l.empty[st.s], st.parity, l.lim))) return;
    if (bytes) expect_tx(&l.full[st.s], bytes);
    const bool second = kb >= kblocks;
    const int k = k_at + (second ? kb - kblocks : kb) * BK, zk = z + (from & planes);
    if (half)  // 64 of its rows (K-major: the map's boxes)
      tma_box(l.ring + st.s * kStage, second ? m1 : m0, l.bars + st.s * 8, MN ? row : k, MN ? k : row, zk);
    else
      load_tile<MN>(l.ring + st.s * kStage, second ? m1 : m0, l.bars + st.s * 8, row, k, zk);
    if (++st.s == kStages) {
      st.s = 0;
      st.parity ^= 1;
    }
  }
}

template <int A_MN, int B_MN>
__device__ __forceinline__ void issue(Ring& st, int count, uint32_t idesc, uint32_t ring, uint64_t* full, uint64_t* empty,
                                      uint32_t d, uint64_t lim) {
  uint32_t more = 0;
  for (; count > 0; --count) {
    if (!(st.ok = mbar_wait(&full[st.s], st.parity, lim))) return;
    tc_fence_after();
    const uint32_t as = ring + st.s * kStage, bs = as + kTile;
#pragma unroll
    for (int kk = 0; kk < BK / 16; ++kk) {
      umma_f16(d, tile_desc<A_MN>(as, kk), tile_desc<B_MN>(bs, kk), idesc, more);
      more = 1;
    }
    commit_pair(&empty[st.s]);
    if (++st.s == kStages) {
      st.s = 0;
      st.parity ^= 1;
    }
  }
}

// Rounds v into this lane's row of a staged block of 32 x 32.
template <typename T>
__device__ __forceinline__ void put(uint8_t* slot, const float (&v)[32], int lane) {
  constexpr int V = 16 / sizeof(T);
#pragma unroll
  for (int u = 0; u < 32 / V; ++u) {
    Pack<T, V> p;
#pragma unroll
    for (int e = 0; e < V; e += 2) from_pair(make_float2(v[u * V + e], v[u * V + e + 1]), p.v + e);
    *reinterpret_cast<Pack<T, V>*>(slot + (sizeof(T) == 4 ? at32(lane, u) : at16(lane, u))) = p;
  }
}

// The upper 8 bits of x's significand as bf16, and what is left in x, kLeast of it at least (of an infinity that, the
// difference of two infinities being a NaN, which fmaxf passes over).
__device__ __forceinline__ float upper(float& x) {
  const float hi = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
  x = copysignf(fmaxf(fabsf(x) - fabsf(hi), fabsf(x) * kLeast), hi);
  return hi;
}

__device__ __forceinline__ void fence_map(const CUtensorMap* m) {
  asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
}

template <int TYPE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    products_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Args a) {
  using T = typename Element<TYPE>::T;
  using O = Order<TYPE>;
  constexpr bool SPLIT = O::kSplit;
  constexpr int kAcc = SPLIT ? 1 : 2;  // accumulators
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* staging = smem + kStages * kStage;
  Unit* units = reinterpret_cast<Unit*>(staging + kEpiWarps * kStaging);
  uint64_t* full = reinterpret_cast<uint64_t*>(units + kKept);
  uint64_t* empty = full + kStages;
  uint64_t* acc_full = empty + kStages;
  uint64_t* acc_empty = acc_full + 2;
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(acc_empty + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_at + 1);
  volatile int* taken = reinterpret_cast<volatile int*>(tmem_at + 2);  // what the pair's first CTA tells the second
  // counts of units: known in this CTA, with their inputs there, begun by the first loading thread, given to the second CTA
  const uint32_t known_at = smem_u32(tmem_at + 2 + kKept), ready_at = known_at + 4, begun_at = known_at + 8,
                 given_at = known_at + 12;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)(blockIdx.x & 1);  // in the pair
  const uint64_t lim = a.wait_ns;          // bound of every wait (for another role of the pair: twice)

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], 2 * kEpiWarps);
    }
    *abort_flag = 0;
    set_ready(known_at, 0);
    set_ready(ready_at, 0);
    set_ready(begun_at, 0);
    set_ready(given_at, 0);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if ((warp == 0 || warp == kLoadB) && lane < 2) {
    const CUtensorMap* const first = warp == 0 ? (lane == 0 ? &maps.a0 : &maps.a1[0])
                                               : (lane == 0 ? &maps.w0[rank] : &maps.w1[0]);
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(first)) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_at)), "r"(512));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // both CTAs' barriers are ready
  tc_fence_after();
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the launch before has ended: so far, nothing of it was read
  const uint32_t tmem = *tmem_at;

  if (warp < kFirstEpi) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegisters));
  if (warp == kScout) {
    bool ok = rank != 0 || !a.hold || flag_wait(a.hold, lim);  // a flag that nothing sets: every role's wait runs out
    const Plan& l = *a.plan;
    // (from memory: working it out here for one group took longer, its instructions being fetched for this once)
    const Head head{l.total, {0, l.first[1], l.first[2]}, {l.tiles[0], l.tiles[1]}, {l.splits[0], l.splits[1]}, l.parts[1]};
    uint32_t peer;
    asm("mapa.shared::cluster.u32 %0, %1, 1;" : "=r"(peer) : "r"(smem_u32(tmem_at + 2)));
    Groups groups;
    groups.load(a);
    // Short units: the next one is taken as this one becomes known, and not only when its loads begin, so that the trip to
    // the list's counter is over by then. (Of long ones a pair would hold one while others end.)
    bool ahead = false;
    int held = -1;
    for (int m = 0; ok; ++m) {
      int p = -1;
      if (lane == 0) {
        if (rank == 0) {
          if ((ok = wait_given(begun_at, ahead ? m - 1 : m, 2 * lim))) {
            p = ahead ? held : atomicAdd(&a.plan->next, 1);
            if (p >= head.total) p = -1;
            asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(peer + 4 * (m % kKept)), "r"(p) : "memory");
            asm volatile("st.release.cluster.shared::cluster.b32 [%0], %1;" ::"r"(peer + 4 * kKept + 12), "r"(m + 1)
                         : "memory");
          }
        } else if ((ok = wait_given(given_at, m + 1, 2 * lim))) {
          p = taken[m % kKept];
        }
        ok = ok && !*abort_flag;
      }
      if (!(ok = __shfl_sync(0xffffffffu, ok, 0))) break;
      p = __shfl_sync(0xffffffffu, p, 0);
      Unit u{};
      if (p < 0)
        u.kind = kEnd;
      else
        u = unit_at(p, a, head, groups);
      if (lane == 0) {
        units[m % kKept] = u;
        set_ready(known_at, m + 1);
        ahead = p >= 0 && (u.s1 - u.s0) * O::kTermsOf <= kShort;
        if (ahead && rank == 0) held = atomicAdd(&a.plan->next, 1);
      }
      const bool free = u.kind < kOut || groups.done(a);
      if (lane == 0) {
        if (!free)
          ok = u.kind == kOut ? wait_done(a.done_row + u.row_tile, a.stored, lim)
                              : wait_done(a.done_group + u.group, a.stored * u.need, lim);
        if (ok) {
          asm volatile("fence.proxy.async;" ::: "memory");  // what other CTAs stored, before copies of it
          set_ready(ready_at, m + 1);
        }
      }
      ok = __shfl_sync(0xffffffffu, ok, 0);
      if (p < 0) break;
    }
    if (!ok) {
      *abort_flag = 1;
      if (lane == 0 && a.status) atomicOr(a.status, kStatusTimeout);
    }
  } else if (warp == 0 || warp == kLoadB) {
    if (lane == 0) {
      const bool is_b = warp == kLoadB;
      Loader l;
      l.st.parity = 1;  // of a slot's release
      l.ring = smem_u32(smem) + (is_b ? kTile : 0);
      l.bars = in_leader(full);
      l.full = full;
      l.empty = empty;
      l.lim = 2 * lim;
      int used = 0;  // slots filled so far (up to kStages)
      for (int m = 0; !*abort_flag; ++m) {
        // weights do not wait for the phase before
        if (!(l.st.ok = wait_ready(known_at, m + 1, 2 * lim))) break;
        const Unit u = units[m % kKept];
        if (u.kind == kEnd) break;
        if ((!is_b || u.kind == kWeight) && !(l.st.ok = wait_ready(ready_at, m + 1, 2 * lim))) break;
        if (!is_b) set_ready(begun_at, m + 1);
        const CUtensorMap *m0, *m1;
        int row, z = 0, planes = 0, kblocks, k_at = 0;
        const int narrow = a.narrow[u.kind == kWeight ? 2 : u.kind == kOut];
        bool mn, of_planes = false;  // whether the planes are this factor's
        if (u.kind == kWeight) {
          const int which = is_b ? a.wb[u.prod] : a.wa[u.prod];
          m0 = m1 = a.clips ? a.clips + u.group * kClips + which : &maps.clip[which];
          if (a.clips) fence_map(m0);
          row = is_b ? u.n0 + rank * (128 >> narrow) : u.m0 + rank * 128;
          of_planes = which >= kInH;
          kblocks = INT_MAX;
          k_at = u.start;
          planes = 1;
          mn = true;
        } else {
          const int phase = u.kind == kOut;
          kblocks = a.kblocks[phase];
          if (!is_b) {
            m0 = phase ? &maps.a1[0] : &maps.a0;
            m1 = phase ? &maps.a1[1] : m0;
            row = u.start + u.m0 + rank * 128;
            planes = 1;
            of_planes = phase;
            mn = false;
          } else {
            m0 = phase ? &maps.w1[0] : &maps.w0[u.kind == kGated ? rank : 0];
            m1 = phase ? &maps.w1[1] : m0;
            row = u.kind == kGated ? u.n0 : u.n0 + rank * (128 >> narrow);
            z = u.group;
            planes = a.groups;
            mn = a.b_columns[phase];
          }
        }
        // (also rows that the group has not in the second CTA's half of the tile: a thread that loads nothing is held back
        // by nothing, and one that falls two rounds of the ring behind takes another round's parity for its own)
        const uint32_t bytes = rank != 0 || is_b ? 0 : 2 * (kTile + (kTile >> narrow));
        const int bits = u.kind >= kOut ? a.plane_bits : 0, plane = of_planes ? bits : 0;
        used = min(used + (u.s1 - u.s0) * O::kTermsOf, kStages);
        for (int kb = u.s0; kb < u.s1 && l.st.ok;) {
          const int to = O::end_of_run(kb, u.s1);
          for (int t = 0; t < O::kTermsOf && l.st.ok; ++t) {
            const int zt = z + (SPLIT ? (is_b ? term_b(t) : term_a(t)) * planes : 0);
            if (mn)
              load_run<1>(l, kb, to, kblocks, k_at, m0, m1, row, zt, bytes, bits, plane, is_b && narrow);
            else
              load_run<0>(l, kb, to, kblocks, k_at, m0, m1, row, zt, bytes, bits, plane, is_b && narrow);
          }
          kb = to;
        }
        if (!l.st.ok) break;
      }
      Ring& st = l.st;
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
        if (!(st.ok = wait_ready(known_at, m + 1, 2 * lim))) break;
        const Unit& u = units[m % kKept];
        const int kind = u.kind, s1 = u.s1;
        int kb = u.s0;
        if (kind == kEnd) break;
        const bool a_mn = kind == kWeight, b_mn = kind == kWeight || a.b_columns[kind == kOut];
        const uint32_t idesc = idesc_16(TYPE != SOAP_F16, a_mn, b_mn, 256 >> a.narrow[kind == kWeight ? 2 : kind == kOut]);
        for (; kb < s1 && st.ok; ++n) {
          const int to = O::end_of_run(kb, s1), ac = n % kAcc, count = (to - kb) * O::kTermsOf;
          if (n >= kAcc && !(st.ok = mbar_wait(&acc_empty[ac], ((n / kAcc) & 1) ^ 1, 2 * lim))) break;
          tc_fence_after();
          const uint32_t d = tmem + static_cast<uint32_t>(ac * 256);
          if (a_mn)
            issue<1, 1>(st, count, idesc, ring, full, empty, d, 2 * lim);
          else if (b_mn)
            issue<0, 1>(st, count, idesc, ring, full, empty, d, 2 * lim);
          else
            issue<0, 0>(st, count, idesc, ring, full, empty, d, 2 * lim);
          if (st.ok) commit_pair(&acc_full[ac]);
          kb = to;
        }
      }
      if (!st.ok) *abort_flag = 1;
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegisters));
    const int q = warp & 3;           // accumulator lanes 32 q .. 32 q + 31
    const int half = (warp - kFirstEpi) / 4;  // of the columns
    uint8_t* stage = staging + (warp - kFirstEpi) * kStaging;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(32 * q) << 16);
    const int pre_cols = (a.width + 31) / 32;  // blocks
    int n = 0;  // accumulators so far
    int k = 0;  // staged blocks so far
    bool ok = true;
    // A place for a block of `half` (2 KB: 16-bit elements) or whole size (fp32), whose copies out have been read: two of
    // one, one of the other, and no copy on its way where one size follows the other.
    bool halves = true;
    auto next_slot = [&](bool half) {
      if (lane == 0) {
        if (half && halves)
          sent_read<1>();
        else
          sent_read<0>();
      }
      halves = half;
      __syncwarp();
      return stage + (half ? (k++ & 1) * 2048 : 0);
    };
    auto send = [&](const CUtensorMap* map, const uint8_t* slot, int x, int y, int z) {
      before_tma();
      __syncwarp();
      if (lane == 0) send_block(map, smem_u32(slot), x, y, z);
    };
    for (int m = 0;; ++m) {
      if (lane == 0) ok = wait_ready(known_at, m + 1, 2 * lim);
      if (!(ok = __shfl_sync(0xffffffffu, ok, 0))) break;
      const Unit u = units[m % kKept];
      if (u.kind == kEnd) break;
      const int r0 = u.m0 + rank * 128 + 32 * q;
      // its columns in blocks of 32 (of g and u 64 each, else 128, or half of that): none below the last row, and to the last column
      const bool gated = u.kind == kGated;
      const int narrow = a.narrow[u.kind == kWeight ? 2 : u.kind == kOut];
      const int most = (gated ? 2 : 4) >> narrow, c0 = u.n0 + 32 * most * half;
      const int blocks = r0 < u.M && c0 < u.N ? min(most, (u.N - c0 + 31) / 32) : 0;
      const uint32_t t0 = lanes + 32 * most * half, u_at = 128 >> narrow;  // (u's columns behind g's)
      const CUtensorMap* const clips = a.clips ? a.clips + u.group * kClips : maps.clip;
      if (a.clips && lane == 0) {
        if (u.kind <= kGrad) fence_map(clips + kH);
        if (u.kind == kGrad) fence_map(clips + kDG), fence_map(clips + kDU);
        if (u.kind == kOut) fence_map(clips + kY);
      }

      // h, dg or du: to the second phase's (and the weights' gradients') operand
      auto to_operand = [&](Clip which, float (&v)[32], int col) {
#pragma unroll 1  // (instructions that are fetched once)
        for (int plane = 0; plane <= (SPLIT ? 2 : a.plane_bits); ++plane) {
          uint8_t* const slot = next_slot(true);
          if constexpr (SPLIT) {
            float w[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) w[j] = upper(v[j]);
            put<__nv_bfloat16>(slot, w, lane);
          } else {
            put<T>(slot, v, lane);
            if (plane < a.plane_bits) {
#pragma unroll
              for (int j = 0; j < 32; ++j) v[j] = rest_of(v[j], from_f32<T>(v[j]));
            }
          }
          send(clips + which, slot, col, u.start + r0, plane);
        }
      };
      auto to_result = [&](const float (&v)[32], int col) {
        uint8_t* const slot = next_slot(sizeof(T) == 2);
        const bool weight = u.kind == kWeight;
        if (weight ? a.dw_tma[u.prod] : a.y_tma) {
          put<T>(slot, v, lane);
          if (weight)
            send(&maps.dw[u.prod], slot, col, r0, u.group);
          else
            send(clips + kY, slot, col, u.start + r0, 0);
        } else {
          if (lane == 0) sent_read<0>();  // (blocks stored here are not counted among the copies)
          __syncwarp();
          T* const to = weight ? static_cast<T*>(a.dw[u.prod]) + (int64_t)u.group * a.stride_dw[u.prod] : static_cast<T*>(a.y);
          const int64_t ld = weight ? a.ld_dw[u.prod] : a.ld_y;
          store_user(slot, v, to + (int64_t)(weight ? r0 : u.start + r0) * ld + col, ld, min(32, u.M - r0),
                     min(32, u.N - col), false, lane);
          before_tma();
        }
      };
      auto pre_at = [&](int which, int col) {
        return reinterpret_cast<float4*>(a.pre) +
               ((((int64_t)u.block + (r0 - u.m0) / 32) * 2 + which) * pre_cols + col / 32) * 256 + lane;
      };
      // block i of g and u
      auto finish_gated = [&](int i, float (&v)[32], float (&w)[32]) {
        const int col = c0 + 32 * i;
        if (a.pre) {
          put_lines(pre_at(0, col), v);
          put_lines(pre_at(1, col), w);
        }
        if (a.act == LAYER_SILU)
          gate<LAYER_SILU>(v, w);
        else
          gate<LAYER_GELU>(v, w);
        to_operand(kH, v, col);
      };
      // block i of dh, whose g and u are in g and up; then the next block's (next, if any) come
      auto finish_grad = [&](int i, float (&v)[32], float (&g)[32], float (&up)[32], int next) {
        const int col = c0 + 32 * i;
        if (a.act == LAYER_SILU)
          gate_back<LAYER_SILU>(g, up, v);
        else
          gate_back<LAYER_GELU>(g, up, v);
        to_operand(kDG, g, col);
        if (next < blocks) get_lines(pre_at(0, c0 + 32 * next), g);
        if (a.params) to_operand(kH, up, col);
        if (next < blocks) get_lines(pre_at(1, c0 + 32 * next), up);
        to_operand(kDU, v, col);
      };
      // Parts along K: each stores its sums, and the one that is the last to store a block adds up all of them in the
      // parts' order. A part begins with a block of its own, so that parts that end together finish different blocks.
      const int phase = u.kind == kWeight ? 2 : u.kind == kOut;
      const int share = rank * kEpiWarps + warp - kFirstEpi;
      auto partial_at = [&](int part, int i) {
        return reinterpret_cast<float4*>(a.partial[phase]) +
               (((int64_t)(u.slot + (part - u.part) * u.tiles) * kPerTile + share) * 4 + i) * 256 + lane;
      };
      auto parts_stored = [&] {  // this part's sums come before its counts
        __threadfence();
        __syncwarp();
      };
      auto last_part = [&](int i) {
        int there = 0;
        if (lane == 0) there = atomicAdd(a.count[phase] + (u.tile * kPerTile + share) * 4 + i, 1);
        __threadfence();
        return __shfl_sync(0xffffffffu, there, 0) == u.splits - 1;
      };
      auto add_parts = [&](int i, float (&v)[32]) {
        get_lines_l2(partial_at(0, i), v);
        int s = 1;
        for (; s + 1 < u.splits; s += 2) {  // (two on their way at a time)
          float x[32], y[32];
          get_lines_l2(partial_at(s, i), x);
          get_lines_l2(partial_at(s + 1, i), y);
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = (v[j] + x[j]) + y[j];
        }
        if (s < u.splits) {
          float x[32];
          get_lines_l2(partial_at(s, i), x);
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] += x[j];
        }
      };
      auto wait_acc = [&](int ac) {
        ok = mbar_wait(&acc_full[ac], (n / kAcc) & 1, 2 * lim) && !*abort_flag;
        tc_fence_after();
        return ok = __all_sync(0xffffffffu, ok);
      };
      auto release_acc = [&](int ac) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0)
          asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_leader(&acc_empty[ac])) : "memory");
      };
      // stored: what waits for these blocks may go on
      auto report = [&](int count) {
        if (u.kind <= kGrad && lane == 0 && count > 0) {
          sent_done<0>();
          asm volatile("fence.acq_rel.gpu;" ::: "memory");  // (once for both)
          asm volatile("red.relaxed.gpu.global.add.s32 [%0], %1;" ::"l"(a.done_row + u.row_tile), "r"(count) : "memory");
          asm volatile("red.relaxed.gpu.global.add.s32 [%0], %1;" ::"l"(a.done_group + u.group), "r"(count) : "memory");
        }
      };
      const int turn = u.splits > 1 && blocks > 0 ? u.part % blocks : 0;
      auto turned = [&](int i) { return i + turn < blocks ? i + turn : i + turn - blocks; };
      int finished = most - blocks;  // (blocks that hold nothing count for the first part)
      if (u.part > 0) finished = 0;
      // fp32: the runs' sums are added up in the tensor memory's other half, 16 columns at a time
      const bool summed = SPLIT && u.s1 - u.s0 > kRun;
      if (summed) {
        for (int kb = u.s0; kb < u.s1; kb = O::end_of_run(kb, u.s1), ++n) {
          if (!wait_acc(n % kAcc)) break;
#pragma unroll 1
          for (int i = 0; i < (gated ? 4 : 2) * blocks; ++i) {
            const uint32_t at = t0 + (gated ? u_at * (i & 1) + 16 * (i >> 1) : 16 * i);
            float v[16], w[16];
            if (kb == u.s0) {
              tmem_ld16(at, v);
            } else {
              tmem_ld16x2(at, at + 256, v, w);
#pragma unroll
              for (int j = 0; j < 16; ++j) v[j] += w[j];
            }
            tmem_st16(at + 256, v);
          }
          release_acc(n % kAcc);
        }
        if (!ok) break;
      }
      const int ac = n % kAcc;
      const uint32_t t = t0 + static_cast<uint32_t>(summed ? 256 : ac * 256);
      const bool whole = u.splits == 1;
      float g[32], up[32];  // of the block that is next
      if (u.kind == kGrad && whole && blocks > 0) {  // (the first block's come while the products are formed)
        get_lines(pre_at(0, c0), g);
        get_lines(pre_at(1, c0), up);
      }
      if (!summed && !wait_acc(ac)) break;
      if (!whole) {
        for (int i = 0; i < (gated ? 2 * blocks : blocks); ++i) {  // (g's and u's blocks in turn)
          float v[32];
          tmem_ld32(t + (gated ? u_at * (i & 1) + 32 * (i >> 1) : 32 * i), v);
          put_lines(partial_at(u.part, i), v);
        }
        if (!summed) release_acc(ac);
        parts_stored();
      } else if (blocks == 0 && !summed) {
        release_acc(ac);
      }
      for (int j = 0; j < blocks; ++j) {
        const int i = turned(j);
        if (!whole && !last_part(i)) continue;
        float v[32];
        if (gated) {
          float w[32];
          if (whole) {
            tmem_ld32x2(t + 32 * i, t + u_at + 32 * i, v, w);
            if (j + 1 == blocks && !summed) release_acc(ac);
          } else {
            add_parts(2 * i, v);
            add_parts(2 * i + 1, w);
          }
          finish_gated(i, v, w);
        } else {
          if (whole) {
            tmem_ld32(t + 32 * i, v);
            if (j + 1 == blocks && !summed) release_acc(ac);
          } else {
            add_parts(i, v);
          }
          if (u.kind == kGrad) {
            if (!whole) {
              get_lines(pre_at(0, c0 + 32 * i), g);
              get_lines(pre_at(1, c0 + 32 * i), up);
            }
            finish_grad(i, v, g, up, whole ? i + 1 : blocks);
          } else {
            to_result(v, c0 + 32 * i);
          }
        }
        ++finished;
      }
      if (!summed) ++n;
      report(finished);
      __syncwarp();
    }
    if (lane == 0) sent_done<0>();
    if (!ok) {
      *abort_flag = 1;
      if (lane == 0 && a.status) atomicOr(a.status, kStatusTimeout);
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
    if (*abort_flag) atomicOr(&a.plan->gave_up, 1);
    __threadfence();  // this CTA's results (and its word) come before its count
    const bool last = atomicAdd(&a.plan->through, 1) == (int)gridDim.x - 1;
    __threadfence();
    *abort_flag = last && atomicOr(&a.plan->gave_up, 0) != 0;
  }
  __syncthreads();
  if (*abort_flag) {
    if (a.pre && !a.backward) {
#pragma unroll 1
      for (int64_t i = threadIdx.x; i < a.pre_elems / 4; i += kThreads)
        reinterpret_cast<float4*>(a.pre)[i] = make_float4(NAN, NAN, NAN, NAN);
    }
    const T nan = from_f32<T>(NAN);
    for (int r = warp; r < a.rows; r += kThreads / 32)
      for (int c = lane; c < a.hidden; c += 32) static_cast<T*>(a.y)[(int64_t)r * a.ld_y + c] = nan;
    for (int p = 0; p < 3 && a.params; ++p)
      for (int g = 0; g < a.groups; ++g)
        for (int r = warp; r < a.wrows[p]; r += kThreads / 32)
          for (int c = lane; c < a.wcols[p]; c += 32)
            static_cast<T*>(a.dw[p])[(int64_t)g * a.stride_dw[p] + (int64_t)r * a.ld_dw[p] + c] = nan;
  }
}

// ---- before the products ----

constexpr int kPrepThreads = 256;

// bounds[g]: the largest of offsets[0 .. g], within 0 .. rows. All of the CTA's threads; a barrier at the end.
__device__ void find_bounds(const Args& a, int (&buf)[2][kMaxGroups + 1], int*& bounds, bool tell) {
  bool off = false;
  for (int i = threadIdx.x; i <= a.groups; i += kPrepThreads) {
    const int v = a.offsets ? a.offsets[i] : i == 0 ? 0 : a.rows;
    off |= v < 0 || v > a.rows || (a.offsets && i > 0 && v < a.offsets[i - 1]);
    buf[0][i] = min(max(v, 0), a.rows);
  }
  if (tell && off && a.status) atomicOr(a.status, kStatusRange);
  int at = 0;
  for (int d = 1; d <= a.groups; d *= 2, at ^= 1) {
    __syncthreads();
    for (int i = threadIdx.x; i <= a.groups; i += kPrepThreads) buf[at ^ 1][i] = max(buf[at][i], i >= d ? buf[at][i - d] : 0);
  }
  __syncthreads();
  bounds = buf[at];
}

template <bool SPLIT>
__device__ __forceinline__ void copy_operands(const CopyJobs& jobs, const int* bounds) {
  for (int j = 0; j < jobs.n; ++j) {
    const CopyJob& c = jobs.job[j];
    const int chunks = c.ld_out / 8;
    const int64_t all = c.matrices * c.rows * chunks;
    for (int64_t i = (int64_t)blockIdx.x * kPrepThreads + threadIdx.x; i < all; i += (int64_t)gridDim.x * kPrepThreads) {
      const int64_t row = i / chunks, m = row / c.rows, r = row - m * c.rows;
      if (c.of_groups && bounds[m + 1] == bounds[m]) continue;  // nothing reads them
      const int col = (int)(i - row * chunks) * 8, n = min(8, c.inner - col);
      const int64_t from = m * c.stride + r * c.ld + col;
      Pack<uint16_t, 8> out[SPLIT ? 3 : 1];
      alignas(16) float in[SPLIT ? 8 : 1];
      if constexpr (SPLIT) {
        const float* const p = static_cast<const float*>(c.src) + from;
        if (n == 8 && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
          *reinterpret_cast<float4*>(in) = *reinterpret_cast<const float4*>(p);
          *reinterpret_cast<float4*>(in + 4) = *reinterpret_cast<const float4*>(p + 4);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) in[e] = e < n ? p[e] : 0.f;
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (SPLIT) {
          float x = in[e];
          // (a NaN's first plane stays one without its lower bits)
          const uint32_t quiet = x != x ? 0x40u : 0u;
#pragma unroll
          for (int p = 0; p < 3; ++p) out[p].v[e] = (uint16_t)((__float_as_uint(upper(x)) >> 16) | (p == 0 ? quiet : 0u));
        } else {
          out[0].v[e] = e < n ? static_cast<const uint16_t*>(c.src)[from + e] : (uint16_t)0;
        }
      }
#pragma unroll
      for (int p = 0; p < (SPLIT ? 3 : 1); ++p)
        *reinterpret_cast<Pack<uint16_t, 8>*>(c.dst + p * c.plane + row * c.ld_out + col) = out[p];
    }
  }
}

// All CTAs: `rows` rows of `cols` elements become 0; from row `first` on those that follow row `last`.
template <typename T>
__device__ __forceinline__ void zero_rows(T* p, int64_t ld, int64_t rows, int cols, int64_t first, int64_t last) {
  const bool whole = reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * sizeof(T) % 16 == 0;
  const int step = whole ? 16 / (int)sizeof(T) : 1;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    T* const row = p + (r < first ? r : r - first + last) * ld;
    for (int c = threadIdx.x * step; c < cols; c += kPrepThreads * step) {
      if (whole && c + step <= cols) {
        *reinterpret_cast<uint4*>(row + c) = make_uint4(0, 0, 0, 0);
      } else {
        for (int e = c; e < min(cols, c + step); ++e) row[e] = from_f32<T>(0.f);
      }
    }
  }
}

// The first CTA: the plan and zeros for the counters. All: the groups' maps, zeros for rows of no group and for the
// gradients of groups without rows.
template <typename T>
__global__ void __launch_bounds__(kPrepThreads) prepare_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Args a, const __grid_constant__ CopyJobs jobs) {
  __shared__ int buf[2][kMaxGroups + 1];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the products' CTAs set themselves up meanwhile
  int* bounds;
  find_bounds(a, buf, bounds, blockIdx.x == 0);
  if (blockIdx.x == 0) {
    Plan& l = *a.plan;
    for (int i = threadIdx.x; i < a.done_words; i += kPrepThreads) a.done_row[i] = 0;
    for (int i = threadIdx.x; i <= a.groups; i += kPrepThreads) l.bounds[i] = bounds[i];
    if (threadIdx.x < 32) {
      const int lane = threadIdx.x;
      auto length = [&](int g) { return g < a.groups ? bounds[g + 1] - bounds[g] : 0; };
      int some = 0;
      for (int g = 0; g < a.groups; g += 32) some += __popc(__ballot_sync(0xffffffffu, length(g + lane) > 0));
      const int each = a.each[0] + a.each[1] + a.each[2], most = some > 0 && each > 0 ? a.pool / some / each : 0;
      int tiles = 0, blocks = 0, parts = 0, slots = 0;  // of the groups before
      for (int g0 = 0; g0 <= a.groups; g0 += 32) {
        const int g = g0 + lane, len = length(g);
        const int n = a.params ? parts_of(up_div(len, BK) << a.plane_bits, most, a.products) : 0;
        int4 v = make_int4(up_div(len, a.row_tile), up_div(len, 32), n, n > 1 ? n : 0);
        const int4 own = v;
        for (int d = 1; d < 32; d *= 2) {
          const int4 o = make_int4(__shfl_up_sync(0xffffffffu, v.x, d), __shfl_up_sync(0xffffffffu, v.y, d),
                                   __shfl_up_sync(0xffffffffu, v.z, d), __shfl_up_sync(0xffffffffu, v.w, d));
          if (lane >= d) v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
        }
        if (g <= a.groups) {
          l.row_tiles[g] = tiles + v.x - own.x;
          l.blocks[g] = blocks + v.y - own.y;
          l.parts[g] = parts + v.z - own.z;
          l.slots[g] = slots + v.w - own.w;
        }
        tiles += __shfl_sync(0xffffffffu, v.x, 31);
        blocks += __shfl_sync(0xffffffffu, v.y, 31);
        parts += __shfl_sync(0xffffffffu, v.z, 31);
        slots += __shfl_sync(0xffffffffu, v.w, 31);
      }
      if (lane == 0) {
        l.next = l.through = l.gave_up = 0;
        const Head h = head_of(a, tiles, parts);
        l.total = h.total;
        for (int p = 0; p < 3; ++p) l.first[p] = h.first[p];
        for (int p = 0; p < 2; ++p) l.tiles[p] = h.tiles[p], l.splits[p] = h.splits[p];
      }
    }
  }
  if (a.clips) {
    const CUtensorMap* const from = maps.clip;
    for (int i = blockIdx.x * kPrepThreads + threadIdx.x; i < a.groups * kClips; i += gridDim.x * kPrepThreads) {
      const int g = i / kClips, c = i - g * kClips;
      if (!a.backward && c > kY) continue;
      const uint4* src = reinterpret_cast<const uint4*>(from + c);
      uint4* dst = reinterpret_cast<uint4*>(const_cast<CUtensorMap*>(a.clips) + i);
#pragma unroll
      for (int w = 0; w < 8; ++w) dst[w] = src[w];
      // rows end with the group's (of a group without rows nothing is ever copied)
      asm volatile("tensormap.replace.tile.global_dim.global.b1024.b32 [%0], 1, %1;" ::"l"(reinterpret_cast<uint64_t>(dst)),
                   "r"(max(bounds[g + 1], 1))
                   : "memory");
      asm volatile("fence.proxy.tensormap::generic.release.gpu;" ::: "memory");
    }
  }
  copy_operands<sizeof(T) == 4>(jobs, bounds);
  if (!a.offsets && a.rows > 0) return;
  const int first = bounds[0], last = bounds[a.groups];
  const int64_t outside = first + (a.rows - last);
  zero_rows(static_cast<T*>(a.y), a.ld_y, outside, a.hidden, first, last);
  if (!a.params) return;
  for (int g = 0; g < a.groups; ++g) {
    if (bounds[g + 1] > bounds[g]) continue;
    for (int p = 0; p < 3; ++p)
      zero_rows(static_cast<T*>(a.dw[p]) + (int64_t)g * a.stride_dw[p], a.ld_dw[p], a.wrows[p], a.wcols[p], a.wrows[p], 0);
  }
}

template <int TYPE>
cudaError_t launch(const Maps& maps, const Args& a, int64_t units, cudaStream_t s) {
  // per device: the pairs that are resident at once, found (with the kernel's shared-memory attribute set) on the
  // first launch there
  static std::atomic<int> pairs_of[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(2);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int pairs = dev < 64 ? pairs_of[dev].load(std::memory_order_relaxed) : 0;
  if (pairs == 0) {
    e = cudaFuncSetAttribute(products_kernel<TYPE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    e = cudaOccupancyMaxActiveClusters(&pairs, products_kernel<TYPE>, &cfg);
    if (e != cudaSuccess) return e;
    if (pairs < 1) return cudaErrorLaunchOutOfResources;
    if (dev < 64) pairs_of[dev].store(pairs, std::memory_order_relaxed);
  }
  cfg.gridDim = dim3((unsigned)(2 * std::max<int64_t>(1, std::min<int64_t>(pairs, units))));
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, products_kernel<TYPE>, maps, a);
}

}  // namespace

cudaError_t prepare(const Maps& maps, const Args& a, const CopyJobs& jobs, int64_t chunks, int type, cudaStream_t s) {
  // dense: nothing but the plan; groups: as many CTAs as rows and gradients to zero can keep busy; copies: as they can
  int64_t ctas = a.offsets || a.rows == 0 ? 304 : 1;
  if (jobs.n > 0) ctas = std::max(ctas, std::min<int64_t>(kSms * 8, (chunks + kPrepThreads - 1) / kPrepThreads));
  if (type == SOAP_F32)
    prepare_kernel<float><<<(unsigned)ctas, kPrepThreads, 0, s>>>(maps, a, jobs);
  else if (type == SOAP_BF16)
    prepare_kernel<__nv_bfloat16><<<(unsigned)ctas, kPrepThreads, 0, s>>>(maps, a, jobs);
  else
    prepare_kernel<__half><<<(unsigned)ctas, kPrepThreads, 0, s>>>(maps, a, jobs);
  return cudaGetLastError();
}

cudaError_t run(const Maps& maps, const Args& a, int type, int64_t units, cudaStream_t s) {
  return type == SOAP_F32    ? launch<SOAP_F32>(maps, a, units, s)
         : type == SOAP_BF16 ? launch<SOAP_BF16>(maps, a, units, s)
                             : launch<SOAP_F16>(maps, a, units, s);
}

}  // namespace ffn
}  // namespace soap
