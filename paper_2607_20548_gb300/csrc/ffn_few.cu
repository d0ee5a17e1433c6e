// The gated feed-forward block's forward pass for few rows (of 16-bit types): a decode batch, or experts with a few
// rows each, bound by the weights' bytes.
//
// The products are turned: a weight's 128 output features are the tensor core's rows, 16 to 128 of the block's rows its
// columns, so that shared memory holds weights and hardly anything else, and every lane of the accumulator holds values
// (with the rows as the tensor core's rows, in ffn_steps.cu, 24 rows of 2048 x 8192 took 48 us in place of 36). In the
// first phase the 128 features are 64 of g and the same 64 of u; the warps that hold u's hand them over through shared
// memory. An MMA that adds to the accumulator of the one before takes 140 cycles however narrow: the slices' four go to
// accumulators of their own, which the epilogue adds up.
//
// Where h is kept as two planes, its rounding to the type and what that leaves, both products come from one load of the
// weights, and h's rounding does not reach y.
//
// A CTA per SM takes units from one list, as in ffn_steps.cu: the first phase's tiles, then parts along K of the
// second's. One warp takes units, one loads weights (which wait for nothing: while the first phase ends, the ring, all
// of shared memory, fills with the second's), one loads rows, one issues the MMAs, four drain the accumulators.
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

enum Kind { kEnd = -1, kGated, kOut };

constexpr int kEpiWarps = 4;
constexpr int kLoadRows = 2 + kEpiWarps, kScout = kLoadRows + 1;  // warps
constexpr int kThreads = 32 * (kScout + 1);
constexpr int kKept = 32;  // units that the roles may be apart, and more: 1 + the ring's slots + 2 + 1

struct Unit {
  int kind, group;
  int n0, m0, M, start;          // first feature, first row in the group; the group's rows, its first
  int s0, s1;                    // slices
  int splits, part, slot, tile;  // parts along K; this one, its place among the partial sums, and its tile's
  int tiles;                     // places between two parts' sums
  int row_tile, block;           // among all groups'
  int pad;
};

template <int NT>
struct Config {
  static constexpr int kRowsTile = NT * 128;           // 64 elements of each of NT rows
  static constexpr int kRing = 204800;
  static constexpr int kMostStages = kRing / (kTile + kRowsTile);
  static constexpr int kAcc = NT <= 64 ? 4 : 2;        // accumulators of a unit
  static constexpr int kChunk = NT < 32 ? NT : 32;     // rows that a thread drains at a time
  static constexpr int kChunks = NT / kChunk;
  static constexpr uint32_t kColumns = 2 * kAcc * NT;  // of tensor memory
  static constexpr int kSmem = 1024 + kRing + 2 * 32 * 32 * 4 + kKept * (int)sizeof(Unit) + 512;
  static_assert(kSmem <= 232448 && kMostStages + 4 <= kKept, "shared memory");
};

__host__ __device__ constexpr uint32_t idesc_few(bool bf16, int a_mn, int n) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (static_cast<uint32_t>(a_mn) << 15) |
         (static_cast<uint32_t>(n >> 3) << 17) | ((128u >> 4) << 24);
}

__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate));
}

__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}

// N columns of this lane's accumulator row.
template <int N>
__device__ __forceinline__ void drain(uint32_t t, float (&v)[N]) {
  if constexpr (N == 32) {
    tmem_ld32(t, v);
  } else {
    tmem_ld16(t, v);
  }
}

// A unit as all lanes of a warp work it out. Units go group by group, and a group's row by row of feature tiles: the
// row tiles of a group with more than one take the same weights one after another.
template <int NT>
__device__ __forceinline__ Unit unit_at(int p, const Args& a, const Head& h, const Groups& c) {
  const Plan& l = *a.plan;
  const bool dense = a.offsets == nullptr;
  Unit u{};
  const int phase = p >= h.first[1];
  int i = phase ? p - h.first[1] : p;
  const int wide = phase ? 128 : 64, N = phase ? a.hidden : a.width;
  u.kind = phase ? kOut : kGated;
  u.splits = phase ? h.splits[1] : 1;
  u.tiles = phase ? h.tiles[1] : h.tiles[0];
  u.slot = i;
  u.part = i / u.tiles;
  i -= u.part * u.tiles;
  u.tile = i;
  const int nn = up_div(N, wide);
  int nm = up_div(a.rows, NT);
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
    nm = up_div(u.M, NT);
    i -= u.row_tile * nn;
  }
  const int n = i / nm, m = i - n * nm;
  u.n0 = n * wide;
  u.m0 = m * NT;
  u.row_tile += m;
  const int slices = a.slices[phase];
  u.s0 = (int)((int64_t)slices * u.part / u.splits);
  u.s1 = (int)((int64_t)slices * (u.part + 1) / u.splits);
  return u;
}

template <int TYPE, int NT>
__global__ void __launch_bounds__(kThreads, 1)
    few_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Args a) {
  using T = typename Element<TYPE>::T;
  using C = Config<NT>;
  constexpr int kAcc = C::kAcc, kChunk = C::kChunk;
  const int planes = 1 + a.plane_bits;  // of h, whose tiles lie beside one another
  const int kStage = kTile + planes * C::kRowsTile, kStages = C::kRing / kStage;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* handed = reinterpret_cast<float*>(smem + C::kRing);  // [2][rows][features]: u's values for a warp of g's
  Unit* units = reinterpret_cast<Unit*>(handed + 2 * 32 * 32);
  uint64_t* full = reinterpret_cast<uint64_t*>(units + kKept);
  uint64_t* empty = full + C::kMostStages;
  uint64_t* acc_full = empty + C::kMostStages;
  uint64_t* acc_empty = acc_full + 2;
  uint64_t* given = acc_empty + 2;  // per half: u's values are there; they have been taken
  uint64_t* got = given + 2;
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(got + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_at + 1);
  // counts of units: known, with their inputs there, begun by the warp that loads weights
  const uint32_t known_at = smem_u32(tmem_at + 2), ready_at = known_at + 4, begun_at = known_at + 8;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint64_t lim = a.wait_ns;  // bound of every wait (for another role: twice)

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], kEpiWarps);
      mbar_init(&given[i], 1);
      mbar_init(&got[i], 1);
    }
    *abort_flag = 0;
    set_ready(known_at, 0);
    set_ready(ready_at, 0);
    set_ready(begun_at, 0);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if ((warp == 0 || warp == kLoadRows) && lane < 2) {
    const CUtensorMap* const first = warp == 0 ? (lane == 0 ? &maps.w0[0] : &maps.w0[1]) : (lane == 0 ? &maps.a0 : &maps.a1[0]);
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(first)) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_at)),
                 "r"(C::kColumns));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the launch before has ended: so far, nothing of it was read
  const uint32_t tmem = *tmem_at;

  if (warp == kScout) {
    bool ok = !a.hold || flag_wait(a.hold, lim);  // a flag that nothing sets: every role's wait runs out
    const Plan& l = *a.plan;
    const Head head{l.total, {0, l.first[1], 0}, {l.tiles[0], l.tiles[1]}, {1, l.splits[1]}, 0};
    Groups groups;
    groups.load(a);
    for (int m = 0; ok; ++m) {
      int p = -1;
      if (lane == 0 && (ok = wait_given(begun_at, m, 2 * lim) && !*abort_flag)) {
        p = atomicAdd(&a.plan->next, 1);
        if (p >= head.total) p = -1;
      }
      if (!(ok = __shfl_sync(0xffffffffu, ok, 0))) break;
      p = __shfl_sync(0xffffffffu, p, 0);
      Unit u{};
      if (p < 0)
        u.kind = kEnd;
      else
        u = unit_at<NT>(p, a, head, groups);
      if (lane == 0) {
        units[m % kKept] = u;
        set_ready(known_at, m + 1);
        if (u.kind == kOut) ok = wait_done(a.done_row + u.row_tile, 2 * up_div(a.width, 64), lim);
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
  } else if (warp == 0 || warp == kLoadRows) {
    if (lane == 0) {
      const bool of_rows = warp == kLoadRows;
      Ring st;
      st.parity = 1;  // of a slot's release
      int used = 0;   // slots filled so far (up to kStages)
      for (int m = 0; !*abort_flag; ++m) {
        if (!(st.ok = wait_ready(of_rows ? ready_at : known_at, m + 1, 2 * lim))) break;
        const Unit u = units[m % kKept];
        if (u.kind == kEnd) break;
        if (!of_rows) set_ready(begun_at, m + 1);
        const int phase = u.kind == kOut;
        const bool mn = a.b_columns[phase];
        const CUtensorMap *m0, *m1;  // of rows; of the first and the second 64 features
        int at0 = u.n0, at1 = u.n0;
        if (of_rows) {
          m0 = m1 = phase ? &maps.a1[0] : &maps.a0;
        } else if (phase) {
          m0 = m1 = &maps.w1[0];
          at1 += 64;
        } else {
          m0 = &maps.w0[0];
          m1 = &maps.w0[1];
        }
        used = min(used + u.s1 - u.s0, kStages);
        for (int kb = u.s0; kb < u.s1; ++kb) {
          if (!(st.ok = mbar_wait(&empty[st.s], st.parity, 2 * lim))) break;
          const uint32_t slot = smem_u32(smem) + st.s * kStage;
          const int k = kb * BK;
          if (of_rows) {
            load_box(slot + kTile, m0, &full[st.s], k, u.start + u.m0, 0);
            if (phase && planes > 1) load_box(slot + kTile + C::kRowsTile, m0, &full[st.s], k, u.start + u.m0, 1);
          } else {
            expect_tx(&full[st.s], kTile + (phase ? planes : 1) * C::kRowsTile);
            load_box(slot, m0, &full[st.s], mn ? at0 : k, mn ? k : at0, u.group);
            load_box(slot + kBox, m1, &full[st.s], mn ? at1 : k, mn ? k : at1, u.group);
          }
          if (++st.s == kStages) {
            st.s = 0;
            st.parity ^= 1;
          }
        }
        if (!st.ok) break;
      }
      // every slice consumed before the shared memory goes away
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
    if (lane == 0) {
      Ring st;
      for (int m = 0; st.ok && !*abort_flag; ++m) {
        if (!(st.ok = wait_ready(known_at, m + 1, 2 * lim))) break;
        const Unit& u = units[m % kKept];
        const int kind = u.kind, count = u.s1 - u.s0;
        if (kind == kEnd) break;
        const bool mn = a.b_columns[kind == kOut];
        const uint32_t idesc = idesc_few(TYPE == SOAP_BF16, mn, NT);
        const int buf = m & 1;
        if (m >= 2 && !(st.ok = mbar_wait(&acc_empty[buf], ((m >> 1) & 1) ^ 1, 2 * lim))) break;
        tc_fence_after();
        const uint32_t d = tmem + static_cast<uint32_t>(buf * kAcc * NT);
        for (int i = 0; i < count; ++i) {
          if (!(st.ok = mbar_wait(&full[st.s], st.parity, 2 * lim))) break;
          tc_fence_after();
          const uint32_t as = smem_u32(smem) + st.s * kStage, bs = as + kTile;
#pragma unroll
          for (int kk = 0; kk < BK / 16; ++kk)
            mma(d + (kk % kAcc) * NT, mn ? tile_desc<1>(as, kk) : tile_desc<0>(as, kk), tile_desc<0>(bs, kk), idesc,
                i > 0 || kk >= kAcc);
          if (kind == kOut && planes > 1) {
#pragma unroll
            for (int kk = 0; kk < BK / 16; ++kk)
              mma(d + (kk % kAcc) * NT, mn ? tile_desc<1>(as, kk) : tile_desc<0>(as, kk),
                  tile_desc<0>(bs + C::kRowsTile, kk), idesc, 1);
          }
          umma_commit(&empty[st.s]);
          if (++st.s == kStages) {
            st.s = 0;
            st.parity ^= 1;
          }
        }
        if (st.ok) umma_commit(&acc_full[buf]);
      }
      if (!st.ok) *abort_flag = 1;
    }
  } else {
    const int q = warp & 3;  // accumulator lanes 32 q .. 32 q + 31
    const uint32_t lanes = tmem + (static_cast<uint32_t>(32 * q) << 16);
    const int pre_cols = (a.width + 31) / 32;  // blocks
    uint32_t turn = 0;                         // parity of given and got
    bool ok = true;
    for (int m = 0;; ++m) {
      if (lane == 0) ok = wait_ready(known_at, m + 1, 2 * lim);
      if (!(ok = __shfl_sync(0xffffffffu, ok, 0))) break;
      const Unit u = units[m % kKept];
      if (u.kind == kEnd) break;
      const int buf = m & 1, rows = min(NT, u.M - u.m0);
      ok = mbar_wait(&acc_full[buf], (m >> 1) & 1, 2 * lim) && !*abort_flag;
      tc_fence_after();
      if (!(ok = __all_sync(0xffffffffu, ok))) break;
      const bool gated = u.kind == kGated, of_u = gated && q >= 2;
      const int f = u.n0 + 32 * (gated ? q & 1 : q) + lane;  // this lane's feature
      const int64_t row0 = (int64_t)u.start + u.m0;
      for (int c = 0; c < C::kChunks; ++c) {
        const int left = rows - c * kChunk;  // rows of this chunk and behind
        if (left <= 0) break;
        float v[kChunk];
        const uint32_t t = lanes + static_cast<uint32_t>(buf * kAcc * NT + c * kChunk);
        drain<kChunk>(t, v);
#pragma unroll
        for (int i = 1; i < kAcc; ++i) {
          float w[kChunk];
          drain<kChunk>(t + i * NT, w);
#pragma unroll
          for (int j = 0; j < kChunk; ++j) v[j] += w[j];
        }
        if (gated) {
          float* const box = handed + (q & 1) * 32 * 32 + lane;
          if (a.pre && f < a.width) {
#pragma unroll
            for (int j = 0; j < kChunk; ++j) {
              const int r = u.m0 + c * kChunk + j;
              if (j < left)
                a.pre[((((int64_t)u.block + r / 32) * 2 + of_u) * pre_cols + f / 32) * 1024 + (f % 32 / 4 * 32 + r % 32) * 4 +
                      f % 4] = v[j];
            }
          }
          if (of_u) {
            // (the last values have been taken: the first time, nothing was there)
            if (lane == 0) ok = mbar_wait(&got[q & 1], turn ^ 1, 2 * lim);
            if (!(ok = __shfl_sync(0xffffffffu, ok, 0))) break;
#pragma unroll
            for (int j = 0; j < kChunk; ++j) box[32 * j] = v[j];
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(&given[q & 1])) : "memory");
          } else {
            ok = mbar_wait(&given[q & 1], turn, 2 * lim);
            if (!(ok = __all_sync(0xffffffffu, ok))) break;
            T* const h = static_cast<T*>(a.h) + (row0 + c * kChunk) * a.ld_h + f;
            float w[kChunk];
#pragma unroll
            for (int j = 0; j < kChunk; ++j) w[j] = box[32 * j];
            if (a.act == LAYER_SILU)
              gate<LAYER_SILU>(v, w);
            else
              gate<LAYER_GELU>(v, w);
#pragma unroll
            for (int j = 0; j < kChunk; ++j)
              if (j < left && f < a.width) {
                const T upper = from_f32<T>(v[j]);
                h[j * a.ld_h] = upper;
                if (planes > 1) h[a.h_plane + j * a.ld_h] = from_f32<T>(rest_of(v[j], upper));
              }
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(&got[q & 1])) : "memory");
          }
          turn ^= 1;
          continue;
        }
        if (u.splits > 1) {
          // each part stores its sums; the one that is the last to store a block adds up all of them in the parts' order
          auto at = [&](int part) {
            return reinterpret_cast<float4*>(a.partial[1]) +
                   (((int64_t)(u.slot + (part - u.part) * u.tiles) * kEpiWarps + q) * C::kChunks + c) * (kChunk * 8) + lane;
          };
#pragma unroll
          for (int j = 0; j < kChunk / 4; ++j)
            at(u.part)[32 * j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
          __threadfence();
          __syncwarp();
          int there = 0;
          if (lane == 0) there = atomicAdd(a.count[1] + (u.tile * kEpiWarps + q) * C::kChunks + c, 1);
          __threadfence();
          if (__shfl_sync(0xffffffffu, there, 0) != u.splits - 1) continue;
#pragma unroll
          for (int j = 0; j < kChunk; ++j) v[j] = 0.f;
#pragma unroll 4
          for (int s = 0; s < u.splits; ++s) {
            const float4* const from = at(s);
#pragma unroll
            for (int j = 0; j < kChunk / 4; ++j) {
              const float4 x = __ldcg(from + 32 * j);
              v[4 * j] += x.x, v[4 * j + 1] += x.y, v[4 * j + 2] += x.z, v[4 * j + 3] += x.w;
            }
          }
        }
        T* const y = static_cast<T*>(a.y) + (row0 + c * kChunk) * a.ld_y + f;
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
          if (j < left && f < a.hidden) y[j * a.ld_y] = from_f32<T>(v[j]);
      }
      if (!ok) break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(&acc_empty[buf])) : "memory");
      if (gated && !of_u) {  // stored: what waits for it may go on
        asm volatile("fence.proxy.async;" ::: "memory");
        __threadfence();
        __syncwarp();
        if (lane == 0)
          asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(a.done_row + u.row_tile) : "memory");
      }
    }
    if (!ok) {
      *abort_flag = 1;
      if (lane == 0 && a.status) atomicOr(a.status, kStatusTimeout);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kColumns));
  }

  // Where a wait gave up, the last CTA makes all results NaN (pre's words are two of T's), so that none is taken for an answer.
  if (threadIdx.x == 0) {
    if (*abort_flag) atomicOr(&a.plan->gave_up, 1);
    __threadfence();  // this CTA's results (and its word) come before its count
    const bool last = atomicAdd(&a.plan->through, 1) == (int)gridDim.x - 1;
    __threadfence();
    *abort_flag = last && atomicOr(&a.plan->gave_up, 0) != 0;
  }
  __syncthreads();
  if (*abort_flag) {
    // (y and, as rows of 8 KB, pre; one loop: with two the calls that do not get here took 0.3 us more)
    const T nan = from_f32<T>(NAN);
#pragma unroll 1
    for (int k = 0; k < (a.pre ? 2 : 1); ++k) {
      T* const p = k ? reinterpret_cast<T*>(a.pre) : static_cast<T*>(a.y);
      const int64_t rows = k ? a.pre_elems / 2048 : a.rows, ld = k ? 2048 * 4 / (int)sizeof(T) : a.ld_y;
      const int cols = k ? 2048 * 4 / (int)sizeof(T) : a.hidden;
#pragma unroll 1
      for (int64_t r = warp; r < rows; r += kThreads / 32)
#pragma unroll 1
        for (int c = lane; c < cols; c += 32) p[r * ld + c] = nan;
    }
  }
}

template <int TYPE, int NT>
cudaError_t launch(const Maps& maps, const Args& a, int64_t units, cudaStream_t s) {
  // per device: the CTAs that are resident at once, found (with the kernel's shared-memory attribute set) on the first
  // launch there
  static std::atomic<int> ctas_of[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  int ctas = dev < 64 ? ctas_of[dev].load(std::memory_order_relaxed) : 0;
  if (ctas == 0) {
    e = cudaFuncSetAttribute(few_kernel<TYPE, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Config<NT>::kSmem);
    if (e != cudaSuccess) return e;
    e = cudaDeviceGetAttribute(&ctas, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    if (dev < 64) ctas_of[dev].store(ctas, std::memory_order_relaxed);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(ctas, units)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Config<NT>::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, few_kernel<TYPE, NT>, maps, a);
}

template <int TYPE>
cudaError_t launch_tile(const Maps& maps, const Args& a, int64_t units, cudaStream_t s) {
  return a.row_tile == 16   ? launch<TYPE, 16>(maps, a, units, s)
         : a.row_tile == 32 ? launch<TYPE, 32>(maps, a, units, s)
         : a.row_tile == 64 ? launch<TYPE, 64>(maps, a, units, s)
                            : launch<TYPE, 128>(maps, a, units, s);
}

}  // namespace

cudaError_t run_few(const Maps& maps, const Args& a, int type, int64_t units, cudaStream_t s) {
  return type == SOAP_BF16 ? launch_tile<SOAP_BF16>(maps, a, units, s) : launch_tile<SOAP_F16>(maps, a, units, s);
}

}  // namespace ffn
}  // namespace soap
