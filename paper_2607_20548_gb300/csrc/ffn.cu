// The gated feed-forward block's C entry points (include/layer.h, layer_ffn_*): checks, the workspace's layout, copies
// of operands that the products cannot read as they lie, tensor maps. The products are ffn_steps.cu's.
#include <algorithm>
#include <cstdint>

#include "../../include/layer.h"
#include "ffn.h"
#include "pair.h"
#include "profile.h"
#include "soap_internal.h"

namespace soap {
namespace {

using namespace ffn;

constexpr int kMaxSide = 65536;
constexpr int64_t kMaxRows = INT32_MAX - 65536;

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }
int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }

bool bad_ptr(const void* p, size_t size) { return p && reinterpret_cast<uintptr_t>(p) % size; }

bool bad_matrix(const layer_matrix_t* m, int64_t rows, int64_t cols, int groups, size_t size) {
  if (!m || !m->data || bad_ptr(m->data, size)) return true;
  const int64_t along = m->columns ? rows : cols, across = m->columns ? cols : rows;
  return m->ld < along || (groups > 1 && m->stride < (across - 1) * m->ld + along);
}

bool bad_sizes(int64_t rows, int64_t hidden, int64_t width, int32_t groups, int32_t type) {
  return rows < 0 || rows > kMaxRows || hidden < 1 || hidden > kMaxSide || width < 1 || width > kMaxSide || groups < 1 ||
         groups > kMaxGroups || type < SOAP_F32 || type > SOAP_F16;
}

// Rows as the products' columns (ffn_few.cu) or rows. Measured, bf16 forward: dense 2048 x 8192 with 24, 64, 96 rows 36,
// 42, 50 us as columns, 48, 45, 46 as rows; 64 groups of 2048 x 768 with 3, 32, 64, 94, 128 rows each 99, 105, 111, 118,
// 127 and 114 (16 rows), 116, 119, 121, 124.
bool few_rows(int64_t rows, int groups, int type, bool backward) {
  return !backward && type != SOAP_F32 && rows <= 64 * (int64_t)groups;
}

// Planes that h, dg and du are kept in: fp32 three of bf16; 16-bit types their rounding and, for few results and small
// weights, where a few latencies set the time, also what that leaves, so that the results' own rounding is all of their
// error (1.0 in place of 1.4 of one rounding in root mean square, whatever the size). Both passes: 1 row of 64 x 64
// bf16 36 us, in one plane 33; 8 rows of 1024 x 1024 64 and 54; 24 rows of 1024 x 1024, which have one plane, 56 and 67 in
// two. A rule on the weights alone would hold every row of a model to the same, at the price of the large calls: up to
// 2^19 elements in two planes, 512 x 512 would take 57 us in place of 48 with 100 rows, 124 in place of 94 with 8192, 299
// in place of 207 with 32768. All others round h, dg and du once, to what the tensor core multiplies: six of
// the nine products of both passes read them, so that a second plane everywhere would be 15 products' work for 9.
int planes_of(int64_t rows, int64_t hidden, int64_t width, int groups, int type) {
  return type == SOAP_F32 ? 3 : rows * hidden <= 16384 && groups * hidden * width <= 1 << 23 ? 2 : 1;
}

// Slices of a tile's sums, per phase (of the weights' gradients: of all rows). Planes of 16-bit types are added one
// after the other, but for few rows, where one load of the weights serves both.
int products_of(int type) { return type == SOAP_F32 ? 6 : 1; }  // of planes, per slice
struct Slices {
  int64_t n[3];
};
Slices slices_of(int64_t rows, int64_t hidden, int64_t width, int groups, int type, bool backward) {
  const bool few = few_rows(rows, groups, type, backward);
  const int twice = !few && type != SOAP_F32 && planes_of(rows, hidden, width, groups, type) == 2 ? 2 : 1;
  return Slices{{up_div(hidden, 64), twice * (backward ? 2 : 1) * (int64_t)up_div(width, 64), twice * (int64_t)up_div(rows, 64)}};
}

// Rows as columns: 64 and 128 features by the rows that a group has on average, and half as many again. Else 256 x 256
// (the first phase forward: 128 of g and of u), or half the columns where that leaves no pair without a tile and sums are
// too short to go in parts: a tile's products take as long, what follows them half as long.
Tiles tiles_of(int64_t rows, int64_t hidden, int64_t width, int groups, int type, bool backward) {
  if (few_rows(rows, groups, type, backward)) {
    const int64_t each = groups == 1 ? rows : (rows + rows / 2) / groups;
    int n = 16;
    while (n < each && n < 128) n *= 2;
    return Tiles{n, {64, 128, 0}, kSms, 128 * n, 4 * std::max(1, n / 32)};
  }
  Tiles t{256, {backward ? 256 : 128, 256, 256}, kSms / 2, 256 * 256, 64};
  const Slices n = slices_of(rows, hidden, width, groups, type, backward);
  const int64_t some = std::min<int64_t>(groups, rows), row_tiles = rows / 256 + some;
  const int64_t tiles[3] = {row_tiles * up_div(width, t.cols[0]), row_tiles * up_div(hidden, 256),
                            some * 3 * up_div(width, 256) * up_div(hidden, 256)};
  for (int p = 0; p < 3; ++p)
    if (2 * tiles[p] <= t.pool && n.n[p] * products_of(type) < kMinParted) t.cols[p] /= 2;
  return t;
}

// Where everything lies in the workspace.
struct Layout {
  int64_t row_tiles;              // at most
  int64_t tiles[3], slots[3];     // at most; of partial sums
  int64_t units;                  // at most
  size_t plan, done, done_words, count[3], clips, partial[3], inter[3], x, dy, w[3], bytes;
  size_t inter_plane, x_plane, w_plane;  // elements of a plane
};

Layout layout_of(int64_t rows, int64_t hidden, int64_t width, int groups, int type, bool copies, bool backward) {
  Layout l{};
  const Tiles t = tiles_of(rows, hidden, width, groups, type, backward);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += up256(bytes);
    return was;
  };
  l.row_tiles = rows / t.rows + std::min<int64_t>(groups, rows);
  l.tiles[0] = l.row_tiles * up_div(width, t.cols[0]);
  l.tiles[1] = l.row_tiles * up_div(hidden, t.cols[1]);
  // (of either order of the weights)
  const int64_t each = backward ? 3 * std::max((int64_t)up_div(width, 256) * up_div(hidden, t.cols[2]),
                                               (int64_t)up_div(width, t.cols[2]) * up_div(hidden, 256)) : 0;
  l.tiles[2] = backward ? std::min<int64_t>(groups, rows) * each : 0;
  const auto [slices] = slices_of(rows, hidden, width, groups, type, backward);
  for (int p = 0; p < 3; ++p) {
    const int64_t parts = slices[p] * products_of(type) < kMinParted ? 1 : slices[p], longest = (slices[p] + kMaxSlices - 1) / kMaxSlices;
    l.units += l.tiles[p] * std::max(parts, longest);
    // parts of tiles that are fewer than the pairs; and of those too long for one accumulator (of the weights' gradients:
    // a group of s > kMaxSlices slices has ceil(s / kMaxSlices) of them, and there are at most `longest` such groups, each
    // of which adds less than one to what all rows together have)
    l.slots[p] = parts > 1 ? std::min<int64_t>(t.pool, l.tiles[p] * parts) : 0;
    if (longest > 1) l.slots[p] += p < 2 ? l.tiles[p] * longest : each * (longest + (groups > 1 ? std::min<int64_t>(groups, longest) : 0));
  }
  l.plan = take(sizeof(Plan));
  l.done = at;
  size_t words = l.row_tiles + groups;
  for (int p = 0; p < 3; ++p) {
    l.count[p] = at + words * 4;
    words += l.slots[p] * t.blocks;
  }
  l.done_words = words;
  take(words * 4);
  l.clips = take((size_t)groups * kClips * sizeof(CUtensorMap));
  for (int p = 0; p < 3; ++p) l.partial[p] = take((size_t)l.slots[p] * t.partial * 4);
  const size_t planes = type == SOAP_F32 ? 3 : 1;
  l.inter_plane = (size_t)rows * up8(width);
  for (int i = 0; i < (backward ? 3 : 1); ++i) l.inter[i] = take(planes_of(rows, hidden, width, groups, type) * l.inter_plane * 2);
  if (copies || type == SOAP_F32) {
    l.x_plane = (size_t)rows * up8(hidden);
    l.x = take(planes * l.x_plane * 2);
    if (backward) l.dy = take(planes * l.x_plane * 2);
    l.w_plane = (size_t)groups * std::max(hidden * up8(width), width * up8(hidden));
    for (int i = 0; i < 3; ++i) l.w[i] = take(planes * l.w_plane * 2);
  }
  l.bytes = at;
  return l;
}

struct Call {
  int64_t rows;
  int hidden, width, groups;
  const int32_t* offsets;
  int type, act;
  const layer_matrix_t* w[3];  // gate, up, down
  int* status;
  uint8_t* ws;
  size_t ws_bytes;
  bool backward;
};

bool units_of_16(const void* p, int64_t ld, int64_t stride, size_t size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * (int64_t)size % 16 == 0 && stride * (int64_t)size % 16 == 0;
}

bool bad_call(const Call& c) {
  const size_t size = dtype_size(c.type);
  return (!c.offsets && c.groups != 1) || bad_ptr(c.offsets, 4) || bad_ptr(c.status, 4) ||
         (c.act != LAYER_SILU && c.act != LAYER_GELU) || bad_matrix(c.w[0], c.hidden, c.width, c.groups, size) ||
         bad_matrix(c.w[1], c.hidden, c.width, c.groups, size) || bad_matrix(c.w[2], c.width, c.hidden, c.groups, size) ||
         !c.w[0]->columns != !c.w[1]->columns || !c.ws || bad_ptr(c.ws, 256);
}

// Whether a call has something to do beside its results: to look at the offsets.
bool tells(const Call& c) { return c.offsets && c.status; }

// What a row-major matrix (or `matrices` of them, or planes) looks like to the copies.
struct View {
  void* p;
  int64_t rows, ld, stride;
  int cols, depth;
};

bool make_map(CUtensorMap* map, const View& v, int type, int box_cols, int box_rows) {
  auto fn = tc::encode_fn();
  if (!fn) return false;
  const size_t size = dtype_size(type);
  const cuuint64_t dims[3] = {(cuuint64_t)v.cols, (cuuint64_t)v.rows, (cuuint64_t)v.depth};
  // (of a single matrix the third step is never taken)
  const cuuint64_t strides[2] = {(cuuint64_t)v.ld * size, (cuuint64_t)(v.depth > 1 ? v.stride : v.ld) * size};
  const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, steps[3] = {1, 1, 1};
  const CUtensorMapDataType t = type == SOAP_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                : type == SOAP_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                    : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return fn(map, t, 3, v.p, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
            box_cols * size == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t compute(const Call& c, const void* x, int64_t ld_x, const void* dy, int64_t ld_dy, float* pre, void* y,
                    int64_t ld_y, const layer_matrix_t* const (&grads)[3], cudaStream_t s) {
  const bool f32 = c.type == SOAP_F32;
  const int etype = f32 ? (int)SOAP_BF16 : c.type, planes = f32 ? 3 : 1;
  const size_t size = dtype_size(c.type);
  const layer_matrix_t& gate = *c.w[0];
  const layer_matrix_t& down = *c.w[2];

  // operands as they lie, or copies
  const void* in[5] = {x, dy, c.w[0]->data, c.w[1]->data, c.w[2]->data};
  bool copy[5];
  bool any = false;
  for (int i = 0; i < 5; ++i) {
    const bool none = i == 1 && !c.backward;
    copy[i] = !none && (f32 || (i < 2 ? !units_of_16(in[i], i ? ld_dy : ld_x, 0, size)
                                      : !units_of_16(in[i], c.w[i - 2]->ld, c.groups > 1 ? c.w[i - 2]->stride : 0, size)));
    any |= copy[i];
  }
  const Layout l = layout_of(c.rows, c.hidden, c.width, c.groups, c.type, any, c.backward);
  if (c.ws_bytes < l.bytes) return cudaErrorInvalidValue;
  const size_t place[5] = {l.x, l.dy, l.w[0], l.w[1], l.w[2]};
  View v[5];
  CopyJobs jobs{};
  int64_t chunks = 0;
  for (int i = 0; i < 5; ++i) {
    if (i == 1 && !c.backward) continue;
    const bool mat = i >= 2;
    const layer_matrix_t* m = mat ? c.w[i - 2] : nullptr;
    const int64_t wr = i == 4 ? c.width : c.hidden, wc = i == 4 ? c.hidden : c.width;
    const int64_t rows = !mat ? c.rows : m->columns ? wc : wr;
    const int cols = (int)(!mat ? c.hidden : m->columns ? wr : wc);
    const int n = mat ? c.groups : 1;
    v[i] = View{const_cast<void*>(in[i]), rows, mat ? m->ld : i ? ld_dy : ld_x, mat ? m->stride : 0, cols, n};
    if (!copy[i] || c.rows == 0) continue;
    CopyJob& j = jobs.job[jobs.n++];
    j = CopyJob{in[i], v[i].ld, v[i].stride, rows, cols, (int)up8(cols), n, mat, reinterpret_cast<uint16_t*>(c.ws + place[i]), 0};
    v[i].p = j.dst;
    v[i].ld = j.ld_out;
    v[i].stride = rows * j.ld_out;
    v[i].depth = n * planes;
    j.plane = n * v[i].stride;
    chunks = std::max(chunks, n * rows * (j.ld_out / 8));
  }

  Args a{};
  a.plan = reinterpret_cast<Plan*>(c.ws + l.plan);
  a.done_row = reinterpret_cast<int*>(c.ws + l.done);
  a.done_group = a.done_row + l.row_tiles;
  a.done_words = (int)l.done_words;
  for (int p = 0; p < 3; ++p) {
    a.count[p] = reinterpret_cast<int*>(c.ws + l.count[p]);
    a.partial[p] = reinterpret_cast<float*>(c.ws + l.partial[p]);
  }
  const Tiles t = tiles_of(c.rows, c.hidden, c.width, c.groups, c.type, c.backward);
  const bool few = few_rows(c.rows, c.groups, c.type, c.backward);
  a.row_tile = t.rows;
  for (int p = 0; p < 3; ++p) {
    a.col_tile[p] = t.cols[p];
    a.narrow[p] = !few && t.cols[p] < (p == 0 && !c.backward ? 128 : 256);
  }
  // every warp of both CTAs counts its share of a tile: blocks of 32 columns of h, or of dg, du and h
  a.stored = 16 * ((c.backward ? 4 : 2) >> a.narrow[0]) * up_div(c.width, t.cols[0]);
  a.pool = t.pool;
  const int kept = planes_of(c.rows, c.hidden, c.width, c.groups, c.type);
  a.plane_bits = c.type != SOAP_F32 && kept == 2;
  if (few) {
    a.h = c.ws + l.inter[0];
    a.ld_h = up8(c.width);
    a.h_plane = (int64_t)l.inter_plane;
  }
  a.clips = c.offsets && c.rows > 0 && !few ? reinterpret_cast<const CUtensorMap*>(c.ws + l.clips) : nullptr;
  a.backward = c.backward;
  a.params = grads[0] != nullptr;
  a.groups = c.groups;
  a.rows = (int)c.rows;
  a.hidden = c.hidden;
  a.width = c.width;
  // the second factor's K runs down its columns: x Wg by hidden, h Wd by width; dy Wd^T by hidden, dg Wg^T by width
  a.b_columns[0] = c.backward ? down.columns != 0 : gate.columns == 0;
  a.b_columns[1] = c.backward ? gate.columns != 0 : down.columns == 0;
  a.kblocks[0] = up_div(c.hidden, 64);
  a.kblocks[1] = up_div(c.width, 64);
  const Slices n = slices_of(c.rows, c.hidden, c.width, c.groups, c.type, c.backward);
  for (int p = 0; p < 2; ++p) a.slices[p] = (int)n.n[p];
  a.products = products_of(c.type);
  // a gradient in its weight's order: of a column-major weight the transposed product
  const int left[3] = {kInX, kInX, kInH}, right[3] = {kInDG, kInDU, kInDY};
  for (int p = 0; p < 3; ++p) {
    const bool turned = c.w[p]->columns;
    a.wa[p] = turned ? right[p] : left[p];
    a.wb[p] = turned ? left[p] : right[p];
    a.wrows[p] = (p == 2) != turned ? c.width : c.hidden;
    a.wcols[p] = (p == 2) != turned ? c.hidden : c.width;
    a.each[p] = c.backward ? up_div(a.wrows[p], 256) * up_div(a.wcols[p], t.cols[2]) : 0;
  }
  a.act = c.act;
  a.pre = pre;
  a.pre_elems = (int64_t)layer_ffn_pre_elems(c.rows, c.width, c.groups);
  a.y = y;
  a.ld_y = ld_y;
  a.status = c.status;
  const WaitLimit w = wait_limit();
  a.wait_ns = w.ns;
  a.hold = w.hold;
  a.offsets = c.offsets;

  Maps maps{};
  if (c.rows > 0) {
    View inter[3];
    for (int i = 0; i < 3; ++i)
      inter[i] = View{c.ws + l.inter[i], c.rows, up8(c.width), (int64_t)l.inter_plane, c.width, kept};
    const int box = few ? t.rows : 128;
    bool ok = make_map(&maps.a0, v[c.backward ? 1 : 0], etype, 64, box) &&
              make_map(&maps.a1[0], inter[c.backward ? 1 : 0], etype, 64, box) &&
              (!c.backward || make_map(&maps.a1[1], inter[2], etype, 64, box));
    for (int i = 0; i < 2; ++i) {
      ok = ok && make_map(&maps.w0[i], v[c.backward ? 4 : 2 + i], etype, 64, few || a.b_columns[0] || a.narrow[0] ? 64 : 128) &&
           ((i == 1 && !c.backward) || make_map(&maps.w1[i], v[c.backward ? 2 + i : 4], etype, 64, few || a.b_columns[1] || a.narrow[1] ? 64 : 128));
    }
    a.y_tma = !few && units_of_16(y, ld_y, 0, size);
    if (!few) ok = ok && make_map(&maps.clip[kH], inter[0], etype, 32, 32);
    if (a.y_tma) ok = ok && make_map(&maps.clip[kY], View{y, c.rows, ld_y, 0, c.hidden, 1}, c.type, 32, 32);
    if (c.backward) {
      ok = ok && make_map(&maps.clip[kDG], inter[1], etype, 32, 32) && make_map(&maps.clip[kDU], inter[2], etype, 32, 32) &&
           make_map(&maps.clip[kInX], v[0], etype, 64, 64) && make_map(&maps.clip[kInDY], v[1], etype, 64, 64) &&
           make_map(&maps.clip[kInH], inter[0], etype, 64, 64) && make_map(&maps.clip[kInDG], inter[1], etype, 64, 64) &&
           make_map(&maps.clip[kInDU], inter[2], etype, 64, 64);
    }
    for (int p = 0; p < 3 && a.params; ++p) {
      const layer_matrix_t& g = *grads[p];
      const int64_t r = p < 2 ? c.hidden : c.width, k = p < 2 ? c.width : c.hidden;
      a.dw_tma[p] = units_of_16(g.data, g.ld, c.groups > 1 ? g.stride : 0, size);
      if (a.dw_tma[p])
        ok = ok && make_map(&maps.dw[p], View{g.data, g.columns ? k : r, g.ld, g.stride, (int)(g.columns ? r : k), c.groups},
                            c.type, 32, 32);
    }
    if (!ok) return cudaErrorInvalidValue;
  }
  for (int p = 0; p < 3 && a.params; ++p) {
    a.dw[p] = grads[p]->data;
    a.ld_dw[p] = grads[p]->ld;
    a.stride_dw[p] = grads[p]->stride;
  }

  const cudaError_t e = prepare(maps, a, jobs, chunks, c.type, s);
  if (e != cudaSuccess || c.rows == 0) return e;
  return few ? run_few(maps, a, c.type, l.units, s) : run(maps, a, c.type, l.units, s);
}

}  // namespace
}  // namespace soap

using namespace soap;

extern "C" {

size_t layer_ffn_pre_elems(int64_t rows, int64_t width, int32_t groups) {
  if (bad_sizes(rows, 1, width, groups, SOAP_F32)) return 0;
  // each group's rows in blocks of 32
  const int64_t blocks = (rows + 31 * std::min<int64_t>(rows, groups)) / 32;
  return (size_t)blocks * 32 * 2 * ((width + 31) / 32 * 32);
}

size_t layer_ffn_workspace_bytes(int64_t rows, int64_t hidden, int64_t width, int32_t groups, int32_t type,
                                 int32_t aligned, int32_t backward) {
  if (bad_sizes(rows, hidden, width, groups, type)) return 0;
  return layout_of(rows, hidden, width, groups, type, !aligned, backward != 0).bytes;
}

soap_status_t layer_ffn_forward(int64_t rows, int64_t hidden, int64_t width, int32_t groups,
                                const int32_t* offsets, const void* x, int64_t ld_x, int32_t type,
                                const layer_matrix_t* gate, const layer_matrix_t* up, const layer_matrix_t* down,
                                int32_t act, void* y, int64_t ld_y, float* pre, int32_t* status, void* workspace,
                                size_t workspace_bytes, soap_stream_t stream) {
  if (bad_sizes(rows, hidden, width, groups, type)) return SOAP_ERR_INVALID_ARG;
  const Call c{rows, (int)hidden, (int)width, groups, offsets, type, act, {gate, up, down}, status,
               static_cast<uint8_t*>(workspace), workspace_bytes, false};
  const size_t size = dtype_size(type);
  if (bad_call(c) || bad_ptr(pre, 16)) return SOAP_ERR_INVALID_ARG;
  if (rows > 0 && (!x || bad_ptr(x, size) || ld_x < hidden || !y || bad_ptr(y, size) || ld_y < hidden))
    return SOAP_ERR_INVALID_ARG;
  if (rows == 0 && !tells(c)) return SOAP_OK;
  cudaStream_t s = (cudaStream_t)stream;
  ProfScope prof(kFamGemmTc, 6.0 * rows * hidden * width, 3.0 * groups * hidden * width * size, s);
  const layer_matrix_t* none[3] = {nullptr, nullptr, nullptr};
  const cudaError_t e = compute(c, x, ld_x, nullptr, 0, pre, y, ld_y, none, s);
  return e == cudaSuccess ? SOAP_OK : e == cudaErrorInvalidValue ? SOAP_ERR_INVALID_ARG : SOAP_ERR_CUDA;
}

soap_status_t layer_ffn_backward(int64_t rows, int64_t hidden, int64_t width, int32_t groups,
                                 const int32_t* offsets, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x,
                                 int32_t type, const layer_matrix_t* gate, const layer_matrix_t* up,
                                 const layer_matrix_t* down, int32_t act, const float* pre, void* dx, int64_t ld_dx,
                                 const layer_matrix_t* d_gate, const layer_matrix_t* d_up,
                                 const layer_matrix_t* d_down, int32_t* status, void* workspace,
                                 size_t workspace_bytes, soap_stream_t stream) {
  if (bad_sizes(rows, hidden, width, groups, type)) return SOAP_ERR_INVALID_ARG;
  const Call c{rows, (int)hidden, (int)width, groups, offsets, type, act, {gate, up, down}, status,
               static_cast<uint8_t*>(workspace), workspace_bytes, true};
  const size_t size = dtype_size(type);
  if (bad_call(c) || bad_ptr(pre, 16)) return SOAP_ERR_INVALID_ARG;
  if (rows > 0 && (!x || bad_ptr(x, size) || ld_x < hidden || !dy || bad_ptr(dy, size) || ld_dy < hidden || !dx ||
                   bad_ptr(dx, size) || ld_dx < hidden || !pre))
    return SOAP_ERR_INVALID_ARG;
  const layer_matrix_t* grads[3] = {d_gate, d_up, d_down};
  if (!d_gate != !d_up || !d_gate != !d_down) return SOAP_ERR_INVALID_ARG;
  if (d_gate)
    for (int i = 0; i < 3; ++i)
      if (bad_matrix(grads[i], i < 2 ? hidden : width, i < 2 ? width : hidden, groups, size) ||
          !grads[i]->columns != !c.w[i]->columns)
        return SOAP_ERR_INVALID_ARG;
  if (rows == 0 && !d_gate && !tells(c)) return SOAP_OK;
  cudaStream_t s = (cudaStream_t)stream;
  ProfScope prof(kFamGemmTc, (d_gate ? 12.0 : 6.0) * rows * hidden * width, 3.0 * groups * hidden * width * size, s);
  const cudaError_t e = compute(c, x, ld_x, dy, ld_dy, const_cast<float*>(pre), dx, ld_dx, grads, s);
  return e == cudaSuccess ? SOAP_OK : e == cudaErrorInvalidValue ? SOAP_ERR_INVALID_ARG : SOAP_ERR_CUDA;
}

}  // extern "C"
