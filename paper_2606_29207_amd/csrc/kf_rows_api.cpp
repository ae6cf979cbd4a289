// C-ABI layer of the operators on whole rows of tokens: host-side argument
// checks, workspace sizing and launches on the caller's stream.  Declarations
// and the contract of every entry point are in include/kf.h.
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "kf.h"
#include "kf_rows.h"

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

// Rows of `len` elements, `stride` apart, in 16-byte pieces.
bool stride_ok(int64_t stride, int64_t len) { return stride >= len && stride % 8 == 0; }

bool fp8_pool(const kf_shape* s) { return s->kv_dtype == KF_KV_FP8_E4M3; }

}  // namespace

namespace kf {

RowsLayout rows_layout(int32_t num_rows, int32_t num_seqs, int32_t num_kv_heads, int32_t group,
                       int64_t cus) {
  RowsLayout l{};
  if (num_kv_heads > kMaxLaunchRoutes) return l;
  // ceil(n_b G / kRowTile) tiles of each sequence that has rows (one, and so a
  // grid, where there are none)
  const int64_t pairs = (int64_t)num_rows * group;
  if (pairs > INT32_MAX - kRowTile) return l;
  const int64_t tiles = pairs / kRowTile + std::max(1, std::min(num_seqs, num_rows));
  int64_t recs = kMaxRecsPerCu * cus / num_kv_heads;
  if (recs < 2) recs = 0;
  if ((tiles + recs) * num_kv_heads > kMaxWgs) return l;
  l.max_tiles = (int32_t)tiles;
  l.max_recs = (int32_t)recs;
  l.rec_rows = (int32_t)std::min<int64_t>(kRowTile, (pairs + 31) / 32 * 32);
  l.tiles_off = 256;
  l.info_off = l.tiles_off + round_up(((size_t)num_seqs + 1) * sizeof(int32_t), 256);
  l.items_off = l.info_off + round_up((size_t)num_seqs * 4 * sizeof(int32_t), 256);
  l.splits_off = l.items_off + round_up((size_t)(tiles + recs) * sizeof(RowsItem), 256);
  l.ml_off = l.splits_off + round_up((size_t)(recs / 2) * sizeof(RowsSplit), 256);
  const size_t rec = (size_t)recs * num_kv_heads * l.rec_rows;
  l.o_off = l.ml_off + round_up(rec * 2 * sizeof(float), 256);
  l.total = l.o_off + rec * kDim * sizeof(float);
  return l;
}

// A plan and the combine of its parts cost 15 to 20 us.  Where the row tiles leave
// workgroups free and an even split of every tile comes to few steps (0.7 us each),
// on the mean or for the longest sequence, sequences of different lengths cost less
// than that, and every workgroup finds its own tile.  With a plan and without, us:
// 64 rows 18.1 and 10.0; 8 drafted tokens over 2K tokens 27.9 and 18.1; 48 of those
// over 300 .. 1500 tokens 69 and 49, over 800 .. 2500 95 and 76 (up to kMostSteps).
int32_t unplanned_parts(const RowsLayout& l, int32_t num_seqs, int32_t num_kv_heads,
                        int32_t num_routes, int32_t num_page_ids, int32_t max_pages_per_route,
                        int64_t slots) {
  const int64_t items = (int64_t)l.max_tiles * num_kv_heads;
  if (num_seqs > 64 || num_seqs < 1 || items > slots) return 0;
  // mean key tiles of a sequence at most, as the page table tells it: pages that are
  // reserved count too.  The parts of a row tile follow its own tokens (tile_parts): 64
  // rows with 8K tokens reserved 14.4 us (24.2 in parts of the reserved pages), 8.9 with
  // none, 8 drafted tokens over 300 14.5 for any reservation.  But launches that take a
  // plan because of it pay for it: 48 trees of 8 over 300 tokens 20 us with a table of
  // their own length, 51 with 8K reserved each and as much in max_pages_per_route.
  const int64_t pages = std::min((int64_t)num_page_ids, (int64_t)num_routes * max_pages_per_route);
  const int64_t keys = (pages * KF_PAGE_SIZE / kKeyTile + num_routes) / num_seqs + 1;
  int64_t parts = std::min(slots / items, (keys + kMinPart - 1) / kMinPart);
  // steps go down with the parts, the combine's turns up: 8 drafted tokens over 8K
  // tokens, 8 KV heads, 24.7 us in parts of kMinPart, 21.9 in 2 sqrt(keys) parts,
  // one KV head over 30K 36 and 29.6
  parts = std::min(parts, (int64_t)(2.0 * sqrt((double)keys)));
  parts = std::max<int64_t>(1, std::min<int64_t>(parts, l.max_recs / l.max_tiles));
  // the longest sequence's at most, where every sequence has a route
  const int64_t most = ((int64_t)max_pages_per_route * KF_PAGE_SIZE / kKeyTile + 1) *
                       std::max(1, num_routes - num_seqs + 1);
  return keys <= kMeanSteps * parts || most <= kMostSteps * parts ? (int32_t)parts : 0;
}

}  // namespace kf

namespace {

// Host checks that the two attention operators share; fills the kernel
// arguments (a.num_rows == 0: nothing to launch).
int prepare_rows(const kf_shape* shape, const void* q, int32_t num_rows, int64_t q_stride,
                 const int32_t* seq_row_begin, const void* k_pool, const void* v_pool,
                 const float* k_scale, const float* v_scale, const kf_route* routes,
                 int32_t num_routes, int32_t max_pages_per_route, const int32_t* page_ids,
                 const int32_t* seq_route_begin, void* out, float* lse, void* workspace,
                 size_t workspace_bytes, int32_t* err_flags, kf::RowsArgs& a) {
  const int st = kf::check_shape(shape);
  if (st != KF_OK) return st;
  if (num_rows < 0 || num_routes < 0 || max_pages_per_route < 0) return KF_ERR_INVALID_ARG;
  if (num_rows == 0) return KF_OK;
  if (!q || !seq_row_begin || !k_pool || !v_pool || !seq_route_begin || !out || !lse ||
      !err_flags || (num_routes > 0 && !routes) || (shape->num_page_ids > 0 && !page_ids))
    return KF_ERR_INVALID_ARG;
  if (fp8_pool(shape) && (!k_scale || !v_scale)) return KF_ERR_INVALID_ARG;
  if (!stride_ok(q_stride, (int64_t)shape->num_q_heads * KF_HEAD_DIM)) return KF_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k_pool, 16) || !aligned(v_pool, 16) || !aligned(out, 16))
    return KF_ERR_INVALID_ARG;
  const void* p4[] = {seq_row_begin, k_scale, v_scale, routes, page_ids, seq_route_begin, lse,
                      err_flags};
  for (const void* p : p4)
    if (p && !aligned(p, 4)) return KF_ERR_INVALID_ARG;
  const int32_t group = shape->num_q_heads / shape->num_kv_heads;
  const int64_t cus = kf::cu_count();
  const kf::RowsLayout l =
      kf::rows_layout(num_rows, shape->num_seqs, shape->num_kv_heads, group, cus);
  if (l.total == 0) return KF_ERR_UNSUPPORTED;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < l.total) return KF_ERR_WORKSPACE;

  a.q = static_cast<const uint16_t*>(q);
  a.q_stride = q_stride;
  a.seq_row_begin = seq_row_begin;
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.routes = routes;
  a.page_ids = page_ids;
  a.seq_route_begin = seq_route_begin;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.err_flags = err_flags;
  a.num_rows = num_rows;
  a.num_seqs = shape->num_seqs;
  a.num_q_heads = shape->num_q_heads;
  a.num_kv_heads = shape->num_kv_heads;
  a.group = group;
  a.num_routes = num_routes;
  a.max_pages_per_route = max_pages_per_route;
  a.num_pages = shape->num_pages;
  a.num_page_ids = shape->num_page_ids;
  a.head_major = shape->kv_layout == KF_KV_HEAD_MAJOR;
  a.scale_log2 = (float)((double)shape->scale * 1.4426950408889634074);
  char* ws = static_cast<char*>(workspace);
  a.head = reinterpret_cast<int32_t*>(ws);
  a.seq_tiles = reinterpret_cast<int32_t*>(ws + l.tiles_off);
  a.seq_info = reinterpret_cast<int32_t*>(ws + l.info_off);
  a.items = reinterpret_cast<kf::RowsItem*>(ws + l.items_off);
  a.splits = reinterpret_cast<kf::RowsSplit*>(ws + l.splits_off);
  a.rec_ml = reinterpret_cast<float*>(ws + l.ml_off);
  a.rec_o = reinterpret_cast<float*>(ws + l.o_off);
  a.max_tiles = l.max_tiles;
  a.max_recs = l.max_recs;
  a.rec_rows = l.rec_rows;
  a.slots = (int32_t)(2 * cus);
  a.parts = kf::unplanned_parts(l, shape->num_seqs, shape->num_kv_heads, num_routes,
                                shape->num_page_ids, max_pages_per_route, a.slots);
  // the row tiles that num_rows comes to if every row belongs to a sequence
  const int64_t tiles = ((int64_t)num_rows * group + kf::kRowTile - 1) / kf::kRowTile;
  a.may_split = l.max_recs > 1 && tiles * shape->num_kv_heads < kf::kSplitSlots * (int64_t)a.slots;
  return KF_OK;
}

}  // namespace

extern "C" {

size_t kf_kv_append_rows_workspace_bytes(int32_t num_routes) {
  if (num_routes < 0) return 0;
  return (size_t)(num_routes > 0 ? num_routes : 1) * 4 * sizeof(int32_t);
}

int kf_kv_append_rows(const kf_shape* shape, void* k_pool, void* v_pool, float* k_scale,
                      float* v_scale, const void* k_rows, const void* v_rows, int32_t num_rows,
                      int64_t row_stride, const int32_t* row_list, int32_t num_entries,
                      const int32_t* route_entry_begin, kf_route* routes, int32_t num_routes,
                      const int32_t* page_ids, void* workspace, size_t workspace_bytes,
                      int32_t* err_flags, void* stream) {
  const int st = kf::check_shape(shape);
  if (st != KF_OK) return st;
  if (num_rows < 0 || num_entries < 0 || num_routes < 0) return KF_ERR_INVALID_ARG;
  if (!row_list && num_entries > num_rows) return KF_ERR_INVALID_ARG;
  if (num_routes == 0 || num_entries == 0) return KF_OK;
  if (!k_pool || !v_pool || !k_rows || !v_rows || !route_entry_begin || !routes || !err_flags ||
      (shape->num_page_ids > 0 && !page_ids))
    return KF_ERR_INVALID_ARG;
  if (fp8_pool(shape) && (!k_scale || !v_scale)) return KF_ERR_INVALID_ARG;
  if (!stride_ok(row_stride, (int64_t)shape->num_kv_heads * KF_HEAD_DIM)) return KF_ERR_INVALID_ARG;
  if (!aligned(k_pool, 16) || !aligned(v_pool, 16) || !aligned(k_rows, 16) || !aligned(v_rows, 16))
    return KF_ERR_INVALID_ARG;
  const void* p4[] = {k_scale, v_scale, row_list, route_entry_begin, routes, page_ids, err_flags};
  for (const void* p : p4)
    if (p && !aligned(p, 4)) return KF_ERR_INVALID_ARG;
  // a wave per (page, KV head, K or V); the pages of num_routes routes
  const int64_t tiles = (int64_t)num_entries / KF_PAGE_SIZE + 2 * (int64_t)num_routes;
  if (num_routes > kf::kMaxLaunchRoutes || shape->num_kv_heads > kf::kMaxLaunchRoutes ||
      tiles * 2 * shape->num_kv_heads > 4 * kf::kMaxWgs)
    return KF_ERR_UNSUPPORTED;
  if (!workspace || !aligned(workspace, 16) ||
      workspace_bytes < kf_kv_append_rows_workspace_bytes(num_routes))
    return KF_ERR_WORKSPACE;
  kf::AppendRowsArgs a{};
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.k_rows = static_cast<const uint16_t*>(k_rows);
  a.v_rows = static_cast<const uint16_t*>(v_rows);
  a.row_stride = row_stride;
  a.row_list = row_list;
  a.entry_begin = route_entry_begin;
  a.routes = routes;
  a.page_ids = page_ids;
  a.plan = static_cast<int32_t*>(workspace);
  a.err_flags = err_flags;
  a.num_rows = num_rows;
  a.num_entries = num_entries;
  a.num_routes = num_routes;
  a.num_seqs = shape->num_seqs;
  a.num_kv_heads = shape->num_kv_heads;
  a.num_pages = shape->num_pages;
  a.num_page_ids = shape->num_page_ids;
  a.head_major = shape->kv_layout == KF_KV_HEAD_MAJOR;
  return kf::launch_append_rows(a, fp8_pool(shape), as_stream(stream)) == hipSuccess ? KF_OK
                                                                                    : KF_ERR_HIP;
}

size_t kf_rows_attn_workspace_bytes(const kf_shape* shape, int32_t num_rows) {
  if (kf::check_shape(shape) != KF_OK || num_rows < 0) return 0;
  return kf::rows_layout(num_rows, shape->num_seqs, shape->num_kv_heads,
                         shape->num_q_heads / shape->num_kv_heads, kf::cu_count())
      .total;
}

int kf_prompt_attn(const kf_shape* shape, const void* q, int32_t num_rows, int64_t q_stride,
                   const int32_t* seq_row_begin, const int32_t* first_pos, const void* k_pool,
                   const void* v_pool, const float* k_scale, const float* v_scale,
                   const kf_route* routes, int32_t num_routes, int32_t max_pages_per_route,
                   const int32_t* page_ids, const int32_t* seq_route_begin, void* out, float* lse,
                   void* workspace, size_t workspace_bytes, int32_t* err_flags, void* stream) {
  kf::RowsArgs a{};
  if (num_rows > 0 && ((shape && shape->num_seqs > 0 && !first_pos) || !aligned(first_pos, 4)))
    return KF_ERR_INVALID_ARG;
  const int st = prepare_rows(shape, q, num_rows, q_stride, seq_row_begin, k_pool, v_pool, k_scale,
                              v_scale, routes, num_routes, max_pages_per_route, page_ids,
                              seq_route_begin, out, lse, workspace, workspace_bytes, err_flags, a);
  if (st != KF_OK || num_rows == 0) return st;
  a.first_pos = first_pos;
  return kf::launch_rows_attn(a, fp8_pool(shape), false, as_stream(stream)) == hipSuccess
             ? KF_OK
             : KF_ERR_HIP;
}

int kf_tree_attn(const kf_shape* shape, const void* q, int32_t num_rows, int64_t q_stride,
                 const void* k_draft, const void* v_draft, int64_t kv_stride,
                 const uint64_t* tree_mask, const int32_t* seq_row_begin, const void* k_pool,
                 const void* v_pool, const float* k_scale, const float* v_scale,
                 const kf_route* routes, int32_t num_routes, int32_t max_pages_per_route,
                 const int32_t* page_ids, const int32_t* seq_route_begin, void* out, float* lse,
                 void* workspace, size_t workspace_bytes, int32_t* err_flags, void* stream) {
  kf::RowsArgs a{};
  const int st = prepare_rows(shape, q, num_rows, q_stride, seq_row_begin, k_pool, v_pool, k_scale,
                              v_scale, routes, num_routes, max_pages_per_route, page_ids,
                              seq_route_begin, out, lse, workspace, workspace_bytes, err_flags, a);
  if (st != KF_OK || num_rows == 0) return st;
  if (!k_draft || !v_draft || !tree_mask || !aligned(k_draft, 16) || !aligned(v_draft, 16) ||
      !aligned(tree_mask, 8) || !stride_ok(kv_stride, (int64_t)shape->num_kv_heads * KF_HEAD_DIM))
    return KF_ERR_INVALID_ARG;
  a.k_draft = static_cast<const uint16_t*>(k_draft);
  a.v_draft = static_cast<const uint16_t*>(v_draft);
  a.kv_stride = kv_stride;
  a.tree_mask = tree_mask;
  return kf::launch_rows_attn(a, fp8_pool(shape), true, as_stream(stream)) == hipSuccess
             ? KF_OK
             : KF_ERR_HIP;
}

}  // extern "C"
