// Internal interface between the C-ABI layer of the row operators
// (kf_rows_api.cpp) and their gfx950 kernels (kf_rows.hip).
#pragma once

#include "kf_internal.h"

namespace kf {

constexpr int kRowTile = 128;     // (row, query head) pairs of one KV head per workgroup
constexpr int kKeyTile = 32;      // tokens per step of a workgroup: two pages
constexpr int kMaxRecsPerCu = 8;  // records of split work items per compute unit
constexpr int kMinPart = 4;       // key tiles of a part at least
constexpr int kUnplannedSteps = 24;  // mean steps of a workgroup up to which a launch needs no plan
constexpr int kSplitSlots = 4;    // (row tile, KV head) pairs per resident workgroup from which on
                                  // a launch splits none
constexpr int kCombineWgsPerSlot = 8;  // workgroups of the combine per resident workgroup at most

// ------------------------------------------------------------------- append
struct AppendRowsArgs {
  void* k_pool;
  void* v_pool;
  float* k_scale;
  float* v_scale;
  const uint16_t* k_rows;
  const uint16_t* v_rows;
  int64_t row_stride;
  const int32_t* row_list;
  const int32_t* entry_begin;  // [num_routes + 1]
  kf_route* routes;
  const int32_t* page_ids;
  int32_t* plan;  // [num_routes][4]: tokens before the append (-1: none is made), first entry,
                  // entries, first page id's index
  int32_t* err_flags;
  int32_t num_rows, num_entries, num_routes, num_seqs, num_kv_heads, num_pages, num_page_ids;
  int32_t head_major;
};

hipError_t launch_append_rows(const AppendRowsArgs& a, bool fp8, hipStream_t stream);

// ---------------------------------------------------------------- attention
// One work item: the keys [key0, key1) (in tiles, over the sequence's visible
// tokens) of one row tile; the last part of a row tile has key1 = INT32_MAX.
struct RowsItem {
  int32_t seq;    // -1 - b: the rows of sequence b become NaN
  int32_t tile;   // row tile of the sequence
  int32_t key0, key1;
  int32_t rec;    // record of a split tile's part, -1: the outputs are written
  int32_t row0, rows, first_pos, route0, route1;  // of the sequence
  int32_t pad[2];
};

// The parts of one split row tile.
struct RowsSplit {
  int32_t seq, tile, rec, parts;
};

struct RowsArgs {
  const uint16_t* q;
  int64_t q_stride;
  const int32_t* seq_row_begin;
  const int32_t* first_pos;    // prompts
  const uint16_t* k_draft;     // trees
  const uint16_t* v_draft;
  int64_t kv_stride;
  const uint64_t* tree_mask;
  const void* k_pool;
  const void* v_pool;
  const float* k_scale;
  const float* v_scale;
  const kf_route* routes;
  const int32_t* page_ids;
  const int32_t* seq_route_begin;
  uint16_t* out;
  float* lse;
  int32_t* err_flags;
  int32_t num_rows, num_seqs, num_q_heads, num_kv_heads, group;
  int32_t num_routes, max_pages_per_route, num_pages, num_page_ids;
  int32_t head_major;
  float scale_log2;
  // workspace
  int32_t* head;        // [0] items (-1: every row becomes NaN), [1] split tiles
  int32_t* seq_tiles;   // [num_seqs + 1] first row tile of each sequence
  int32_t* seq_info;    // [num_seqs][4] tokens, smallest tok_begin, bad
  RowsItem* items;
  RowsSplit* splits;
  float* rec_ml;        // [records][Hkv][rec_rows][2] (max, sum), base 2
  float* rec_o;         // [records][Hkv][rec_rows][kDim], not normalised
  int32_t max_tiles;    // row tiles at most
  int32_t max_recs;     // records per KV head
  int32_t rec_rows;     // rows of a record
  int32_t slots;        // resident workgroups
  int32_t parts;        // > 0: no plan; every row tile in so many parts
  int32_t may_split;    // a plan may split row tiles: a combine follows
};

struct RowsLayout {
  size_t tiles_off, info_off, items_off, splits_off, ml_off, o_off, total;
  int32_t max_tiles, max_recs, rec_rows;
};
// total 0: more than a launch takes.
RowsLayout rows_layout(int32_t num_rows, int32_t num_seqs, int32_t num_kv_heads, int32_t group,
                       int64_t cus);

// Parts per row tile of a launch that runs without a plan, 0 with one.
int32_t unplanned_parts(const RowsLayout& l, int32_t num_seqs, int32_t num_kv_heads,
                        int32_t num_routes, int32_t num_page_ids, int64_t slots);

hipError_t launch_rows_attn(const RowsArgs& a, bool fp8, bool tree, hipStream_t stream);

}  // namespace kf
