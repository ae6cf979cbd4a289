// Internal interface between the C-ABI layer of the row operators
// (kf_rows_api.cpp) and their gfx950 kernels (kf_rows.hip).
#pragma once

#include "kf_internal.h"

namespace kf {

constexpr int kRowTile = 128;     // (row, query head) pairs of one KV head per workgroup
constexpr int kKeyTile = 32;      // tokens per step of a workgroup: two pages
constexpr int kMaxRecsPerCu = 8;  // records of split work items per compute unit, 136 MB at most (with
                                  // 4, 3 chunks of 512 rows behind 30K tokens 915 us instead of
                                  // 816, 7 of them 1928 and 1864; with 16 the same within 1.5 %)
constexpr int kMinPart = 4;       // key tiles of a part at least: 8 drafted tokens over 700 tokens
                                  // 15.4 us, 18.2 in parts of 8; over 300 14.3 in parts of 2, but
                                  // 64 rows over 1000 26.1 instead of 21.3
constexpr int kMeanSteps = 24;    // steps of a workgroup up to which a launch needs no plan:
constexpr int kMostSteps = 96;    // mean, and at most
constexpr int kWindowSteps = 512; // (with a window that the mean sequence fills)
constexpr int kSplitSlots = 4;    // (row tile, KV head) pairs per resident workgroup from which on
                                  // a launch splits none (2, 4 and 8: prompts of 6K .. 16K tokens
                                  // the same within 1 %; 8 packed ones 145, 144 and 148 us)
// Key tiles from which on tiles of one length are split for a shorter last round: 5
// chunks of 512 rows behind 30K tokens 1743 -> 1314 us, behind 1.7K (54 tiles and on)
// 144 -> 127; 80 trees of 32 rows over 8K 566 -> 520, over 1.5K (48) 136 -> 133; but
// over 1K (33) 103 -> 110.
constexpr int kEqualSteps = 48;
constexpr int64_t kMaxWgs = 0xFFFFFF;  // of 256 threads, in a launch: 32 bits of threads
constexpr int kCombineWgsPerSlot = 8;  // workgroups of the combine per resident workgroup at most
                                       // (2 and 32: the same)
// One launch appends up to kDirectEntries entries, and up to kDirectMean a route (a
// workgroup each): 1 row 7.3 us, 8.7 with a plan; a row for each of 16 routes 7.4 and
// 9.0, of 64 7.7 and 9.7, three for each of 16 9.1 and 10.1 (fp8); but 16 rows of one
// route 11.1 and 9.1, two for each of 64 12.0 and 10.6 (fp8).
constexpr int kDirectEntries = 64;
constexpr int kDirectMean = 3;
// The one launch has a workgroup per route, each of whose waves reads the whole table
// of entries, up to kDirectRoutes routes, and from there on a workgroup per entry that
// reads it once: 64 entries in 64 routes 8.4 us and 8.9, in 128 9.1 and 9.0, in 256 10.5
// and 9.0, in 1024 28 and 9.0, in 65535 32,000 and 20.
constexpr int kDirectRoutes = 128;
// The plan's workgroups, one a route, read the table each up to kPlanRoutes routes; from
// there on a launch before it does: 200 entries in 1024 routes 15.2 and 17.5, in 2048
// 18.0 and 17.7, in 4096 25 and 18, in 65535 1820 and 53.
constexpr int kPlanRoutes = 2048;
// Most of so many routes take few rows or none, and their workgroups are a wave each; of
// four waves above kWaveEntries entries, where one route may take thousands: 16K listed
// rows of one route among 4096 63 us (113 with one wave, 62 with eight), spread over all
// of them 91 (87, 98); 1000 of one route 21 with one wave and with four.
constexpr int kWaveEntries = 1024;

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
  int32_t tok_begin, tok_end, page_base;          // of its first route
  int32_t pad[3];
};

// The parts of one split row tile.
struct RowsSplit {
  int32_t tile, rec, parts, row0, rows;
  int32_t pad[3];
};

struct RowsArgs {
  const uint16_t* q;
  int64_t q_stride;
  const int32_t* seq_row_begin;
  const int32_t* first_pos;    // prompts, rows with a window
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
  int32_t* head;        // [0] items (-1: every row becomes NaN), [1] split tiles,
                        // [2] (row, head) pairs of the largest
  int32_t* seq_tiles;   // [num_seqs + 1] first row tile of each sequence
  int32_t* seq_info;    // [num_seqs][4] key tiles, smallest tok_begin, bad, largest tok_end
  RowsItem* items;
  RowsSplit* splits;
  float* rec_ml;        // [records][Hkv][rec_rows][2] (max, sum), base 2
  float* rec_o;         // [records][Hkv][rec_rows][kDim], not normalised
  int32_t max_tiles;    // row tiles at most
  int32_t max_recs;     // records per KV head
  int32_t rec_rows;     // rows of a record
  int32_t slots;        // resident workgroups
  int32_t parts;        // > 0: no plan; every row tile in so many parts at most
  int32_t may_split;    // a plan may split row tiles: a combine follows
  int32_t sinks, window;  // window < 0: none (last: the kernels' arguments before them keep
                          // their places, and with those the scalar registers of their loads)
};

struct RowsLayout {
  size_t tiles_off, info_off, items_off, splits_off, ml_off, o_off, total;
  int32_t max_tiles, max_recs, rec_rows;
};
// total 0: more than a launch takes.
RowsLayout rows_layout(int32_t num_rows, int32_t num_seqs, int32_t num_kv_heads, int32_t group,
                       int64_t cus);

// Parts per row tile, at most, of a launch that runs without a plan, 0 with one.
// most_keys: key tiles that a row tile sees at most, whatever the cache holds.
int32_t unplanned_parts(const RowsLayout& l, int32_t num_seqs, int32_t num_kv_heads,
                        int32_t num_routes, int32_t num_page_ids, int32_t max_pages_per_route,
                        int64_t most_keys, int64_t slots);

hipError_t launch_rows_attn(const RowsArgs& a, bool fp8, bool tree, hipStream_t stream);

}  // namespace kf
