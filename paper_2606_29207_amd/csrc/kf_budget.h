// Internal interface between the C-ABI layer of the cache-budget operators
// (kf_budget_api.cpp) and their gfx950 kernels (kf_budget.hip).
#pragma once

#include "kf_internal.h"

namespace kf {

constexpr int64_t kMaxBudgetWgs = 0xFFFFFF;  // workgroups of a launch: 32 bits of threads

// ------------------------------------------------------------- attn_weights
constexpr int kFewColumns = 64;    // (row, head) pairs of a sequence that stay in registers
constexpr int kHeldColumns = 256;  // ... in LDS
// Workgroups that share more columns than that, and 32 columns steps of each at least.
// With 1, 4, 8 and 16, us: prompts of 500 rows 60, 27, 20 and 17, of 2000 183, 65, 54 and
// 66, of 10K 949, 556, 518 and 521, 16 of 300 .. 1500 190, 165, 181 and 239 (5 by the rule).
constexpr int kMaxSegments = 8;
constexpr int64_t kSegmentSteps = 4;
constexpr int64_t kSegmentWgs = 8;  // workgroups of a launch at most, per resident one

struct AttnWeightsArgs {
  const uint16_t* q;
  int64_t q_stride;
  const float* lse;
  const int32_t* seq_row_begin;
  const int32_t* first_pos;
  const void* k_pool;
  const float* k_scale;
  const kf_route* routes;
  const int32_t* page_ids;
  float* weights;  // [num_pages][Hkv][kPage]
  int32_t* err_flags;
  float decay, scale_log2;
  int32_t num_rows, num_seqs, num_q_heads, num_kv_heads, group;
  int32_t num_routes, max_pages_per_route, num_pages, num_page_ids;
  int32_t head_major;
  int32_t chunk_pages, chunks;  // pages of a workgroup, workgroups of a route and KV head
  int32_t segments;  // workgroups that share the columns of the same keys
  float* sums;       // workspace: [segments][num_routes][chunks * Hkv][256 tokens], if they are
                     // several
};

// How a launch is dealt out, by what the host knows; and its workspace (0: none).
void plan_attn_weights(AttnWeightsArgs& a, int64_t slots);
inline size_t attn_weights_bytes(const AttnWeightsArgs& a) {
  return a.segments == 1 ? 0 : (size_t)a.segments * a.num_routes * a.chunks * a.num_kv_heads *
                                   256 * sizeof(float);
}

hipError_t launch_attn_weights(const AttnWeightsArgs& a, bool fp8, hipStream_t stream);

// -------------------------------------------------------------------- evict
constexpr int kPartTokens = 8192;  // of a part of a sequence whose tokens are told apart by several
                                   // workgroups, and the most parts
constexpr int kMaxParts = 32;
constexpr int64_t kOneWorkgroup = 40 * 1024;  // tokens of a sequence up to which one does, and
constexpr int64_t kHeldTokens = 64 * 1024;    // where the parts would be more than kFewParts
constexpr int64_t kFewParts = 256;
constexpr size_t kMostParts = 4096;  // of a launch: 100 MB of bins

struct EvictArgs {
  void* k_pool;
  void* v_pool;
  float* k_scale;
  float* v_scale;
  float* weights;
  kf_route* routes;
  const int32_t* page_ids;
  const int32_t* seq_route_begin;
  const int32_t* into;
  const int32_t* keep;
  int32_t* err_flags;
  int32_t num_seqs, num_kv_heads, num_routes, max_pages_per_route, num_pages, num_page_ids;
  int32_t head_major;
  int32_t max_keep, keep_first, keep_last;
  // workspace
  int32_t* plan;  // [num_seqs][2]: tokens kept (-1: the sequence is left alone), index of the
                  // first page id that they go to
  int32_t* list;  // [num_seqs][Hkv][max_keep]: page * kPage + slot of each, in order
  // several workgroups for a sequence and KV head
  int32_t parts;   // 1: one does
  uint32_t* rows;  // [num_seqs][Hkv][parts][3 passes][2048 bins]
  int32_t* state;  // [num_seqs][Hkv][parts][4]: the threshold's bits, how many equal ones are
                   // wanted, larger keys of the part, a bad page among its own
};

// The workspace of an eviction.
struct EvictLayout {
  size_t list_off, state_off, rows_off, total;
  int32_t parts;
};
EvictLayout evict_layout(const kf_shape& s, int32_t max_keep);

hipError_t launch_evict(const EvictArgs& a, bool fp8, hipStream_t stream);

}  // namespace kf
