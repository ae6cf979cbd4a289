// C-ABI layer of the operators that keep a cache within a budget: host-side
// argument checks, workspace sizing and launches on the caller's stream.
// Declarations and the contract of every entry point are in include/kf.h.
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "kf.h"
#include "kf_budget.h"

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bool fp8_pool(const kf_shape* s) { return s->kv_dtype == KF_KV_FP8_E4M3; }

hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

int64_t div_up(int64_t x, int64_t y) { return (x + y - 1) / y; }

// A page and a slot of it share 31 bits of the list of what stays.
bool pages_fit(const kf_shape* s) { return s->num_pages <= INT32_MAX / KF_PAGE_SIZE; }

// The columns of a launch, and a workgroup per route and KV head.
bool weights_fit(const kf_shape* s, int32_t num_rows, int32_t num_routes) {
  return num_routes <= kf::kMaxLaunchRoutes &&
         (int64_t)num_rows * (s->num_q_heads / s->num_kv_heads) <= (1 << 28) - 256 &&
         (int64_t)num_routes * s->num_kv_heads <= kf::kMaxBudgetWgs;
}

}  // namespace

extern "C" {

size_t kf_attn_weights_workspace_bytes(const kf_shape* shape, int32_t num_rows, int32_t num_routes,
                                       int32_t max_pages_per_route) {
  if (kf::check_shape(shape) != KF_OK || num_rows < 0 || num_routes < 0 ||
      max_pages_per_route < 0 || !weights_fit(shape, num_rows, num_routes))
    return 0;
  kf::AttnWeightsArgs a{};
  a.num_rows = num_rows;
  a.num_seqs = shape->num_seqs;
  a.num_kv_heads = shape->num_kv_heads;
  a.group = shape->num_q_heads / shape->num_kv_heads;
  a.num_routes = std::max(1, num_routes);
  a.max_pages_per_route = max_pages_per_route;
  a.num_page_ids = shape->num_page_ids;
  kf::plan_attn_weights(a, 2 * (int64_t)kf::cu_count());
  return std::max<size_t>(256, kf::attn_weights_bytes(a));
}

int kf_attn_weights(const kf_shape* shape, const void* q, int32_t num_rows, int64_t q_stride,
                    const float* lse, const int32_t* seq_row_begin, const int32_t* first_pos,
                    const void* k_pool, const float* k_scale, const kf_route* routes,
                    int32_t num_routes, int32_t max_pages_per_route, const int32_t* page_ids,
                    float decay, float* weights, void* workspace, size_t workspace_bytes,
                    int32_t* err_flags, void* stream) {
  const int st = kf::check_shape(shape);
  if (st != KF_OK) return st;
  if (num_rows < 0 || num_routes < 0 || max_pages_per_route < 0 || !isfinite(decay))
    return KF_ERR_INVALID_ARG;
  if (num_rows == 0 || num_routes == 0 || shape->num_seqs == 0) return KF_OK;
  if (!q || !lse || !seq_row_begin || !first_pos || !k_pool || !routes || !weights || !err_flags ||
      (shape->num_page_ids > 0 && !page_ids) || (fp8_pool(shape) && !k_scale))
    return KF_ERR_INVALID_ARG;
  if (q_stride < (int64_t)shape->num_q_heads * KF_HEAD_DIM || q_stride % 8 != 0)
    return KF_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k_pool, 16)) return KF_ERR_INVALID_ARG;
  const void* p4[] = {lse, seq_row_begin, first_pos, k_scale, routes, page_ids, weights, err_flags};
  for (const void* p : p4)
    if (p && !aligned(p, 4)) return KF_ERR_INVALID_ARG;
  const int32_t H = shape->num_kv_heads, group = shape->num_q_heads / H;
  if (!weights_fit(shape, num_rows, num_routes)) return KF_ERR_UNSUPPORTED;

  kf::AttnWeightsArgs a{};
  a.q = static_cast<const uint16_t*>(q);
  a.q_stride = q_stride;
  a.lse = lse;
  a.seq_row_begin = seq_row_begin;
  a.first_pos = first_pos;
  a.k_pool = k_pool;
  a.k_scale = k_scale;
  a.routes = routes;
  a.page_ids = page_ids;
  a.weights = weights;
  a.err_flags = err_flags;
  a.decay = decay;
  a.scale_log2 = (float)((double)shape->scale * 1.4426950408889634074);
  a.num_rows = num_rows;
  a.num_seqs = shape->num_seqs;
  a.num_q_heads = shape->num_q_heads;
  a.num_kv_heads = H;
  a.group = group;
  a.num_routes = num_routes;
  a.max_pages_per_route = max_pages_per_route;
  a.num_pages = shape->num_pages;
  a.num_page_ids = shape->num_page_ids;
  a.head_major = shape->kv_layout == KF_KV_HEAD_MAJOR;
  kf::plan_attn_weights(a, 2 * (int64_t)kf::cu_count());
  const size_t need = kf::attn_weights_bytes(a);
  if (need > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < need))
    return KF_ERR_WORKSPACE;
  a.sums = static_cast<float*>(workspace);
  return kf::launch_attn_weights(a, fp8_pool(shape), as_stream(stream)) == hipSuccess ? KF_OK
                                                                                     : KF_ERR_HIP;
}

size_t kf_kv_evict_workspace_bytes(const kf_shape* shape, int32_t max_keep) {
  if (kf::check_shape(shape) != KF_OK || max_keep < 0) return 0;
  if (shape->num_seqs > kf::kMaxLaunchRoutes || shape->num_kv_heads > kf::kMaxLaunchRoutes) return 0;
  return kf::evict_layout(*shape, max_keep).total;
}

int kf_kv_evict(const kf_shape* shape, void* k_pool, void* v_pool, float* k_scale, float* v_scale,
                float* weights, kf_route* routes, int32_t num_routes, int32_t max_pages_per_route,
                const int32_t* page_ids, const int32_t* seq_route_begin, const int32_t* into,
                const int32_t* keep, int32_t max_keep, int32_t keep_first, int32_t keep_last,
                void* workspace, size_t workspace_bytes, int32_t* err_flags, void* stream) {
  const int st = kf::check_shape(shape);
  if (st != KF_OK) return st;
  if (num_routes < 0 || max_pages_per_route < 0 || max_keep < 0 || keep_first < 0 || keep_last < 0)
    return KF_ERR_INVALID_ARG;
  if (shape->num_seqs == 0 || num_routes == 0) return KF_OK;
  if (!k_pool || !v_pool || !weights || !routes || !seq_route_begin || !into || !keep ||
      !err_flags || (shape->num_page_ids > 0 && !page_ids))
    return KF_ERR_INVALID_ARG;
  if (fp8_pool(shape) && (!k_scale || !v_scale)) return KF_ERR_INVALID_ARG;
  if (!aligned(k_pool, 16) || !aligned(v_pool, 16)) return KF_ERR_INVALID_ARG;
  const void* p4[] = {k_scale, v_scale, weights, routes, page_ids, seq_route_begin, into, keep,
                      err_flags};
  for (const void* p : p4)
    if (p && !aligned(p, 4)) return KF_ERR_INVALID_ARG;
  const int64_t pages = div_up(max_keep, KF_PAGE_SIZE);
  const size_t need = kf_kv_evict_workspace_bytes(shape, max_keep);
  const kf::EvictLayout l = kf::evict_layout(*shape, max_keep);
  if (need == 0 || !pages_fit(shape) ||
      (div_up(pages * 2 * shape->num_kv_heads, 4) + 1) * shape->num_seqs > kf::kMaxBudgetWgs ||
      (int64_t)shape->num_kv_heads * shape->num_seqs * 4 * l.parts > kf::kMaxBudgetWgs)
    return KF_ERR_UNSUPPORTED;
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < need) return KF_ERR_WORKSPACE;

  kf::EvictArgs a{};
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.weights = weights;
  a.routes = routes;
  a.page_ids = page_ids;
  a.seq_route_begin = seq_route_begin;
  a.into = into;
  a.keep = keep;
  a.err_flags = err_flags;
  a.num_seqs = shape->num_seqs;
  a.num_kv_heads = shape->num_kv_heads;
  a.num_routes = num_routes;
  a.max_pages_per_route = max_pages_per_route;
  a.num_pages = shape->num_pages;
  a.num_page_ids = shape->num_page_ids;
  a.head_major = shape->kv_layout == KF_KV_HEAD_MAJOR;
  a.max_keep = max_keep;
  a.keep_first = keep_first;
  a.keep_last = keep_last;
  char* ws = static_cast<char*>(workspace);
  a.plan = reinterpret_cast<int32_t*>(ws);
  a.list = reinterpret_cast<int32_t*>(ws + l.list_off);
  a.parts = l.parts;
  a.state = reinterpret_cast<int32_t*>(ws + l.state_off);
  a.rows = reinterpret_cast<uint32_t*>(ws + l.rows_off);
  return kf::launch_evict(a, fp8_pool(shape), as_stream(stream)) == hipSuccess ? KF_OK : KF_ERR_HIP;
}

}  // extern "C"

namespace kf {

// Sequences of many tokens, on the mean of what the table reserves (the pages that what
// stays goes to among it), are told apart by several workgroups each; by one, which reads
// their weights once, up to kHeldTokens, but where the parts are few.  By one and by
// several, 8 KV heads, 64 tokens kept, the whole call, us: one of 30K tokens 52 and 61, of
// 40K 67 and 60, of 64K 92 and 52; 8 of 40K 70 and 70, of 64K 96 and 84, 16 of 64K 98 and
// 151; 48 of 2K .. 64K 116 and 196; 4 of 128K 347 and 86, 16 of them 361 and 284.  With
// 4096 kept, one of 30K 62 and 58, of 40K 80 and 61, 8 of 64K 258 and 242, 16 of them 420
// and 472: those of 64K count as 68K and go by several, 16 of them to their loss.  The mean
// less max_keep would send these by one, but 8 of 64K and one of 40K too.  (The sequences'
// own tokens are not known here: where they differ much, or two routes of full length take
// turns, the mean is not theirs.)
EvictLayout evict_layout(const kf_shape& s, int32_t max_keep) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  EvictLayout l{};
  const int64_t tokens = (int64_t)s.num_page_ids * KF_PAGE_SIZE / std::max(1, s.num_seqs);
  const size_t units = (size_t)s.num_seqs * s.num_kv_heads;
  l.parts = (int32_t)std::min<int64_t>(kMaxParts, tokens / kPartTokens);
  if (tokens < kOneWorkgroup || (tokens <= kHeldTokens && units * l.parts > kFewParts)) l.parts = 1;
  while (l.parts > 1 && units * l.parts > kMostParts) --l.parts;
  l.list_off = up((size_t)s.num_seqs * 2 * sizeof(int32_t)) + 256;
  l.state_off = l.list_off + up(units * max_keep * sizeof(int32_t));
  const size_t parts = l.parts > 1 ? units * l.parts : 0;
  l.rows_off = l.state_off + up(parts * 4 * sizeof(int32_t));
  l.total = l.rows_off + parts * 3 * 2048 * sizeof(uint32_t);
  return l;
}

// By the (row, head) pairs of a sequence on the mean, and the workgroups of 256 keys
// that the table has room for.
void plan_attn_weights(AttnWeightsArgs& a, int64_t slots) {
  const int64_t most = std::max(1, std::min(a.max_pages_per_route, a.num_page_ids));
  const int64_t columns = (int64_t)a.num_rows * a.group / std::max(1, a.num_seqs);
  // A workgroup's pages: 16 (one decode row over 32K tokens of bf16, 16 sequences, 190 us; 8
  // and 32 212 and 195, 64 204, 128 222, 256 195), where the columns stay in LDS twice as many
  // (74 us, 80 with 16, 77 with 64).
  int64_t chunk = columns > kFewColumns && columns <= kHeldColumns ? 32 : 16;
  while (div_up(most, chunk) * a.num_kv_heads * a.num_routes > kMaxBudgetWgs) chunk *= 2;
  a.chunk_pages = (int32_t)std::min<int64_t>(chunk, INT32_MAX / 2);
  a.chunks = (int32_t)div_up(most, a.chunk_pages);
  // A prompt's first keys are seen by all of its rows, its last ones by a few: in one
  // workgroup each, the first ones would end last.
  const int64_t wgs = (int64_t)a.chunks * a.num_kv_heads * a.num_routes;
  const int64_t steps = (int64_t)a.num_rows * a.group / 32;
  a.segments = 1;
  if (columns > kHeldColumns && chunk == 16 && wgs < kSegmentWgs * slots)
    a.segments = (int32_t)std::max<int64_t>(
        1, std::min<int64_t>({kMaxSegments, kSegmentWgs * slots / wgs, steps / kSegmentSteps}));
}

}  // namespace kf
