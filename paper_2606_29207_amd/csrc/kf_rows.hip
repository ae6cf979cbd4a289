// gfx950 kernels of the operators on whole rows of tokens:
//   append_plan_kernel, append_tile_kernel -- rows of K/V into the paged cache
//   rows_plan_kernel     -- work items of an attention launch
//   rows_kernel          -- attention of prompt rows, of rows with a window, or of
//                           drafted trees over it
//   rows_combine_kernel  -- reduction of the row tiles whose keys were split
#include "kf_device.h"
#include "kf_rows.h"

namespace kf {
namespace {

constexpr float kLn2 = 0.69314718055994530942f;

// ------------------------------------------------------------------- append
// Appends move 512 bytes in and 512 (fp8 256) out per token and KV head, and nothing
// else: memory bounds them.  A wave takes one page of one KV head, K or V, so that the
// whole page is written at once (V's rows of sixteen slots turn around in registers)
// and its fp8 scale is one wave's decision.  16K rows of 8 KV heads (134 MB): 28 us,
// 4.9 TB/s, a copy's rate; prompts into fp8 pages (260 MB) 48 .. 58 us, 4.5 .. 5.4
// TB/s; the plan before them 5 us.  Appends of a few rows are one launch, bound by its
// chain of loads (7.3 us a pass).

// Whether row i of the table of entries decreases or leaves [0, num_entries].
__device__ __forceinline__ bool bad_entries(const AppendRowsArgs& a, int i) {
  const int x = a.entry_begin[i], y = a.entry_begin[i + 1];
  return x < 0 || y < x || y > a.num_entries;
}

// One route's check: its tokens before the append, or -1 if it takes no rows (flag
// says why).  WHOLE: by the workgroup together; else by every wave for itself, for
// calls of a few rows, which are a chain of loads.  TABLE: the table of entries too.
template <bool WHOLE, bool TABLE>
__device__ int append_check(const AppendRowsArgs& a, int r, int& flag) {
  const int lane = WHOLE ? threadIdx.x : threadIdx.x & 63, step = WHOLE ? blockDim.x : 64;
  // page ids and listed rows read at a time (a few waves: more; 1 row 7.1 us, 7.4 with 4)
  constexpr int kAtOnce = WHOLE && !TABLE ? 4 : 1;
  auto any = [](bool x) -> bool { return WHOLE ? __syncthreads_or(x) : __ballot(x) != 0; };
  const int e0 = a.entry_begin[r], n = a.entry_begin[r + 1] - e0;
  const int32_t* rp = reinterpret_cast<const int32_t*>(a.routes + r);
  const int seq = rp[0], tb = rp[2], te = rp[3], base = rp[4], cap = rp[5];
  flag = 0;
  if (TABLE) {
    bool bad = false;
    for (int i = lane; i < a.num_routes; i += step) bad |= bad_entries(a, i);
    flag = any(bad) ? KF_EFLAG_BAD_ROUTE : 0;
  }
  if (flag || n == 0) return -1;
  const int64_t j0 = (int64_t)te - tb, last = (j0 + n - 1) / kPage;
  if (seq < 0 || seq >= a.num_seqs || j0 < 0 || (int64_t)te + n > INT32_MAX || j0 + n > INT32_MAX)
    flag = KF_EFLAG_BAD_ROUTE;
  else if (last >= cap)
    flag = KF_EFLAG_TAIL_FULL;
  else if (base < 0 || base + last >= a.num_page_ids)
    flag = KF_EFLAG_BAD_ROUTE;
  if (flag) return -1;
  bool page = false, row = false;
#pragma unroll kAtOnce
  for (int64_t p = j0 / kPage + lane; p <= last; p += step)
    page |= (uint32_t)a.page_ids[base + p] >= (uint32_t)a.num_pages;
  if (a.row_list)
#pragma unroll kAtOnce
    for (int i = lane; i < n; i += step) row |= (uint32_t)a.row_list[e0 + i] >= (uint32_t)a.num_rows;
  flag = any(page) ? KF_EFLAG_BAD_PAGE : any(row) ? KF_EFLAG_BAD_ROUTE : 0;
  return flag ? -1 : (int)j0;
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Sizes of the two bf16 of x as integers, which order as the values do (an
// infinity is 0x7F80, a NaN more); the larger of two such pairs, place by place.
__device__ __forceinline__ uint32_t sizes(uint32_t x) { return x & 0x7FFF7FFFu; }
__device__ __forceinline__ uint32_t larger(uint32_t x, uint32_t y) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x),
                                                                __builtin_bit_cast(u16x2, y)));
}
__device__ __forceinline__ uint32_t both_places(uint32_t x) { return larger(x, x >> 16) & 0xFFFFu; }

// The scale of an fp8 page after an append, if its rule is one scale for all of
// the call's tokens: sizes of the token at slot 0 (first, if the page begins with
// the call) and of all of them (most).  Negative where it is not: a token beyond
// 448 times the scale re-encodes the page; and where the quick quotient below is
// not exact: infinities, NaN, scales near the ends of float32.
__device__ __forceinline__ float one_scale(bool begins, uint32_t first, uint32_t most,
                                           const float* scale_at) {
  float scale;
  if (begins) {
    const float amax = __builtin_bit_cast(float, first << 16);
    scale = amax > 0.0f ? amax / 28.0f : 1.0f;
  } else {
    scale = *scale_at;
  }
  const bool ok = most < 0x7F80u && __builtin_bit_cast(float, most << 16) <= 448.0f * scale &&
                  scale >= 0x1p-60f && scale <= 0x1p60f;
  return ok ? scale : -1.0f;
}

// x / scale, correctly rounded, clamped to +-448: inv is 1 / scale, correctly
// rounded, so that one step from x inv by its remainder gives the nearest float
// (Markstein).  Remainders stay in range where the quotient is not far below
// E4M3's smallest value; there any quotient rounds to the same zero.  The remainder
// of -0 is +0, and +0 - 0 is +0: the sign is x's own (scales are positive).
__device__ __forceinline__ float quotient(float x, float scale, float inv) {
  const float q = x * inv;
  const float y = __builtin_fmaf(__builtin_fmaf(-q, scale, x), inv, q);
  return __builtin_copysignf(fminf(fabsf(y), 448.0f), x);
}
__device__ __forceinline__ float lo_bf16(uint32_t x) { return __builtin_bit_cast(float, x << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t x) {
  return __builtin_bit_cast(float, x & 0xFFFF0000u);
}

// The slots [s0, s1) of one page of one KV head, K or V, filled from the rows of
// entries e0 .. by one wave.
template <bool FP8>
__device__ void append_page(const AppendRowsArgs& a, int page, int g, bool is_v, int s0, int s1,
                            int e0, uint16_t* lds) {
  const int lane = threadIdx.x & 63, H = a.num_kv_heads;
  const size_t head = slice_of(page, g, H, a.num_pages, a.head_major);
  const uint16_t* rows = (is_v ? a.v_rows : a.k_rows) + (size_t)g * kDim;
  auto row_of = [&](int s) -> int64_t {
    const int e = e0 + s - s0;
    return (a.row_list ? a.row_list[e] : e) * a.row_stride;
  };
  if (!FP8 && !is_v) {  // sixteen lanes a row
    uint16_t* k = static_cast<uint16_t*>(a.k_pool) + head * (kPage * kDim);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = 4 * i + (lane >> 4);
      if (s >= s0 && s < s1)
        *reinterpret_cast<u32x4*>(k + s * kDim + 8 * (lane & 15)) =
            ld16(rows + row_of(s) + 8 * (lane & 15));
    }
    return;
  }
  uint8_t* pool = FP8 ? static_cast<uint8_t*>(is_v ? a.v_pool : a.k_pool) + head * (kPage * kDim)
                      : nullptr;
  float* scale_at = FP8 ? (is_v ? a.v_scale : a.k_scale) + (size_t)page * H + g : nullptr;
  if (FP8 && !is_v) {  // four lanes a row: eight dims of every 32
    const int s = lane >> 2, c = lane & 3;
    const bool mine = s >= s0 && s < s1;
    u32x4 x[4] = {};
    if (mine) {
      const uint16_t* row = rows + row_of(s);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = ld16(row + 32 * i + 8 * c);
    }
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) most = larger(most, sizes(x[i][k]));
    most = both_places(most);
    most |= s == 0 ? most << 16 : 0;  // the token at slot 0 in the upper half
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) most = larger(most, (uint32_t)__shfl_xor((int)most, m));
    const float scale = one_scale(s0 == 0, most >> 16, most & 0xFFFFu, scale_at);
    if (scale > 0.0f) {
      const float inv = 1.0f / scale;
      if (mine) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u32x2 codes;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t u = x[i][2 * k], v = x[i][2 * k + 1];
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(lo_bf16(u), scale, inv),
                                                    quotient(hi_bf16(u), scale, inv), 0, false);
            w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(lo_bf16(v), scale, inv),
                                                quotient(hi_bf16(v), scale, inv), w, true);
            codes[k] = (uint32_t)w;
          }
          *reinterpret_cast<u32x2*>(pool + kDim * s + 32 * i + 8 * c) = codes;
        }
      }
      if (lane == 0) *scale_at = scale;
      return;
    }
  }
  uint32_t x[kPage];  // dims 2 lane, 2 lane + 1 of each token
#pragma unroll
  for (int s = 0; s < kPage; ++s)
    x[s] = s >= s0 && s < s1 ? reinterpret_cast<const uint32_t*>(rows + row_of(s))[lane] : 0;
  if constexpr (!FP8) {  // two rows of sixteen slots a lane
    u32x4* v = reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.v_pool) + head * (kPage * kDim)) +
               4 * lane;
    u32x4 r[4] = {};
    if (s1 - s0 < kPage) {
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = v[i];
    }
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int s = 0; s < kPage; ++s) {
        const uint32_t bits = (d ? x[s] >> 16 : x[s] & 0xFFFFu) << (16 * (s & 1));
        const uint32_t keep = s & 1 ? 0xFFFFu : 0xFFFF0000u;
        const int at = 2 * d + (s >> 3), wd = (s & 7) >> 1;
        if (s >= s0 && s < s1) r[at][wd] = (r[at][wd] & keep) | bits;
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = r[i];
    return;
  }
  u32x4 old[2] = {};  // V: the lane's two rows of sixteen slots
  if (FP8 && is_v) {
    if (s1 - s0 < kPage) {
#pragma unroll
      for (int d = 0; d < 2; ++d) old[d] = ld16(pool + (2 * lane + d) * kPage);
    }
    uint32_t most = 0;
#pragma unroll
    for (int s = 0; s < kPage; ++s) most = larger(most, sizes(x[s]));
    most = both_places(most) | both_places(sizes(x[0])) << 16;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) most = larger(most, (uint32_t)__shfl_xor((int)most, m));
    const float scale = one_scale(s0 == 0, most >> 16, most & 0xFFFFu, scale_at);
    if (scale > 0.0f) {
      const float inv = 1.0f / scale;
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float q[4];
          uint32_t keep = 0;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int s = 4 * i + k;
            q[k] = quotient(d ? hi_bf16(x[s]) : lo_bf16(x[s]), scale, inv);
            if (s < s0 || s >= s1) keep |= 0xFFu << (8 * k);
          }
          int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
          w = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
          r[i] = ((uint32_t)w & ~keep) | (old[d][i] & keep);
        }
        *reinterpret_cast<u32x4*>(pool + (2 * lane + d) * kPage) = r;
      }
      if (lane == 0) *scale_at = scale;
      return;
    }
  }
  if constexpr (FP8) {
    // The E4M3 append rule, token after token, in float32: the token at slot 0
    // sets scale = amax / 28; a later one beyond 448 scale re-encodes the slots
    // before it to amax / 28; each is stored as RNE(x / scale).
    uint16_t* codes = lds + lane;  // [slot][lane]: the code pairs of this lane's dims
    if (is_v) {
#pragma unroll
      for (int s = 0; s < kPage; ++s)
        codes[64 * s] = (uint16_t)((old[0][s >> 2] >> (8 * (s & 3)) & 0xFFu) |
                                   (old[1][s >> 2] >> (8 * (s & 3)) & 0xFFu) << 8);
    } else {
      for (int s = 0; s < s0; ++s) codes[64 * s] = reinterpret_cast<uint16_t*>(pool)[64 * s + lane];
    }
    float scale = s0 > 0 ? *scale_at : 0.0f;
#pragma unroll
    for (int s = 0; s < kPage; ++s) {
      if (s < s0 || s >= s1) continue;
      const float x0 = lo_bf16(x[s]), x1 = hi_bf16(x[s]);
      const float amax = wave_max(fmaxf(fabsf(x0), fabsf(x1)));
      if (s == 0) {
        scale = amax > 0.0f ? amax / 28.0f : 1.0f;
      } else if (amax > 448.0f * scale) {
        const float fresh = amax / 28.0f;
#pragma unroll 1
        for (int t = 0; t < s; ++t) {
          const f32x2 was = e4m3_values(codes[64 * t]);
          codes[64 * t] = (uint16_t)e4m3_pair(was.x * scale / fresh, was.y * scale / fresh);
        }
        scale = fresh;
      }
      codes[64 * s] = (uint16_t)e4m3_pair(x0 / scale, x1 / scale);
    }
    if (is_v) {
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        u32x4 r = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < kPage; ++s)
          r[s >> 2] |= (uint32_t)((codes[64 * s] >> (8 * d)) & 0xFFu) << (8 * (s & 3));
        *reinterpret_cast<u32x4*>(pool + (2 * lane + d) * kPage) = r;
      }
    } else {
      for (int s = 0; s < s1; ++s) reinterpret_cast<uint16_t*>(pool)[64 * s + lane] = codes[64 * s];
    }
    if (lane == 0) *scale_at = scale;
  }
}

// The table of entries of a call of many routes, by one workgroup, before the plan:
// -1 into every route's row of it, or 0.
__global__ __launch_bounds__(1024) void append_table_kernel(AppendRowsArgs a) {
  bool bad = false;
#pragma unroll 8
  for (int i = threadIdx.x; i < a.num_routes; i += 1024) bad |= bad_entries(a, i);
  bad = __syncthreads_or(bad);
  for (int i = threadIdx.x; i < a.num_routes; i += 1024) a.plan[4 * i] = bad ? -1 : 0;
  if (bad && threadIdx.x == 0) atomicOr(a.err_flags, KF_EFLAG_BAD_ROUTE);
}

// One workgroup per route: the check; the plan of its pages, or with DIRECT the
// pages themselves; the route's new end.  MANY routes: the table of entries has been
// read before, or with DIRECT there is a workgroup per entry, which reads it once, and
// the first one of a route works on it.
template <bool FP8, bool DIRECT, bool MANY>
__global__ __launch_bounds__(1024) void append_plan_kernel(AppendRowsArgs a) {
  __shared__ uint16_t lds[FP8 && DIRECT ? 16 * kPage * 64 : 1];
  int r = blockIdx.x;
  if constexpr (DIRECT && MANY) {
    __shared__ int s_route;
    if (threadIdx.x == 0) s_route = -1;
    __syncthreads();
    bool bad = false;
#pragma unroll 4
    for (int i = threadIdx.x; i < a.num_routes; i += 1024) {
      const int x = a.entry_begin[i], y = a.entry_begin[i + 1];
      bad |= x < 0 || y < x || y > a.num_entries;
      if (x == (int)blockIdx.x && y > x) s_route = i;  // (one, in a table that does not decrease)
    }
    bad = __syncthreads_or(bad);
    if (bad && threadIdx.x == 0) atomicOr(a.err_flags, KF_EFLAG_BAD_ROUTE);
    r = bad ? -1 : s_route;
    if (r < 0) return;
  } else if (MANY) {
    if (a.plan[4 * r] < 0) return;
  }
  int flag = 0;
  const int j0 = append_check<!DIRECT, !MANY>(a, r, flag);
  if (threadIdx.x == 0 && flag) atomicOr(a.err_flags, flag);
  if (!DIRECT && threadIdx.x == 0) a.plan[4 * r] = j0;
  if (j0 < 0) return;
  const int e0 = a.entry_begin[r], n = a.entry_begin[r + 1] - e0;
  const int base = a.routes[r].page_base;
  if constexpr (DIRECT) {
    const int p0 = j0 / kPage, pages = (j0 + n - 1) / kPage - p0 + 1, w = threadIdx.x >> 6;
    const int units = 2 * a.num_kv_heads;
    for (int64_t u = w; u < (int64_t)pages * units; u += 16) {
      const int p = p0 + (int)(u / units), k = (int)(u % units);
      const int s0 = p == p0 ? j0 % kPage : 0;
      const int s1 = min(kPage, j0 + n - p * kPage);
      append_page<FP8>(a, uniform(a.page_ids[base + p]), k >> 1, k & 1, s0, s1,
                       e0 + p * kPage + s0 - j0, lds + (FP8 ? w * kPage * 64 : 0));
    }
  } else if (threadIdx.x == 0) {
    a.plan[4 * r + 1] = e0;
    a.plan[4 * r + 2] = n;
    a.plan[4 * r + 3] = base;
  }
  __syncthreads();  // every thread has read tok_end before it moves
  if (threadIdx.x == 0) a.routes[r].tok_end += n;
}

// First page tile of route r, whose first entry is `entry`: its n / 16 + 2 pages fit
// before the next route's, as at most min(r, entry) routes before it have entries.
__host__ __device__ __forceinline__ int64_t append_first_tile(int entry, int r) {
  return (int64_t)(entry / kPage) + 2 * (int64_t)(r < entry ? r : entry);
}

// One wave per (page tile, KV head, K or V).
template <bool FP8>
__global__ __launch_bounds__(256) void append_tile_kernel(AppendRowsArgs a) {
  __shared__ uint16_t lds[FP8 ? 4 * kPage * 64 : 1];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t unit = (int64_t)blockIdx.x * 4 + w;
  const int units = 2 * a.num_kv_heads;
  const int64_t tile = unit / units;
  const int k = (int)(unit % units);
  // the last route whose first tile is at most `tile`: 64 probes a step
  int lo = 0, hi = a.num_routes;  // first(lo) <= tile < first(hi)
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, at = lo + lane * step;
    const bool in = at < hi && append_first_tile(a.entry_begin[at], at) <= tile;
    const uint64_t v = __ballot(in);
    // a table that decreases can answer anything; a plan is then never made
    const int last = v ? 63 - __builtin_clzll(v) : 0;
    lo += last * step;
    hi = min(hi, lo + step);
  }
  const int j0 = a.plan[4 * lo];
  if (j0 < 0) return;
  const int e0 = a.plan[4 * lo + 1], n = a.plan[4 * lo + 2], base = a.plan[4 * lo + 3];
  const int p0 = j0 / kPage;
  const int64_t p = p0 + tile - append_first_tile(e0, lo);
  if (p < p0 || p > (j0 + n - 1) / kPage) return;
  const int s0 = p == p0 ? j0 % kPage : 0;
  const int s1 = (int)min((int64_t)kPage, j0 + n - p * kPage);
  append_page<FP8>(a, uniform(a.page_ids[base + p]), k >> 1, k & 1, s0, s1,
                   (int)(e0 + p * kPage + s0 - j0), lds + (FP8 ? w * kPage * 64 : 0));
}

// --------------------------------------------------------------------- plan
__device__ __forceinline__ bool route_ok(const RowsArgs& a, int b, const int32_t* rp) {
  const int64_t n = (int64_t)rp[3] - rp[2], pages = n > 0 ? (n + kPage - 1) / kPage : 0;
  return rp[0] == b && n >= 0 && n <= INT32_MAX && rp[4] >= 0 && pages <= rp[5] &&
         pages <= a.max_pages_per_route && rp[4] + pages <= a.num_page_ids;
}

// Key tiles of a route's tokens.
__device__ __forceinline__ int64_t route_tiles(const int32_t* rp) {
  const int64_t n = (int64_t)rp[3] - rp[2];
  return n > 0 ? (n + kKeyTile - 1) / kKeyTile : 0;
}
constexpr int kMostKeys = 1 << 26;  // key tiles of a sequence that a plan tells apart

__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor((long long)x, m);
  return x;
}

// Key tiles of row tile t of a sequence whose first row sits at pos and whose routes
// hold `tiles` of them, of tokens first .. last - 1 (prompts that see a part of them: an
// estimate where the routes leave gaps or part-filled tiles).  Tokens / 32 would leave
// the tiles of short routes to the last part: 16 trees of 8 over 8K tokens in routes of
// 16 tokens 278 us, 599 that way, of 48 tokens 145 and 223, of 256 the same.
// (With a window: the tokens of the sinks and from the first row's window on, in the
// same proportion, and two tiles at their ends.)
template <bool TREE, bool WINDOW>
__device__ __forceinline__ int key_tiles(const RowsArgs& a, int pos, int t, int n, int tiles,
                                         int first, int last) {
  if (TREE) return tiles + (n + kKeyTile - 1) / kKeyTile;
  const int64_t rows = ((int64_t)(t + 1) * kRowTile - 1) / a.group;
  const int64_t end = pos + (rows < n ? rows : n - 1) + 1 - first, span = (int64_t)last - first;
  if (end <= 0 || span <= 0) return 0;
  if (WINDOW) {
    const int64_t e = end < span ? end : span;
    const int64_t row0 = (int64_t)t * kRowTile / a.group;
    int64_t lo = pos + row0 - a.window + 1 - first, si = (int64_t)a.sinks - first;
    lo = lo < 0 ? 0 : lo < e ? lo : e;
    si = si < 0 ? 0 : si < lo ? si : lo;
    const int64_t k = ((e - lo + si) * tiles + span - 1) / span + 2;
    return (int)(k < tiles ? k : tiles);
  }
  if (end >= span) return tiles;
  const int64_t plain = (span + kKeyTile - 1) / kKeyTile;
  return (int)(tiles == plain ? (end + kKeyTile - 1) / kKeyTile : (end * tiles + span - 1) / span);
}

// One workgroup: the row tiles of every sequence, cut into parts of at most `cap` key
// tiles, largest first (the grid is dealt out in order, so the last ones are small).
// Up to kPlanSeqs sequences are gathered by a thread per route and kept in LDS: 9 to
// 13 us, a chain of table reads, scans and one write.  More are read from memory by a
// wave per sequence: trees of 1000 sequences 588 us that way and 504 with a thread per
// route, of 64 267 and 262.
constexpr int kPlanSeqs = 1024;

template <bool TREE, bool WINDOW>
__global__ __launch_bounds__(1024) void rows_plan_kernel(RowsArgs a) {
  __shared__ unsigned long long s_work;
  __shared__ int s_most, s_least, s_recs, s_parts, s_splits, s_pairs;
  __shared__ int s_count[64], s_scan[16];
  __shared__ unsigned long long l_keys[kPlanSeqs];
  __shared__ int l_tiles[kPlanSeqs + 1], l_info[4 * kPlanSeqs], l_begin[kPlanSeqs + 1];
  __shared__ int l_route[kPlanSeqs + 1], l_pos[kPlanSeqs], l_seen[kPlanSeqs];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, B = a.num_seqs;
  const bool small = B <= kPlanSeqs;
  int* const tiles_of = small ? l_tiles : a.seq_tiles;  // first row tile of each sequence
  int* const info = small ? l_info : a.seq_info;        // key tiles, first and last token's end, bad
  const int* const begin = small ? l_begin : a.seq_row_begin;
  const int* const route = small ? l_route : a.seq_route_begin;
  const int* const pos = small ? l_pos : a.first_pos;
  int bad = 0, r0 = 0, r1 = 0;
  // the first route of a thread, on its way with the tables
  kf_route own{-1, 0, 0, 0, 0, 0};
  if (small && tid < a.num_routes) own = a.routes[tid];
  for (int b = tid; b <= B; b += 1024) {
    const int v = a.seq_row_begin[b];
    bad |= v < 0 || v > a.num_rows || (b > 0 && a.seq_row_begin[b - 1] > v);
    if (small) {
      l_begin[b] = v;
      l_route[b] = a.seq_route_begin[b];
      if (!TREE && b < B) l_pos[b] = a.first_pos[b];
    }
  }
  if (small && tid < B) {
    r0 = a.seq_route_begin[tid];
    r1 = a.seq_route_begin[tid + 1];
    const bool wrong = r0 < 0 || r1 < r0 || r1 > a.num_routes;
    l_keys[tid] = 0;
    l_seen[tid] = 0;
    l_info[4 * tid + 1] = INT32_MAX;
    l_info[4 * tid + 2] = wrong;
    l_info[4 * tid + 3] = INT32_MIN;
  }
  if (tid == 0) s_work = 0, s_most = 0, s_least = INT32_MAX;
  if (tid < 64) s_count[tid] = 0;
  if (__syncthreads_or(bad)) {
    if (tid == 0) {
      a.head[0] = -1;
      a.head[1] = 0;
      a.head[2] = 1;
      atomicOr(a.err_flags, KF_EFLAG_BAD_ROUTE);
    }
    return;
  }
  // the key tiles of the sequences' routes: a thread per route, or a wave per sequence
  if (small) {
    for (int r = tid; r < a.num_routes; r += 1024) {
      if (r != tid) own = a.routes[r];
      const int32_t* rp = reinterpret_cast<const int32_t*>(&own);
      const int b = rp[0];
      if (b < 0 || b >= B || r < l_route[b] || r >= l_route[b + 1]) continue;
      if (route_ok(a, b, rp)) {
        atomicAdd(&l_seen[b], 1);
        atomicAdd(&l_keys[b], (unsigned long long)route_tiles(rp));
        if (rp[3] > rp[2]) {
          atomicMin(&l_info[4 * b + 1], rp[2]);
          atomicMax(&l_info[4 * b + 3], rp[3]);
        }
      }
    }
    __syncthreads();
    if (tid < B) {
      const int n = l_begin[tid + 1] - l_begin[tid];
      // each of its routes has to have been seen
      const bool wrong = l_info[4 * tid + 2] || l_seen[tid] != r1 - r0 ||
                         (TREE && n > KF_MAX_DRAFT);
      l_info[4 * tid] = (int)min(l_keys[tid], (unsigned long long)kMostKeys);
      l_info[4 * tid + 2] = wrong;
      if (wrong && n > 0) atomicOr(a.err_flags, KF_EFLAG_BAD_ROUTE);
    }
  } else {
    for (int b = w; b < B; b += 16) {
      const int n = begin[b + 1] - begin[b];
      if (n == 0) continue;
      const int q0 = a.seq_route_begin[b], q1 = a.seq_route_begin[b + 1];
      bool wrong = q0 < 0 || q1 < q0 || q1 > a.num_routes || (TREE && n > KF_MAX_DRAFT);
      int64_t keys = 0;
      int first = INT32_MAX, last = INT32_MIN;
      if (!wrong) {
        bool mine = true;
        for (int r = q0 + lane; r < q1; r += 64) {
          const int32_t* rp = reinterpret_cast<const int32_t*>(a.routes + r);
          mine &= route_ok(a, b, rp);
          keys += route_tiles(rp);
          if (rp[3] > rp[2]) {
            first = min(first, rp[2]);
            last = max(last, rp[3]);
          }
        }
        wrong = __ballot(!mine) != 0;
      }
      keys = wave_sum(keys);
#pragma unroll
      for (int m = 32; m >= 1; m >>= 1) {
        first = min(first, __shfl_xor(first, m));
        last = max(last, __shfl_xor(last, m));
      }
      if (lane == 0) {
        info[4 * b] = (int)min(keys, (int64_t)kMostKeys);
        info[4 * b + 1] = first;
        info[4 * b + 2] = wrong;
        info[4 * b + 3] = last;
        if (wrong) atomicOr(a.err_flags, KF_EFLAG_BAD_ROUTE);
      }
    }
  }
  // their first row tiles
  int sum = 0;
  for (int b0 = 0; b0 < B; b0 += 1024) {
    const int b = b0 + tid;
    const int64_t n = b < B ? begin[b + 1] - begin[b] : 0;
    const int mine = (int)((n * a.group + kRowTile - 1) / kRowTile);
    int x = mine;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int y = __shfl_up(x, m);
      if (lane >= m) x += y;
    }
    if (lane == 63) s_scan[w] = x;
    __syncthreads();
    int before = sum;
    for (int i = 0; i < 16; ++i) {
      if (i < w) before += s_scan[i];
      sum += s_scan[i];
    }
    if (b < B) tiles_of[b] = before + x - mine;
    __syncthreads();
  }
  if (tid == 0) tiles_of[B] = sum;
  __syncthreads();
  const int T = min(sum, a.max_tiles);
  // a tile's sequence and key tiles; a bad sequence's tile has one
  auto search = [&](int t, int& b, bool& wrong) -> int {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      (tiles_of[mid] <= t ? lo : hi) = mid;
    }
    b = lo;
    wrong = info[4 * b + 2] != 0;
    if (wrong) return 1;
    const int k = key_tiles<TREE, WINDOW>(a, TREE ? 0 : pos[b], t - tiles_of[b],
                                          begin[b + 1] - begin[b], info[4 * b], info[4 * b + 1],
                                          info[4 * b + 3]);
    return k > 0 ? k : 1;
  };
  int own_b = 0, own_k = 0;  // this thread's first tile
  bool own_wrong = false;
  if (tid < T) own_k = search(tid, own_b, own_wrong);
  auto look = [&](int t, int& b, bool& wrong) -> int {
    if (t >= 1024) return search(t, b, wrong);
    b = own_b;
    wrong = own_wrong;
    return own_k;
  };
  unsigned long long work = 0;
  int most = 0, least = INT32_MAX;
  for (int t = tid; t < T; t += 1024) {
    int b;
    bool wrong;
    const int k = look(t, b, wrong);
    work += k;
    most = max(most, k);
    least = min(least, k);
  }
  if (64 * w < T) {
    if (a.may_split) work = (unsigned long long)wave_sum((int64_t)work);
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
      most = max(most, __shfl_xor(most, m));
      least = min(least, __shfl_xor(least, m));
    }
    if (lane == 0) {
      atomicAdd(&s_work, work);
      atomicMax(&s_most, most);
      atomicMin(&s_least, least);
    }
  }
  __syncthreads();
  most = s_most;
  least = s_least;
  int cap = most;
  const bool may_split = a.may_split && (int64_t)T * a.num_kv_heads < kSplitSlots * (int64_t)a.slots;
  // Tiles of much the same length that do not fill whole rounds of the workgroups:
  // the rounds' tiles stay whole and the others (all of them, below one round) are cut
  // into `tail` parts, so that the last round is a shorter one.
  const int round = max(1, a.slots / a.num_kv_heads), whole = T / round * round;
  int tail = 1;
  if (may_split && least >= kEqualSteps && (int64_t)least * 4 >= (int64_t)most * 3) {
    const int r = T / round, left = T - whole;
    int turns = left > 0;  // of the last round, in parts
    for (int p = 2; p <= 8 && left * p <= a.max_recs; ++p) {
      const int n = (left * p + round - 1) / round;
      if (n * tail < turns * p) turns = n, tail = p;
    }
    if ((r * tail + turns) * 10 > 9 * (r + 1) * tail) tail = 1;
  }
  if (may_split && tail == 1) {
    const unsigned long long share = (s_work * a.num_kv_heads + a.slots - 1) / a.slots;
    cap = (int)min((unsigned long long)most, max(share, (unsigned long long)kMinPart));
    // An even share per workgroup, in one round.  Where that leaves more parts than
    // workgroups (tiles of different lengths), smaller ones pack better: 48 agentic
    // trees 817 us with the share itself, 736 with 1/2 of it, 688 with 5/8, 694 with
    // 11/16, 699 with 3/4; 40 short prompts over 1K .. 30K tokens 359 (9/16) and 345
    // (5/8).  With as many tiles as workgroups (multi-head prompts) halves cost
    // 94 -> 131.
    bool cut = (int64_t)T * a.num_kv_heads >= a.slots;
    for (;;) {  // until the records of split tiles fit
      __syncthreads();
      if (tid == 0) s_recs = s_parts = 0;
      __syncthreads();
      int64_t recs = 0;
      int whole = 0;
      for (int t = tid; t < T; t += 1024) {
        int b;
        bool wrong;
        const int k = look(t, b, wrong);
        if (k > cap)
          recs += (k + cap - 1) / cap;
        else
          ++whole;
      }
      if (64 * w < T) {
        recs = min(wave_sum(recs), (int64_t)1 << 24);
        whole = (int)wave_sum(whole);
        if (lane == 0) {
          atomicAdd(&s_recs, (int)recs);
          atomicAdd(&s_parts, (int)recs + whole);
        }
      }
      __syncthreads();
      const bool more = (int64_t)s_parts * a.num_kv_heads > a.slots;
      if (!cut && more && cap > kMinPart)
        cap = max((int)((int64_t)cap * 5 / 8), kMinPart);
      else if (s_recs <= a.max_recs)
        break;
      else
        cap += cap / 4 + 1;
      cut = true;
    }
  }
  __syncthreads();
  if (tid == 0) s_recs = 0, s_splits = 0, s_pairs = 1;
  const int per = max(1, min(cap, most));
  // by size of their parts, largest first; prompts that stay whole sequence after
  // sequence, the longest first, so that the tiles that run at a time read the same
  // tokens (64 prompts of 420 tokens 249 -> 237 us, of 128 tokens 65 -> 60,
  // 16 of 100 .. 2000 tokens the same within 2 %)
  const bool by_seq = !TREE && small && cap >= most && tail == 1;
  auto place = [&](int part) { return 63 - (int)((int64_t)part * 63 / per); };
  int own_size = 0;  // by_seq: of this thread's sequence
  if (by_seq) {
    if (tid < B && l_tiles[tid + 1] > l_tiles[tid]) {
      int b;
      bool wrong;
      own_size = search(min(l_tiles[tid + 1], T) - 1, b, wrong);
      atomicAdd(&s_count[place(own_size)], l_tiles[tid + 1] - l_tiles[tid]);
    }
  } else {
    for (int t = tid; t < T; t += 1024) {
      int b;
      bool wrong;
      const int k = look(t, b, wrong), parts = (k + per - 1) / per;
      atomicAdd(&s_count[place((k + parts - 1) / parts)], parts);
    }
  }
  __syncthreads();
  if (w == 0) {
    const int mine = s_count[lane];
    int x = mine;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int y = __shfl_up(x, m);
      if (lane >= m) x += y;
    }
    s_count[lane] = x - mine;
    if (lane == 63) a.head[0] = x + (tail - 1) * (T - whole);
  }
  __syncthreads();
  if (by_seq) {
    // l_keys: where a sequence's items begin
    if (own_size > 0)
      l_keys[tid] = atomicAdd(&s_count[place(own_size)], l_tiles[tid + 1] - l_tiles[tid]);
    __syncthreads();
  }
  for (int t = tid; t < T; t += 1024) {
    int b;
    bool wrong;
    const int k = look(t, b, wrong);
    int parts = (k + per - 1) / per;
    int at;
    if (tail > 1) {
      // Every tile is whole but for the last round's.  Which ones those are must not
      // follow from the order of atomics: a split rounds its sums in another order.
      // Last tile first, as a prompt's later rows see more: 5 chunks of 1024 rows
      // behind 30K tokens 2598 us, first tile first 2624.
      at = T - 1 - t;
      if (at >= whole) {
        parts = tail;
        at = whole + (at - whole) * tail;
      }
    } else {
      at = by_seq ? (int)l_keys[b] + l_tiles[b + 1] - 1 - t
                  : atomicAdd(&s_count[place((k + parts - 1) / parts)], parts);
    }
    RowsItem it;
    it.seq = wrong ? -1 - b : b;
    it.tile = t - tiles_of[b];
    it.rec = -1;
    it.row0 = begin[b];
    it.rows = begin[b + 1] - begin[b];
    it.first_pos = TREE ? 0 : pos[b];
    it.route0 = route[b];
    it.route1 = route[b + 1];
    it.tok_begin = it.tok_end = it.page_base = 0;
    if (!wrong && it.route0 < it.route1) {
      const kf_route& first = a.routes[it.route0];
      it.tok_begin = first.tok_begin;
      it.tok_end = first.tok_end;
      it.page_base = first.page_base;
    }
    it.pad[0] = it.pad[1] = it.pad[2] = 0;
    if (parts > 1) {
      it.rec = atomicAdd(&s_recs, parts);
      const int64_t pairs = (int64_t)it.rows * a.group - (int64_t)it.tile * kRowTile;
      a.splits[atomicAdd(&s_splits, 1)] =
          RowsSplit{it.tile, it.rec, parts, it.row0, it.rows, {0, 0, 0}};
      atomicMax(&s_pairs, (int)min(pairs, (int64_t)kRowTile));
    }
    for (int p = 0; p < parts; ++p) {
      it.key0 = (int)((int64_t)k * p / parts);
      it.key1 = p + 1 < parts ? (int)((int64_t)k * (p + 1) / parts) : INT32_MAX;
      a.items[at + p] = it;
      if (parts > 1) it.rec += 1;
    }
  }
  __syncthreads();
  if (tid == 0) {
    a.head[1] = s_splits;
    a.head[2] = s_pairs;
  }
}

// Without a plan (a.parts > 0: launches of up to 64 sequences and little work):
// row tile `tile` of the launch, looked up by a wave.  -1: a bad table of rows;
// 0: there is no such tile; 1: b and its own tile.
__device__ __forceinline__ int find_tile(const RowsArgs& a, int tile, int lane, int& b, int& own,
                                         int& row0, int& rows) {
  int n = 0, i0 = 0;
  bool bad = false;
  if (lane < a.num_seqs) {
    i0 = a.seq_row_begin[lane];
    const int i1 = a.seq_row_begin[lane + 1];
    bad = i0 < 0 || i1 < i0 || i1 > a.num_rows;
    n = bad ? 0 : i1 - i0;
  }
  if (__ballot(bad)) return -1;
  const int mine = (n * a.group + kRowTile - 1) / kRowTile;
  int x = mine;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int y = __shfl_up(x, m);
    if (lane >= m) x += y;
  }
  const uint64_t found = __ballot(x > tile);
  if (!found) return 0;
  b = uniform(__builtin_ctzll(found));
  own = tile - __builtin_amdgcn_readlane(x - mine, b);
  row0 = __builtin_amdgcn_readlane(i0, b);
  rows = __builtin_amdgcn_readlane(n, b);
  return 1;
}

// Parts of a row tile of `all` key tiles, of `most` for which the launch has
// workgroups: its page table may reserve many times what it holds.
__device__ __forceinline__ int tile_parts(int most, int64_t all) {
  const float by_turns = 2.0f * __builtin_sqrtf((float)all);
  return max(1, min(most, min((int)((all + kMinPart - 1) / kMinPart), (int)by_turns)));
}

// ---------------------------------------------------------------- attention
// The x of the lower and of the upper of this lane and the one 32 away.  (The
// compiler's builtin for this instruction returns its first result twice.)
__device__ __forceinline__ f32x2 both_halves(float x) {
  float lo = x, hi = x;
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(lo), "+v"(hi));
  return f32x2{lo, hi};
}
__device__ __forceinline__ float max_halves(float x) {
  const f32x2 u = both_halves(x);
  return fmaxf(u.x, u.y);
}
__device__ __forceinline__ float sum_halves(float x) {
  const f32x2 u = both_halves(x);
  return u.x + u.y;
}

// The visible tokens of a sequence as tiles of 32, route after route.
struct Walk {
  int r, r_end;   // current route, the sequence's last + 1
  int base, n;    // its first page id's index, its tokens that the row tile sees (with a
                  // window: those before the tile's last row, in its window or not)
  int tb;         // its first token
  int j, tiles;   // next tile of the route, its tiles (with a window and no JUMP: those up to
                  // the end of its sinks, then all of them)
  int from, to;   // JUMP: the tile behind the sinks, where the window begins
  int pid[2];     // page ids of that tile (sent for a step ahead, awaited at its barrier)
};

// One tile: its first token's position (of drafted tokens: its first row) and how
// many of its tokens there are (0: there is no such tile).
struct Tile {
  int pos0, left;
  int kind;  // bits 0 and 1: its pages outside the pool; kDraft, kPart
};
constexpr int kDraft = 4;  // drafted tokens
constexpr int kPart = 8;   // fewer than 32 tokens
// Its pages (0 for one outside the pool), and where they begin in the pools, in
// bytes.
struct Pages {
  int pid[2];
  uint64_t at[2];
};

__device__ __forceinline__ int visible(int begin, int end, int last_pos) {
  const int64_t n = (int64_t)end - begin, see = (int64_t)last_pos + 1 - begin;
  return (int)(see < 0 ? 0 : see < n ? see : n);
}

__device__ __forceinline__ void walk_ids(const RowsArgs& a, Walk& w) {
  const int last = (w.n - 1) / kPage;
#pragma unroll
  for (int i = 0; i < 2; ++i) w.pid[i] = fixed(a.page_ids)[w.base + min(2 * w.j + i, last)];
}

// The tokens that a row tile sees: those up to its last row's position; with a window
// those before low (where its first row's window begins) only if they are sinks.
struct Sight {
  int last_pos, low, sinks;
};

// The first token of the window of a row at first_pos + i.
__device__ __forceinline__ int window_begin(const RowsArgs& a, int first_pos, int i) {
  const int64_t x = (int64_t)first_pos + i - a.window + 1;
  return (int)max((int64_t)INT32_MIN, min((int64_t)INT32_MAX, x));
}

// A route's tokens begin .. end - 1 in that sight: n, and its tiles [0, from) and
// [to, tiles).
template <bool WINDOW>
__device__ __forceinline__ void route_sight(const Sight& s, int begin, int end, int& n, int& from,
                                            int& to, int& tiles) {
  n = visible(begin, end, s.last_pos);
  tiles = (n + kKeyTile - 1) / kKeyTile;
  from = to = 0;
  if (WINDOW) {
    const int64_t before = (int64_t)s.low - begin;  // tokens before the window
    if (before >= n)
      to = tiles;
    else
      to = before <= 0 ? 0 : (int)before / kKeyTile;
    from = (visible(begin, end, min(s.last_pos, s.sinks - 1)) + kKeyTile - 1) / kKeyTile;
    to = max(to, from);
    if (to == tiles) to = tiles = from;
  }
}
template <bool WINDOW>
__device__ __forceinline__ int sight_tiles(const Sight& s, int begin, int end) {
  int n, from, to, tiles;
  route_sight<WINDOW>(s, begin, end, n, from, to, tiles);
  return tiles - to + from;
}

// With a window, the walk gets from a route's sinks to its window either by a look at
// every tile (JUMP) or as it gets to another route, from the route's row.  bf16's kernel
// has the scalar registers for the former, fp8's has not: 16K-token prompts, window 2048,
// 609 us and 625; fp8 chunks, window 8000, 819 and 740.
// Enters the route begin .. end - 1 at the k-th of its visible tiles.
template <bool WINDOW, bool JUMP>
__device__ __forceinline__ void walk_route(Walk& w, const Sight& s, int begin, int end, int base,
                                           int k) {
  int from, to;
  route_sight<WINDOW>(s, begin, end, w.n, from, to, w.tiles);
  w.tb = begin;
  w.base = base;
  w.j = k;
  if (WINDOW && k >= from)
    w.j = k - from + to;
  else if (WINDOW && !JUMP && from < to)
    w.tiles = from;
  if (JUMP) {
    w.from = from;
    w.to = to;
  }
}

// Behind a route's last tile: the next route that has any.
template <bool WINDOW, bool JUMP>
__device__ __forceinline__ void walk_on(const RowsArgs& a, Walk& w, const Sight& s) {
  while (w.j >= w.tiles && w.r < w.r_end) {
    if (WINDOW && !JUMP) {  // from the sinks to the window of the same route
      const auto* rp = fixed(reinterpret_cast<const int32_t*>(a.routes)) + 6 * (int64_t)w.r;
      int n, from, to, tiles;
      route_sight<WINDOW>(s, rp[2], rp[3], n, from, to, tiles);
      if (w.tiles == from && from < to) {
        w.j = to;
        w.tiles = tiles;
        break;
      }
    }
    if (++w.r < w.r_end) {
      const auto* rp = fixed(reinterpret_cast<const int32_t*>(a.routes)) + 6 * (int64_t)w.r;
      if (WINDOW) {
        walk_route<WINDOW, JUMP>(w, s, rp[2], rp[3], rp[4], 0);
      } else {
        w.n = visible(rp[2], rp[3], s.last_pos);
        w.tb = rp[2];
        w.base = rp[4];
        w.tiles = (w.n + kKeyTile - 1) / kKeyTile;
        w.j = 0;
      }
    }
  }
  if (w.r < w.r_end) walk_ids(a, w);
}

// The visible tiles of a sequence's routes; -1 if one of them is bad.  The first
// route of a sequence goes into its item.
template <bool WINDOW>
__device__ __forceinline__ int count_tiles(const RowsArgs& a, int b, int r0, int r1, const Sight& s,
                                           int lane, RowsItem& it) {
  it.tok_begin = it.tok_end = it.page_base = 0;
  int64_t tiles = 0;
  bool bad = r0 < 0 || r1 < r0 || r1 > a.num_routes;
  if (bad) return -1;
  if (r1 > r0) {
    const auto* at = fixed(reinterpret_cast<const int32_t*>(a.routes)) + 6 * (int64_t)r0;
    const int32_t row[6] = {at[0], at[1], at[2], at[3], at[4], at[5]};
    it.tok_begin = row[2];
    it.tok_end = row[3];
    it.page_base = row[4];
    if (r1 - r0 == 1)
      return route_ok(a, b, row) ? sight_tiles<WINDOW>(s, row[2], row[3]) : -1;
  }
  for (int r = r0 + lane; r < r1; r += 64) {
    const int32_t* rp = reinterpret_cast<const int32_t*>(a.routes + r);
    bad |= !route_ok(a, b, rp);
    tiles += sight_tiles<WINDOW>(s, rp[2], rp[3]);
  }
  return __ballot(bad) ? -1 : uniform((int)min(wave_sum(tiles), (int64_t)1 << 30));
}

// Positions the walk at key tile k of the sequence; tiles of a route: its
// visible tokens / 32, rounded up.  Sixty-four routes at a time.
template <bool WINDOW, bool JUMP>
__device__ __forceinline__ void walk_to(const RowsArgs& a, Walk& w, int r0, int r1, const Sight& s,
                                        int64_t k, int lane) {
  w.r = w.r_end = r1;
  w.j = w.tiles = 0;
  w.from = w.to = 0;
  w.base = w.n = w.tb = w.pid[0] = w.pid[1] = 0;
  for (int r = r0; r < r1; r += 64) {
    int n = 0, tb = 0, te = 0, base = 0;
    if (r + lane < r1) {
      const kf_route& row = a.routes[r + lane];
      tb = row.tok_begin;
      te = row.tok_end;
      base = row.page_base;
      if (!WINDOW) n = visible(tb, te, s.last_pos);
    }
    const int tiles = WINDOW ? sight_tiles<WINDOW>(s, tb, te) : (n + kKeyTile - 1) / kKeyTile;
    int64_t x = tiles;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int64_t y = __shfl_up((long long)x, m);
      if (lane >= m) x += y;
    }
    const uint64_t found = __ballot(x > k);
    if (found) {
      const int at = uniform(__builtin_ctzll(found));
      w.r = r + at;
      if (WINDOW) {
        const int j = uniform((int)(k - __shfl((long long)(x - tiles), at)));
        walk_route<WINDOW, JUMP>(w, s, __builtin_amdgcn_readlane(tb, at),
                                 __builtin_amdgcn_readlane(te, at),
                                 __builtin_amdgcn_readlane(base, at), j);
      } else {
        w.n = __builtin_amdgcn_readlane(n, at);
        w.tb = __builtin_amdgcn_readlane(tb, at);
        w.base = __builtin_amdgcn_readlane(base, at);
        w.tiles = __builtin_amdgcn_readlane(tiles, at);
        w.j = uniform((int)(k - __shfl((long long)(x - tiles), at)));
      }
      walk_ids(a, w);
      return;
    }
    k -= __shfl((long long)x, 63);
  }
}

// Byte offset of 16-byte chunk c of token row `row` in a K tile in LDS: the
// exclusive or spreads the rows that a matrix operand reads at once over all
// banks.
__device__ __forceinline__ int k_at(int row, int c) { return row * 256 + ((c ^ (row & 15)) << 4); }
// ... of half hh (slots 8 hh ..) of row d of page `page` in a V tile: the order
// in which the lanes of a matrix operand read it.
__device__ __forceinline__ int v_at(int page, int d, int hh) {
  return page * 4096 + (d >> 5) * 1024 + hh * 512 + (d & 31) * 16;
}

// 16 bytes a lane from memory straight into LDS, 1 KiB a wave.  ONCE: nothing else
// will read them soon (the non-temporal hint): a tree's cache is read by one
// workgroup, or by two beside each other, a prompt's by many one after another.
// Agentic trees 888 -> 824 us, 32-row trees over 32K 433 -> 425 with the hint; a
// 16K-token prompt would go 2307 -> 2456.  Decode steps of 48 sequences, window 4096,
// 153 -> 130, prompts with a window of 2048 611 -> 680.
template <bool ONCE>
__device__ __forceinline__ void to_lds(const char* g, char* l) {
  __builtin_amdgcn_global_load_lds(
      (const __attribute__((address_space(1))) uint32_t*)g,
      (__attribute__((address_space(3))) uint32_t*)(__attribute__((address_space(3))) void*)l, 16,
      0, ONCE ? 2 : 0);
}

// 4 bytes each of four lanes into LDS.
__device__ __forceinline__ void to_lds4(const float* g, float* l) {
  __builtin_amdgcn_global_load_lds(
      (const __attribute__((address_space(1))) uint32_t*)g,
      (__attribute__((address_space(3))) uint32_t*)(__attribute__((address_space(3))) void*)l, 4, 0,
      0);
}

// A barrier for what the waves wrote to LDS themselves.  (__syncthreads waits
// for loads on their way into LDS too.)
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Which of 8 bf16 are infinite or NaN: their bits set.
__device__ __forceinline__ u32x4 not_finite(u32x4 x) {
  u32x4 m;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m[i] = ((x[i] & 0x7F80u) == 0x7F80u ? 0x0000FFFFu : 0u) |
           ((x[i] & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
  return m;
}

// The chunks tid, tid + 256 of a V tile in LDS: zeroes the slots from `left` on
// (they may hold anything, and a weight of 0 does not undo an infinity); whether
// the others hold infinities or NaN.
__device__ __forceinline__ bool cut_tile(int left, int tid, char* lv) {
  u32x4 odd = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    u32x4* v = reinterpret_cast<u32x4*>(lv + 4096 * i) + tid;
    u32x4 x = *v;
    const int first = 16 * i + 8 * ((tid >> 5) & 1);
    if (left < kKeyTile) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        x[k] &= (first + 2 * k < left ? 0x0000FFFFu : 0u) |
                (first + 2 * k + 1 < left ? 0xFFFF0000u : 0u);
      *v = x;
    }
    odd |= not_finite(x);
  }
  return (odd[0] | odd[1] | odd[2] | odd[3]) != 0;
}

// The same chunks: zeroes infinities and NaN.
__device__ __forceinline__ void tame_tile(int tid, char* lv) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    u32x4* v = reinterpret_cast<u32x4*>(lv + 4096 * i) + tid;
    *v &= ~not_finite(*v);
  }
}

// The drafted tokens t0 .. of a sequence as a tile of K, and of V, which is turned
// around on its way.
__device__ __forceinline__ u32x4 draft_chunk(const RowsArgs& a, const uint16_t* x, int row0,
                                             int row, int n, int g, int c) {
  return row < n ? ld16(x + (size_t)(row0 + row) * a.kv_stride + (size_t)g * kDim + 8 * c)
                 : u32x4{0, 0, 0, 0};
}
__device__ __forceinline__ void draft_k(const RowsArgs& a, int row0, int t0, int n, int g, int tid,
                                        char* lk) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = 16 * i + (tid >> 4), c = tid & 15;
    *reinterpret_cast<u32x4*>(lk + k_at(row, c)) =
        draft_chunk(a, a.k_draft, row0, t0 + row, n, g, c);
  }
  // so that no later register waits for these loads, and with them for all that
  // are on their way into LDS
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
}
__device__ __forceinline__ void draft_v(const RowsArgs& a, int row0, int t0, int n, int g, int tid,
                                        char* lv) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int slot = tid >> 4, c = tid & 15;
    const u32x4 v = draft_chunk(a, a.v_draft, row0, t0 + 16 * i + slot, n, g, c);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      *reinterpret_cast<uint16_t*>(lv + v_at(i, 8 * c + e, slot >> 3) + 2 * (slot & 7)) =
          (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);
}

// Softmax state of one (row, head) per lane column q = lane % 32, shared by the
// two half waves: lane (half, q) holds dims 32 dt + 8 i + 4 half + j at
// o[dt][4 i + j], m is the running reference (base 2), l the lane's own sum.
struct State {
  f32x16 o[4];
  float m, l;
};

// A tile's scores, S^T = K Q^T: matrix row 8 i + 4 half + j of 32 is token
// 16 (i / 2) + 8 half + 4 (i % 2) + j, so that a lane's 16 results are the 8 slots
// 8 half .. of two pages: just the p that the lane feeds to O^T += V^T P^T, whose
// depth of 16 is one page.  No value crosses lanes between the products.
__device__ __forceinline__ f32x16 scores(const u32x4 (&k)[8], const u32x4 (&q)[8]) {
  f32x16 s;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s = mfma32(k[i], q[i], s);
  return s;
}
__device__ __forceinline__ void load_v(const char* lv, int lane, u32x4 (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const u32x4*>(lv + 16 * lane + 1024 * i);
}
__device__ __forceinline__ void load_k(const char* lk, int ka, u32x4 (&k)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) k[i] = *reinterpret_cast<const u32x4*>(lk + (ka ^ (32 * i)));
}

// Infinities and NaN of a V tile into the outputs of the rows that see them (a
// product would spread them to all 32 rows, whose weights of 0 do not undo them).
__device__ __forceinline__ void add_odd(const char* lv, uint32_t sees, const u32x4 (&p)[2], int lane,
                                        State& st) {
  const int half = lane >> 5;
#pragma unroll 1
  for (int t = 0; t < kKeyTile; ++t) {
    uint32_t two = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i == (t >> 4) * 4 + ((t & 7) >> 1)) two = p[i >> 2][i & 3];
    const uint32_t w = (uint32_t)__shfl((int)two, (lane & 31) + 32 * ((t >> 3) & 1));
    const float pt = __builtin_bit_cast(float, t & 1 ? w & 0xFFFF0000u : w << 16);
    const bool see = sees >> t & 1;
    const char* col = lv + v_at(t >> 4, 4 * half, (t >> 3) & 1) + 2 * (t & 7);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int k = 0; k < 16; ++k) {  // dim 32 dt + 8 (k / 4) + 4 half + k % 4
        if (k % 4 == 0) asm volatile("" ::: "memory");  // few loads at a time: registers
        const uint32_t x = *reinterpret_cast<const uint16_t*>(
            col + 1024 * dt + 16 * (8 * (k >> 2) + (k & 3)));
        if (see && (x & 0x7F80u) == 0x7F80u)
          st.o[dt][k] += pt * __builtin_bit_cast(float, x << 16);
      }
  }
}

// NaN into the outputs of the (row, head) pairs [m0, m1) of KV head g of rows
// row0 ...
__device__ __forceinline__ void fill_nan(const RowsArgs& a, int row0, int64_t m0, int64_t m1, int g, int tid,
                         int nt) {
  const int G = a.group;
  for (int64_t x = m0 * 16 + tid; x < m1 * 16; x += nt) {
    const int64_t m = x >> 4, at = (row0 + m / G) * a.num_q_heads + g * G + m % G;
    *reinterpret_cast<u32x4*>(a.out + at * kDim + 8 * (x & 15)) =
        u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
    if ((x & 15) == 0) a.lse[at] = qnan();
  }
}

// One work item of one KV head: four waves of 32 (row, head) pairs each, over
// K/V tiles of 32 tokens that they share through LDS, three tiles on their way
// while one is worked on.  The scores of a tile are computed a step before its
// weights, beside the weights of the tile before it: the matrix cores take the
// one while the vector units take the other.  bf16 pages go from memory into
// their tile.  fp8 pages go into rings of their own (4 KiB); the lanes that loaded
// a chunk widen it into one of two tiles a step before it is needed.
//
// One pass over the keys: m is a reference near the largest score so far, l = sum
// 2^(s - m), o = sum 2^(s - m) v, scores in units of log2; out = o / l, lse =
// (m + log2 l) ln 2.  l and o are float32; the weights are rounded to bf16 for their
// product with V, each by at most 2^-8 of it, the output's own rounding, and
// independently of each other.
//
// 128 pairs a workgroup and two workgroups a compute unit: the outputs, scores and
// operands of 32 pairs a wave take 248 of 256 registers, and the rings 64 of 80 KiB.
// A step of 64 tokens (one buffer) took 2500 us where this takes 2200, rings of five
// tiles the same.  16K-token prompt, 32 / 8 heads: 2150 .. 2330 us on different
// cards, 0.95 .. 1.02 PFLOP/s of its causal work, where the largest plain product
// reaches 1.28 .. 1.40.  A wave's step issues 106 vector, 85 scalar, 16 LDS and 16
// matrix instructions; the matrix cores are busy 49 % of the time.  In every step the
// wave waits for the page ids that it has just sent for (scalar loads count with LDS,
// whose counter the barrier waits for) and for all sixteen operands before its first
// product.  fp8 chunks over 32K tokens, 64 / 8 heads: 2690 .. 2800 us, 0.80 PFLOP/s: 155
// vector, 89 scalar and 23 LDS instructions a step with the widening, whose stores
// conflict (0.7 cycles per LDS instruction), and V's operands are read in pairs behind
// the softmax.  fp8 trees have scalar registers spilled in the loop as well (some 140;
// 120 scalar instructions a step).  bf16 trees of few rows wait for memory: 48 over 2K ..
// 64K tokens, 4.1 GB, 678 us, 6.0 TB/s.
template <bool FP8, bool TREE, bool WINDOW, bool ONCE>
struct Work {
  static constexpr bool kJump = WINDOW && !FP8;
  const RowsArgs& a;
  int tid, lane, wave, g;
  int row0, n_rows;
  bool any;                  // the wave has rows
  float c;
  u32x4 q[8];
  // positions: the lane's row, the wave's and the workgroup's first, the workgroup's last
  int pos, pos_min, tile_min, last_pos;
  // with a window, where it begins: of the lane's row, of the workgroup's last and first
  int low, tile_low, first_low;
  uint64_t draft;            // drafted rows that the lane's row sees
  Walk walk;
  int left;                  // tiles of this part still to come
  int drafts;                // drafted tokens still to come
  Pages pages;               // of the last tile (bf16: whose V is still to be sent for)
  uint64_t head_at;          // the KV head in page 0, and the distance of two pages
  uint32_t page_bytes;
  uint32_t koff, voff;
  const float* scale_of_head;  // of page 0: lanes 0 and 1 K's, 2 and 3 V's
  int ka;
  f32x16 s;                  // scores of the next tile
  State st;
  int flag, steps;
  int* odd_step;             // LDS: the last step whose tile holds infinities or NaN

  // The next tile; the page ids of the one behind it are sent for.
  __device__ __forceinline__ Tile take(Pages& pg) {
    Tile t{0, 0, 0};
    if (__builtin_expect(left > 0 && walk.r < walk.r_end, 1)) {
      --left;  // (from INT32_MAX, where the part has no end, it never comes to 0)
      const int tok0 = walk.j * kKeyTile;
      t.pos0 = walk.tb + tok0;
      t.left = walk.n - tok0;
      if (t.left < kKeyTile) t.kind = kPart;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int pid = walk.pid[i];
        if (__builtin_expect((uint32_t)pid >= (uint32_t)a.num_pages, 0)) {
          pid = 0;
          if (kPage * i < t.left) t.kind |= 1 << i;
        }
        pg.at[i] = head_at + (uint64_t)(uint32_t)pid * page_bytes;
        pg.pid[i] = pid;
      }
      ++walk.j;
      if (kJump && walk.j == walk.from) walk.j = walk.to;
      if (__builtin_expect(walk.j < walk.tiles, 1))
        walk_ids(a, walk);
      else
        walk_on<WINDOW, kJump>(a, walk, Sight{last_pos, first_low, a.sinks});
    } else if (TREE && drafts > 0) {
      t.pos0 = n_rows - drafts;
      t.left = drafts;
      t.kind = kDraft;
      drafts -= kKeyTile;
    }
    return t;
  }

  // Whether some token of the tile is no sink (0 or 1: joined without a branch).
  __device__ __forceinline__ int not_sinks(const Tile& t) const {
    return __builtin_elementwise_sub_sat(a.sinks, t.pos0) < kKeyTile;
  }

  __device__ __forceinline__ static bool paged(const Tile& t) {
    return TREE ? t.left > 0 && !(t.kind & kDraft) : t.left > 0;
  }

  // The loads of one operand of tile t into l, for fp8 into its ring.
  __device__ __forceinline__ void start(const Tile& t, const Pages& pg, const void* pool,
                                        uint32_t off, char* __restrict__ l) {
    if (__builtin_expect(!paged(t), 0)) return;
    const char* from = static_cast<const char*>(pool);
    // Its place in LDS, added up anew every time: the sixteen of the bf16 rings, kept,
    // would cost the scalar registers that the walk needs (16K-token prompts 2200 ->
    // 2146 us); the eight of fp8 fit (chunks 2790, 2846 with it).
    int own = 1024 * wave;
    if constexpr (!FP8) asm volatile("" : "+s"(own));
    l += own;
    if constexpr (!FP8) {
      to_lds<ONCE>(from + pg.at[0] + off, l);
      to_lds<ONCE>(from + pg.at[1] + off, l + 4096);
    } else {  // two waves a page
      const uint64_t x = pg.at[0], y = pg.at[1];
      to_lds<ONCE>(from + (wave >> 1 ? y : x) + off, l);
    }
  }
  // fp8: the scales of tile t, every wave a copy: K of both pages, then V.
  __device__ __forceinline__ void start_scales(const Tile& t, const Pages& pg,
                                               float* __restrict__ ls) {
    const int x = pg.pid[0], y = pg.pid[1];
    if (paged(t) && lane < 4)
      to_lds4(scale_of_head + (size_t)(lane & 1 ? y : x) * a.num_kv_heads, ls + 4 * wave);
  }

  // Waits until at most n loads of this wave are out.
  template <int n>
  __device__ __forceinline__ void wait() {
    __builtin_amdgcn_s_waitcnt(0x0F70 | n);  // vmcnt(n)
    asm volatile("" ::: "memory");
  }

  // fp8: the lane's chunk of a ring widened into a tile.
  __device__ __forceinline__ u32x4 chunk(const char* __restrict__ ring) const {
    return *(reinterpret_cast<const u32x4*>(ring) + tid);
  }
  __device__ __forceinline__ void widen_k(u32x4 x, char* __restrict__ lk) {
    const int t7 = tid & 127, row = 16 * (tid >> 7) + (t7 >> 3);
    u32x4 lo, hi;
    widen(x, lo, hi);
    *reinterpret_cast<u32x4*>(lk + k_at(row, 2 * (t7 & 7))) = lo;
    *reinterpret_cast<u32x4*>(lk + k_at(row, 2 * (t7 & 7) + 1)) = hi;
  }
  __device__ __forceinline__ void widen_v(u32x4 x, char* __restrict__ lv) {
    u32x4 lo, hi;
    widen(x, lo, hi);
    *reinterpret_cast<u32x4*>(lv + v_at(tid >> 7, tid & 127, 0)) = lo;
    *reinterpret_cast<u32x4*>(lv + v_at(tid >> 7, tid & 127, 1)) = hi;
  }

  __device__ __forceinline__ void first_scores(const char* __restrict__ lk) {
    u32x4 k[8];
    load_k(lk, ka, k);
    s = scores(k, q);
  }

  // Works on tile t, whose scores are in s and whose V is in lv; the next tile's
  // K is in lk.
  __device__ __forceinline__ void work(const Tile& t, const char* __restrict__ lk,
                                       char* __restrict__ lv, f32x4 scales) {
    ++steps;
    bool odd = false;
    // (what a window adds stands in statements of its own: as terms of these two
    // conditions, false at compile time, it cost the tree kernels 217 scalar registers)
    bool partly = t.kind || __builtin_elementwise_sub_sat(tile_min, t.pos0) < kKeyTile - 1;
    if constexpr (WINDOW) partly |= (int)(t.pos0 < tile_low) & not_sinks(t);
    if (__builtin_expect(partly, 0)) {
      // some row of the workgroup does not see all of it
      if (cut_tile(t.left, tid, lv)) *odd_step = steps;
      lds_barrier();
      odd = uniform(*odd_step) == steps;
      if (t.kind & 3) flag = KF_EFLAG_BAD_PAGE;
    }
    if (!any) {
      if (odd) {
        lds_barrier();
        tame_tile(tid, lv);
        lds_barrier();
      }
      return;
    }
    // what a score is multiplied by, page by page: c, with the K scale of an fp8 page
    float cs[2] = {c, c};
    if constexpr (FP8) {
      if (TREE && (t.kind & kDraft)) scales = f32x4{1.0f, 1.0f, 1.0f, 1.0f};
      cs[0] *= scales[0];
      cs[1] *= scales[1];
      if (__builtin_expect(__ballot(!(cs[0] > 0.0f && cs[1] > 0.0f)) != 0, 0)) {
        // the largest score is not the largest product's: multiply first
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] *= cs[i >> 3];
        cs[0] = cs[1] = 1.0f;
      }
    }
    const int half = lane >> 5;
    uint32_t sees = ~0u;
    bool mask = t.kind || __builtin_elementwise_sub_sat(pos_min, t.pos0) < kKeyTile - 1;
    if constexpr (WINDOW) mask |= (int)(__ballot(t.pos0 < low) != 0) & not_sinks(t);
    if (__builtin_expect(mask, 0)) {
      const int e = min(__builtin_elementwise_sub_sat(pos, t.pos0), t.left - 1);
      sees = e < 0 ? 0 : e >= 31 ? ~0u : (2u << e) - 1;
      if (TREE && (t.kind & kDraft)) sees = (uint32_t)(draft >> t.pos0);
      if (WINDOW) {
        auto below = [](int n) -> uint32_t { return n <= 0 ? 0 : n >= 32 ? ~0u : (1u << n) - 1; };
        sees &= ~below(__builtin_elementwise_sub_sat(low, t.pos0)) |
                below(__builtin_elementwise_sub_sat(a.sinks, t.pos0));
      }
      const uint32_t mine = sees >> (8 * half);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (t.kind >> (i >> 3) & 1) s[i] = qnan();
        if (!(mine >> (16 * (i >> 3) + (i & 7)) & 1)) s[i] = neg_inf();
      }
    }
    u32x4 k[8], v[8];
    load_k(lk, ka, k);
    if constexpr (!FP8) load_v(lv, lane, v);  // (fp8: no registers for it beside K's)
    float top = neg_inf(), top1 = neg_inf();
    if constexpr (FP8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        top = fmaxf(top, s[i]);
        top1 = fmaxf(top1, s[8 + i]);
      }
      top = max_halves(fmaxf(top * cs[0], top1 * cs[1]));
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[i]);
      top = max_halves(top) * c;
    }
    // The reference moves only when a score exceeds it by 2^8: exp2 and the sums
    // stay in range, and most tiles leave the outputs unscaled.
    if (__builtin_expect(__ballot(top > st.m + 8.0f) != 0, 0)) {
      const float m = fmaxf(st.m, top);
      const float f = m == neg_inf() ? 1.0f : exp2_fast(st.m - m);
      st.m = m;
      st.l *= f;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) st.o[dt][i] *= f;
    }
    const float m = st.m == neg_inf() ? 0.0f : st.m;
    u32x4 p[2];
    // The waves of a SIMD take turns better where the one in its products goes
    // first: fp8 chunks 2820 -> 2727 us, bf16 the same.
    __builtin_amdgcn_s_setprio(1);
    const f32x16 next = scores(k, q);
#pragma unroll
    for (int page = 0; page < 2; ++page)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x0 = s[8 * page + 2 * i], x1 = s[8 * page + 2 * i + 1];
        const float e0 = exp2_fast(__builtin_fmaf(x0, cs[page], -m));
        const float e1 = exp2_fast(__builtin_fmaf(x1, cs[page], -m));
        st.l += e0 + e1;
        p[page][i] = FP8 ? pack_bf16(e0 * scales[2 + page], e1 * scales[2 + page])
                         : pack_bf16(e0, e1);
      }
    s = next;
    if (__builtin_expect(mask, 0)) {
      if constexpr (FP8) {  // a hidden token weighs nothing, whatever its page's scale
        const uint32_t mine = sees >> (8 * half);
#pragma unroll
        for (int page = 0; page < 2; ++page)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t two = mine >> (16 * page + 2 * i) & 3u;
            p[page][i] &= (two & 1 ? 0x0000FFFFu : 0u) | (two & 2 ? 0xFFFF0000u : 0u);
          }
      }
    }
    if (__builtin_expect(odd, 0)) {
      add_odd(lv, sees, p, lane, st);
      lds_barrier();
      tame_tile(tid, lv);
      lds_barrier();
      if constexpr (!FP8) load_v(lv, lane, v);
    }
    if constexpr (FP8) load_v(lv, lane, v);
#pragma unroll
    for (int page = 0; page < 2; ++page)
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) st.o[dt] = mfma32(v[4 * page + dt], p[page], st.o[dt]);
    __builtin_amdgcn_s_setprio(0);
  }

  // bf16: tile t, whose place t4 takes, V in lv; the next tile's K in lk.  The
  // loads of t4's K go into k0, where t's was, those of t3's V into v3; drafted
  // tokens are written a step before they are needed (k2, v1).
  __device__ __forceinline__ bool step(Tile& t, const Tile& t1, const Tile& t2, const Tile& t3,
                                       const char* __restrict__ lk, char* __restrict__ lv,
                                       char* __restrict__ k0, char* __restrict__ v3,
                                       char* __restrict__ k2, char* __restrict__ v1) {
    Pages pg4;
    const Tile t4 = take(pg4);
    // V of t1, K and V of t2, K of t3 may still be out
    if (__builtin_expect(paged(t3), 1))
      wait<8>();
    else
      wait<0>();
    lds_barrier();
    start(t3, pages, a.v_pool, voff, v3);
    start(t4, pg4, a.k_pool, koff, k0);
    pages = pg4;
    work(t, lk, lv, f32x4{1.0f, 1.0f, 1.0f, 1.0f});
    if (TREE && (t2.kind & kDraft)) draft_k(a, row0, t2.pos0, n_rows, g, tid, k2);
    if (TREE && (t1.kind & kDraft)) draft_v(a, row0, t1.pos0, n_rows, g, tid, v1);
    t = t4;
    return t1.left > 0;
  }

  // fp8: tile t, whose place t4 takes, V in lv; the next tile's K in lk.  t2's K is
  // widened into k2, t1's V into v1, from their rings; the loads of t4 go into the
  // rings' places of t.
  __device__ __forceinline__ bool step8(Tile& t, const Tile& t1, const Tile& t2, const Tile& t3,
                                        const char* __restrict__ lk, char* __restrict__ lv,
                                        char* __restrict__ k2, char* __restrict__ v1,
                                        const char* __restrict__ rk2, const char* __restrict__ rv1,
                                        char* __restrict__ rk0, char* __restrict__ rv0,
                                        float* __restrict__ s0) {
    Pages pg4;
    const Tile t4 = take(pg4);
    // the rings are each wave's own: what stood in t's places has been read
    const f32x4 scales = *reinterpret_cast<const f32x4*>(s0 + 4 * wave);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    start(t4, pg4, a.k_pool, koff, rk0);
    start(t4, pg4, a.v_pool, koff, rv0);
    start_scales(t4, pg4, s0);
    if (__builtin_expect(paged(t4), 1))
      wait<6>();
    else
      wait<0>();
    const u32x4 ck = chunk(rk2), cv = chunk(rv1);
    lds_barrier();
    if (TREE && (t2.kind & kDraft))
      draft_k(a, row0, t2.pos0, n_rows, g, tid, k2);
    else if (t2.left > 0)
      widen_k(ck, k2);
    if (TREE && (t1.kind & kDraft))
      draft_v(a, row0, t1.pos0, n_rows, g, tid, v1);
    else if (t1.left > 0)
      widen_v(cv, v1);
    work(t, lk, lv, scales);
    t = t4;
    return t1.left > 0;
  }
};

template <bool FP8, bool TREE, bool WINDOW, bool ONCE>
__global__ __launch_bounds__(256, 2) void rows_kernel(RowsArgs a) {
  // K and V: four tiles each (bf16), or two tiles and a ring of four (fp8)
  constexpr int kTile = kKeyTile * kDim * 2, kRing = FP8 ? kKeyTile * kDim : 16;
  __shared__ __align__(16) char k0[kTile], v0[kTile], k1[kTile], v1[kTile];
  __shared__ __align__(16) char k2[FP8 ? kRing : kTile], v2[FP8 ? kRing : kTile];
  __shared__ __align__(16) char k3[FP8 ? kRing : kTile], v3[FP8 ? kRing : kTile];
  __shared__ __align__(16) char k4[kRing], v4[kRing], k5[kRing], v5[kRing];
  __shared__ __align__(16) float s0[16], s1[16], s2[16], s3[16];
  __shared__ int odd_step;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int H = a.num_kv_heads, G = a.group;
  const int g = blockIdx.x % H, item = blockIdx.x / H;
  RowsItem it;
  int found = 1;
  if (a.parts > 0) {
    const int tile = item % a.max_tiles;
    found = find_tile(a, tile, lane, it.seq, it.tile, it.row0, it.rows);
    if (found > 0) {
      it.first_pos = TREE ? 0 : fixed(a.first_pos)[it.seq];
      it.route0 = fixed(a.seq_route_begin)[it.seq];
      it.route1 = fixed(a.seq_route_begin)[it.seq + 1];
    }
    it.rec = a.parts > 1 ? tile * a.parts + item / a.max_tiles : -1;
  } else {
    const int items = fixed(a.head)[0];
    const auto* at = fixed(reinterpret_cast<const int32_t*>(a.items + item));
    it.seq = at[0];
    it.tile = at[1];
    it.key0 = at[2];
    it.key1 = at[3];
    it.rec = at[4];
    it.row0 = at[5];
    it.rows = at[6];
    it.first_pos = at[7];
    it.route0 = at[8];
    it.route1 = at[9];
    it.tok_begin = at[10];
    it.tok_end = at[11];
    it.page_base = at[12];
    found = items < 0 ? -1 : item < items;
  }
  if (found < 0) {  // no row's sequence is known
    for (int r = item; r < a.num_rows; r += gridDim.x / H) fill_nan(a, r, 0, G, g, tid, 256);
    if (a.parts > 0 && item == 0 && tid == 0) atomicOr(a.err_flags, KF_EFLAG_BAD_ROUTE);
    return;
  }
  if (found == 0) return;
  const int b = uniform(it.seq < 0 ? -1 - it.seq : it.seq);
  const int row0 = it.row0, n_rows = it.rows;
  const int m0 = it.tile * kRowTile, m1 = min(n_rows * G, m0 + kRowTile);  // (row, head) pairs
  // no token lies behind INT32_MAX
  const int p0 = it.first_pos;
  auto position = [&](int pair) {
    return TREE ? INT32_MAX
                : __builtin_elementwise_add_sat(p0, (int)((uint32_t)min(pair, m1 - 1) / (uint32_t)G));
  };
  Sight sight{uniform(position(m1 - 1)), INT32_MIN, 0};
  if (WINDOW) {
    sight.low = uniform(window_begin(a, p0, (int)((uint32_t)m0 / (uint32_t)G)));
    sight.sinks = a.sinks;
  }
  const int route0 = it.route0, route1 = it.route1;
  if (a.parts > 0) {
    const int k = TREE && n_rows > KF_MAX_DRAFT
                      ? -1 : count_tiles<WINDOW>(a, b, route0, route1, sight, lane, it);
    if (k < 0) {
      it.seq = -1 - b;
      if (tid == 0) atomicOr(a.err_flags, KF_EFLAG_BAD_ROUTE);
    } else {
      const int64_t all = k + (TREE ? (n_rows + kKeyTile - 1) / kKeyTile : 0);
      const int part = item / a.max_tiles;
      const int parts = tile_parts(a.parts, all);  // those behind them are empty
      it.key0 = uniform((int)(all * part / parts));
      it.key1 = part + 1 != parts ? uniform((int)(all * (part + 1) / parts)) : INT32_MAX;
    }
  }
  if (it.seq < 0) {
    if (it.rec < 0)
      fill_nan(a, row0, m0, m1, g, tid, 256);
    else if (tid < m1 - m0)  // a sum of NaN makes the outputs NaN
      *reinterpret_cast<f32x2*>(a.rec_ml + 2 * (((size_t)it.rec * H + g) * a.rec_rows + tid)) =
          f32x2{0.0f, qnan()};
    return;
  }
  // this lane's row and head
  const int m = m0 + 32 * wave + l32;
  const bool mine = m < m1;
  const uint32_t mc = mine ? m : m1 - 1;
  const int row = mc / (uint32_t)G, h = g * G + mc % (uint32_t)G;
  const float c0 = a.scale_log2;
  Work<FP8, TREE, WINDOW, ONCE> w{a};
  w.tid = tid;
  w.lane = lane;
  w.wave = wave;
  w.g = g;
  w.row0 = row0;
  w.n_rows = n_rows;
  w.any = m0 + 32 * wave < m1;
  w.c = c0 == 0.0f ? 1.0f : fabsf(c0);
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    w.q[ks] = ld16(a.q + (row0 + row) * a.q_stride + (size_t)h * kDim + 16 * ks + 8 * half);
  }
  w.pos = w.pos_min = w.tile_min = INT32_MAX;
  w.last_pos = sight.last_pos;
  w.low = w.tile_low = w.first_low = sight.low;
  w.draft = 0;
  if constexpr (TREE) {
    w.draft = mine ? a.tree_mask[row0 + row] : 0;
    if (n_rows < 64) w.draft &= ((uint64_t)1 << n_rows) - 1;
  } else {
    w.pos = position(m);
    w.pos_min = uniform(position(m0 + 32 * wave));
    w.tile_min = uniform(position(m0));
    if (WINDOW) {
      auto begins = [&](int pair) {
        return window_begin(a, p0, (int)((uint32_t)min(pair, m1 - 1) / (uint32_t)G));
      };
      w.low = begins(m);
      w.tile_low = uniform(begins(m1 - 1));
    }
  }
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) w.st.o[dt][i] = 0.0f;
  w.st.m = neg_inf();
  w.st.l = 0.0f;
  w.flag = w.steps = 0;
  w.odd_step = &odd_step;
  if (tid == 0) odd_step = 0;
  const uint32_t head_bytes = kPage * kDim * (FP8 ? 1 : 2);
  w.page_bytes = a.head_major ? head_bytes : H * head_bytes;
  w.head_at = (uint64_t)(a.head_major ? (int64_t)g * a.num_pages : g) * head_bytes;
  const int krow = 4 * wave + (lane >> 4);  // of a page
  w.koff = FP8 ? 1024 * (wave & 1) + 16 * lane : 256 * krow + 16 * ((lane & 15) ^ krow);
  w.voff = 1024 * wave + 32 * l32 + 16 * half;
  {
    const uintptr_t ks = reinterpret_cast<uintptr_t>(a.k_scale);
    const uintptr_t vs = reinterpret_cast<uintptr_t>(a.v_scale);
    w.scale_of_head = reinterpret_cast<const float*>((lane & 2 ? vs : ks)) + g;
  }
  w.ka = k_at(16 * (l32 >> 4) + 8 * ((l32 >> 2) & 1) + 4 * ((l32 >> 3) & 1) + (l32 & 3), half);
  // (the pages of the first tile are on their way before q is waited for)
  // A part that begins in its sequence's first route has that in its item (packed
  // prompts 183 -> 180 us, one short one 8.9 -> 8.0; fp8's kernel has no registers for
  // it, chunks 2704 -> 2779).
  const int see = route0 < route1 ? visible(it.tok_begin, it.tok_end, sight.last_pos) : 0;
  const int first_tiles = !WINDOW          ? (see + kKeyTile - 1) / kKeyTile
                          : route0 < route1 ? sight_tiles<WINDOW>(sight, it.tok_begin, it.tok_end)
                                            : 0;
  if (!FP8 && it.key0 < first_tiles) {
    w.walk.r = route0;
    w.walk.r_end = route1;
    if (WINDOW) {
      walk_route<WINDOW, WINDOW && !FP8>(w.walk, sight, it.tok_begin, it.tok_end, it.page_base,
                                         it.key0);
    } else {
      w.walk.n = see;
      w.walk.tb = it.tok_begin;
      w.walk.base = it.page_base;
      w.walk.tiles = (see + kKeyTile - 1) / kKeyTile;
      w.walk.j = it.key0;
    }
    walk_ids(a, w.walk);
  } else {
    walk_to<WINDOW, WINDOW && !FP8>(a, w.walk, route0, route1, sight, it.key0, lane);
  }
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    if (c0 < 0.0f) w.q[ks] ^= 0x80008000u;                 // a negative scale turns the row around
    if (c0 == 0.0f || !mine) w.q[ks] = u32x4{0, 0, 0, 0};  // a zero one makes all scores equal
  }
  w.left = it.key1 == INT32_MAX ? INT32_MAX : it.key1 - it.key0;
  w.drafts = TREE && it.key1 == INT32_MAX ? n_rows : 0;

  Tile t0, t1, t2, t3;
  if constexpr (!FP8) {
    t0 = w.take(w.pages);
    w.start(t0, w.pages, a.k_pool, w.koff, k0);
    w.start(t0, w.pages, a.v_pool, w.voff, v0);
    t1 = w.take(w.pages);
    w.start(t1, w.pages, a.k_pool, w.koff, k1);
    w.start(t1, w.pages, a.v_pool, w.voff, v1);
    t2 = w.take(w.pages);
    w.start(t2, w.pages, a.k_pool, w.koff, k2);
    w.start(t2, w.pages, a.v_pool, w.voff, v2);
    t3 = w.take(w.pages);
    w.start(t3, w.pages, a.k_pool, w.koff, k3);
    if (t0.left > 0) {
      if (w.paged(t3))
        w.template wait<12>();
      else
        w.template wait<0>();
      if (TREE && (t0.kind & kDraft)) {
        draft_k(a, row0, t0.pos0, n_rows, g, tid, k0);
        draft_v(a, row0, t0.pos0, n_rows, g, tid, v0);
      }
      if (TREE && (t1.kind & kDraft)) draft_k(a, row0, t1.pos0, n_rows, g, tid, k1);
      lds_barrier();
      w.first_scores(k0);
      while (w.step(t0, t1, t2, t3, k1, v0, k0, v3, k2, v1) &&
             w.step(t1, t2, t3, t0, k2, v1, k1, v0, k3, v2) &&
             w.step(t2, t3, t0, t1, k3, v2, k2, v1, k0, v3) &&
             w.step(t3, t0, t1, t2, k0, v3, k3, v2, k1, v0)) {
      }
    }
  } else {
    auto start = [&](char* rk, char* rv, float* ls) __attribute__((always_inline)) {
      const Tile t = w.take(w.pages);
      w.start(t, w.pages, a.k_pool, w.koff, rk);
      w.start(t, w.pages, a.v_pool, w.koff, rv);
      w.start_scales(t, w.pages, ls);
      return t;
    };
    t0 = start(k2, v2, s0);
    t1 = start(k3, v3, s1);
    t2 = start(k4, v4, s2);
    t3 = start(k5, v5, s3);
    if (t0.left > 0) {
      if (w.paged(t3))
        w.template wait<6>();
      else
        w.template wait<0>();
      if (TREE && (t0.kind & kDraft)) {
        draft_k(a, row0, t0.pos0, n_rows, g, tid, k0);
        draft_v(a, row0, t0.pos0, n_rows, g, tid, v0);
      } else {
        w.widen_k(w.chunk(k2), k0);
        w.widen_v(w.chunk(v2), v0);
      }
      if (TREE && (t1.kind & kDraft))
        draft_k(a, row0, t1.pos0, n_rows, g, tid, k1);
      else if (t1.left > 0)
        w.widen_k(w.chunk(k3), k1);
      lds_barrier();
      w.first_scores(k0);
      while (w.step8(t0, t1, t2, t3, k1, v0, k0, v1, k4, v3, k2, v2, s0) &&
             w.step8(t1, t2, t3, t0, k0, v1, k1, v0, k5, v4, k3, v3, s1) &&
             w.step8(t2, t3, t0, t1, k1, v0, k0, v1, k2, v5, k4, v4, s2) &&
             w.step8(t3, t0, t1, t2, k0, v1, k1, v0, k3, v2, k5, v5, s3)) {
      }
    }
  }
  if (w.flag && tid == 0) atomicOr(a.err_flags, w.flag);
  if (!mine) return;
  const State& st = w.st;
  const float l = sum_halves(st.l);
  if (it.rec >= 0) {
    const size_t rec = ((size_t)it.rec * H + g) * a.rec_rows + (m - m0);
    if (half == 0) *reinterpret_cast<f32x2*>(a.rec_ml + 2 * rec) = f32x2{st.m, l};
    if (l == 0.0f) return;  // the combine does not read it
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(a.rec_o + rec * kDim + 32 * dt + 8 * i + 4 * half) =
            f32x4{st.o[dt][4 * i], st.o[dt][4 * i + 1], st.o[dt][4 * i + 2], st.o[dt][4 * i + 3]};
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const size_t at = (size_t)(row0 + row) * a.num_q_heads + h;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<u32x2*>(a.out + at * kDim + 32 * dt + 8 * i + 4 * half) =
          u32x2{pack_bf16(st.o[dt][4 * i] * inv, st.o[dt][4 * i + 1] * inv),
                pack_bf16(st.o[dt][4 * i + 2] * inv, st.o[dt][4 * i + 3] * inv)};
  if (half == 0) a.lse[at] = l == 0.0f ? neg_inf() : (st.m + __log2f(l)) * kLn2;
}

// The parts of a split row tile into its outputs: a wave per (row, head), a lane
// per part's maximum and sum, then the parts' outputs, eight on their way at a time.
// A part whose sum is 0 has written none.
// Bound by its chain of loads: 4 us for one tile, 8 us for 48 trees in 2 to 4 parts,
// 14 .. 18 us for 128 and 256 full tiles in 4 and 2.
__global__ __launch_bounds__(256) void rows_combine_kernel(RowsArgs a) {
  const int H = a.num_kv_heads, G = a.group;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const bool planned = a.parts == 0;
  const int splits = planned ? fixed(a.head)[1] : a.max_tiles;
  const int pairs = planned ? fixed(a.head)[2] : a.rec_rows;  // of a tile at most
  const size_t stride = (size_t)H * a.rec_rows;
  // (records per compute unit and workgroups are few: all of this fits 32 bits)
  for (uint32_t u = blockIdx.x * 4 + wave; u < (uint32_t)splits * H * pairs; u += gridDim.x * 4) {
    const int rm = (int)(u % (uint32_t)pairs), g = (int)(u / (uint32_t)pairs % (uint32_t)H);
    const int split = uniform((int)(u / ((uint32_t)pairs * (uint32_t)H)));
    RowsSplit sp;
    if (planned) {
      const auto* at = fixed(reinterpret_cast<const int32_t*>(a.splits + split));
      sp.tile = at[0];
      sp.rec = at[1];
      sp.parts = at[2];
      sp.row0 = at[3];
      sp.rows = at[4];
    } else {
      int b;
      sp.rec = split * a.parts;
      sp.parts = a.parts;
      if (find_tile(a, split, lane, b, sp.tile, sp.row0, sp.rows) <= 0) return;
    }
    const int row0 = sp.row0, m = sp.tile * kRowTile + rm;
    if (m >= sp.rows * G) continue;
    const size_t rec = ((size_t)sp.rec * H + g) * a.rec_rows + rm;
    const float* ml = a.rec_ml + 2 * rec;
    const f32x2* ro = reinterpret_cast<const f32x2*>(a.rec_o + rec * kDim) + lane;
    float ref = neg_inf();  // the largest maximum so far
    float l = 0.0f;
    f32x2 o = {0.0f, 0.0f};
    for (int p = 0; p < sp.parts; p += 64) {
      const int n = min(64, sp.parts - p);
      f32x2 y[8];
      auto load = [&](int i0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = ro[(size_t)(p + min(i0 + i, n - 1)) * stride * (kDim / 2)];
      };
      load(0);
      f32x2 x = {neg_inf(), 0.0f};  // of part p + lane
      if (lane < n) x = *reinterpret_cast<const f32x2*>(ml + (size_t)(p + lane) * stride * 2);
      const uint64_t some = __ballot(x.y != 0.0f);  // parts with outputs
      const float top = fmaxf(ref, wave_max(x.x));
      const float base = top == neg_inf() ? 0.0f : top;
      const float f = exp2_fast(ref - base), e = exp2_fast(x.x - base);
      ref = top;
      float sum = e * x.y;
#pragma unroll
      for (int k = 32; k >= 1; k >>= 1) sum += __shfl_xor(sum, k);
      l = __builtin_fmaf(l, f, sum);
      o.x *= f;
      o.y *= f;
      for (int i0 = 0;;) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (!(some >> (i0 + i) & 1)) continue;
          const float w = __builtin_bit_cast(
              float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, e), i0 + i));
          o.x = __builtin_fmaf(w, y[i].x, o.x);
          o.y = __builtin_fmaf(w, y[i].y, o.y);
        }
        if ((i0 += 8) >= n || !(some >> i0)) break;
        load(i0);
      }
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const size_t at = (size_t)(row0 + m / G) * a.num_q_heads + g * G + m % G;
    reinterpret_cast<uint32_t*>(a.out + at * kDim)[lane] = pack_bf16(o.x * inv, o.y * inv);
    if (lane == 0) a.lse[at] = l == 0.0f ? neg_inf() : (ref + __log2f(l)) * kLn2;
  }
}

}  // namespace

hipError_t launch_append_rows(const AppendRowsArgs& a, bool fp8, hipStream_t stream) {
  if (a.num_entries <= kDirectEntries && a.num_entries <= kDirectMean * a.num_routes) {
    const bool many = a.num_routes > kDirectRoutes;
    if (fp8 && many)
      append_plan_kernel<true, true, true><<<a.num_entries, 1024, 0, stream>>>(a);
    else if (fp8)
      append_plan_kernel<true, true, false><<<a.num_routes, 1024, 0, stream>>>(a);
    else if (many)
      append_plan_kernel<false, true, true><<<a.num_entries, 1024, 0, stream>>>(a);
    else
      append_plan_kernel<false, true, false><<<a.num_routes, 1024, 0, stream>>>(a);
    return hipGetLastError();
  }
  hipError_t st;
  if (a.num_routes > kPlanRoutes) {
    append_table_kernel<<<1, 1024, 0, stream>>>(a);
    if ((st = hipGetLastError()) != hipSuccess) return st;
    append_plan_kernel<false, false, true>
        <<<a.num_routes, a.num_entries > kWaveEntries ? 256 : 64, 0, stream>>>(a);
  } else {
    append_plan_kernel<false, false, false><<<a.num_routes, 512, 0, stream>>>(a);
  }
  if ((st = hipGetLastError()) != hipSuccess) return st;
  const int64_t tiles = append_first_tile(a.num_entries, a.num_routes);
  const int64_t grid = (tiles * 2 * a.num_kv_heads + 3) / 4;
  if (fp8)
    append_tile_kernel<true><<<(uint32_t)grid, 256, 0, stream>>>(a);
  else
    append_tile_kernel<false><<<(uint32_t)grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

template <bool TREE, bool WINDOW, bool ONCE>
hipError_t launch_rows(const RowsArgs& a, bool fp8, hipStream_t stream) {
  hipError_t st;
  if (a.parts == 0) {
    rows_plan_kernel<TREE, WINDOW><<<1, 1024, 0, stream>>>(a);
    if ((st = hipGetLastError()) != hipSuccess) return st;
  }
  // (a workgroup without an item still takes its place on a compute unit)
  const int items = a.parts > 0 ? a.max_tiles * a.parts : a.max_tiles + (a.may_split ? a.max_recs : 0);
  const uint32_t grid = (uint32_t)items * a.num_kv_heads;
  if (fp8)
    rows_kernel<true, TREE, WINDOW, ONCE><<<grid, 256, 0, stream>>>(a);
  else
    rows_kernel<false, TREE, WINDOW, ONCE><<<grid, 256, 0, stream>>>(a);
  st = hipGetLastError();
  if (st != hipSuccess || a.parts == 1 || (a.parts == 0 && !a.may_split)) return st;
  // a wave per (row, head) and turn; most splits at most
  const int64_t splits = a.parts > 0 ? a.max_tiles : min(a.max_tiles, a.max_recs / 2);
  const int64_t waves = splits * a.num_kv_heads * a.rec_rows;
  const uint32_t wgs = (uint32_t)min((waves + 3) / 4, (int64_t)kCombineWgsPerSlot * a.slots);
  rows_combine_kernel<<<wgs, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_rows_attn(const RowsArgs& a, bool fp8, bool tree, hipStream_t stream) {
  if (tree) return launch_rows<true, false, true>(a, fp8, stream);
  if (a.window < 0) return launch_rows<false, false, false>(a, fp8, stream);
  // rows of one row tile a sequence (decode steps): no other workgroup reads their tokens
  return (int64_t)a.num_rows * a.group <= (int64_t)kRowTile * a.num_seqs
             ? launch_rows<false, true, true>(a, fp8, stream)
             : launch_rows<false, true, false>(a, fp8, stream);
}

}  // namespace kf
