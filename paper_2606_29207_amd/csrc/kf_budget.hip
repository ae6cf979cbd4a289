// gfx950 kernels of the operators that keep a cache within a budget:
//   attn_weights_kernel -- the attention weight that every token receives
//   evict_select_kernel -- which tokens of a sequence and KV head stay
//   evict_move_kernel   -- those tokens into the pages of another route
#include "kf_budget.h"
#include "kf_device.h"

namespace kf {
namespace {

// A route's row (seq, part, tok_begin, tok_end, page_base, page_cap) is sound.
__device__ __forceinline__ bool route_row_ok(int tok_begin, int tok_end, int base, int cap,
                                             int max_pages, int num_page_ids) {
  const int64_t n = (int64_t)tok_end - tok_begin, pages = n > 0 ? (n + kPage - 1) / kPage : 0;
  return n >= 0 && n <= INT32_MAX && base >= 0 && pages <= cap && pages <= max_pages &&
         base + pages <= num_page_ids;
}

// ------------------------------------------------------------- attn_weights
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// 16 bytes a lane from memory straight into LDS, 1 KiB a wave.
__device__ __forceinline__ void to_lds16(const uint16_t* g, char* l) {
  __builtin_amdgcn_global_load_lds(
      (const __attribute__((address_space(1))) uint32_t*)g,
      (__attribute__((address_space(3))) uint32_t*)(__attribute__((address_space(3))) void*)l, 16,
      0, 0);
}

// One route and KV head as a workgroup sees it.  The (row, query head) pairs of the
// sequence are its columns: column c is row c / G, head g G + c % G.
struct Seen {
  int row0, rows, g;
  int n, base;        // the route's tokens, its first page id's index
  int64_t first;      // the first row's position less tok_begin
  int p0, p1;         // the workgroup's pages
};

// How far the row at place i sees into the route: its last token's index.
__device__ __forceinline__ int reach(const Seen& s, int64_t i) {
  const int64_t x = s.first + i;
  return (int)(x < -1 ? -1 : x > INT32_MAX ? INT32_MAX : x);
}
// Whether a row has a softmax: it saw a token, and its lse is a number.
__device__ __forceinline__ bool has_softmax(float lse) { return lse > neg_inf(); }

// Few columns (a decode step, a small tree): they stay in registers, 16 a matrix
// product, and the keys stream past, a page of 16 per product of depth 32.
template <bool FP8, int NC>
__device__ __forceinline__ void few_columns(const AttnWeightsArgs& a, const Seen& s, int& flag) {
  constexpr int kBatch = NC == 1 ? 4 : 2;  // pages on their way at a time
  constexpr int kLoads = FP8 ? 2 : 4;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int n16 = lane & 15, grp = lane >> 4, H = a.num_kv_heads, G = a.group;
  const uint32_t C = (uint32_t)s.rows * G;
  u32x4 q[NC][4];
  float lse[NC][4];
  int sees[NC][4];
#pragma unroll
  for (int t = 0; t < NC; ++t) {
    const uint32_t c = 16 * t + n16, cc = c < C ? c : C - 1;
    const uint16_t* row = a.q + (s.row0 + (int64_t)(cc / G)) * a.q_stride +
                          (size_t)(s.g * G + cc % G) * kDim;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      q[t][k] = ld16(row + (FP8 ? 64 * (k >> 1) + 16 * grp + 8 * (k & 1) : 32 * k + 8 * grp));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t m = 16 * t + 4 * grp + i, mm = m < C ? m : C - 1;
      const float x = a.lse[(s.row0 + (int64_t)(mm / G)) * a.num_q_heads + s.g * G + mm % G];
      lse[t][i] = x * kLog2e;
      sees[t][i] = m < C && has_softmax(x) ? reach(s, mm / G) : -1;
    }
  }
  const size_t head_bytes = kPage * kDim * (FP8 ? 1 : 2);
  const char* pool = static_cast<const char*>(a.k_pool);
  const uint32_t at = FP8 ? n16 * kDim + 16 * grp : 2 * (n16 * kDim + 8 * grp);

  struct Batch {
    u32x4 k[kBatch][kLoads];
    float scale[kBatch], old[kBatch];
    int pid[kBatch];
  };
  auto load = [&](Batch& b, int p) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (p + i >= s.p1) break;
      int pid = fixed(a.page_ids)[s.base + p + i];
      b.pid[i] = pid;
      if ((uint32_t)pid >= (uint32_t)a.num_pages) pid = 0;
      const char* from = pool + slice_of(pid, s.g, H, a.num_pages, a.head_major) * head_bytes + at;
#pragma unroll
      for (int k = 0; k < kLoads; ++k)
        b.k[i][k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from + 64 * k));
      b.scale[i] = FP8 ? a.k_scale[(size_t)pid * H + s.g] : 1.0f;
      b.old[i] = 0.0f;
      if (a.decay != 0.0f) b.old[i] = a.weights[((size_t)pid * H + s.g) * kPage + n16];
    }
  };
  auto work = [&](const Batch& b, int p) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (p + i >= s.p1) break;
      u32x4 k[4];
      if constexpr (FP8) {
        widen(b.k[i][0], k[0], k[1]);
        widen(b.k[i][1], k[2], k[3]);
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) k[u] = b.k[i][u];
      }
      const float c = a.scale_log2 * b.scale[i];
      const int j = (p + i) * kPage + n16;
      float sum = 0.0f;
#pragma unroll
      for (int t = 0; t < NC; ++t) {
        f32x4 d = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < 4; ++u) d = mfma16(q[t][u], k[u], d);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const float e = exp2_fast(__builtin_fmaf(d[m], c, -lse[t][m]));
          sum += j <= sees[t][m] ? e : 0.0f;
        }
      }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      const int pid = b.pid[i];
      if ((uint32_t)pid >= (uint32_t)a.num_pages)
        flag |= KF_EFLAG_BAD_PAGE;
      else if (grp == 0 && j < s.n)
        a.weights[((size_t)pid * H + s.g) * kPage + n16] =
            j < s.first && a.decay != 0.0f ? __builtin_fmaf(a.decay, b.old[i], sum) : sum;
    }
  };
  constexpr int kStep = 4 * kBatch;  // the four waves take batches in turn
  int p = s.p0 + kBatch * wave;
  if (p >= s.p1) return;
  Batch x, y;
  load(x, p);
  for (;;) {
    if (p + kStep < s.p1) load(y, p + kStep);
    work(x, p);
    if ((p += kStep) >= s.p1) break;
    if (p + kStep < s.p1) load(x, p + kStep);
    work(y, p);
    if ((p += kStep) >= s.p1) break;
  }
}

// Many columns (prompts): 64 keys a wave stay in registers, the columns that see them
// stream past through LDS, 32 a matrix product.  KW waves lie along the keys, 4 / KW
// along the columns of a step.
template <bool FP8, int KW>
__device__ __forceinline__ void many_columns(const AttnWeightsArgs& a, const Seen& s, char* lds,
                                             float* red, int& flag) {
  constexpr int RW = 4 / KW, kCols = 32 * RW, kPieces = 2 * RW;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int kw = wave % KW, rw = wave / KW;
  const int H = a.num_kv_heads, G = a.group;
  const size_t head_bytes = kPage * kDim * (FP8 ? 1 : 2);
  const uint16_t* q = a.q + s.row0 * a.q_stride + (size_t)s.g * G * kDim;
  const float* lse = a.lse + (int64_t)s.row0 * a.num_q_heads + s.g * G;
  const int last = (s.n - 1) / kPage;
  const int turn = kCols / G, rest = kCols % G;  // rows and heads that a step moves on by
  for (int p = s.p0; p < s.p1; p += 4 * KW) {
    // keys 32 kt + l32 of the wave's 64
    const int pk = p + 4 * kw;
    u32x4 k[2][8];
    float c[2][2];
    int pid[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      pid[kt] = a.page_ids[s.base + min(pk + 2 * kt + (l32 >> 4), last)];
      const int id = (uint32_t)pid[kt] < (uint32_t)a.num_pages ? pid[kt] : 0;
      const char* from = static_cast<const char*>(a.k_pool) +
                         slice_of(id, s.g, H, a.num_pages, a.head_major) * head_bytes;
      if constexpr (FP8) {
        from += (l32 & 15) * kDim + 16 * half;
        u32x4 x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = ld16(from + 32 * u);
#pragma unroll
        for (int u = 0; u < 4; ++u) widen(x[u], k[kt][2 * u], k[kt][2 * u + 1]);
        const float sc = a.scale_log2 * a.k_scale[(size_t)id * H + s.g];
        c[kt][0] = __shfl(sc, 0);
        c[kt][1] = __shfl(sc, 16);
      } else {
        from += 2 * ((l32 & 15) * kDim + 8 * half);
#pragma unroll
        for (int u = 0; u < 8; ++u) k[kt][u] = ld16(from + 32 * u);
        c[kt][0] = c[kt][1] = a.scale_log2;
      }
    }
    // the first row that sees the first of the workgroup's keys, and its columns
    const int64_t before = (int64_t)p * kPage - s.first;
    const int i0 = (int)max((int64_t)0, min((int64_t)s.rows, before));
    const int C = (s.rows - i0) * G, steps = (C + kCols - 1) / kCols;
    // staged pieces: column 4 piece + lane / 16 of the step
    int64_t off[kPieces];
    int hh[kPieces];
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
      const uint32_t col = 4 * (kPieces * wave + u) + (lane >> 4);
      hh[u] = col % (uint32_t)G;
      off[u] = (i0 + (int64_t)(col / (uint32_t)G)) * a.q_stride + hh[u] * kDim;
    }
    const int64_t off_last = (s.rows - 1) * a.q_stride + (G - 1) * kDim;
    const int64_t off_turn = turn * a.q_stride + rest * kDim, off_wrap = a.q_stride - G * kDim;
    int left = C;  // columns not staged yet
    auto stage = [&](char* to) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < kPieces; ++u) {
        const int col = 4 * (kPieces * wave + u) + (lane >> 4);
        const int64_t o = col < left ? off[u] : off_last;
        to_lds16(q + o + 8 * ((lane & 15) ^ (col & 15)), to + 1024 * (kPieces * wave + u));
        off[u] += off_turn;
        hh[u] += rest;
        if (hh[u] >= G) {
          hh[u] -= G;
          off[u] += off_wrap;
        }
      }
      left -= kCols;
    };
    // the lane's column of a product: 32 rw + l32 of the step
    int col_left = C - (32 * rw + l32), ch = (32 * rw + l32) % G, ci = i0 + (32 * rw + l32) / G;
    float next_lse = 0.0f;
    int next_sees = -1;
    auto column = [&]() __attribute__((always_inline)) {
      next_sees = col_left > 0 ? reach(s, ci) : -1;
      next_lse = col_left > 0 ? lse[(int64_t)ci * a.num_q_heads + ch] : neg_inf();
      col_left -= kCols;
      ci += turn;
      ch += rest;
      if (ch >= G) {
        ch -= G;
        ++ci;
      }
    };
    f32x16 acc[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[kt][i] = 0.0f;
    const int j0 = pk * kPage;
    if (steps > 0) {
      stage(lds);
      column();
    }
    for (int st = 0; st < steps; ++st) {
      char* now = lds + (st & 1) * (kCols * 256);
      __syncthreads();  // this step's columns are there, and the other buffer is free
      const float z = next_lse * kLog2e;
      const int sees = has_softmax(next_lse) ? next_sees : -1;
      if (st + 1 < steps) {
        stage(lds + (~st & 1) * (kCols * 256));
        column();
      }
      if (__ballot(sees >= j0) == 0) continue;
      u32x4 b[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int chunk = FP8 ? 4 * (u >> 1) + 2 * half + (u & 1) : 2 * u + half;
        b[u] = *reinterpret_cast<const u32x4*>(now + (32 * rw + l32) * 256 +
                                               ((chunk ^ (l32 & 15)) << 4));
      }
      f32x16 d[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
        for (int i = 0; i < 16; ++i) d[kt][i] = 0.0f;
#pragma unroll
        for (int u = 0; u < 8; ++u) d[kt] = mfma32(k[kt][u], b[u], d[kt]);
      }
      if (__ballot(sees - 63 < j0) == 0) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            acc[kt][i] += exp2_fast(__builtin_fmaf(d[kt][i], c[kt][i >> 3], -z));
      } else {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int j = j0 + 32 * kt + 8 * (i >> 2) + 4 * half + (i & 3);
            const float e = exp2_fast(__builtin_fmaf(d[kt][i], c[kt][i >> 3], -z));
            acc[kt][i] += j <= sees ? e : 0.0f;
          }
      }
    }
    // The sums over the 32 columns of a half wave: lane l32 ends with that of value
    // 16 kt + i = l32.  In every turn a lane gives half of its values away.
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = acc[i >> 4][i & 15];
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1)
#pragma unroll
      for (int i = 0; i < m; ++i) {
        const float give = lane & m ? v[i] : v[i + m], keep = lane & m ? v[i + m] : v[i];
        v[i] = keep + __shfl_xor(give, m);
      }
    float sum = v[0];
    const int kt = l32 >> 4, i = l32 & 15;
    const int m = 32 * kt + 8 * (i >> 2) + 4 * half + (i & 3);  // of the wave's 64 keys
    const int id0 = __shfl(pid[0], m & 16), id1 = __shfl(pid[1], m & 16);
    const int id = kt ? id1 : id0, j = j0 + m;
    float* at = a.weights + ((size_t)id * H + s.g) * kPage + (m & 15);
    const bool mine = rw == 0 && j < s.n && pk + (m >> 4) < s.p1;
    const float old = mine && a.decay != 0.0f && (uint32_t)id < (uint32_t)a.num_pages ? *at : 0.0f;
    if constexpr (RW > 1) {
      red[64 * wave + m] = sum;
      __syncthreads();
      sum = 0.0f;
#pragma unroll
      for (int w = 0; w < RW; ++w) sum += red[64 * (kw + KW * w) + m];
    }
    if (mine) {
      if ((uint32_t)id >= (uint32_t)a.num_pages)
        flag |= KF_EFLAG_BAD_PAGE;
      else
        *at = j < s.first && a.decay != 0.0f ? __builtin_fmaf(a.decay, old, sum) : sum;
    }
    __syncthreads();  // (the next keys' first columns go where this step's may still be read)
  }
}

template <bool FP8, int KW>
__global__ __launch_bounds__(256, 2) void attn_weights_kernel(AttnWeightsArgs a) {
  constexpr int kCols = 32 * (4 / KW);
  __shared__ __align__(16) char lds[2 * kCols * 256];
  __shared__ float red[256];
  const int H = a.num_kv_heads, r = blockIdx.y;
  const int g = blockIdx.x % H, chunk = blockIdx.x / H;
  const auto* rp = fixed(reinterpret_cast<const int32_t*>(a.routes)) + 6 * (int64_t)r;
  const int seq = rp[0], tb = rp[2], te = rp[3], base = rp[4], cap = rp[5];
  Seen s;
  bool bad = seq < 0 || seq >= a.num_seqs;
  if (!bad) {
    s.row0 = fixed(a.seq_row_begin)[seq];
    const int end = fixed(a.seq_row_begin)[seq + 1];
    s.rows = end - s.row0;
    bad = s.row0 < 0 || end < s.row0 || end > a.num_rows;
    if (!bad && s.rows == 0) return;  // not looked at
    bad = bad || !route_row_ok(tb, te, base, cap, a.max_pages_per_route, a.num_page_ids);
  }
  if (bad) {
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.err_flags, KF_EFLAG_BAD_ROUTE);
    return;
  }
  s.g = g;
  s.n = te - tb;
  s.base = base;
  s.first = (int64_t)fixed(a.first_pos)[seq] - tb;
  const int pages = (int)(((int64_t)s.n + kPage - 1) / kPage);
  if ((int64_t)chunk * a.chunk_pages >= pages) return;
  s.p0 = chunk * a.chunk_pages;
  s.p1 = (int)min((int64_t)pages, (int64_t)s.p0 + a.chunk_pages);
  int flag = 0;
  const int64_t C = (int64_t)s.rows * a.group;
  if (C <= 16)
    few_columns<FP8, 1>(a, s, flag);
  else if (C <= kFewColumns)
    few_columns<FP8, kFewColumns / 16>(a, s, flag);
  else
    many_columns<FP8, KW>(a, s, lds, red, flag);
  if (__ballot(flag != 0) && (threadIdx.x & 63) == 0) atomicOr(a.err_flags, KF_EFLAG_BAD_PAGE);
}

// -------------------------------------------------------------------- evict
constexpr int kKeysInLds = 34 * 1024;   // tokens of a sequence whose keys stay in LDS
constexpr int kEvictRoutes = 1024;      // routes of a sequence at most

// Orders as the weights do; NaN before all others, zeros equal.
__device__ __forceinline__ uint32_t order_key(float w) {
  if (w != w) return 0;
  const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.0f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// The tokens of a sequence and KV head that stay: of its L tokens, in the order of its
// routes, the first and the last ones, and of the others those of the largest keys, the
// earlier of equal ones.  A threshold by radix, 11, 11 and 10 bits a pass over the keys.
// Each wave has a stretch of the tokens of its own, so that a place's rank is its
// wave's first rank and a count of ballots.
__global__ __launch_bounds__(1024) void evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t keys[kKeysInLds];
  __shared__ uint32_t hist[2048];
  __shared__ int pre[kEvictRoutes + 1], pbase[kEvictRoutes];
  __shared__ int s_scan[2][16], s_bin, s_want;
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  const int g = blockIdx.x, b = blockIdx.y, H = a.num_kv_heads;
  int32_t* plan = a.plan + 2 * b;
  const int into = a.into[b];
  if (into == -1) {
    if (g == 0 && tid == 0) plan[0] = -1;
    return;
  }
  const int r0 = a.seq_route_begin[b], r1 = a.seq_route_begin[b + 1], keep = a.keep[b];
  auto fail = [&](int flag) {
    if (tid == 0) {
      if (g == 0) {
        plan[0] = -1;
        atomicOr(a.err_flags, flag);
      }
    }
  };
  if (r0 < 0 || r1 < r0 || r1 > a.num_routes || r1 - r0 > kEvictRoutes || into < r0 || into >= r1 ||
      keep < 0 || keep > a.max_keep)
    return fail(KF_EFLAG_BAD_ROUTE);
  // the routes' tokens, and where each one's begin among the sequence's
  const int R = r1 - r0;
  int n = 0;
  bool bad = false;
  if (tid < R) {
    const kf_route row = a.routes[r0 + tid];
    bad = row.seq != b || !route_row_ok(row.tok_begin, row.tok_end, row.page_base, row.page_cap,
                                        a.max_pages_per_route, a.num_page_ids);
    n = bad ? 0 : row.tok_end - row.tok_begin;
    if (r0 + tid == into) bad = bad || n != 0;
    pbase[tid] = row.page_base;
  }
  int64_t x = n;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int64_t y = __shfl_up((long long)x, m);
    if (lane >= m) x += y;
  }
  // (sums beyond 32 bits are refused: each wave's is below 2^37)
  __shared__ int64_t s_sum[16];
  if (lane == 63) s_sum[w] = x;
  if (__syncthreads_or(bad)) return fail(KF_EFLAG_BAD_ROUTE);
  int64_t before = 0, all = 0;
  for (int i = 0; i < 16; ++i) {
    if (i < w) before += s_sum[i];
    all += s_sum[i];
  }
  if (all > INT32_MAX - 1024) return fail(KF_EFLAG_BAD_ROUTE);
  if (tid < R) pre[tid] = (int)(before + x) - n;
  if (tid == 0) pre[R] = (int)all;
  __syncthreads();
  const int L = (int)all, K = min(L, keep);
  const int first = min(K, a.keep_first), last = min(K - first, a.keep_last);
  // where they go
  const kf_route to = a.routes[into];
  const int64_t pages = ((int64_t)K + kPage - 1) / kPage;
  if (pages > to.page_cap) return fail(KF_EFLAG_TAIL_FULL);
  if ((int64_t)to.tok_begin + K > INT32_MAX || to.page_base + pages > a.num_page_ids)
    return fail(KF_EFLAG_BAD_ROUTE);
  for (int64_t p = tid; p < pages; p += 1024)
    bad |= (uint32_t)a.page_ids[to.page_base + p] >= (uint32_t)a.num_pages;

  // this wave's stretch, and a walk over the places lo .. hi - 1 of it, eight at a time a
  // lane: f(place, token, its weight) with the token's page * 16 + slot
  const int per = ((L + 1023) / 1024) * 64, lo = min(L, w * per), hi = min(L, lo + per);
  auto walk = [&](bool want_weights, auto f) __attribute__((always_inline)) {
    int r = 0;
    {  // the route of place lo + lane
      const int e = min(lo + lane, L - 1);
      int top = R;
      while (top - r > 1) {
        const int mid = (r + top) >> 1;
        (pre[mid] <= e ? r : top) = mid;
      }
    }
    for (int e0 = lo; e0 < hi; e0 += 512) {
      int at[8];
      float wt[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = e0 + 64 * i + lane;
        at[i] = 0;
        if (e < hi) {
          while (e >= pre[r + 1]) ++r;
          const int j = e - pre[r], pid = a.page_ids[pbase[r] + j / kPage];
          if ((uint32_t)pid < (uint32_t)a.num_pages)
            at[i] = pid * kPage + j % kPage;
          else
            at[i] = -1;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        wt[i] = 0.0f;
        if (want_weights && e0 + 64 * i + lane < hi && at[i] >= 0)
          wt[i] = a.weights[((size_t)(at[i] >> 4) * H + g) * kPage + (at[i] & 15)];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) f(e0 + 64 * i + lane, at[i], wt[i]);
    }
  };
  const bool in_lds = L <= kKeysInLds;
  walk(in_lds, [&](int e, int at, float wt) {
    if (e >= hi) return;
    bad |= at < 0;
    if (in_lds) keys[e] = order_key(wt);
  });
  if (__syncthreads_or(bad)) return fail(KF_EFLAG_BAD_PAGE);

  const int c0 = first, c1 = L - last;  // the places that compete
  int want = K - first - last;          // and how many of them stay
  uint32_t top = 0;                     // the threshold's bits so far
  const bool none = want == 0, every = want == c1 - c0;
  if (!none && !every) {
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
      const int above = pass == 0 ? 32 : pass == 1 ? 21 : 10;
      hist[tid] = hist[tid + 1024] = 0;
      __syncthreads();
      auto count = [&](int e, uint32_t key) __attribute__((always_inline)) {
        const bool mine = e >= max(lo, c0) && e < min(hi, c1) &&
                          (pass == 0 || key >> above == top >> above);
        const uint64_t who = __ballot(mine);
        if (!who) return;
        const uint32_t bin = (key >> shift) & (bins - 1);
        const int lead = __builtin_ctzll(who);
        const uint32_t one = __builtin_amdgcn_readlane(bin, lead);
        if (__ballot(mine && bin == one) == who) {  // many weights are alike
          if (lane == lead) atomicAdd(&hist[one], (uint32_t)__builtin_popcountll(who));
        } else if (mine) {
          atomicAdd(&hist[bin], 1u);
        }
      };
      if (in_lds) {
        for (int e = lo + lane; e < lo + per; e += 64) count(e, e < hi ? keys[e] : 0);
      } else {
        walk(true, [&](int e, int, float wt) { count(e, order_key(wt)); });
      }
      __syncthreads();
      // the bin in which the want-th largest lies: thread t has bins 2 t and 2 t + 1 from
      // the top
      const int bin = bins - 1 - 2 * tid;
      const int h0 = bin > 0 ? (int)hist[bin] : 0, h1 = bin > 0 ? (int)hist[bin - 1] : 0;
      int y = h0 + h1;
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const int z = __shfl_up(y, m);
        if (lane >= m) y += z;
      }
      if (lane == 63) s_scan[0][w] = y;
      __syncthreads();
      int under = y - h0 - h1;
      for (int i = 0; i < w; ++i) under += s_scan[0][i];
      if (under < want && under + h0 + h1 >= want) {
        const bool upper = under + h0 >= want;
        s_bin = upper ? bin : bin - 1;
        s_want = want - under - (upper ? 0 : h0);
      }
      __syncthreads();
      top |= (uint32_t)s_bin << shift;
      want = s_want;
      __syncthreads();
    }
  }
  // A place stays if it is one of the first or last ones, if its key is larger than
  // top, or if it is one of the first `want` equal ones.
  auto kind = [&](int e, uint32_t key, bool& equal) -> bool {
    equal = false;
    if (e >= hi) return false;
    if (e < c0 || e >= c1) return true;
    if (none) return false;
    if (every) return true;
    equal = key == top;
    return key > top;
  };
  int sure = 0, equals = 0;
  auto tally = [&](int e, uint32_t key) {
    bool eq;
    const bool yes = kind(e, key, eq);
    sure += __builtin_popcountll(__ballot(yes));
    equals += __builtin_popcountll(__ballot(eq));
  };
  if (in_lds) {
    for (int e = lo + lane; e < lo + per; e += 64) tally(e, e < hi ? keys[e] : 0);
  } else {
    walk(true, [&](int e, int, float wt) { tally(e, order_key(wt)); });
  }
  if (lane == 0) {
    s_scan[0][w] = sure;
    s_scan[1][w] = equals;
  }
  __syncthreads();
  sure = equals = 0;
  for (int i = 0; i < w; ++i) {
    sure += s_scan[0][i];
    equals += s_scan[1][i];
  }
  if (none || every) want = 0;
  int32_t* list = a.list + ((size_t)b * H + g) * a.max_keep;
  const uint64_t lower = ((uint64_t)1 << lane) - 1;
  walk(!in_lds, [&](int e, int at, float wt) {
    bool eq;
    const uint32_t key = in_lds ? (e < hi ? keys[e] : 0) : order_key(wt);
    const bool yes = kind(e, key, eq);
    const uint64_t ys = __ballot(yes), es = __ballot(eq);
    const int eq_rank = equals + __builtin_popcountll(es & lower);
    const int rank = sure + __builtin_popcountll(ys & lower) + min(eq_rank, want);
    if (yes || (eq && eq_rank < want)) list[rank] = at;
    sure += __builtin_popcountll(ys);
    equals += __builtin_popcountll(es);
  });
  if (g == 0 && tid == 0) {
    plan[0] = K;
    plan[1] = to.page_base;
  }
}

// A code of a page of scale was as one of a page of scale now: the nearest to
// value * was / now, in 32 bits; a NaN's stays.
__device__ __forceinline__ uint32_t recode4(uint32_t codes, float was, float now) {
  const f32x2 lo = e4m3_values(codes & 0xFFFFu), hi = e4m3_values(codes >> 16);
  uint32_t out = e4m3_pair(lo.x * was / now, lo.y * was / now) |
                 e4m3_pair(hi.x * was / now, hi.y * was / now) << 16;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if ((codes >> (8 * i) & 0x7Fu) == 0x7Fu)
      out = (out & ~(0xFFu << (8 * i))) | (codes & 0xFFu << (8 * i));
  return out;
}

// Dword d (uniform) of two vectors.
__device__ __forceinline__ uint32_t pick(u32x4 a, u32x4 b, int d) {
  const u32x4 x = d & 4 ? b : a;
  const uint32_t y = d & 1 ? x[1] : x[0], z = d & 1 ? x[3] : x[2];
  return d & 2 ? z : y;
}

// A wave moves one page of one KV head, K or V, of what stays.  V's rows of sixteen
// slots are read whole: a token's own two bytes of each come with the other 30.
template <bool FP8>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int H = a.num_kv_heads, b = blockIdx.y;
  const int kept = a.plan[2 * b];
  if (kept < 0) return;
  if (blockIdx.x == 0) {  // the routes: all others are empty now
    const int into = a.into[b], r1 = a.seq_route_begin[b + 1];
    for (int r = a.seq_route_begin[b] + threadIdx.x; r < r1; r += 256)
      a.routes[r].tok_end = a.routes[r].tok_begin + (r == into ? kept : 0);
  }
  const int64_t item = (int64_t)blockIdx.x * 4 + wave;
  const bool is_v = item & 1;
  const int g = (int)((item >> 1) % H), p = (int)((item >> 1) / H);
  const int n = min(kPage, kept - p * kPage);  // (max_keep bounds p)
  if (n <= 0) return;
  const int page = a.page_ids[a.plan[2 * b + 1] + p];
  const int32_t* list = a.list + ((size_t)b * H + g) * a.max_keep + p * kPage;
  const int mine = list[min(lane & 15, n - 1)];  // token lane % 16's page * 16 + slot
  const int esz = FP8 ? 1 : 2;
  char* pool = static_cast<char*>(is_v ? a.v_pool : a.k_pool);
  auto slice = [&](int pg) {
    return pool + slice_of(pg, g, H, a.num_pages, a.head_major) * (size_t)(kPage * kDim * esz);
  };
  char* out = slice(page);
  float was = 1.0f, now = 1.0f;
  bool same = true;
  if constexpr (FP8) {
    float* scales = is_v ? a.v_scale : a.k_scale;
    was = scales[(size_t)(mine >> 4) * H + g];
    const uint32_t bits = __builtin_bit_cast(uint32_t, was);
    same = __ballot(bits != (uint32_t)uniform((int)bits)) == 0;
    now = same ? was : wave_max(fabsf(was));
    if (lane == 0) scales[(size_t)page * H + g] = now;
  }
  if (!is_v) {
    if (lane < n)
      a.weights[((size_t)page * H + g) * kPage + lane] =
          a.weights[((size_t)(mine >> 4) * H + g) * kPage + (mine & 15)];
    constexpr int kLanes = FP8 ? 8 : 16, kRows = 64 / kLanes;  // lanes a row, rows a load
    u32x4 x[kPage / kRows];
#pragma unroll
    for (int i = 0; i < kPage / kRows; ++i) {
      const int from = __shfl(mine, kRows * i + lane / kLanes);
      x[i] = ld16(slice(from >> 4) + ((from & 15) * kDim * esz + 16 * (lane % kLanes)));
    }
#pragma unroll
    for (int i = 0; i < kPage / kRows; ++i) {
      const int s = kRows * i + lane / kLanes;
      if constexpr (FP8) {
        const float sc = __shfl(was, s);
        if (!same && sc != now) {
#pragma unroll
          for (int k = 0; k < 4; ++k) x[i][k] = recode4(x[i][k], sc, now);
        }
      }
      if (s < n) *reinterpret_cast<u32x4*>(out + s * kDim * esz + 16 * (lane % kLanes)) = x[i];
    }
    return;
  }
  // V: dims 2 lane and 2 lane + 1, two rows of sixteen slots
  constexpr int kVecs = FP8 ? 2 : 4;
  const size_t mine_at = (size_t)lane * 2 * kPage * esz;
  u32x4 y[kVecs] = {};
  if (n < kPage) {  // slots behind the last one stay as they were
#pragma unroll
    for (int i = 0; i < kVecs; ++i) y[i] = ld16(out + mine_at + 16 * i);
  }
#pragma unroll
  for (int s0 = 0; s0 < kPage; s0 += 4) {
    u32x4 x[4][kVecs];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s0 + s >= n) break;
      const int from = __builtin_amdgcn_readlane(mine, s0 + s);
#pragma unroll
      for (int i = 0; i < kVecs; ++i) x[s][i] = ld16(slice(from >> 4) + mine_at + 16 * i);
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s0 + s >= n) break;
      const int slot = __builtin_amdgcn_readlane(mine, s0 + s) & 15, to = s0 + s;
      if constexpr (FP8) {
        uint32_t two = 0;
#pragma unroll
        for (int d = 0; d < 2; ++d)
          two |= (pick(x[s][d], x[s][d], slot >> 2) >> (8 * (slot & 3)) & 0xFFu) << (8 * d);
        const float sc = __shfl(was, to);
        if (!same && sc != now) two = recode4(two, sc, now);
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const uint32_t z = y[d][to >> 2] & ~(0xFFu << (8 * (to & 3)));
          y[d][to >> 2] = z | (two >> (8 * d) & 0xFFu) << (8 * (to & 3));
        }
      } else {
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const uint32_t v =
              pick(x[s][2 * d], x[s][2 * d + 1], slot >> 1) >> (16 * (slot & 1)) & 0xFFFFu;
          const int vec = 2 * d + (to >> 3), dw = (to & 7) >> 1;
          y[vec][dw] = (y[vec][dw] & ~(0xFFFFu << (16 * (to & 1)))) | v << (16 * (to & 1));
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kVecs; ++i) *reinterpret_cast<u32x4*>(out + mine_at + 16 * i) = y[i];
}

}  // namespace

hipError_t launch_attn_weights(const AttnWeightsArgs& a, bool fp8, hipStream_t stream) {
  const dim3 grid((uint32_t)a.chunks * a.num_kv_heads, a.num_routes);
  if (fp8 && a.key_waves == 1)
    attn_weights_kernel<true, 1><<<grid, 256, 0, stream>>>(a);
  else if (fp8 && a.key_waves == 2)
    attn_weights_kernel<true, 2><<<grid, 256, 0, stream>>>(a);
  else if (fp8)
    attn_weights_kernel<true, 4><<<grid, 256, 0, stream>>>(a);
  else if (a.key_waves == 1)
    attn_weights_kernel<false, 1><<<grid, 256, 0, stream>>>(a);
  else if (a.key_waves == 2)
    attn_weights_kernel<false, 2><<<grid, 256, 0, stream>>>(a);
  else
    attn_weights_kernel<false, 4><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_evict(const EvictArgs& a, bool fp8, hipStream_t stream) {
  evict_select_kernel<<<dim3(a.num_kv_heads, a.num_seqs), 1024, 0, stream>>>(a);
  const hipError_t st = hipGetLastError();
  if (st != hipSuccess) return st;
  const int64_t pages = ((int64_t)a.max_keep + kPage - 1) / kPage;
  const int64_t wgs = (pages * 2 * a.num_kv_heads + 3) / 4;
  const dim3 grid((uint32_t)(wgs > 0 ? wgs : 1), a.num_seqs);
  if (fp8)
    evict_move_kernel<true><<<grid, 256, 0, stream>>>(a);
  else
    evict_move_kernel<false><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace kf
