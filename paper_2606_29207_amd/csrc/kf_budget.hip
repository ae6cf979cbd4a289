// gfx950 kernels of the operators that keep a cache within a budget:
//   attn_weights_kernel -- the attention weight that every token receives
//   evict_select_kernel -- which tokens of a sequence and KV head stay, by one workgroup
//   evict_count_kernel, evict_list_kernel -- the same by several, a launch for each pass
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
constexpr int kKeysInLds = 34 * 1024;  // tokens of a sequence whose keys stay in LDS
constexpr int kEvictRoutes = 1024;     // routes of a sequence at most
constexpr int kBins = 2048;            // of a pass of 11 bits

// Orders as the weights do; NaN before all others, zeros equal.
__device__ __forceinline__ uint32_t order_key(float w) {
  if (w != w) return 0;
  const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.0f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// The bits of a key that a pass counts: 11, 11 and 10 from the top.
__device__ __forceinline__ int pass_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ int pass_bins(int pass) { return pass == 2 ? kBins / 2 : kBins; }
// Whether a key has the threshold's bits above those.
__device__ __forceinline__ bool pass_takes(int pass, uint32_t key, uint32_t top) {
  return pass == 0 || ((key ^ top) >> (pass == 1 ? 21 : 10)) == 0;
}

// Sum over the waves before this one of x[0 .. 15], and over all.
template <class T>
__device__ __forceinline__ T waves_before(const T* x, int w, T& all) {
  T before = 0;
  all = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (i < w) before += x[i];
    all += x[i];
  }
  return before;
}
template <class T>
__device__ __forceinline__ T wave_scan(T x, int lane) {  // inclusive
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const T y = (T)__shfl_up((long long)x, m);
    if (lane >= m) x += y;
  }
  return x;
}
template <>
__device__ __forceinline__ int wave_scan(int x, int lane) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int y = __shfl_up(x, m);
    if (lane >= m) x += y;
  }
  return x;
}

// A sequence's tokens, route after route, and what stays of them.
struct EvictSeq {
  int status;      // 0, -1: left alone, or the error's flag
  int routes;      // its routes
  int L, K;        // its tokens, and those that stay
  int c0, c1;      // the places that compete; those before and behind stay
  int base;        // index of the first page id that they go to
};
struct EvictShared {
  int pre[kEvictRoutes + 1], base[kEvictRoutes];  // of its routes: first place, first page id's
                                                  // index
  int64_t sum[16];
  int scan[2][16];
  int bin, want;
};

// Checked by every workgroup (1024 threads) for itself, but for the page ids.
__device__ __forceinline__ EvictSeq evict_sequence(const EvictArgs& a, int b, EvictShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  EvictSeq s{};
  const int into = a.into[b], keep = a.keep[b];
  const int r0 = a.seq_route_begin[b], r1 = a.seq_route_begin[b + 1];
  s.status = -1;
  if (into == -1) return s;
  s.status = KF_EFLAG_BAD_ROUTE;
  if (r0 < 0 || r1 < r0 || r1 > a.num_routes || r1 - r0 > kEvictRoutes || into < r0 || into >= r1 ||
      keep < 0 || keep > a.max_keep)
    return s;
  s.routes = r1 - r0;
  const kf_route to = a.routes[into];
  int n = 0;
  bool bad = false;
  if (tid < s.routes) {
    const kf_route row = a.routes[r0 + tid];
    bad = row.seq != b || !route_row_ok(row.tok_begin, row.tok_end, row.page_base, row.page_cap,
                                        a.max_pages_per_route, a.num_page_ids);
    n = bad ? 0 : row.tok_end - row.tok_begin;
    bad = bad || (r0 + tid == into && n != 0);
    sh.base[tid] = row.page_base;
  }
  // (64 bits: a route has up to 2^31 - 1 tokens)
  const int64_t x = wave_scan((int64_t)n, lane);
  if (lane == 63) sh.sum[w] = x;
  if (__syncthreads_or(bad)) return s;
  int64_t all;
  const int64_t before = waves_before(sh.sum, w, all);
  if (all > INT32_MAX - 1024) return s;
  if (tid < s.routes) sh.pre[tid] = (int)(before + x) - n;
  if (tid == 0) sh.pre[s.routes] = (int)all;
  s.L = (int)all;
  s.K = min(s.L, keep);
  s.base = to.page_base;
  const int64_t pages = ((int64_t)s.K + kPage - 1) / kPage;
  if ((int64_t)to.tok_begin + s.K > INT32_MAX || to.page_base + pages > a.num_page_ids) return s;
  s.status = pages > to.page_cap ? KF_EFLAG_TAIL_FULL : 0;
  const int first = min(s.K, a.keep_first), last = min(s.K - first, a.keep_last);
  s.c0 = first;
  s.c1 = s.L - last;
  __syncthreads();
  return s;
}

// Whether an id of the pages that they go to is bad (this thread's share).
__device__ __forceinline__ bool evict_bad_target(const EvictArgs& a, const EvictSeq& s) {
  bool bad = false;
  for (int p = threadIdx.x; p < (s.K + kPage - 1) / kPage; p += 1024)
    bad |= (uint32_t)a.page_ids[s.base + p] >= (uint32_t)a.num_pages;
  return bad;
}

// The places lo .. hi - 1, eight at a time a lane, 64 beside each other: f(place, at,
// weight) with at = the token's page * 16 + slot, -1 for a page outside the pool.
// Lanes beyond hi call f too.
template <class F>
__device__ __forceinline__ void evict_walk(const EvictArgs& a, const EvictSeq& s,
                                           const EvictShared& sh, int g, int lo, int hi,
                                           bool want_weights, F f) {
  const int lane = threadIdx.x & 63;
  int r = 0;
  {  // the route of place lo + lane
    const int e = min(lo + lane, s.L - 1);
    int top = s.routes;
    while (top - r > 1) {
      const int mid = (r + top) >> 1;
      (sh.pre[mid] <= e ? r : top) = mid;
    }
  }
  int begin = sh.pre[r], end = sh.pre[r + 1], base = sh.base[r];
  for (int e0 = lo; e0 < hi; e0 += 512) {
    int at[8];
    float wt[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = e0 + 64 * i + lane;
      at[i] = 0;
      if (e < hi) {
        if (e >= end) {
          do ++r;
          while (e >= sh.pre[r + 1]);
          begin = sh.pre[r];
          end = sh.pre[r + 1];
          base = sh.base[r];
        }
        at[i] = a.page_ids[base + (e - begin) / kPage];
      }
      wt[i] = __builtin_bit_cast(float, begin);  // (the slot follows from it)
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = e0 + 64 * i + lane, slot = (e - __builtin_bit_cast(int, wt[i])) & (kPage - 1);
      wt[i] = 0.0f;
      if (e < hi) {
        at[i] = (uint32_t)at[i] < (uint32_t)a.num_pages ? at[i] * kPage + slot : -1;
        if (want_weights && at[i] >= 0)
          wt[i] = a.weights[((size_t)(at[i] >> 4) * a.num_kv_heads + g) * kPage + slot];
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) f(e0 + 64 * i + lane, at[i], wt[i]);
  }
}

// One more of a bin, for the lanes that say so.  Many weights are alike: one lane
// counts for all of one bin.
__device__ __forceinline__ void evict_count(uint32_t* hist, bool mine, uint32_t bin) {
  const uint64_t who = __ballot(mine);
  if (!who) return;
  const int lane = threadIdx.x & 63, lead = __builtin_ctzll(who);
  const uint32_t one = __builtin_amdgcn_readlane(bin, lead);
  if (__ballot(mine && bin == one) == who) {
    if (lane == lead) atomicAdd(&hist[one], (uint32_t)__builtin_popcountll(who));
  } else if (mine) {
    atomicAdd(&hist[bin], 1u);
  }
}

// The bin in which the want-th largest lies, and how many of that bin are wanted.
// Thread t has h0 of bin bins - 1 - 2 t and h1 of the one below.
__device__ __forceinline__ void evict_find(EvictShared& sh, int bins, int h0, int h1, int& bin,
                                           int& want) {
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  const int y = wave_scan(h0 + h1, lane);
  if (lane == 63) sh.scan[0][w] = y;
  __syncthreads();
  int all;
  const int above = waves_before(sh.scan[0], w, all) + y - h0 - h1;
  if (above < want && above + h0 + h1 >= want) {
    const bool upper = above + h0 >= want;
    sh.bin = bins - 1 - 2 * tid - (upper ? 0 : 1);
    sh.want = want - above - (upper ? 0 : h0);
  }
  __syncthreads();
  bin = sh.bin;
  want = sh.want;
}

// What a place is: it stays for sure (one of the first or last ones, or its key is
// larger than the threshold), or its key equals it, and it stays if it is one of the
// first of these that are wanted.
struct EvictRule {
  int c0, c1;
  bool none, every;  // none or all of those that compete stay
  uint32_t top;
  __device__ __forceinline__ bool sure(int e, uint32_t key) const {
    return e < c0 || e >= c1 || every || (!none && key > top);
  }
  __device__ __forceinline__ bool equal(int e, uint32_t key) const {
    return e >= c0 && e < c1 && !none && !every && key == top;
  }
};

// Which tokens of a sequence and KV head stay, by one workgroup: a threshold by radix
// over their keys, which stay in LDS, up to 34K of them.  Each wave has a stretch of the
// places of its own, so that a place's rank is its wave's first rank and a count of
// ballots.
__global__ __launch_bounds__(1024) void evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t keys[kKeysInLds];
  __shared__ uint32_t hist[kBins];
  __shared__ EvictShared sh;
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  const int g = blockIdx.x, b = blockIdx.y;
  int32_t* plan = a.plan + 2 * b;
  EvictSeq s = evict_sequence(a, b, sh);
  const int per = (s.L + 1023) / 1024 * 64;
  const int lo = min(s.L, w * per), hi = min(s.L, lo + per);
  const bool in_lds = s.L <= kKeysInLds;
  if (s.status == 0) {
    bool bad = evict_bad_target(a, s);
    evict_walk(a, s, sh, g, lo, hi, in_lds, [&](int e, int at, float wt) {
      if (e >= hi) return;
      bad |= at < 0;
      if (in_lds) keys[e] = order_key(wt);
    });
    if (__syncthreads_or(bad)) s.status = KF_EFLAG_BAD_PAGE;
  }
  if (g == 0 && tid == 0) {
    plan[0] = s.status ? -1 : s.K;
    plan[1] = s.base;
    if (s.status > 0) atomicOr(a.err_flags, s.status);
  }
  if (s.status) return;

  // the keys of this wave's places, eight at a time a lane
  auto each = [&](auto f) __attribute__((always_inline)) {
    if (!in_lds) {
      evict_walk(a, s, sh, g, lo, hi, true, [&](int e, int at, float wt) { f(e, order_key(wt)); });
      return;
    }
    for (int e0 = lo; e0 < hi; e0 += 512) {
      uint32_t k[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) k[i] = keys[min(e0 + 64 * i + lane, s.L - 1)];
#pragma unroll
      for (int i = 0; i < 8; ++i) f(e0 + 64 * i + lane, k[i]);
    }
  };
  int want = s.K - s.c0 - (s.L - s.c1);  // of those that compete
  EvictRule rule{s.c0, s.c1, want == 0, want == s.c1 - s.c0, 0};
  if (!rule.none && !rule.every) {
    const int from = max(lo, s.c0), till = min(hi, s.c1);
    for (int pass = 0; pass < 3; ++pass) {
      const int bins = pass_bins(pass);
      hist[tid] = hist[tid + 1024] = 0;
      __syncthreads();
      each([&](int e, uint32_t key) {
        evict_count(hist, e >= from && e < till && pass_takes(pass, key, rule.top),
                    key >> pass_shift(pass) & (bins - 1));
      });
      __syncthreads();
      const int at = bins - 1 - 2 * tid;
      int bin;
      evict_find(sh, bins, at > 0 ? hist[at] : 0, at > 0 ? hist[at - 1] : 0, bin, want);
      rule.top |= (uint32_t)bin << pass_shift(pass);
    }
  } else {
    want = 0;
  }
  int sure = 0, equals = 0;
  each([&](int e, uint32_t key) {
    sure += __builtin_popcountll(__ballot(e < hi && rule.sure(e, key)));
    equals += __builtin_popcountll(__ballot(e < hi && rule.equal(e, key)));
  });
  __syncthreads();
  if (lane == 0) {
    sh.scan[0][w] = sure;
    sh.scan[1][w] = equals;
  }
  __syncthreads();
  int all;
  sure = waves_before(sh.scan[0], w, all);
  equals = waves_before(sh.scan[1], w, all);
  int32_t* list = a.list + ((size_t)b * a.num_kv_heads + g) * a.max_keep;
  const uint64_t lower = ((uint64_t)1 << lane) - 1;
  evict_walk(a, s, sh, g, lo, hi, !in_lds, [&](int e, int at, float wt) {
    const uint32_t key = in_lds ? keys[min(e, s.L - 1)] : order_key(wt);
    const bool yes = e < hi && rule.sure(e, key), eq = e < hi && rule.equal(e, key);
    const uint64_t ys = __ballot(yes), es = __ballot(eq);
    const int eq_rank = equals + __builtin_popcountll(es & lower);
    if (yes || (eq && eq_rank < want))
      list[sure + __builtin_popcountll(ys & lower) + min(eq_rank, want)] = at;
    sure += __builtin_popcountll(ys);
    equals += __builtin_popcountll(es);
  });
}

// The same by several workgroups of a sequence and KV head, a launch for each pass:
// each has a part of the places and counts it into a row of bins of its own, and the
// launch behind adds up the rows.
struct EvictPart {
  int parts, lo, hi;  // parts that the sequence has, this one's places
};
__device__ __forceinline__ EvictPart evict_part(const EvictArgs& a, const EvictSeq& s, int p) {
  EvictPart x;
  x.parts = max(1, min(a.parts, (s.L + kPartTokens - 1) / kPartTokens));
  const int per = ((s.L + x.parts - 1) / x.parts + 1023) / 1024 * 1024;
  x.lo = (int)min((int64_t)s.L, (int64_t)p * per);
  x.hi = (int)min((int64_t)s.L, (int64_t)x.lo + per);
  return x;
}
// Row of bins of part p in a pass.
__device__ __forceinline__ uint32_t* evict_row(const EvictArgs& a, int b, int g, int p, int pass) {
  return a.rows + ((((size_t)b * a.num_kv_heads + g) * a.parts + p) * 3 + pass) * kBins;
}
__device__ __forceinline__ int32_t* evict_state(const EvictArgs& a, int b, int g, int p) {
  return a.state + (((size_t)b * a.num_kv_heads + g) * a.parts + p) * 4;
}

// Adds up the rows of a pass, finds the bin, and returns the keys above it in part p
// (MINE), or in the parts before it, with those in the bin in `same`.
template <bool MINE>
__device__ __forceinline__ int evict_next(const EvictArgs& a, EvictShared& sh, int b, int g, int p,
                                          int parts, int pass, uint32_t& top, int& want,
                                          int& same) {
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  const int bins = pass_bins(pass), at = bins - 1 - 2 * tid;
  int h0 = 0, h1 = 0, x0 = 0, x1 = 0;
  if (at > 0) {
#pragma unroll 4
    for (int i = 0; i < parts; ++i) {
      const u32x2 h = *reinterpret_cast<const u32x2*>(evict_row(a, b, g, i, pass) + at - 1);
      h0 += h.y;
      h1 += h.x;
      if (MINE ? i == p : i < p) {
        x0 += h.y;
        x1 += h.x;
      }
    }
  }
  int bin;
  evict_find(sh, bins, h0, h1, bin, want);
  top |= (uint32_t)bin << pass_shift(pass);
  int above = (at > bin ? x0 : 0) + (at - 1 > bin ? x1 : 0);
  int in_bin = at == bin ? x0 : at - 1 == bin ? x1 : 0;
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    above += __shfl_xor(above, m);
    in_bin += __shfl_xor(in_bin, m);
  }
  __syncthreads();
  if (lane == 0) {
    sh.scan[0][w] = above;
    sh.scan[1][w] = in_bin;
  }
  __syncthreads();
  waves_before(sh.scan[1], w, same);
  waves_before(sh.scan[0], w, above);
  return above;
}

template <int PASS>
__global__ __launch_bounds__(1024) void evict_count_kernel(EvictArgs a) {
  __shared__ uint32_t hist[kBins];
  __shared__ EvictShared sh;
  const int tid = threadIdx.x, w = uniform(tid >> 6);
  const int p = blockIdx.x % a.parts, g = blockIdx.x / a.parts, b = blockIdx.y;
  const EvictSeq s = evict_sequence(a, b, sh);
  if (s.status) return;
  const EvictPart part = evict_part(a, s, p);
  if (p >= part.parts) return;
  int want = s.K - s.c0 - (s.L - s.c1);
  const bool counts = want != 0 && want != s.c1 - s.c0;
  if (PASS > 0 && !counts) return;
  int32_t* state = evict_state(a, b, g, p);
  uint32_t top = 0;
  if constexpr (PASS > 0) {
    int same;
    if (PASS > 1) {  // (the first part's: the launch before wrote the same to all)
      top = state[0];
      want = state[1];
    }
    const int above = evict_next<true>(a, sh, b, g, p, part.parts, PASS - 1, top, want, same);
    if (tid == 0) {
      state[0] = top;
      state[1] = want;
      state[2] = above + (PASS > 1 ? state[2] : 0);
    }
  }
  hist[tid] = hist[tid + 1024] = 0;
  __syncthreads();
  const int per = (part.hi - part.lo + 1023) / 1024 * 64;
  const int lo = min(part.hi, part.lo + w * per), hi = min(part.hi, lo + per);
  const int from = max(lo, s.c0), till = min(hi, s.c1);
  bool bad = false;
  evict_walk(a, s, sh, g, lo, hi, counts, [&](int e, int at, float wt) {
    if (e < hi) bad |= at < 0;
    const uint32_t key = order_key(wt);
    evict_count(hist, counts && e >= from && e < till && pass_takes(PASS, key, top),
                key >> pass_shift(PASS) & (pass_bins(PASS) - 1));
  });
  if constexpr (PASS == 0) {
    if (p == 0) bad |= evict_bad_target(a, s);
    bad = __syncthreads_or(bad);
    if (tid == 0) state[3] = bad;
  } else {
    __syncthreads();
  }
  reinterpret_cast<u32x2*>(evict_row(a, b, g, p, PASS))[tid] =
      *reinterpret_cast<const u32x2*>(hist + 2 * tid);
}

__global__ __launch_bounds__(1024) void evict_list_kernel(EvictArgs a) {
  __shared__ EvictShared sh;
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  const int p = blockIdx.x % a.parts, g = blockIdx.x / a.parts, b = blockIdx.y;
  EvictSeq s = evict_sequence(a, b, sh);
  const EvictPart part = evict_part(a, s, p);
  if (s.status == 0) {
    bool bad = false;
    for (int i = lane; i < part.parts; i += 64) bad |= evict_state(a, b, g, i)[3] != 0;
    if (__ballot(bad)) s.status = KF_EFLAG_BAD_PAGE;
  }
  if (blockIdx.x == 0 && tid == 0) {
    int32_t* plan = a.plan + 2 * b;
    plan[0] = s.status ? -1 : s.K;
    plan[1] = s.base;
    if (s.status > 0) atomicOr(a.err_flags, s.status);
  }
  if (s.status || p >= part.parts) return;
  int want = s.K - s.c0 - (s.L - s.c1);
  EvictRule rule{s.c0, s.c1, want == 0, want == s.c1 - s.c0, 0};
  // those that stay before this part: first and last ones, larger keys, equal ones
  int sure = min(part.lo, s.c0) + max(0, part.lo - s.c1), equals = 0;
  const bool counts = !rule.none && !rule.every;
  if (counts) {
    int32_t* state = evict_state(a, b, g, 0);
    rule.top = state[0];
    want = state[1];
    sure += evict_next<false>(a, sh, b, g, p, part.parts, 2, rule.top, want, equals);
    for (int i = 0; i < p; ++i) sure += evict_state(a, b, g, i)[2];
  } else {
    if (rule.every) sure += max(0, min(part.lo, s.c1) - s.c0);
    want = 0;
  }
  const int per = (part.hi - part.lo + 1023) / 1024 * 64;
  const int lo = min(part.hi, part.lo + w * per), hi = min(part.hi, lo + per);
  int mine = 0, alike = 0;
  evict_walk(a, s, sh, g, lo, hi, counts, [&](int e, int at, float wt) {
    const uint32_t key = order_key(wt);
    mine += __builtin_popcountll(__ballot(e < hi && rule.sure(e, key)));
    alike += __builtin_popcountll(__ballot(e < hi && rule.equal(e, key)));
  });
  __syncthreads();
  if (lane == 0) {
    sh.scan[0][w] = mine;
    sh.scan[1][w] = alike;
  }
  __syncthreads();
  int all;
  sure += waves_before(sh.scan[0], w, all);
  equals += waves_before(sh.scan[1], w, all);
  int32_t* list = a.list + ((size_t)b * a.num_kv_heads + g) * a.max_keep;
  const uint64_t lower = ((uint64_t)1 << lane) - 1;
  evict_walk(a, s, sh, g, lo, hi, counts, [&](int e, int at, float wt) {
    const uint32_t key = order_key(wt);
    const bool yes = e < hi && rule.sure(e, key), eq = e < hi && rule.equal(e, key);
    const uint64_t ys = __ballot(yes), es = __ballot(eq);
    const int eq_rank = equals + __builtin_popcountll(es & lower);
    if (yes || (eq && eq_rank < want))
      list[sure + __builtin_popcountll(ys & lower) + min(eq_rank, want)] = at;
    sure += __builtin_popcountll(ys);
    equals += __builtin_popcountll(es);
  });
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
  if (a.parts > 1) {
    const dim3 grid((uint32_t)a.num_kv_heads * a.parts, a.num_seqs);
    evict_count_kernel<0><<<grid, 1024, 0, stream>>>(a);
    evict_count_kernel<1><<<grid, 1024, 0, stream>>>(a);
    evict_count_kernel<2><<<grid, 1024, 0, stream>>>(a);
    evict_list_kernel<<<grid, 1024, 0, stream>>>(a);
  } else {
    evict_select_kernel<<<dim3(a.num_kv_heads, a.num_seqs), 1024, 0, stream>>>(a);
  }
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
