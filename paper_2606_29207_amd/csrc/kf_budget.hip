// gfx950 kernels of the operators that keep a cache within a budget:
//   attn_weights_kernel -- the attention weight that every token receives
//   attn_weights_join_kernel -- its sums where several workgroups shared the columns
//   evict_select_kernel -- which tokens of a sequence and KV head stay, by one workgroup
//   evict_count_kernel, evict_list_kernel -- the same by several, a launch for each pass
//   evict_move_kernel   -- those tokens into the pages of another route
#include <type_traits>

#include "kf_budget.h"
#include "kf_device.h"

namespace kf {
namespace {

// The tokens of a route, and of a sequence that is evicted: places a workgroup's tile
// behind the last one still fit in 32 bits.
constexpr int kMostTokens = INT32_MAX - 1024;

// A route's row (seq, part, tok_begin, tok_end, page_base, page_cap) is sound.
__device__ __forceinline__ bool route_row_ok(int tok_begin, int tok_end, int base, int cap,
                                             int max_pages, int num_page_ids) {
  const int64_t n = (int64_t)tok_end - tok_begin, pages = n > 0 ? (n + kPage - 1) / kPage : 0;
  return n >= 0 && n <= kMostTokens && base >= 0 && pages <= cap && pages <= max_pages &&
         base + pages <= num_page_ids;
}

// ------------------------------------------------------------- attn_weights
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
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

// 16 bytes a lane from memory straight into LDS, 1 KiB a wave.
__device__ __forceinline__ void to_lds16(const char* g, char* l) {
  __builtin_amdgcn_global_load_lds(
      (const __attribute__((address_space(1))) uint32_t*)g,
      (__attribute__((address_space(3))) uint32_t*)(__attribute__((address_space(3))) void*)l, 16,
      0, 2);  // once: the non-temporal hint (32K-token decode 204 us without it, 189 with)
}

// Few columns (a decode step, a small tree): they stay in registers, 16 a matrix
// product, and the keys stream past, a page of 16 per product of depth 32.  Pages go
// through LDS, where each wave has two buffers of 8 KiB of its own: loads of 1 KiB in a
// row, where the operands' own places are 64 bytes of each key's 256.
template <bool FP8, int NC>
__device__ __forceinline__ void few_columns(const AttnWeightsArgs& a, const Seen& s,
                                            char* __restrict__ buf_x, char* __restrict__ buf_y,
                                            int& flag) {
  constexpr int kBatch = FP8 ? 4 : 2;                 // pages of a buffer
  constexpr int kPageBytes = kPage * kDim * (FP8 ? 1 : 2), kLoads = kPageBytes / 1024;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int n16 = lane & 15, grp = lane >> 4, H = a.num_kv_heads, G = a.group;
  const uint32_t C = (uint32_t)s.rows * G;
  // The four waves take batches in turn (of a workgroup's 16 pages: bf16 two a wave, fp8
  // one, whose second buffer is not used then).
  constexpr int kStep = 4 * kBatch;
  int p = s.p0 + kBatch * wave;
  if (p >= s.p1) return;
  buf_x += 8192 * wave;
  buf_y += 8192 * wave;
  // Chunk c (16 bytes) of row r lies at chunk c ^ r (fp8: of its row of two, c ^ r / 2):
  // the sixteen rows that an operand reads at once cover all banks.
  uint32_t from[kLoads];  // in a page, of the lane's chunk of each load
#pragma unroll
  for (int k = 0; k < kLoads; ++k) {
    const int x = 64 * k + lane;  // chunk of the page
    from[k] = 16 * (FP8 ? (x & ~7) | ((x ^ (x >> 4)) & 7) : (x & ~15) | ((x ^ (x >> 4)) & 15));
  }
  const char* pool = static_cast<const char*>(a.k_pool);

  struct Batch {
    float scale[kBatch], old[kBatch];
    int pid[kBatch];
  };
  auto load = [&](Batch& b, int p, char* __restrict__ buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (p + i >= s.p1) break;
      int pid = fixed(a.page_ids)[s.base + p + i];
      b.pid[i] = pid;
      if ((uint32_t)pid >= (uint32_t)a.num_pages) pid = 0;
      const char* page = pool + slice_of(pid, s.g, H, a.num_pages, a.head_major) * kPageBytes;
#pragma unroll
      for (int k = 0; k < kLoads; ++k) to_lds16(page + from[k], buf + kPageBytes * i + 1024 * k);
      b.scale[i] = FP8 ? fixed(a.k_scale)[(size_t)pid * H + s.g] : 1.0f;
      b.old[i] = 0.0f;
      if (a.decay != 0.0f) b.old[i] = a.weights[((size_t)pid * H + s.g) * kPage + n16];
    }
  };
  Batch x, y;
  load(x, p, buf_x);
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
      const float z = a.lse[(s.row0 + (int64_t)(mm / G)) * a.num_q_heads + s.g * G + mm % G];
      lse[t][i] = z * kLog2e;
      sees[t][i] = m < C && has_softmax(z) ? reach(s, mm / G) : -1;
    }
  }
  auto work = [&](const Batch& b, int p, const char* __restrict__ buf)
      __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (p + i >= s.p1) break;
      const char* page = buf + kPageBytes * i;
      u32x4 k[4];
      if constexpr (FP8) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
          widen(*reinterpret_cast<const u32x4*>(page + 128 * n16 +
                                                16 * ((4 * u + grp) ^ (n16 >> 1))),
                k[2 * u], k[2 * u + 1]);
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
          k[u] = *reinterpret_cast<const u32x4*>(page + 256 * n16 + 16 * ((4 * u + grp) ^ n16));
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
  // Waits for a batch: the loads of the next one, if it is whole, may still be out (8 of
  // its pages, and what its tokens' weights were; ids and scales are scalar loads).
  auto wait = [&](int next) __attribute__((always_inline)) {
    static_assert(kBatch * kLoads == 8, "");
    asm volatile("" ::: "memory");
    if (next + kBatch > s.p1)
      __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    else if (a.decay != 0.0f)
      __builtin_amdgcn_s_waitcnt(0x0F70 | (8 + kBatch));
    else
      __builtin_amdgcn_s_waitcnt(0x0F70 | 8);
    asm volatile("" ::: "memory");
  };
  auto read = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };  // what the wave reads
  __builtin_amdgcn_s_waitcnt(0x0F70);  // the columns: or every step would wait for them
  // (One function with both buffers, so that the reads of one are known not to wait for
  // loads into the other.)
  auto step = [&](const Batch& now, const char* __restrict__ buf_now, Batch& next,
                  char* __restrict__ buf_next) __attribute__((always_inline)) {
    if (p + kStep < s.p1) load(next, p + kStep, buf_next);
    wait(p + kStep);
    work(now, p, buf_now);
    read();
    p += kStep;
    return p < s.p1;
  };
  while (step(x, buf_x, y, buf_y) && step(y, buf_y, x, buf_x)) {
  }
}

__device__ __forceinline__ void lds_barrier() {  // for LDS that the waves wrote themselves
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Many columns (prompts, the last rows of one): 64 keys a wave and 256 a workgroup stay
// in registers, the columns that see them stream past through LDS, 32 a matrix product
// and a step.
//
// A product of 32 keys and 32 columns takes the matrix unit 256 cycles, and its 1024
// exponentials take the vector unit as many.  So a product is issued between the
// exponentials of the one before it, two a step in turn, with its own columns in
// registers, those behind them in LDS and others on their way.  2000 rows behind 30K
// tokens, 32 / 8 heads: 540 us, 0.94 PFLOP/s (the largest plain product reaches 1.19).
// 40 vector registers are spilled (fp8 43), most of them outside the loops; the loop of
// columns that some keys are hidden from reloads three.  With 64 and 128 keys a workgroup
// (its waves then also beside each other along the columns) 690 and 585, with eight waves
// 550 .. 680.
template <bool FP8>
struct Columns {
  static constexpr int kCols = 32, kStep = kCols * 256;  // bytes of a step in LDS
  const AttnWeightsArgs& a;
  const Seen& s;
  int tid, lane, wave, half, l32;
  uint32_t magic, single;  // 2^32 / G, rounded up; G = 1: 0 and all bits
  const uint16_t* q;
  const float* lse;
  int all;         // columns of the sequence
  int front;       // the first row's position less tok_begin, in 32 bits
  // the wave's keys: 32 t + l32 of 64
  u32x4 k[2][8];
  float c[2][2], key_scale[2];
  int pid[2];
  f32x16 acc[2];
  int j0;          // index of its first key
  // columns on their way to LDS
  u32x4 piece[2];
  float piece_lse;
  bool even;                     // a step is a whole number of rows
  uint32_t piece_at[2], lse_at;  // the lane's places in a step, in elements

  __device__ __forceinline__ void begin() {
    tid = threadIdx.x;
    lane = tid & 63;
    wave = uniform(tid >> 6);
    half = lane >> 5;
    l32 = lane & 31;
    const int G = a.group;
    magic = G == 1 ? 0 : 0xFFFFFFFFu / (uint32_t)G + 1;
    single = G == 1 ? ~0u : 0;
    q = a.q + s.row0 * a.q_stride + (size_t)s.g * G * kDim;
    lse = a.lse + (int64_t)s.row0 * a.num_q_heads + s.g * G;
    all = s.rows * G;
    front = (int)max((int64_t)INT32_MIN, min((int64_t)INT32_MAX, s.first));
    even = kCols % G == 0 && a.q_stride <= 1 << 24;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t col = 8 * wave + 4 * u + (lane >> 4);
      piece_at[u] = col / (uint32_t)G * (uint32_t)a.q_stride + col % (uint32_t)G * kDim +
                    8 * (lane & 15);
    }
    lse_at = l32 / G * a.num_q_heads + l32 % G;
  }

  __device__ __forceinline__ int row_of(int col) const {  // col < 2^28
    return (int)(__umulhi((uint32_t)col, magic) + ((uint32_t)col & single));
  }
  // The columns of step st: all of a sequence's workgroups begin at its last one, so
  // that those of a KV head read the same ones at a time.
  __device__ __forceinline__ int step_begin(int st) const { return all - (st + 1) * kCols; }
  // Sends for them (the first one in place of those before it).  FAST: a step is a whole
  // number of rows and this one is all there: a lane's places in it are the same as in
  // all others, and a scalar address moves, where the others divide for every column.
  // (No branch in any of these: the compiler would move exponentials past it.)
  template <bool FAST>
  __device__ __forceinline__ void send(int st) {
    const int first = step_begin(st);
    if constexpr (FAST) {
      const int64_t row = row_of(first);
      const uint16_t* from = q + row * a.q_stride;
#pragma unroll
      for (int u = 0; u < 2; ++u) piece[u] = ld16(from + piece_at[u]);
      piece_lse = lse[row * a.num_q_heads + lse_at];
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int x = max(first + 8 * wave + 4 * u + (lane >> 4), 0), i = row_of(x);
        piece[u] = ld16(q + i * a.q_stride + (x - i * a.group) * kDim + 8 * (lane & 15));
        __builtin_amdgcn_sched_barrier(0);  // one address at a time: registers
      }
      const int x = max(first + l32, 0), i = row_of(x);
      piece_lse = lse[(int64_t)i * a.num_q_heads + (x - i * a.group)];
    }
  }
  // A column's 16-byte chunks lie in the order of chunk ^ column % 16: the columns that
  // an operand reads at once then cover all banks.  (Every wave writes all the lse: the
  // same values.)
  __device__ __forceinline__ void put(char* to, float* to_lse) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int col = 8 * wave + 4 * u + (lane >> 4);
      *reinterpret_cast<u32x4*>(to + col * 256 + (((lane & 15) ^ (col & 15)) << 4)) = piece[u];
    }
    to_lse[l32] = piece_lse;
  }
  __device__ __forceinline__ u32x4 get(const char* from, int u) const {
    const int chunk = FP8 ? 4 * (u >> 1) + 2 * half + (u & 1) : 2 * u + half;
    return *reinterpret_cast<const u32x4*>(from + l32 * 256 + ((chunk ^ (l32 & 15)) << 4));
  }
  // The lse of the lane's column, in units of log2, and the last token that its row sees
  // (-1: none).
  __device__ __forceinline__ float column(const float* from_lse) const {
    return from_lse[l32] * kLog2e;
  }
  __device__ __forceinline__ int last_seen(int st, float z) const {
    const int x = step_begin(st) + l32;
    return x >= 0 && has_softmax(z) ? max(-1, __builtin_elementwise_add_sat(front, row_of(x))) : -1;
  }
  // Whether every column of the steps up to st sees all of the wave's keys.
  __device__ __forceinline__ bool sees_all(int st) const {
    const int at = step_begin(st);
    return at >= 0 && reach(s, row_of(at)) - 63 >= j0;
  }

  // Keys t of the wave's from `page` on: bf16 straight into their operand, fp8 codes into
  // half of it, to be widened when they are there.
  template <int t>
  __device__ __forceinline__ void load_keys(int page) {
    const int H = a.num_kv_heads, last = (s.n - 1) / kPage;
    const size_t head_bytes = kPage * kDim * (FP8 ? 1 : 2);
    pid[t] = a.page_ids[s.base + min(page + 2 * t + (l32 >> 4), last)];
    const int id = (uint32_t)pid[t] < (uint32_t)a.num_pages ? pid[t] : 0;
    const char* from = static_cast<const char*>(a.k_pool) +
                       slice_of(id, s.g, H, a.num_pages, a.head_major) * head_bytes +
                       (FP8 ? (l32 & 15) * kDim + 16 * half : 2 * ((l32 & 15) * kDim + 8 * half));
#pragma unroll
    for (int u = 0; u < (FP8 ? 4 : 8); ++u) k[t][u] = ld16(from + 32 * u);
    key_scale[t] = FP8 ? a.k_scale[(size_t)id * H + s.g] : 1.0f;
  }
  template <int t>
  __device__ __forceinline__ void take_keys() {
    if constexpr (FP8) {
      u32x4 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = k[t][u];
#pragma unroll
      for (int u = 0; u < 4; ++u) widen(x[u], k[t][2 * u], k[t][2 * u + 1]);
      const float sc = a.scale_log2 * key_scale[t];
      c[t][0] = __shfl(sc, 0);
      c[t][1] = __shfl(sc, 16);
    } else {
      c[t][0] = c[t][1] = a.scale_log2;
    }
  }

  // The product of keys kk and the columns b, between the exponentials of `was`, that of
  // keys T and the columns of step st, which see some of them (MASK) or all.  READ: each
  // operand makes room for the next step's, in `from`.
  template <int T, bool READ, bool MASK>
  __device__ __forceinline__ void turn(const u32x4 (&kk)[8], u32x4 (&b)[8], f32x16& d,
                                       const f32x16& was, float z, int st, const char* from) {
    const int up_to = MASK ? last_seen(st, z) - (j0 + 32 * T + 4 * half) : 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) d[i] = 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      d = mfma32(kk[u], b[u], d);
      if constexpr (READ) b[u] = get(from, u);
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const int i = 2 * u + v;
        float e = exp2_fast(__builtin_fmaf(was[i], c[T][i >> 3], -z));
        if (MASK) e = 8 * (i >> 2) + (i & 3) <= up_to ? e : 0.0f;
        acc[T][i] += e;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // The exponentials of the last product, of keys 1.
  __device__ __forceinline__ void last_turn(const f32x16& was, float z, int st) {
    const int up_to = last_seen(st, z) - (j0 + 32 + 4 * half);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float e = exp2_fast(__builtin_fmaf(was[i], c[1][i >> 3], -z));
      acc[1][i] += 8 * (i >> 2) + (i & 3) <= up_to ? e : 0.0f;
    }
  }
  __device__ __forceinline__ void first_product(const char* from, u32x4 (&b)[8], f32x16& d) {
#pragma unroll
    for (int u = 0; u < 8; ++u) b[u] = get(from, u);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[t][i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) d[i] = 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u) d = mfma32(k[0][u], b[u], d);
  }

  // The sums over the 32 columns of a half wave: lane l32 ends with that of value
  // 16 t + i = l32.  In every turn a lane gives half of its values away.
  template <int M>
  __device__ __forceinline__ void halve(float (&v)[32]) const {
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const float give = l32 & M ? v[i] : v[i + M], keep = l32 & M ? v[i + M] : v[i];
      v[i] = keep + __shfl_xor(give, M);
    }
    if constexpr (M > 1) halve<M / 2>(v);
  }
  __device__ __forceinline__ float reduce() const {
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = acc[i >> 4][i & 15];
    halve<16>(v);
    return v[0];
  }
  // Which of the wave's 64 keys that is.
  __device__ __forceinline__ int key_of_lane() const {
    return 32 * (l32 >> 4) + 8 * ((l32 >> 2) & 3) + 4 * half + (l32 & 3);
  }

  // The sums of the wave's keys, whose page ids id0 and id1 hold as pid does, into their
  // tokens' weights.
  __device__ __forceinline__ void write(float sum, int id0, int id1, int& flag) {
    const int m = key_of_lane(), j = j0 + m;
    const int x = __shfl(id0, m & 16), y = __shfl(id1, m & 16), id = m & 32 ? y : x;
    if (j0 / kPage + (m >> 4) >= s.p1 || j >= s.n) return;
    if ((uint32_t)id >= (uint32_t)a.num_pages) {
      flag |= KF_EFLAG_BAD_PAGE;
      return;
    }
    float* at = a.weights + ((size_t)id * a.num_kv_heads + s.g) * kPage + (m & 15);
    *at = j < s.first && a.decay != 0.0f ? __builtin_fmaf(a.decay, *at, sum) : sum;
  }

  // Columns that all fit in LDS (the last rows of a prompt): they are put there once, and
  // each wave takes its share of the pages, four at a time, without a barrier.  The last
  // 32 rows of 8 prompts of 2K .. 32K tokens, 64 / 8 heads, fp8: 74 us, 84 with the
  // columns put there anew for every 256 keys.
  __device__ __forceinline__ void run_resident(char* lds_x, char* lds_y, float* lds_lse,
                                               int& flag) {
    begin();
    const int steps = (all + kCols - 1) / kCols;
    constexpr int kInX = kHeldColumns / 2 / kCols;  // steps in lds_x
    auto place = [&](int st) {
      return st < kInX ? lds_x + st * kStep : lds_y + (st - kInX) * kStep;
    };
    int p = s.p0 + 4 * wave;
    if (p < s.p1) {
      load_keys<0>(p);
      load_keys<1>(p);
    }
    for (int st = 0; st < steps; ++st) {
      send<false>(st);
      put(place(st), lds_lse + st * kCols);
    }
    lds_barrier();
    u32x4 b[8];
    f32x16 d0, d1;
    for (; p < s.p1; p += 16) {
      j0 = p * kPage;
      take_keys<0>();
      take_keys<1>();
      const int id0 = pid[0], id1 = pid[1];
      first_product(lds_x, b, d0);
      int st = 0;
      auto body = [&](auto mask) __attribute__((always_inline)) {
        constexpr bool MASK = decltype(mask)::value;
        const float z = column(lds_lse + st * kCols);
        turn<0, true, MASK>(k[1], b, d1, d0, z, st, place(st + 1));
        turn<1, false, MASK>(k[0], b, d0, d1, z, st, nullptr);
        ++st;
      };
      auto whole = [&]() {
        return sees_all(st) && __ballot(!has_softmax(column(lds_lse + st * kCols))) == 0;
      };
      while (st + 1 < steps) {  // (two loops: see run)
        while (st + 1 < steps && whole()) body(std::false_type{});
        while (st + 1 < steps && !whole()) body(std::true_type{});
      }
      // the last step: no product of other columns follows, and the next keys are sent for
      // where these have been used
      const float z = column(lds_lse + st * kCols);
      turn<0, false, true>(k[1], b, d1, d0, z, st, nullptr);
      if (p + 16 < s.p1) {
        load_keys<0>(p + 16);
        load_keys<1>(p + 16);
      }
      last_turn(d1, z, st);
      write(reduce(), id0, id1, flag);
    }
  }

  // Columns beyond that.  segment: which part of the steps, where several workgroups
  // share the columns; their sums then go to `sums` (256 of a workgroup).
  __device__ __forceinline__ void run(char* lds, float* lds_lse, int segment, float* sums,
                                      int& flag) {
    begin();
    char* buf[2] = {lds, lds + kStep};
    float* buf_lse[2] = {lds_lse, lds_lse + kCols};
    const int most = (all + kCols - 1) / kCols;
    const int per = a.segments == 1 ? most : 2 * ((most + 2 * a.segments - 1) / (2 * a.segments));
    for (int p = s.p0; p < s.p1; p += 16) {
      // the first row that sees the first of the workgroup's keys, and its columns
      const int64_t before = (int64_t)p * kPage - s.first;
      const int first = (int)max((int64_t)0, min((int64_t)s.rows, before)) * a.group;
      const int steps = min((all - first + kCols - 1) / kCols, (segment + 1) * per);
      const int from = segment * per;
      j0 = (p + 4 * wave) * kPage;
      float sum = 0.0f;
      if (from < steps) {
        send<false>(from);
        load_keys<0>(p + 4 * wave);
        load_keys<1>(p + 4 * wave);
        take_keys<0>();
        take_keys<1>();
        // Step st works on columns in b, which it replaces by those of step st + 1 from
        // LDS; those of st + 2 are put there, and those of st + 3 sent for.
        u32x4 b[8];
        f32x16 d0, d1;
        put(buf[0], buf_lse[0]);
        send<false>(from + 1);
        lds_barrier();
        first_product(buf[0], b, d0);
        float z = column(buf_lse[0]), next_z = 0.0f;
        put(buf[1], buf_lse[1]);
        send<false>(from + 2);
        // (the products behind the last step's are not used)
        auto step = [&](auto mode, auto odd, int st) __attribute__((always_inline)) {
          constexpr bool MASK = decltype(mode)::value == 0, FAST = decltype(mode)::value == 2;
          constexpr int S = decltype(odd)::value, R = S ^ 1;
          const float z2 = column(buf_lse[R]);
          put(buf[S], buf_lse[S]);
          send<FAST>(st + 3);
          turn<0, true, MASK>(k[1], b, d1, d0, z, st, buf[R]);
          turn<1, false, MASK>(k[0], b, d0, d1, z, st, nullptr);
          z = z2;
          lds_barrier();  // the columns that the next step reads are there, these are free
        };
        // Two steps at a time, and loops of their own for steps that some column does not
        // see whole (or none of: it lies before the first one, or its row has no softmax)
        // and for all others: a branch in the loop has the sums copied back and forth.
        lds_barrier();
        auto whole = [&](int st) {
          if (!sees_all(st + 1)) return false;
          next_z = column(buf_lse[1]);
          return __ballot(!has_softmax(z) || !has_softmax(next_z)) == 0;
        };
        auto fast = [&](int st) { return even && step_begin(st + 4) >= 0; };
        auto body = [&](auto mode, int& st) __attribute__((always_inline)) {
          step(mode, std::integral_constant<int, 0>{}, st);
          step(mode, std::integral_constant<int, 1>{}, st + 1);
          st += 2;
        };
        for (int st = from; st < steps;) {
          while (st < steps && fast(st) && whole(st)) body(std::integral_constant<int, 2>{}, st);
          while (st < steps && !fast(st) && whole(st)) body(std::integral_constant<int, 1>{}, st);
          while (st < steps && !whole(st)) body(std::integral_constant<int, 0>{}, st);
        }
        sum = reduce();
      } else if (!sums) {  // (nothing sees these keys; their pages count all the same)
        load_keys<0>(p + 4 * wave);
        load_keys<1>(p + 4 * wave);
      }
      if (sums)
        sums[64 * wave + key_of_lane()] = sum;
      else
        write(sum, pid[0], pid[1], flag);
      lds_barrier();  // the next keys' columns go where these may still be read
    }
  }
};

// The route of a workgroup and the pages that are its own; whether there are any.
__device__ __forceinline__ bool find_keys(const AttnWeightsArgs& a, Seen& s) {
  const int H = a.num_kv_heads, r = blockIdx.y;
  const int chunk = (int)(blockIdx.x / H);
  const auto* rp = fixed(reinterpret_cast<const int32_t*>(a.routes)) + 6 * (int64_t)r;
  const int seq = rp[0], tb = rp[2], te = rp[3], cap = rp[5];
  s.g = blockIdx.x % H;
  s.base = rp[4];
  bool bad = seq < 0 || seq >= a.num_seqs;
  if (!bad) {
    s.row0 = fixed(a.seq_row_begin)[seq];
    const int end = fixed(a.seq_row_begin)[seq + 1];
    s.first = (int64_t)fixed(a.first_pos)[seq] - tb;
    s.rows = end - s.row0;
    bad = s.row0 < 0 || end < s.row0 || end > a.num_rows;
    if (!bad && s.rows == 0) return false;  // not looked at
    bad = bad || !route_row_ok(tb, te, s.base, cap, a.max_pages_per_route, a.num_page_ids);
  }
  if (bad) {
    if (blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x == 0)
      atomicOr(a.err_flags, KF_EFLAG_BAD_ROUTE);
    return false;
  }
  s.n = te - tb;
  const int pages = (int)(((int64_t)s.n + kPage - 1) / kPage);
  if ((int64_t)chunk * a.chunk_pages >= pages) return false;
  s.p0 = chunk * a.chunk_pages;
  s.p1 = (int)min((int64_t)pages, (int64_t)s.p0 + a.chunk_pages);
  return true;
}
// The sums of a workgroup's keys over segment `segment` of the columns.
__device__ __forceinline__ float* sums_of(const AttnWeightsArgs& a, int segment) {
  return a.sums + 256 * (((size_t)segment * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x);
}

template <bool FP8>
__global__ __launch_bounds__(256, 2) void attn_weights_kernel(AttnWeightsArgs a) {
  constexpr int kHalf = kHeldColumns * 128;
  __shared__ __align__(16) char lds_x[kHalf], lds_y[kHalf];
  __shared__ float lds_lse[kHeldColumns];
  Seen s;
  if (!find_keys(a, s)) return;
  const int segment = blockIdx.z;
  const int64_t C = (int64_t)s.rows * a.group;
  if (segment > 0 && C <= kHeldColumns) return;
  int flag = 0;
  if (C <= 16) {
    few_columns<FP8, 1>(a, s, lds_x, lds_y, flag);
  } else if (C <= kFewColumns) {
    few_columns<FP8, kFewColumns / 16>(a, s, lds_x, lds_y, flag);
  } else {
    Columns<FP8> x{a, s};
    if (C <= kHeldColumns)
      x.run_resident(lds_x, lds_y, lds_lse, flag);
    else
      x.run(lds_x, lds_lse, segment, a.segments > 1 ? sums_of(a, segment) : nullptr, flag);
  }
  if (__ballot(flag != 0) && (threadIdx.x & 63) == 0) atomicOr(a.err_flags, KF_EFLAG_BAD_PAGE);
}

// The segments' sums, in order, into the tokens' weights: a thread a token.
__global__ __launch_bounds__(256) void attn_weights_join_kernel(AttnWeightsArgs a) {
  Seen s;
  if (!find_keys(a, s)) return;
  const int j = s.p0 * kPage + threadIdx.x;
  if ((int64_t)s.rows * a.group <= kHeldColumns || j >= s.n) return;
  const int id = a.page_ids[s.base + j / kPage];
  float x[kMaxSegments];
#pragma unroll
  for (int i = 0; i < kMaxSegments; ++i)
    x[i] = i < a.segments ? sums_of(a, i)[threadIdx.x] : 0.0f;
  if ((uint32_t)id >= (uint32_t)a.num_pages) {
    atomicOr(a.err_flags, KF_EFLAG_BAD_PAGE);
    return;
  }
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kMaxSegments; ++i) sum += x[i];
  float* at = a.weights + ((size_t)id * a.num_kv_heads + s.g) * kPage + j % kPage;
  *at = j < s.first && a.decay != 0.0f ? __builtin_fmaf(a.decay, *at, sum) : sum;
}

// -------------------------------------------------------------------- evict
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
  // Up to 64 routes are looked at by every wave for itself, without a barrier.
  const bool few = s.routes <= 64;
  const int own = few ? lane : tid;
  int n = 0;
  bool bad = false;
  if (own < s.routes) {
    const kf_route row = a.routes[r0 + own];
    bad = row.seq != b || !route_row_ok(row.tok_begin, row.tok_end, row.page_base, row.page_cap,
                                        a.max_pages_per_route, a.num_page_ids);
    n = bad ? 0 : row.tok_end - row.tok_begin;
    bad = bad || (r0 + own == into && n != 0);
    if (!few || w == 0) sh.base[own] = row.page_base;
  }
  // (64 bits: a route has up to kMostTokens, a sequence many of them)
  const int64_t x = wave_scan((int64_t)n, lane);
  int64_t all = __shfl((long long)x, 63), before = 0;
  if (few) {
    if (__ballot(bad)) return s;
  } else {
    if (lane == 63) sh.sum[w] = x;
    if (__syncthreads_or(bad)) return s;
    before = waves_before(sh.sum, w, all);
  }
  if (all > kMostTokens) return s;
  if (own < s.routes && (!few || w == 0)) sh.pre[own] = (int)(before + x) - n;
  if (tid == 0) sh.pre[s.routes] = (int)all;
  s.L = (int)all;
  s.K = min(s.L, keep);
  s.base = to.page_base;
  const int64_t pages = ((int64_t)s.K + kPage - 1) / kPage;
  // (first of these: a full target is full wherever its reservation lies in the table)
  if (pages > to.page_cap) {
    s.status = KF_EFLAG_TAIL_FULL;
    return s;
  }
  // the row that it leaves: as sound as those it came from
  if ((int64_t)to.tok_begin + s.K > INT32_MAX || pages > a.max_pages_per_route ||
      to.page_base + pages > a.num_page_ids)
    return s;
  s.status = 0;
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

// Eight places a lane, 64 beside each other: place e0 + 64 i + lane's page * 16 + slot
// (-1 for a page outside the pool) and weight.
struct EvictBatch {
  int at[8];
  float weight[8];
};
// A lane's way through the routes of its places.
struct EvictWalk {
  int r, begin, end, base;  // the route, its places, its first page id's index
};
__device__ __forceinline__ EvictWalk evict_enter(const EvictSeq& s, const EvictShared& sh, int lo) {
  const int e = min(lo + (int)(threadIdx.x & 63), s.L - 1);
  int r = 0, top = s.routes;
  while (top - r > 1) {
    const int mid = (r + top) >> 1;
    (sh.pre[mid] <= e ? r : top) = mid;
  }
  return EvictWalk{r, sh.pre[r], sh.pre[r + 1], sh.base[r]};
}
__device__ __forceinline__ void evict_load(const EvictArgs& a, const EvictShared& sh, int g,
                                           EvictWalk& w, int e0, int hi, bool want_weights,
                                           EvictBatch& x) {
  const int lane = threadIdx.x & 63;
  int slot[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = e0 + 64 * i + lane;
    x.at[i] = 0;
    slot[i] = 0;
    if (e < hi) {
      if (e >= w.end) {
        do ++w.r;
        while (e >= sh.pre[w.r + 1]);
        w.begin = sh.pre[w.r];
        w.end = sh.pre[w.r + 1];
        w.base = sh.base[w.r];
      }
      x.at[i] = a.page_ids[w.base + (e - w.begin) / kPage];
      slot[i] = (e - w.begin) & (kPage - 1);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x.weight[i] = 0.0f;
    if (e0 + 64 * i + lane < hi) {
      x.at[i] = (uint32_t)x.at[i] < (uint32_t)a.num_pages ? x.at[i] * kPage + slot[i] : -1;
      if (want_weights && x.at[i] >= 0)
        x.weight[i] = a.weights[((size_t)(x.at[i] >> 4) * a.num_kv_heads + g) * kPage + slot[i]];
    }
  }
}
// The places lo .. hi - 1: f(place, at, weight), lanes beyond hi too.
template <class F>
__device__ __forceinline__ void evict_walk(const EvictArgs& a, const EvictSeq& s,
                                           const EvictShared& sh, int g, int lo, int hi,
                                           bool want_weights, F f) {
  if (lo >= hi) return;
  EvictWalk w = evict_enter(s, sh, lo);
  for (int e0 = lo; e0 < hi; e0 += 512) {
    EvictBatch x;
    evict_load(a, sh, g, w, e0, hi, want_weights, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) f(e0 + 64 * i + (int)(threadIdx.x & 63), x.at[i], x.weight[i]);
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

// The keys of a wave's places lo .. hi - 1 in registers, at most N batches of 512, with
// AT also where they are in the pool (every index is known at compile time).  All page
// ids are sent for before the first weight.  N = 0: none, they are read anew.
template <int N, bool AT>
struct EvictHeld {
  const EvictArgs& a;
  const EvictSeq& s;
  const EvictShared& sh;
  int g, lo, hi;
  uint32_t x[8 * N + 1];
  int at[AT ? 8 * N : 1];

  template <class F>
  __device__ __forceinline__ void batches(F f) const {
#pragma unroll
    for (int b = 0; b < N; ++b)
      if (lo + 512 * b < hi) f(b, lo + 512 * b + (int)(threadIdx.x & 63));
  }
  // Whether a place lies in a page outside the pool.
  __device__ __forceinline__ bool load() {
    bool bad = false;
    if constexpr (N == 0) {
      evict_walk(a, s, sh, g, lo, hi, false,
                 [&](int e, int at, float wt) { bad |= e < hi && at < 0; });
      return bad;
    }
    if (lo >= hi) return false;
    uint32_t slots[N + 1];
    EvictWalk w = evict_enter(s, sh, lo);
    batches([&](int b, int e0) __attribute__((always_inline)) {
      slots[b] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = min(e0 + 64 * i, hi - 1);
        if (e >= w.end) {
          do ++w.r;
          while (e >= sh.pre[w.r + 1]);
          w.begin = sh.pre[w.r];
          w.end = sh.pre[w.r + 1];
          w.base = sh.base[w.r];
        }
        x[8 * b + i] = a.page_ids[w.base + (e - w.begin) / kPage];
        slots[b] |= (uint32_t)((e - w.begin) & (kPage - 1)) << (4 * i);
      }
    });
    batches([&](int b, int) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t id = x[8 * b + i];
        const uint32_t slot = slots[b] >> (4 * i) & (kPage - 1);
        bad |= id >= (uint32_t)a.num_pages;
        id = id < (uint32_t)a.num_pages ? id : 0;
        if constexpr (AT) at[8 * b + i] = (int)(id * kPage + slot);
        x[8 * b + i] = __builtin_bit_cast(
            uint32_t, a.weights[((size_t)id * a.num_kv_heads + g) * kPage + slot]);
      }
    });
    batches([&](int b, int) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        x[8 * b + i] = order_key(__builtin_bit_cast(float, x[8 * b + i]));
    });
    return bad;
  }
  // f(place, key), places beyond hi too.
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    if constexpr (N == 0)
      evict_walk(a, s, sh, g, lo, hi, true, [&](int e, int at, float wt) { f(e, order_key(wt)); });
    batches([&](int b, int e0) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f(e0 + 64 * i, x[8 * b + i]);
    });
  }
  // f(place, where it is, key)
  template <class F>
  __device__ __forceinline__ void each_at(F f) const {
    if constexpr (N == 0) {
      evict_walk(a, s, sh, g, lo, hi, true,
                 [&](int e, int at, float wt) { f(e, at, order_key(wt)); });
    } else if constexpr (AT) {
      batches([&](int b, int e0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f(e0 + 64 * i, at[8 * b + i], x[8 * b + i]);
      });
    } else if (lo < hi) {
      EvictWalk w = evict_enter(s, sh, lo);
      batches([&](int b, int e0) __attribute__((always_inline)) {
        EvictBatch there;
        evict_load(a, sh, g, w, lo + 512 * b, hi, false, there);
#pragma unroll
        for (int i = 0; i < 8; ++i) f(e0 + 64 * i, there.at[i], x[8 * b + i]);
      });
    }
  }
};

// Which tokens of a sequence and KV head stay, by one workgroup: a threshold by radix
// over their keys.  Each wave has a stretch of the places of its own, so that a place's
// rank is its wave's first rank and a count of ballots.
// The keys of up to 64K tokens stay in registers: 48 sequences of 2K .. 64K tokens 110 us,
// 191 with those of up to 34K in LDS and a wait for ids and weights every 512 places; 16 of
// 16K 30 and 41.  Code for each size: 700 tokens 13.9 us, 19 in the largest one's.
template <int N, bool AT>
__device__ __forceinline__ void evict_select(const EvictArgs& a, EvictSeq& s, EvictShared& sh,
                                             uint32_t* hist, int per) {
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  const int g = blockIdx.x, b = blockIdx.y;
  const int lo = min(s.L, w * per), hi = min(s.L, lo + per);
  EvictHeld<N, AT> own{a, s, sh, g, lo, hi};
  if (s.status == 0) {
    bool bad = evict_bad_target(a, s);
    bad |= own.load();
    if (__syncthreads_or(bad)) s.status = KF_EFLAG_BAD_PAGE;
  }
  if (g == 0 && tid == 0) {
    int32_t* plan = a.plan + 2 * b;
    plan[0] = s.status ? -1 : s.K;
    plan[1] = s.base;
    if (s.status > 0) atomicOr(a.err_flags, s.status);
  }
  if (s.status) return;

  int want = s.K - s.c0 - (s.L - s.c1);  // of those that compete
  EvictRule rule{s.c0, s.c1, want == 0, want == s.c1 - s.c0, 0};
  if (!rule.none && !rule.every) {
    const int from = max(lo, s.c0), till = min(hi, s.c1);
    for (int pass = 0; pass < 3; ++pass) {
      const int bins = pass_bins(pass);
      hist[tid] = hist[tid + 1024] = 0;
      __syncthreads();
      own.each([&](int e, uint32_t key) {
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
  own.each([&](int e, uint32_t key) {
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
  own.each_at([&](int e, int at, uint32_t key) __attribute__((always_inline)) {
    const bool yes = e < hi && rule.sure(e, key), eq = e < hi && rule.equal(e, key);
    const uint64_t ys = __ballot(yes), es = __ballot(eq);
    const int eq_rank = equals + __builtin_popcountll(es & lower);
    if (yes || (eq && eq_rank < want))
      list[sure + __builtin_popcountll(ys & lower) + min(eq_rank, want)] = at;
    sure += __builtin_popcountll(ys);
    equals += __builtin_popcountll(es);
  });
}

__global__ __launch_bounds__(1024) void evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t hist[kBins];
  __shared__ EvictShared sh;
  EvictSeq s = evict_sequence(a, blockIdx.y, sh);
  const int per = (s.L + 1023) / 1024 * 64;  // places of a wave
  if (per <= 512)
    evict_select<1, true>(a, s, sh, hist, per);
  else if (per <= 512 * 4)
    evict_select<4, true>(a, s, sh, hist, per);
  else if (per <= 512 * 8)
    evict_select<8, false>(a, s, sh, hist, per);
  else
    evict_select<0, false>(a, s, sh, hist, per);
}

// The same by several workgroups of a sequence and KV head, a launch for each pass:
// each has a part of the places and counts it into a row of bins of its own, and the
// launch behind adds up the rows.
struct EvictPart {
  int parts, lo, hi;  // parts that the sequence has, this one's places
};
__device__ __forceinline__ EvictPart evict_part(const EvictArgs& a, const EvictSeq& s, int p) {
  EvictPart x;
  x.parts = min(a.parts, (s.L - 1) / kPartTokens + 1);
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
  auto tally = [&](int e, float wt) __attribute__((always_inline)) {
    const uint32_t key = order_key(wt);
    mine += __builtin_popcountll(__ballot(e < hi && rule.sure(e, key)));
    alike += __builtin_popcountll(__ballot(e < hi && rule.equal(e, key)));
  };
  const bool in_regs = per <= 512;  // one batch, and its places are read once
  EvictBatch own;
  if (!in_regs) {
    evict_walk(a, s, sh, g, lo, hi, counts, [&](int e, int at, float wt) { tally(e, wt); });
  } else if (lo < hi) {
    EvictWalk walk = evict_enter(s, sh, lo);
    evict_load(a, sh, g, walk, lo, hi, counts, own);
#pragma unroll
    for (int i = 0; i < 8; ++i) tally(lo + 64 * i + lane, own.weight[i]);
  }
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
  auto enlist = [&](int e, int at, float wt) __attribute__((always_inline)) {
    const uint32_t key = order_key(wt);
    const bool yes = e < hi && rule.sure(e, key), eq = e < hi && rule.equal(e, key);
    const uint64_t ys = __ballot(yes), es = __ballot(eq);
    const int eq_rank = equals + __builtin_popcountll(es & lower);
    if (yes || (eq && eq_rank < want))
      list[sure + __builtin_popcountll(ys & lower) + min(eq_rank, want)] = at;
    sure += __builtin_popcountll(ys);
    equals += __builtin_popcountll(es);
  };
  if (!in_regs) {
    evict_walk(a, s, sh, g, lo, hi, counts, enlist);
  } else if (lo < hi) {
#pragma unroll
    for (int i = 0; i < 8; ++i) enlist(lo + 64 * i + lane, own.at[i], own.weight[i]);
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

// Dword d (uniform) of a vector.
__device__ __forceinline__ uint32_t pick(u32x4 x, int d) {
  const uint32_t y = d & 1 ? x[1] : x[0], z = d & 1 ? x[3] : x[2];
  return d & 2 ? z : y;
}

// One page of one KV head, K or V, of what stays, by a wave: n tokens, token lane % 16's
// page * 16 + slot in `mine`, into page `page`.  V's rows of sixteen slots are read
// whole: a token's own two bytes of each come with the other 30.
template <bool FP8, bool V>
__device__ __forceinline__ void evict_page(const EvictArgs& a, int g, int page, int mine, int n) {
  constexpr int esz = FP8 ? 1 : 2;
  const int lane = threadIdx.x & 63, H = a.num_kv_heads;
  char* pool = static_cast<char*>(V ? a.v_pool : a.k_pool);
  auto slice = [&](int pg) {
    return pool + slice_of(pg, g, H, a.num_pages, a.head_major) * (size_t)(kPage * kDim * esz);
  };
  char* out = slice(page);
  float was = 1.0f, now = 1.0f;
  bool same = true;
  if constexpr (FP8) {
    float* scales = V ? a.v_scale : a.k_scale;
    was = scales[(size_t)(mine >> 4) * H + g];
    const uint32_t bits = __builtin_bit_cast(uint32_t, was);
    same = __ballot(bits != (uint32_t)uniform((int)bits)) == 0;
    now = same ? was : wave_max(fabsf(was));
    if (lane == 0) scales[(size_t)page * H + g] = now;
  }
  if constexpr (!V) {
    float weight = 0.0f;
    if (lane < n) weight = a.weights[((size_t)(mine >> 4) * H + g) * kPage + (mine & 15)];
    constexpr int kLanes = FP8 ? 8 : 16, kRows = 64 / kLanes;  // lanes a row, rows a load
    u32x4 x[kPage / kRows];
#pragma unroll
    for (int i = 0; i < kPage / kRows; ++i) {
      const int from = __shfl(mine, kRows * i + lane / kLanes);
      x[i] = ld16(slice(from >> 4) + ((from & 15) * kDim * esz + 16 * (lane % kLanes)));
    }
    if (lane < n) a.weights[((size_t)page * H + g) * kPage + lane] = weight;
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
  } else {
    // 1 KiB in a row a load: bf16 eight slots, 8 (lane % 2) .., of dim 32 i + lane / 2, fp8
    // the sixteen of dim 64 i + lane.
    constexpr int kVecs = FP8 ? 2 : 4;
    u32x4 y[kVecs] = {};
    if (n < kPage) {  // slots behind the last one stay as they were
#pragma unroll
      for (int i = 0; i < kVecs; ++i) y[i] = ld16(out + 1024 * i + 16 * lane);
    }
    // Tokens come in the order of their pages.  bf16: a page is read once for all of its
    // own, two tokens at a time (48 agentic requests moved in 528 us, 537 with four, 547
    // with one, 640 anew for every token); fp8, whose pages are half as large, anew for
    // every token, four at a time (16 sequences 16K -> 3000 tokens 87 us, 101 .. 122 the
    // other way).
    constexpr int kTogether = FP8 ? 4 : 2;
    auto fresh = [&](int s) {
      return FP8 || s == 0 || (__builtin_amdgcn_readlane(mine, s) ^
                               __builtin_amdgcn_readlane(mine, s - 1)) >> 4 != 0;
    };
    u32x4 last[kVecs] = {};  // the page of the token before
#pragma unroll
    for (int s0 = 0; s0 < kPage; s0 += kTogether) {
      u32x4 x[kTogether][kVecs];
#pragma unroll
      for (int s = 0; s < kTogether; ++s) {
        if (s0 + s < n && fresh(s0 + s)) {
          const char* from = slice(__builtin_amdgcn_readlane(mine, s0 + s) >> 4) + 16 * lane;
#pragma unroll
          for (int i = 0; i < kVecs; ++i) x[s][i] = ld16(from + 1024 * i);
        }
      }
#pragma unroll
      for (int s = 0; s < kTogether; ++s) {
        if (s0 + s >= n) break;
        const int slot = __builtin_amdgcn_readlane(mine, s0 + s) & 15, to = s0 + s;
        if (fresh(to)) {
#pragma unroll
          for (int i = 0; i < kVecs; ++i) last[i] = x[s][i];
        }
        if constexpr (FP8) {
          uint32_t two = 0;
#pragma unroll
          for (int i = 0; i < 2; ++i)
            two |= (pick(last[i], slot >> 2) >> (8 * (slot & 3)) & 0xFFu) << (8 * i);
          const float sc = __shfl(was, to);
          if (!same && sc != now) two = recode4(two, sc, now);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t z = y[i][to >> 2] & ~(0xFFu << (8 * (to & 3)));
            y[i][to >> 2] = z | (two >> (8 * i) & 0xFFu) << (8 * (to & 3));
          }
        } else {
          const bool turn = (slot ^ to) & 8;  // the slot is in the neighbour's half
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t v = pick(last[i], (slot & 7) >> 1) >> (16 * (slot & 1)) & 0xFFFFu;
            if (turn) v = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);
            const int dw = (to & 7) >> 1;
            const uint32_t z =
                (y[i][dw] & ~(0xFFFFu << (16 * (to & 1)))) | v << (16 * (to & 1));
            y[i][dw] = (lane & 1) == to >> 3 ? z : y[i][dw];
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) *reinterpret_cast<u32x4*>(out + 1024 * i + 16 * lane) = y[i];
  }
}

// What stays of every sequence into its new pages, K and V of a page by waves beside each
// other.  Bound by memory: whole sequences (48 of 4096 tokens) move at 4.6 TB/s, a copy's
// rate, and where a part of a page stays its V is read all the same: 48 sequences of 2K ..
// 64K tokens to 4096, 1.6 GB, 528 us, 5.5 TB/s of the 2.9 GB that takes.  (Several pages a
// wave, the next one's list on its way: the same.)
template <bool FP8>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int H = a.num_kv_heads, b = blockIdx.y;
  const int kept = fixed(a.plan)[2 * b];
  if (kept < 0) return;
  if (blockIdx.x == 0) {  // the routes: all others are empty now
    const int into = a.into[b], r1 = a.seq_route_begin[b + 1];
    for (int r = a.seq_route_begin[b] + threadIdx.x; r < r1; r += 256)
      a.routes[r].tok_end = a.routes[r].tok_begin + (r == into ? kept : 0);
  }
  const uint32_t item = blockIdx.x * 4 + wave;
  const int g = (int)((item >> 1) % (uint32_t)H), p = (int)((item >> 1) / (uint32_t)H);
  const int n = min(kPage, kept - p * kPage);  // (max_keep bounds p)
  if (n <= 0) return;
  const int page = fixed(a.page_ids)[fixed(a.plan)[2 * b + 1] + p];
  const int32_t* list = a.list + ((size_t)b * H + g) * a.max_keep + p * kPage;
  const int mine = list[min(lane & 15, n - 1)];
  if (item & 1)
    evict_page<FP8, true>(a, g, page, mine, n);
  else
    evict_page<FP8, false>(a, g, page, mine, n);
}

}  // namespace

hipError_t launch_attn_weights(const AttnWeightsArgs& a, bool fp8, hipStream_t stream) {
  const dim3 grid((uint32_t)a.chunks * a.num_kv_heads, a.num_routes, a.segments);
  if (fp8)
    attn_weights_kernel<true><<<grid, 256, 0, stream>>>(a);
  else
    attn_weights_kernel<false><<<grid, 256, 0, stream>>>(a);
  const hipError_t st = hipGetLastError();
  if (st != hipSuccess || a.segments == 1) return st;
  attn_weights_join_kernel<<<dim3(grid.x, grid.y), 256, 0, stream>>>(a);
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
