// Host check of the row operators' C-ABI layer (kf_rows_api.cpp built against the
// HIP test double): over random shapes on devices of 1 to 1024 compute units, a
// workspace of the queried size is accepted and every region of it lies inside
// and apart from the others; the row tiles of any table of rows fit the bound;
// unplanned launches stay within their records and their grid; arbitrary
// arguments give a known status.
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <random>
#include <vector>

#include "kf.h"
#include "kf_rows.h"

static int g_cus = 256;
hipError_t hipGetDevice(int* d) { *d = 0; return hipErrorNoDevice; }  // asked anew every time
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = g_cus; return hipSuccess; }

static std::mt19937_64 rng(11);
static int64_t rnd(int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); }
static bool coin() { return rnd(0, 1); }

static unsigned char* g_ws;
static size_t g_bytes;
static int g_launches, g_errors;
#define CHECK(c)                                             \
  do {                                                       \
    if (!(c) && ++g_errors < 20) printf("line %d: %s\n", __LINE__, #c); \
  } while (0)

static void touch(const void* p, size_t n) {
  unsigned char* c = (unsigned char*)p;
  if (n == 0) return;
  CHECK(c >= g_ws && c + n <= g_ws + g_bytes);
  c[0] = c[n - 1] = 0x5a;
}

namespace kf {
hipError_t launch_append(const AppendArgs&, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_partial(const PartialArgs&, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_merge(const MergeArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_gather(const PartialArgs&, bool, int, int, void*, void*, hipStream_t) { return hipSuccess; }
hipError_t scratch_address(void** out) { *out = nullptr; return hipSuccess; }

hipError_t launch_append_rows(const AppendRowsArgs& a, bool fp8, hipStream_t) {
  ++g_launches;
  CHECK(a.num_entries > 0 && a.num_routes > 0 && a.row_stride % 8 == 0);
  CHECK(!fp8 || (a.k_scale && a.v_scale));
  touch(a.plan, (size_t)a.num_routes * 16);
  const int64_t tiles = (int64_t)a.num_entries / kPage + 2 * (int64_t)a.num_routes;
  // threads of a grid fit 32 bits
  CHECK((tiles * 2 * a.num_kv_heads + 3) / 4 * 256 <= UINT32_MAX);
  CHECK((int64_t)a.num_routes * 1024 <= UINT32_MAX);
  return hipSuccess;
}

hipError_t launch_rows_attn(const RowsArgs& a, bool fp8, bool tree, hipStream_t) {
  ++g_launches;
  CHECK(!fp8 || (a.k_scale && a.v_scale));
  CHECK(tree ? a.k_draft && a.v_draft && a.tree_mask : a.first_pos != nullptr);
  CHECK(a.parts >= 0 && (a.parts == 0 || a.num_seqs <= 64));
  CHECK(a.parts <= 1 || (int64_t)a.parts * a.max_tiles <= a.max_recs);
  const int64_t items = a.parts > 0 ? (int64_t)a.max_tiles * a.parts : (int64_t)a.max_tiles + a.max_recs;
  CHECK(items > 0 && items * a.num_kv_heads * 256 <= UINT32_MAX);
  if (a.may_split) CHECK(a.max_tiles > 0 && a.max_recs > 1);  // the combine's grid
  CHECK(a.rec_rows >= 1 && a.rec_rows <= kRowTile && a.rec_rows % 32 == 0);
  const size_t rec = (size_t)a.max_recs * a.num_kv_heads * a.rec_rows;
  struct { const void* p; size_t n; } part[] = {
      {a.head, 8}, {a.seq_tiles, ((size_t)a.num_seqs + 1) * 4}, {a.seq_info, (size_t)a.num_seqs * 16},
      {a.items, ((size_t)a.max_tiles + a.max_recs) * sizeof(RowsItem)},
      {a.splits, (size_t)(a.max_recs / 2) * sizeof(RowsSplit)}, {a.rec_ml, rec * 8}, {a.rec_o, rec * 512}};
  for (auto& x : part) touch(x.p, x.n);
  for (int i = 0; i + 1 < 7; ++i)
    CHECK((const char*)part[i].p + part[i].n <= (const char*)part[i + 1].p);
  CHECK((uintptr_t)a.items % 16 == 0 && (uintptr_t)a.rec_ml % 8 == 0 && (uintptr_t)a.rec_o % 16 == 0);
  return hipSuccess;
}
}  // namespace kf

static void* const P = (void*)0x10000;

int main() {
  for (int it = 0; it < 3000; ++it) {
    g_cus = (int)rnd(1, 1024);
    kf_shape s{};
    const int G = (int)rnd(1, 16);
    s.num_kv_heads = (int)(coin() ? rnd(1, 16) : rnd(1, 3000));
    s.num_q_heads = s.num_kv_heads * G;
    s.num_seqs = (int)(coin() ? rnd(0, 80) : rnd(0, 5000));
    s.head_dim = 128;
    s.page_size = 16;
    s.kv_dtype = (int)rnd(0, 1);
    s.num_pages = (int)rnd(1, 1 << 20);
    s.num_page_ids = (int)rnd(0, 1 << 20);
    s.scale = 0.1f;
    s.kv_layout = (int)rnd(0, 1);
    const int rows = (int)(coin() ? rnd(0, 300) : rnd(0, 200000));
    const size_t need = kf_rows_attn_workspace_bytes(&s, rows);
    if (need == 0 || need > (size_t)3 << 30) continue;
    // any table of rows has at most max_tiles row tiles
    const kf::RowsLayout l = kf::rows_layout(rows, s.num_seqs, s.num_kv_heads, G, 256);
    std::vector<int> cut(s.num_seqs + 1);
    for (int& c : cut) c = (int)rnd(0, rows);
    std::sort(cut.begin(), cut.end());
    int64_t tiles = 0;
    for (int b = 0; b < s.num_seqs; ++b)
      tiles += ((int64_t)(cut[b + 1] - cut[b]) * G + kf::kRowTile - 1) / kf::kRowTile;
    CHECK(tiles <= l.max_tiles);
    g_bytes = need;
    g_ws = (unsigned char*)aligned_alloc(256, (need + 255) / 256 * 256);  // touched at the ends only
    const bool tree = coin();
    const int before = g_launches, routes = (int)rnd(0, 5000);
    const int64_t qs = (int64_t)s.num_q_heads * 128 + 8 * rnd(0, 9), ks = (int64_t)s.num_kv_heads * 128;
    void* sc = s.kv_dtype ? P : nullptr;
    auto call = [&](size_t bytes) {
      return tree ? kf_tree_attn(&s, P, rows, qs, P, P, ks, (uint64_t*)P, (int*)P, P, P, (float*)sc,
                                 (float*)sc, (kf_route*)P, routes, 100, (int*)P, (int*)P, P, (float*)P,
                                 g_ws, bytes, (int*)P, nullptr)
                  : kf_prompt_attn(&s, P, rows, qs, (int*)P, (int*)P, P, P, (float*)sc, (float*)sc,
                                   (kf_route*)P, routes, 100, (int*)P, (int*)P, P, (float*)P, g_ws,
                                   bytes, (int*)P, nullptr);
    };
    CHECK(call(need) == KF_OK);
    CHECK(g_launches == before + (rows > 0));
    if (rows > 0) CHECK(call(need - 1) == KF_ERR_WORKSPACE && g_launches == before + 1);
    free(g_ws);
    // appends
    const int nr = (int)rnd(0, 4000), entries = (int)rnd(0, 100000);
    g_bytes = kf_kv_append_rows_workspace_bytes(nr);
    g_ws = (unsigned char*)aligned_alloc(256, (g_bytes + 255) / 256 * 256);
    const int b2 = g_launches;
    const int st = kf_kv_append_rows(&s, P, P, (float*)sc, (float*)sc, P, P, entries, ks, nullptr,
                                     entries, (int*)P, (kf_route*)P, nr, (int*)P, g_ws, g_bytes,
                                     (int*)P, nullptr);
    const bool large = ((int64_t)entries / 16 + 2 * nr) * 2 * s.num_kv_heads > 4 * kf::kMaxWgs;
    CHECK(st == (large && nr > 0 && entries > 0 ? KF_ERR_UNSUPPORTED : KF_OK));
    CHECK(g_launches == b2 + (nr > 0 && entries > 0 && !large));
    free(g_ws);
  }
  // arbitrary arguments: a known status
  g_bytes = 0;
  for (int it = 0; it < 200000; ++it) {
    kf_shape s;
    int* f = (int*)&s;
    for (size_t i = 0; i < sizeof s / 4; ++i) f[i] = (int)(coin() ? rnd(-2, 20) : rnd(INT32_MIN, INT32_MAX));
    if (coin()) s.head_dim = 128, s.page_size = 16, s.kv_dtype = 0, s.kv_layout = 0, s.scale = 1.0f;
    auto n = [] { return (int)(coin() ? rnd(-2, 50) : rnd(INT32_MIN, INT32_MAX)); };
    auto p = [] { return coin() ? P : coin() ? nullptr : (void*)(uintptr_t)rnd(1, 1 << 20); };
    const int st = kf_prompt_attn(&s, p(), n(), n(), (int*)p(), (int*)p(), p(), p(), (float*)p(),
                                  (float*)p(), (kf_route*)p(), n(), n(), (int*)p(), (int*)p(), p(),
                                  (float*)p(), nullptr, 0, (int*)p(), nullptr);
    CHECK(st <= 0 && st >= -3);
    const int st2 = kf_kv_append_rows(&s, p(), p(), (float*)p(), (float*)p(), p(), p(), n(), n(),
                                      (int*)p(), n(), (int*)p(), (kf_route*)p(), n(), (int*)p(), nullptr,
                                      0, (int*)p(), nullptr);
    CHECK(st2 <= 0 && st2 >= -3);
    (void)kf_rows_attn_workspace_bytes(&s, n());
    (void)kf_kv_append_rows_workspace_bytes(n());
  }
  if (g_errors) return 1;
  printf("rows_stress ok\n");
  return 0;
}
