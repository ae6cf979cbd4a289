// Host check of the C-ABI layer of the operators of a budget (kf_budget_api.cpp built
// against the HIP test double): over random shapes on devices of 1 to 1024 compute
// units, a workspace of the queried size is accepted and every region of it lies
// inside, aligned, and apart from the others; grids fit; arbitrary arguments give a
// known status.
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <random>

#include "kf.h"
#include "kf_budget.h"

static int g_cus = 256;
hipError_t hipGetDevice(int* d) { *d = 0; return hipErrorNoDevice; }  // asked anew every time
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = g_cus; return hipSuccess; }

static std::mt19937_64 rng(7);
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

hipError_t launch_attn_weights(const AttnWeightsArgs& a, bool fp8, hipStream_t) {
  ++g_launches;
  CHECK(!fp8 || a.k_scale);
  CHECK(a.chunk_pages >= 16 && a.chunks >= 1);
  // every page of a route has a workgroup, and a join's thread per token
  CHECK((int64_t)a.chunks * a.chunk_pages >= std::min(a.max_pages_per_route, a.num_page_ids));
  CHECK(a.segments >= 1 && a.segments <= kMaxSegments);
  CHECK(a.segments == 1 || a.chunk_pages == 16);
  const int64_t wgs = (int64_t)a.chunks * a.num_kv_heads * a.num_routes;
  CHECK(wgs <= kMaxBudgetWgs && a.num_routes <= 65535);
  if (a.segments > 1) touch(a.sums, (size_t)wgs * a.segments * 1024);
  return hipSuccess;
}
hipError_t launch_evict(const EvictArgs& a, bool fp8, hipStream_t) {
  ++g_launches;
  CHECK(!fp8 || (a.k_scale && a.v_scale));
  const size_t units = (size_t)a.num_seqs * a.num_kv_heads, parts = a.parts > 1 ? units * a.parts : 0;
  CHECK(a.parts >= 1 && a.parts <= kMaxParts && parts <= kMostParts);
  struct { const void* p; size_t n; } part[] = {{a.plan, (size_t)a.num_seqs * 8},
                                                {a.list, units * a.max_keep * 4},
                                                {a.state, parts * 16}, {a.rows, parts * 3 * 8192}};
  for (auto& x : part) touch(x.p, x.n);
  for (int i = 0; i + 1 < 4; ++i)
    CHECK((const char*)part[i].p + part[i].n <= (const char*)part[i + 1].p);
  CHECK((uintptr_t)a.rows % 8 == 0);
  CHECK(a.num_seqs <= 65535 && (int64_t)units * a.parts * 1024 <= UINT32_MAX);
  CHECK(((int64_t)a.max_keep / 16 + 1) * 2 * a.num_kv_heads / 4 * 256 <= UINT32_MAX);
  return hipSuccess;
}
}  // namespace kf

static void* const P = (void*)0x10000;

int main() {
  for (int it = 0; it < 4000; ++it) {
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
    const int rows = (int)(coin() ? rnd(0, 300) : rnd(0, 200000));
    const int routes = (int)(coin() ? rnd(0, 300) : rnd(0, 65535)), maxp = (int)rnd(0, 1 << (int)rnd(1, 20));
    const size_t need = kf_attn_weights_workspace_bytes(&s, rows, routes, maxp);
    if (need > 0) {
      g_bytes = need;
      g_ws = (unsigned char*)aligned_alloc(256, (need + 255) / 256 * 256);
      const int st = kf_attn_weights(&s, P, rows, s.num_q_heads * 128, (float*)P, (int32_t*)P, (int32_t*)P,
                                     P, (float*)P, (kf_route*)P, routes, maxp, (int32_t*)P, 0.5f,
                                     (float*)P, g_ws, need, (int32_t*)P, nullptr);
      CHECK(st == KF_OK);
      free(g_ws);
    }
    const int keep = (int)(coin() ? rnd(0, 300) : rnd(0, 1 << 17));
    const size_t en = kf_kv_evict_workspace_bytes(&s, keep);
    if (en > 0 && en < (size_t)2 << 30) {
      g_bytes = en;
      g_ws = (unsigned char*)aligned_alloc(256, (en + 255) / 256 * 256);
      const int st = kf_kv_evict(&s, P, P, (float*)P, (float*)P, (float*)P, (kf_route*)P, routes, maxp,
                                 (int32_t*)P, (int32_t*)P, (int32_t*)P, (int32_t*)P, keep, (int)rnd(0, 9),
                                 (int)rnd(0, 9), g_ws, en, (int32_t*)P, nullptr);
      CHECK(st == KF_OK || st == KF_ERR_UNSUPPORTED);
      free(g_ws);
    }
    // arbitrary arguments, none of them launched
    kf_shape t = s;
    if (coin()) t.num_seqs = (int)rnd(INT32_MIN, INT32_MAX);
    if (coin()) t.num_kv_heads = (int)rnd(INT32_MIN, INT32_MAX);
    if (coin()) t.num_q_heads = (int)rnd(INT32_MIN, INT32_MAX);
    const int before = g_launches;
    auto any = [] { return (int)rnd(INT32_MIN, INT32_MAX); };
    kf_attn_weights_workspace_bytes(&t, any(), any(), any());
    kf_kv_evict_workspace_bytes(&t, any());
    const int a = kf_attn_weights(&t, P, any(), rnd(-9, 1 << 20), (float*)P, (int32_t*)P, (int32_t*)P, P,
                                  (float*)P, (kf_route*)P, any(), any(), (int32_t*)P, 1.0f, (float*)P,
                                  nullptr, 0, nullptr, nullptr);
    const int b = kf_kv_evict(&t, P, P, (float*)P, (float*)P, (float*)P, (kf_route*)P, any(), any(),
                              (int32_t*)P, (int32_t*)P, (int32_t*)P, (int32_t*)P, any(), any(), any(),
                              nullptr, 0, nullptr, nullptr);
    CHECK(a <= KF_OK && a >= KF_ERR_SCRATCH_LIMIT && b <= KF_OK && b >= KF_ERR_SCRATCH_LIMIT);
    CHECK(g_launches == before);
  }
  if (g_errors || g_launches < 1000) return printf("%d errors, %d launches\n", g_errors, g_launches), 1;
  printf("budget_stress ok (%d launches)\n", g_launches);
  return 0;
}
