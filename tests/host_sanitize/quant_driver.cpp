// The argument checks and launch plans of the operators of quantised inference on the host, over random arguments
// with bad ones among them: what reaches a launcher fits what the kernels assume, what does not says why, and nothing
// is launched for an empty or a refused call.  Launchers are stand-ins that check and count.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <random>

#include "awe_quant.h"

namespace {
int g_launches = 0, g_failures = 0;
void expect(bool ok, const char* what) {
  if (!ok) {
    ++g_failures;
    std::printf("failed: %s\n", what);
  }
}
}  // namespace

namespace awe {
awe_status launch_w4(const W4Launch& g, hipStream_t) {
  ++g_launches;
  expect(g.M > 0 && g.N > 0 && g.K >= 0 && g.y != nullptr && g.ldy >= g.N, "w4 sizes");
  if (g.K > 0) {
    const int64_t groups = (g.K + g.group - 1) / g.group, e = g.x_type == AWE_I8 ? 1 : 2, se = g.s_type == AWE_F32 ? 4 : 2;
    expect(g.group % 32 == 0 || g.group >= g.K, "w4 group");
    expect(g.ldx >= g.K && g.ldw >= (g.K + 1) / 2 && g.lds >= groups && (!g.zeros || g.ldz >= groups), "w4 rows");
    // a tile's rows are reached by 32 bits: 64 of X and of a wave's W, 256 scales and zero points
    expect(64 * g.ldx * e < (int64_t(1) << 31) && 64 * g.ldw < (int64_t(1) << 31) && 255 * g.lds * se < (int64_t(1) << 32) &&
               (!g.zeros || 255 * g.ldz < (int64_t(1) << 32)),
           "w4 offsets");
  }
  return AWE_OK;
}
static void expect_batch(const awe_cache& c, const awe_batch& b) {
  expect(b.sequences > 0 && b.rows > 0 && b.max_rows > 0 && b.ld_blocks * c.block >= b.max_length, "batch");
  expect((std::min(b.rows, b.max_rows) / c.block + 2) * 256 < (int64_t(1) << 32), "grid");
}
awe_status launch_cache_store(const CacheLaunch& g, hipStream_t) {
  ++g_launches;
  expect_batch(g.c, g.b);
  return AWE_OK;
}
awe_status launch_cache_load(const CacheLaunch& g, hipStream_t) {
  ++g_launches;
  expect_batch(g.c, g.b);
  for (const Rows* r : {&g.k, &g.v})
    expect(g.c.heads == 1 || r->head >= g.c.head_dim || g.c.head_dim == 0, "distinct heads");
  return AWE_OK;
}
awe_status launch_cache_attend(const AttendLaunch& g, hipStream_t) {
  ++g_launches;
  expect_batch(g.c, g.b);
  const AttendPlan p = plan_attend(g.c, g.b, g.q_heads);
  const int64_t cols = std::min(g.b.rows, g.b.max_rows) * (g.q_heads / g.c.heads);
  if (p.own_columns) {
    expect((int64_t)p.groups * kRowsColumns >= cols && p.splits == 1 && p.workspace == 0, "plan of many columns");
  } else {
    expect((int64_t)p.groups * 16 >= cols && p.chunk > 0 && p.chunk % 256 == 0, "plan of few columns");
    expect((int64_t)p.splits * p.chunk >= g.b.max_length, "splits cover the tokens");
    const size_t need = p.splits == 1 ? 0 : (size_t)g.b.sequences * g.c.heads * cols * p.splits * (g.c.head_dim + 4) * 4;
    expect(p.workspace == need && (need == 0 || g.ws != nullptr), "workspace holds every part");
    expect((int64_t)p.groups * p.splits * 256 < (int64_t(1) << 32), "grid of few columns");
  }
  return AWE_OK;
}
}  // namespace awe

int main() {
  std::mt19937_64 rng(7);
  auto pick = [&](std::initializer_list<int64_t> v) { return *(v.begin() + rng() % v.size()); };
  void* p = reinterpret_cast<void*>(uintptr_t(1) << 40);
  void* odd = reinterpret_cast<void*>((uintptr_t(1) << 40) + 1);
  auto ptr = [&] { return rng() % 40 == 0 ? (rng() % 2 ? nullptr : odd) : p; };
  int calls = 0, ok = 0;
  for (int i = 0; i < 200000; ++i, ++calls) {
    const int before = g_launches;
    awe_status st;
    const awe_dtype t = (awe_dtype)pick({3, 4, 5, 4, 5, 2, 0, 1});
    if (i % 2) {
      const int64_t M = pick({-1, 0, 1, 33, 5000, 1 << 20, int64_t(1) << 33}), N = pick({0, 1, 77, 8192, -3, int64_t(1) << 31}),
                    K = pick({0, 1, 31, 4097, 1 << 22, 1 << 25, -9});
      const int64_t group = pick({32, 64, 128, 96, 48, 0, -32, 1 << 26, K}), groups = group > 0 ? (K + group - 1) / group : 1;
      st = awe_gemm_w4(M, N, K, ptr(), K + pick({0, 0, 5, -1}), (awe_dtype)pick({4, 5, 2, 2, 3}), (const float*)(rng() % 3 ? nullptr : p),
                       (const uint8_t*)p, (K + 1) / 2 + pick({0, 0, 7, -1, 1 << 25}), ptr(), groups + pick({0, 0, 1, -1}), t,
                       (const uint8_t*)(rng() % 2 ? nullptr : p), groups + pick({0, 2, -1}), group, ptr(), N + pick({0, 0, 3, -1}),
                       (awe_dtype)pick({3, 4, 5, 1}), nullptr);
    } else {
      awe_cache c{(int8_t*)ptr(), (int8_t*)ptr(), (float*)ptr(), (float*)ptr(), pick({0, 1, 100, -1, int64_t(1) << 32}),
                  (int32_t)pick({1, 2, 8, 8, 0, 70000}), (int32_t)pick({64, 128, 256, 128, 96}), (int32_t)pick({16, 32, 64, 128, 64, 20})};
      const int64_t length = pick({0, 1, 100, 65536, 1 << 20, 0x7fffff00, -1});
      awe_batch b{(int32_t)pick({0, 1, 7, 64, 100000, -1}), (int32_t*)ptr(), (int32_t*)ptr(), (int32_t*)ptr(), length / 16 + pick({0, 1, 1, -1}),
                  pick({0, 1, 64, 5000, 1 << 20, -1, 1 << 28}), pick({1, 1, 64, 5000, 1 << 20, 0, 1 << 28}), length};
      const int64_t head = pick({128, 256, 64, 0, -1}), row = pick({4096, 2048, 128, 1 << 20, 0, int64_t(1) << 41});
      int32_t* flag = (int32_t*)(rng() % 3 ? nullptr : ptr());
      if (i % 3 == 0) {
        st = awe_cache_store(rng() % 50 ? &c : nullptr, rng() % 50 ? &b : nullptr, ptr(), row, head, ptr(), row, head, t, flag, nullptr);
      } else if (i % 3 == 1) {
        st = awe_cache_load(&c, &b, ptr(), row, head, ptr(), row, head, t, flag, nullptr);
      } else {
        const int32_t heads = (int32_t)pick({1, 2, 8, 64, 40, 0, 70000});
        size_t n = 0;
        const awe_status q = awe_cache_attend_workspace_bytes(&c, &b, heads, &n);
        const size_t given = rng() % 4 ? n : n / 2;
        st = awe_cache_attend(&c, &b, ptr(), row, head, heads, t, 0.1f, (int32_t)(rng() % 2), ptr(), row, head, rng() % 9 ? p : nullptr,
                              given, flag, nullptr);
        expect(st != AWE_OK || q == AWE_OK, "workspace of an accepted call");
        expect(!(st == AWE_OK && g_launches > before && given < n), "small workspace");
      }
    }
    expect(st == AWE_OK || g_launches == before, "refused and launched");
    expect(st == AWE_OK || std::strlen(awe_last_error()) > 0, "refused without a word");
    ok += g_launches > before;
  }
  std::printf("calls %d launched %d failures %d\n", calls, ok, g_failures);
  return g_failures ? 1 : 0;
}
