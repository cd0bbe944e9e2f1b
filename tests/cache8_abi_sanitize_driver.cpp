// Host-side driver of the 8-bit paged cache's entry points for the sanitizer build (tests/test_cache8_abi_sanitized.py):
// sizes that would overflow careless arithmetic, refusals, and, only when the HIP runtime sees no device,
// well-formed calls of many shapes, whose plans and offset tables all run before the launch fails.  Fake device
// pointers are never dereferenced by correct host code.  Exit status 0 when every check holds.
#include <hip/hip_runtime_api.h>

#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <random>
#include <vector>

#include "taskpress.h"

namespace {

int failures = 0, checks = 0;

void expect(tp_status got, tp_status want, const char* what, int line) {
  ++checks;
  if (got != want || (want != TP_OK && std::strlen(tp_last_error()) == 0)) {
    std::fprintf(stderr, "line %d: %s returned %d, expected %d (%s)\n", line, what, got, want, tp_last_error());
    ++failures;
  }
}
#define EXPECT(call, want) expect((call), (want), #call, __LINE__)

char* fake() { return reinterpret_cast<char*>(0x10000); }

tp_cache8 cache_of(int32_t batch, int32_t page_tokens = 64, int32_t max_pages = 16, int64_t num_pages = 100, int32_t qfmt = 0) {
  return tp_cache8{{fake(), (const int32_t*)fake(), (const int32_t*)fake(), num_pages, page_tokens, max_pages, batch}, qfmt};
}

}  // namespace

int main() {
  int devices = 0;
  const bool have_device = hipGetDeviceCount(&devices) == hipSuccess && devices > 0;
  const tp_dims d = {2, 8, 2, 128};
  size_t n = 0;

  // sizes at the ends of their types
  for (int32_t total : {1, 64, INT32_MAX})
    for (int32_t most : {1, 5, 1000, INT32_MAX})
      for (int64_t len : {(int64_t)1, (int64_t)512, (int64_t)1 << 20, (int64_t)1 << 30, INT64_MAX}) {
        const tp_cache8 c = cache_of(65535, 256, 1 << 22, INT32_MAX);
        const tp_step s = {(const int32_t*)fake(), total, most};
        const tp_status r = tp_cache8_workspace_size(&d, &c, &s, len, &n);
        expect(r == TP_OK || r == TP_ERR_UNSUPPORTED || r == TP_ERR_SHAPE ? TP_OK : r, TP_OK, "size", __LINE__);
      }
  for (int32_t x : {INT32_MIN, -1, 0, 7, INT32_MAX}) {
    const tp_step s = {(const int32_t*)fake(), 64, 1};
    for (int field = 0; field < 4; ++field) {
      tp_cache8 c = cache_of(64);
      (field == 0 ? c.cache.page_tokens : field == 1 ? c.cache.max_pages : field == 2 ? c.cache.batch : c.qfmt) = x;
      (void)tp_cache8_workspace_size(&d, &c, &s, 64, &n);
    }
    for (int field = 0; field < 4; ++field) {
      tp_dims e = d;
      (field == 0 ? e.num_layers : field == 1 ? e.num_q_heads : field == 2 ? e.num_kv_heads : e.head_dim) = x;
      const tp_cache8 c = cache_of(64);
      (void)tp_cache8_workspace_size(&e, &c, &s, 64, &n);
      (void)tp_cache8_page_bytes(&e, 64);
    }
    (void)tp_cache8_page_bytes(&d, x);
  }
  // strides whose extents would overflow
  const tp_cache8 c3 = cache_of(3);
  const tp_step s3 = {(const int32_t*)fake(), 7, 4};
  for (int64_t x : {INT64_MIN, (int64_t)-8, (int64_t)0, (int64_t)8, (int64_t)1 << 60, INT64_MAX, INT64_MAX - 7}) {
    for (int field = 0; field < 3; ++field) {
      tp_rows r = {fake(), 7 * 1024, 1024, 128};
      (field == 0 ? r.layer_stride : field == 1 ? r.token_stride : r.head_stride) = x;
      EXPECT(tp_cache8_attention(&d, &c3, &s3, &r, -1.0f, 64, &r, nullptr, nullptr, 0, nullptr) == TP_OK ? TP_OK : TP_ERR_HIP,
             TP_ERR_HIP);  // refused for one reason or another
      (void)tp_cache8_append(&d, &c3, &s3, &r, &r, nullptr, nullptr, &r, &r, nullptr);
    }
  }
  // offsets
  const std::vector<std::vector<int64_t>> offsets = {
      {0, INT64_MAX, INT64_MAX, INT64_MAX}, {0, 5, INT64_MIN, 7}, {INT64_MIN, 0, 1, 2}, {0, 1, 2, (int64_t)1 << 62}};
  for (const auto& off : offsets) {
    const tp_batch b = {3, off.data(), nullptr};
    EXPECT(tp_cache8_load(&d, &c3, off.data(), fake(), fake(), (float*)fake(), 4, nullptr), TP_ERR_SHAPE);
    EXPECT(tp_cache8_read(&d, &c3, &b, nullptr, fake(), fake(), nullptr), TP_ERR_SHAPE);
  }
  const int64_t none[4] = {0, 0, 0, 0}, some[4] = {0, 5, 5, 40};
  const tp_batch some_b = {3, some, nullptr};
  for (int64_t f : {INT64_MIN, (int64_t)-1, ((int64_t)1 << 30) + 1, INT64_MAX}) {
    const int64_t first[3] = {0, 0, f};
    EXPECT(tp_cache8_read(&d, &c3, &some_b, first, fake(), fake(), nullptr), TP_ERR_SHAPE);
  }
  EXPECT(tp_cache8_load(&d, &c3, none, fake(), fake(), (float*)fake(), 4, nullptr), TP_OK);
  std::vector<int64_t> many(66, 0);
  const tp_cache8 c65 = cache_of(65);
  EXPECT(tp_cache8_load(&d, &c65, many.data(), fake(), fake(), (float*)fake(), 4, nullptr), TP_ERR_UNSUPPORTED);

  if (!have_device) {
    std::mt19937 rng(7);
    const auto pick = [&](int lo, int hi) { return (int)(lo + rng() % (uint32_t)(hi - lo + 1)); };
    for (int i = 0; i < 3000; ++i) {
      const int hkv = pick(1, 9), L = pick(1, 4);
      const tp_dims e = {L, hkv * pick(1, 17), hkv, pick(0, 1) ? 64 : 128};
      const int batch = pick(1, 64), most = pick(0, 2) ? pick(1, 9) : pick(1, 900);
      const tp_cache8 c = cache_of(batch, 32 << pick(0, 3), pick(1, 2000), 100, pick(0, 1));
      const bool single = most == 1 && pick(0, 1);
      const tp_step s = {single ? nullptr : (const int32_t*)fake(), batch * most, most};
      const int64_t kv = (int64_t)e.num_kv_heads * e.head_dim, q = (int64_t)e.num_q_heads * e.head_dim;
      const tp_rows rk = {fake(), kv * s.total, kv, e.head_dim}, rq = {fake(), q * s.total, q, e.head_dim};
      const int64_t len = pick(1, c.cache.max_pages * c.cache.page_tokens);
      EXPECT(tp_cache8_workspace_size(&e, &c, &s, len, &n), TP_OK);
      EXPECT(tp_cache8_attention(&e, &c, &s, &rq, 0.1f, len, &rq, (float*)fake(), fake(), n, nullptr), TP_ERR_HIP);
      if (n > 0) EXPECT(tp_cache8_attention(&e, &c, &s, &rq, 0.1f, len, &rq, nullptr, fake(), n - 1, nullptr), TP_ERR_WORKSPACE);
      const tp_rope rope = {(const float*)fake(), pick(1, 1 << 20), 16 * pick(1, e.head_dim / 16), pick(0, 1)};
      EXPECT(tp_cache8_append(&e, &c, &s, &rk, &rk, (const int32_t*)fake(), &rope, &rq, &rq, nullptr), TP_ERR_HIP);
      EXPECT(tp_cache8_append(&e, &c, &s, &rk, &rk, nullptr, nullptr, nullptr, nullptr, nullptr), TP_ERR_HIP);
      std::vector<int64_t> off(batch + 1, 0), first(batch);
      for (int b = 0; b < batch; ++b) {
        off[b + 1] = off[b] + pick(b == 0 ? 1 : 0, std::min(500, c.cache.max_pages * c.cache.page_tokens));
        first[b] = pick(0, 1000);
      }
      const tp_batch bt = {batch, off.data(), nullptr};
      EXPECT(tp_cache8_load(&e, &c, off.data(), fake(), fake(), (float*)fake(), pick(2, 8), nullptr), TP_ERR_HIP);
      EXPECT(tp_cache8_read(&e, &c, &bt, pick(0, 1) ? first.data() : nullptr, fake(), fake(), nullptr), TP_ERR_HIP);
    }
  }
  std::printf("%d checks, %d failures\n", checks, failures);
  return failures == 0 ? 0 : 1;
}
