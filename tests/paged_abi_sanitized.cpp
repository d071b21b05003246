// Host-side exercise of the paged cache's C ABI for a build with the address and undefined-behaviour sanitizers on the host code
// (tests/test_paged_host_sanitized.py compiles and runs it): configurations up to their limits, sizes, refusals.  No call here
// reaches a launch.  Exit code 0 = all expectations held.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <limits>

#include "rf2.h"

static int failures = 0;
#define EXPECT(cond)                                                        \
  do {                                                                      \
    if (!(cond)) { std::printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); ++failures; } \
  } while (0)

static rf2_paged_config base() {
  rf2_paged_config c;
  std::memset(&c, 0, sizeof c);
  c.heads = 8; c.kv_heads = 2; c.head_dim = 64; c.page = 64; c.n_pages = 10; c.max_seqs = 4; c.max_pages = 5; c.max_tokens = 32;
  return c;
}

static int create(const rf2_paged_config& c) {
  rf2_paged_plan* p = (rf2_paged_plan*)1;
  const int rc = rf2_paged_plan_create(&c, &p);
  EXPECT((rc == RF2_OK) == (p != nullptr));
  if (rc != RF2_OK) return rc;
  rf2_paged_info in;
  EXPECT(rf2_paged_plan_info(p, &in) == RF2_OK);
  EXPECT(in.cache_elements == (int64_t)c.n_pages * c.kv_heads * c.page * c.head_dim);
  EXPECT(in.workspace_bytes > 0 && in.workspace_bytes < (int64_t)1 << 28);
  EXPECT(rf2_paged_attn(p, 1, 1, nullptr, 0, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) == RF2_ERR_INVALID_ARG);
  EXPECT(rf2_paged_store(p, 1, nullptr, 0, nullptr, 0, nullptr, nullptr, nullptr, nullptr) == RF2_ERR_INVALID_ARG);
  EXPECT(rf2_paged_release(p, 1, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) == RF2_ERR_INVALID_ARG);
  EXPECT(rf2_paged_append(p, 1, 1, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) == RF2_ERR_INVALID_ARG);
  // strides and sizes at the ends of their types
  void* const at = (void*)(uintptr_t)4096;
  int32_t* const ints = (int32_t*)at;
  for (int64_t stride : {std::numeric_limits<int64_t>::min(), (int64_t)-8, (int64_t)0, (int64_t)7, std::numeric_limits<int64_t>::max()})
    if (c.max_tokens > 1) {
      EXPECT(rf2_paged_store(p, 2, at, stride, at, stride, ints, at, at, nullptr) == RF2_ERR_INVALID_ARG);
      EXPECT(rf2_paged_attn(p, 1, 2, at, stride, at, at, ints, ints, ints, at, at, nullptr, nullptr) == RF2_ERR_INVALID_ARG);
    }
  for (int32_t n : {std::numeric_limits<int32_t>::min(), -1, c.max_seqs + 1, std::numeric_limits<int32_t>::max()}) {
    EXPECT(rf2_paged_append(p, n, 1, ints, ints, ints, ints, ints, ints, ints, ints, ints, ints, nullptr) == RF2_ERR_INVALID_ARG);
    EXPECT(rf2_paged_release(p, n, (const uint8_t*)at, ints, ints, ints, ints, ints, ints, ints, nullptr) == RF2_ERR_INVALID_ARG);
    EXPECT(rf2_paged_attn(p, n, 1, at, 4096, at, at, ints, ints, ints, at, at, nullptr, nullptr) == RF2_ERR_INVALID_ARG);
  }
  EXPECT(rf2_paged_plan_destroy(p) == RF2_OK);
  return rc;
}

int main() {
  rf2_paged_config c = base();
  EXPECT(create(c) == RF2_OK);
  for (int kv : {1, 2, 4, 8}) { c.kv_heads = kv; EXPECT(create(c) == RF2_OK); }
  c = base(); c.heads = c.kv_heads = 512; EXPECT(create(c) == RF2_OK);
  c = base(); c.max_seqs = 4096; c.max_tokens = 1 << 20; EXPECT(create(c) == RF2_OK);
  c = base(); c.page = 256; c.head_dim = 128; c.n_pages = 1 << 22; c.max_pages = 1 << 16; c.heads = c.kv_heads = 512; EXPECT(create(c) == RF2_OK);
  c.n_pages += 1; EXPECT(create(c) == RF2_ERR_UNSUPPORTED);
  const int32_t extremes[] = {std::numeric_limits<int32_t>::min(), -1, 0, std::numeric_limits<int32_t>::max()};
  for (int field = 0; field < 10; ++field)
    for (int32_t x : extremes) {
      c = base();
      (&c.heads)[field] = x;
      const int rc = create(c);
      const bool zero_is_fine = field == 8 || field == 9;          // dtype, causal
      EXPECT((rc == RF2_OK) == (x == 0 && zero_is_fine));
    }
  for (float s : {-1.0f, std::numeric_limits<float>::quiet_NaN(), std::numeric_limits<float>::infinity()}) {
    c = base();
    c.scale = s;
    EXPECT(create(c) == RF2_ERR_INVALID_ARG);
  }
  if (failures == 0) std::printf("PAGED ABI CHECK PASSED\n");
  return failures != 0;
}
