// Host-side exercise of the norms' and rotations' C ABI for a build with the address and undefined-behaviour sanitizers on the host code
// (tests/test_rope_host_sanitized.py compiles and runs it): configurations up to their limits, frequencies, strides and sizes at the ends of
// their types, refusals.  No call here reaches a launch.  Exit code 0 = all expectations held.
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

static rf2_rope_config base() {
  rf2_rope_config c;
  std::memset(&c, 0, sizeof c);
  c.heads = 4; c.kv_heads = 2; c.head_dim = 64; c.norm = RF2_NORM_RMS; c.eps = 1e-6f; c.axes = 3; c.theta = 10000.0;
  c.axis_dim[0] = 16; c.axis_dim[1] = 24; c.axis_dim[2] = 24;
  return c;
}

static int create(const rf2_rope_config& c, const double* table = nullptr) {
  rf2_rope_plan* p = (rf2_rope_plan*)1;
  const int rc = rf2_rope_plan_create(&c, table, &p);
  EXPECT((rc == RF2_OK) == (p != nullptr));
  if (rc != RF2_OK) return rc;
  rf2_rope_info in;
  EXPECT(rf2_rope_plan_info(p, &in) == RF2_OK);
  EXPECT((in.workspace_bytes > 0) == (c.norm == RF2_NORM_RMS) && in.workspace_bytes < (int64_t)1 << 24);
  const void* const at = (void*)(uintptr_t)4096;
  int32_t* const ints = (int32_t*)at;
  float* const floats = (float*)at;
  const void* const w = c.norm == RF2_NORM_RMS ? at : nullptr;
  float* const dw = c.norm == RF2_NORM_RMS ? floats : nullptr;
  const int64_t least = std::numeric_limits<int64_t>::min(), most = std::numeric_limits<int64_t>::max();
  for (int64_t stride : {least, (int64_t)-8, (int64_t)0, (int64_t)7, (int64_t)8, most - 7, most}) {
    const rf2_rows good{at, 3 * c.heads * c.head_dim, (int64_t)c.heads * c.head_dim, c.head_dim}, none{nullptr, 0, 0, 0};
    for (int field = 0; field < 3; ++field) {
      rf2_rows bad = good;
      (field == 0 ? bad.batch : field == 1 ? bad.token : bad.head) = stride;
      const rf2_rope_tensors in_place{good, none, bad, none}, from{bad, none, good, none};
      const bool read_fits = stride == 0 || stride == 8;
      // rows that are written may not share memory: an axis of several has a stride of a row at least
      const bool axis_of_one = field == 2 && c.heads == 1;
      EXPECT(rf2_rope_apply(p, 2, 3, &in_place, ints, 0, w, nullptr, nullptr) == (axis_of_one ? RF2_ERR_HIP : RF2_ERR_INVALID_ARG));
      EXPECT(rf2_rope_apply(p, 2, 3, &from, ints, 0, w, nullptr, nullptr) == (read_fits || axis_of_one ? RF2_ERR_HIP : RF2_ERR_INVALID_ARG));
      const rf2_rope_gradients gradients{good, none, good, none, bad, none};
      EXPECT(rf2_rope_backward(p, 2, 3, &gradients, ints, 0, w, nullptr, dw, nullptr, floats, nullptr) == (axis_of_one ? RF2_ERR_HIP : RF2_ERR_INVALID_ARG));
    }
    const rf2_rope_tensors fine{good, none, good, none};
    EXPECT(rf2_rope_apply(p, 2, 3, &fine, ints, stride, w, nullptr, nullptr) == (stride == 0 || stride == 7 || stride == 8 ? RF2_ERR_HIP : RF2_ERR_INVALID_ARG));
  }
  const rf2_rope_tensors all{{at, 0, 8, 8}, {at, 0, 8, 8}, {at, 0, 8, 8}, {at, 0, 8, 8}};
  for (int32_t n : {std::numeric_limits<int32_t>::min(), -1, std::numeric_limits<int32_t>::max()}) {
    EXPECT(rf2_rope_apply(p, n, 1, &all, ints, 0, w, w, nullptr) != RF2_OK);
    EXPECT(rf2_rope_apply(p, 1, n, &all, ints, 0, w, w, nullptr) != RF2_OK);
    EXPECT(rf2_rope_apply(p, n, n, &all, ints, 0, w, w, nullptr) != RF2_OK);
  }
  EXPECT(rf2_rope_plan_destroy(p) == RF2_OK);
  return rc;
}

int main() {
  rf2_rope_config c = base();
  EXPECT(create(c) == RF2_OK);
  for (int32_t d : {64, 128}) for (int32_t norm : {0, 1}) for (int32_t halves : {0, 1}) for (int32_t type : {0, 1}) {
    c = base(); c.head_dim = d; c.norm = norm; c.pairing = halves; c.dtype = type; c.weight_dtype = halves ? RF2_DTYPE_F32 : type;
    EXPECT(create(c) == RF2_OK);
  }
  c = base(); c.heads = 1; c.kv_heads = 65535; EXPECT(create(c) == RF2_OK);
  c = base(); c.axes = 4; for (int a = 0; a < 4; ++a) c.axis_dim[a] = 16;
  EXPECT(create(c) == RF2_OK);
  c = base(); c.axes = 0; EXPECT(create(c) == RF2_OK);
  const int32_t extremes[] = {std::numeric_limits<int32_t>::min(), -1, std::numeric_limits<int32_t>::max()};
  for (int32_t x : extremes)
    for (int field = 0; field < 9; ++field) {
      c = base();
      int32_t* const fields[] = {&c.heads, &c.kv_heads, &c.head_dim, &c.dtype, &c.weight_dtype, &c.norm, &c.pairing, &c.axes, &c.axis_dim[1]};
      *fields[field] = x;
      EXPECT(create(c) != RF2_OK);
    }
  for (float eps : {0.0f, -1.0f, 1e-38f, 2.0f, std::numeric_limits<float>::quiet_NaN(), std::numeric_limits<float>::infinity()}) {
    c = base(); c.eps = eps; EXPECT(create(c) == RF2_ERR_INVALID_ARG);
  }
  for (double theta : {0.0, -1.0, std::numeric_limits<double>::quiet_NaN(), std::numeric_limits<double>::infinity(), std::numeric_limits<double>::denorm_min()}) {
    c = base(); c.theta = theta; EXPECT(create(c) == RF2_ERR_INVALID_ARG);
  }
  for (double theta : {1e-2, 1.0, 1e6, std::numeric_limits<double>::max()}) { c = base(); c.theta = theta; EXPECT(create(c) == RF2_OK); }
  // frequencies whose fractions of a turn lie at the ends of what is kept of them: whole and half turns, next to them, none
  constexpr double turn = 6.283185307179586476925286766559;
  double table[32] = {};
  for (double f : {0.0, turn, turn / 2, -turn / 2, 1.5 * turn, 65536.0, -65536.0, 1e-300, -5e-324, turn * (0.5 - 0x1p-33), turn * (0.5 + 0x1p-33), turn * 0x1p-33, turn * 1.5 * 0x1p-32,
                   turn * (0x1p-33 - 0x1p-65), turn * 3 * 0x1p-65}) {
    for (double& t : table) t = f;
    EXPECT(create(base(), table) == RF2_OK);
    table[31] = 65537.0; EXPECT(create(base(), table) == RF2_ERR_INVALID_ARG);
    table[31] = std::numeric_limits<double>::quiet_NaN(); EXPECT(create(base(), table) == RF2_ERR_INVALID_ARG);
    table[31] = std::numeric_limits<double>::infinity(); EXPECT(create(base(), table) == RF2_ERR_INVALID_ARG);
  }
  if (failures == 0) std::printf("ROPE ABI CHECK PASSED\n");
  return failures != 0;
}
