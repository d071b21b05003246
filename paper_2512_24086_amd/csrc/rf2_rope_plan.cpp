// Host side of the norms and rotations of Q and K: configuration checks, frequencies, sizes.
#include "rf2_rope.h"

#include <cmath>
#include <new>

namespace {

// Turns of a frequency, f / 2 pi, |f| <= 2^16, in units of 2^-64, whole turns left out, to the nearest.  f has 64 bits, 1 / 2 pi here 126: the product
// in whole numbers is 2^16 2^64 2^-128 units off at most.  (A quotient of 64 bits loses of the fraction what the whole turns take, and a
// position multiplies it.)
uint64_t fraction_of_turns(long double f) {
  typedef unsigned __int128 u128;
  constexpr uint64_t HIGH = 0x28be60db9391054a, LOW = 0x7f09d5f47d4d3770;             // 2^128 / 2 pi
  int e = 0;
  const uint64_t m = (uint64_t)ldexpl(frexpl(fabsl(f), &e), 64);                      // |f| = m 2^(e - 64)
  if (e <= -64) return 0;                                                             // (less than half a unit)
  const u128 product = (u128)m * HIGH + ((u128)m * LOW >> 64);                        // of m 2^64 / 2 pi
  const uint64_t turns = (uint64_t)((product + ((u128)1 << (63 - e))) >> (64 - e));
  return f < 0 ? 0 - turns : turns;
}

}  // namespace

extern "C" {

int rf2_rope_plan_create(const rf2_rope_config* cfg, const double* inv_freq_host, rf2_rope_plan** out) {
  if (!cfg || !out) return RF2_ERR_INVALID_ARG;
  *out = nullptr;
  const rf2_rope_config& c = *cfg;
  if (c.heads < 1 || c.kv_heads < 1) return RF2_ERR_INVALID_ARG;
  if (c.dtype != RF2_DTYPE_BF16 && c.dtype != RF2_DTYPE_F16) return RF2_ERR_INVALID_ARG;
  if (c.weight_dtype != c.dtype && c.weight_dtype != RF2_DTYPE_F32) return RF2_ERR_INVALID_ARG;
  if (c.norm != RF2_NORM_NONE && c.norm != RF2_NORM_RMS) return RF2_ERR_INVALID_ARG;
  if (c.norm == RF2_NORM_RMS && !(c.eps >= 1e-30f && c.eps <= 1.0f)) return RF2_ERR_INVALID_ARG;  // also rejects NaN
  if (c.pairing != RF2_ROPE_PAIRS && c.pairing != RF2_ROPE_HALVES) return RF2_ERR_INVALID_ARG;
  if (c.axes < 0 || c.axes > 4 || (c.axes == 0 && c.norm == RF2_NORM_NONE)) return RF2_ERR_INVALID_ARG;
  if (c.head_dim != 64 && c.head_dim != 128) return RF2_ERR_UNSUPPORTED;
  if (c.heads > 65535 || c.kv_heads > 65535) return RF2_ERR_UNSUPPORTED;
  int64_t dims = 0;
  for (int a = 0; a < c.axes; ++a) {
    if (c.axis_dim[a] < 0 || c.axis_dim[a] % 2 != 0) return RF2_ERR_INVALID_ARG;
    dims += c.axis_dim[a];
  }
  if (dims > c.head_dim) return RF2_ERR_INVALID_ARG;
  if (c.axes > 0 && !inv_freq_host && !(c.theta > 0.0 && std::isfinite(c.theta))) return RF2_ERR_INVALID_ARG;

  // turns per position of each pair; pairs behind the last axis do not turn
  rf2_rope_table tables[2] = {};
  int i = 0;
  for (int a = 0; a < c.axes; ++a)
    for (int j = 0; j < c.axis_dim[a] / 2; ++j, ++i) {
      const long double f = inv_freq_host ? (long double)inv_freq_host[i] : powl((long double)c.theta, -2.0L * j / c.axis_dim[a]);
      if (!(fabsl(f) <= 65536.0L)) return RF2_ERR_INVALID_ARG;
      for (int way = 0; way < 2; ++way) {
        const uint64_t turns = fraction_of_turns(way == 0 ? f : -f);
        const int32_t rest = (int32_t)(uint32_t)turns;                 // with a sign: what is left is a multiple of 2^32 again
        tables[way].turns[i] = (int32_t)(uint32_t)((turns - (uint64_t)(int64_t)rest) >> 32);
        tables[way].rest[i] = rest;
      }
      tables[0].axis[i] = tables[1].axis[i] = (uint8_t)a;
    }

  rf2_rope_plan* p = new (std::nothrow) rf2_rope_plan();
  if (!p) return RF2_ERR_ALLOC;
  p->cfg = c;
  p->d_table = nullptr;
  p->info.workspace_bytes = c.norm == RF2_NORM_RMS ? rf2_rope_workspace(c.head_dim) : 0;
  int n_dev = 0;
  if (hipGetDeviceCount(&n_dev) != hipSuccess || n_dev == 0) {
    (void)hipGetLastError();
    p->device = -1;
    *out = p;
    return RF2_OK;
  }
  hipError_t e = hipGetDevice(&p->device);
  if (e == hipSuccess) e = hipMalloc((void**)&p->d_table, sizeof tables);
  if (e == hipSuccess) e = hipMemcpy(p->d_table, tables, sizeof tables, hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    const int rc = e == hipErrorOutOfMemory ? ((void)hipGetLastError(), (int)RF2_ERR_ALLOC) : rf2_note_hip_error(e);
    rf2_rope_plan_destroy(p);
    return rc;
  }
  *out = p;
  return RF2_OK;
}

int rf2_rope_plan_destroy(rf2_rope_plan* plan) {
  if (!plan) return RF2_OK;
  if (plan->d_table) (void)hipFree(plan->d_table);
  delete plan;
  return RF2_OK;
}

int rf2_rope_plan_info(const rf2_rope_plan* plan, rf2_rope_info* out) {
  if (!plan || !out) return RF2_ERR_INVALID_ARG;
  *out = plan->info;
  return RF2_OK;
}

}  // extern "C"
