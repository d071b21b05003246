// Host side of the paged cache: configuration checks and sizes.
#include "rf2_paged.h"

#include <cmath>
#include <new>

extern "C" {

int rf2_paged_plan_create(const rf2_paged_config* cfg, rf2_paged_plan** out) {
  if (!cfg || !out) return RF2_ERR_INVALID_ARG;
  *out = nullptr;
  const rf2_paged_config& c = *cfg;
  if (c.heads < 1 || c.kv_heads < 1 || c.heads % c.kv_heads != 0) return RF2_ERR_INVALID_ARG;
  if (c.n_pages < 1 || c.max_seqs < 1 || c.max_pages < 1 || c.max_tokens < 1) return RF2_ERR_INVALID_ARG;
  if (c.dtype != RF2_DTYPE_BF16 && c.dtype != RF2_DTYPE_F16) return RF2_ERR_INVALID_ARG;
  if (c.causal != 0 && c.causal != 1) return RF2_ERR_INVALID_ARG;
  if (!(c.scale >= 0.0f && std::isfinite(c.scale))) return RF2_ERR_INVALID_ARG;  // also rejects NaN
  if (c.head_dim != 64 && c.head_dim != 128) return RF2_ERR_UNSUPPORTED;
  if (c.page != 32 && c.page != 64 && c.page != 128 && c.page != 256) return RF2_ERR_UNSUPPORTED;
  if (c.heads > 512 || c.max_seqs > RF2_PAGED_MAX_SEQS || c.max_tokens > 1 << 20) return RF2_ERR_UNSUPPORTED;
  if ((int64_t)c.n_pages * c.page > (int64_t)1 << 30) return RF2_ERR_UNSUPPORTED;    // slots in int32
  if ((int64_t)c.max_pages * c.page > (int64_t)1 << 24) return RF2_ERR_UNSUPPORTED;  // 16 Mi tokens, as a layer has at most
  if ((int64_t)c.max_seqs * c.max_pages > (int64_t)1 << 30) return RF2_ERR_UNSUPPORTED;    // entries of the table in int32

  const double scale = c.scale > 0.0f ? (double)c.scale : 1.0 / std::sqrt((double)c.head_dim);
  const float scale_log2 = (float)(scale * 1.4426950408889634);
  if (!std::isfinite(scale_log2)) return RF2_ERR_INVALID_ARG;      // (infinity times a logit of 0 is not a number)

  rf2_paged_plan* p = new (std::nothrow) rf2_paged_plan();
  if (!p) return RF2_ERR_ALLOC;
  p->cfg = c;
  p->scale_log2 = scale_log2;
  p->info.cache_elements = (int64_t)c.n_pages * c.kv_heads * c.page * c.head_dim;
  p->info.workspace_bytes = rf2_paged_workspace(c);
  int n_dev = 0;
  if (hipGetDeviceCount(&n_dev) != hipSuccess || n_dev == 0) {
    (void)hipGetLastError();
    p->device = -1;
  } else if (const hipError_t e = hipGetDevice(&p->device)) {
    delete p;
    return rf2_note_hip_error(e);
  }
  *out = p;
  return RF2_OK;
}

int rf2_paged_plan_destroy(rf2_paged_plan* plan) {
  delete plan;
  return RF2_OK;
}

int rf2_paged_plan_info(const rf2_paged_plan* plan, rf2_paged_info* out) {
  if (!plan || !out) return RF2_ERR_INVALID_ARG;
  *out = plan->info;
  return RF2_OK;
}

}  // extern "C"
