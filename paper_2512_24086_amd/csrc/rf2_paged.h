// Internal declarations of the paged cache (not installed).
#pragma once
#include <algorithm>

#include "rf2_internal.h"

struct rf2_paged_plan {
  rf2_paged_config cfg;
  rf2_paged_info info;
  int device;
  float scale_log2;  // scale * log2(e)
};

constexpr int RF2_PAGED_MAX_SEQS = 4096;

// Attention launches are cut into parts (rf2_paged_attn.hip): as many as this are aimed at, in all K/V heads together.
constexpr int RF2_PAGED_PARTS = 1024;
// Query rows of a workgroup where a sequence has many (16 or 32 where it has few).
constexpr int RF2_PAGED_ROWS_MANY = 128;
// Groups of rows of a tile whose parts are added together (32 bytes each).
constexpr int RF2_PAGED_JOINTS = 16;

inline int rf2_paged_parts_per_head(int kv_heads) { return std::max(1, RF2_PAGED_PARTS / kv_heads); }

// Bytes of the partial results of a launch: sequences that are cut have fewer than twice as many parts as are aimed at, each of
// `rows` rows of head_dim sums and two numbers more, and at most as many tiles, with 32 bytes for every 8 rows
// (rf2_paged_attn.hip).
inline int64_t rf2_paged_parts_bytes(const rf2_paged_config& c) {
  const int64_t aimed = (int64_t)rf2_paged_parts_per_head(c.kv_heads) * c.kv_heads;
  return 2 * aimed * RF2_PAGED_ROWS_MANY * (c.head_dim + 2) * 4 + 32 * (aimed * RF2_PAGED_JOINTS + 1);
}

// Launches of more sequences than this add up their shares first: 16 bytes each, and 16 more.
constexpr int RF2_PAGED_SURVEY = 256;
inline int64_t rf2_paged_workspace(const rf2_paged_config& c) {
  return rf2_paged_parts_bytes(c) + (c.max_seqs > RF2_PAGED_SURVEY ? 16 * ((int64_t)c.max_seqs + 1) : 0);
}

inline bool rf2_aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

inline int rf2_check_paged_device(const rf2_paged_plan* plan) {
  if (plan->device < 0) return rf2_note_hip_error(hipErrorNoDevice);
  int current = -1;
  const hipError_t e = hipGetDevice(&current);
  if (e != hipSuccess) return rf2_note_hip_error(e);
  return current == plan->device ? RF2_OK : RF2_ERR_INVALID_ARG;
}
