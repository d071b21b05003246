// New tokens of a paged cache, one launch: Q normalised and rotated, K too and into the cache's operand tiles, V into its own (gfx950).
//
// HBM bound, or by the launch where tokens are few: every row is read once and written once.  The first workgroups do K and V as rf2_paged_store
// does (a row of K passes through its lanes' registers on the way into LDS), the others Q as rf2_rope_apply does.
#include "rf2_paged_store.h"
#include "rf2_rope.h"

namespace {

struct StoreRopeArgs {
  const uint16_t *k, *v;
  int64_t k_stride, v_stride;
  const int32_t* slots;
  int n_tokens, page_shift, kv_heads;
  int64_t n_slots;
  unsigned windows, run;
  uint16_t *k_cache, *v_cache;
  RopeArgs rope;
  const int32_t* pos;
  const void* wk;
  int norm;
  const int32_t* n_live;             // tokens that are not padding, or NULL
  RopeSide q;
};

template <class T, int D, bool HALVES, bool KEEP>
__global__ void __launch_bounds__(256) store_rope_kernel(StoreRopeArgs a) {
  if (blockIdx.x < 8 * a.run) {
    const auto prepare = [&](const u32x4& row, int64_t token, int c) {
      const RopeLane angles = rope_lane<D, HALVES>(a.rope, c);
      const RopePlace place = rope_place(a.rope, angles, a.pos + token * a.rope.axes);
      float A[8], B[8], x[8];
      T::unpack(row, x);
      if (a.norm) {
        rope_factors<T, D, HALVES, true>(a.rope, angles, place, a.wk, c, A, B);
        rope_row<D, HALVES, true>(a.rope, A, B, x);
      } else {
        rope_factors<T, D, HALVES, false>(a.rope, angles, place, nullptr, c, A, B);
        rope_row<D, HALVES, false>(a.rope, A, B, x);
      }
      return T::pack(x);
    };
    store_rows<D>(a.k, a.v, a.k_stride, a.v_stride, a.slots, a.n_tokens, a.n_slots, a.page_shift, a.kv_heads, a.windows, a.run, a.k_cache, a.v_cache,
                  blockIdx.x, prepare);
    return;
  }
  const uint32_t live = a.n_live ? (uint32_t)min(max(*a.n_live, 0), a.n_tokens) : (uint32_t)a.n_tokens;
  const RopeTokens tokens{a.pos, 0, live, live};
  if (a.norm) rope_apply_rows<T, D, HALVES, true, KEEP>(a.rope, tokens, a.q, blockIdx.x - 8 * a.run);
  else rope_apply_rows<T, D, HALVES, false, KEEP>(a.rope, tokens, a.q, blockIdx.x - 8 * a.run);
}

}  // namespace

extern "C" int rf2_paged_store_rope(const rf2_paged_plan* plan, const rf2_rope_plan* rope, int32_t n_tokens, const void* q, int64_t q_stride, const void* k,
                                    int64_t k_stride, const void* v, int64_t v_stride, const int32_t* pos, const void* wq, const void* wk,
                                    const int32_t* slots, const int32_t* n_live, void* k_cache, void* v_cache, void* q_out, int64_t q_out_stride,
                                    void* stream) {
  if (!plan || !rope || n_tokens < 0 || n_tokens > plan->cfg.max_tokens || !k_cache || !v_cache) return RF2_ERR_INVALID_ARG;
  const rf2_paged_config& c = plan->cfg;
  const rf2_rope_config& r = rope->cfg;
  if (r.heads != c.heads || r.kv_heads != c.kv_heads || r.head_dim != c.head_dim || r.dtype != c.dtype || rope->device != plan->device)
    return RF2_ERR_INVALID_ARG;
  if (n_tokens > 0 && (!q || !k || !v || !slots || !q_out)) return RF2_ERR_INVALID_ARG;
  const int64_t row = (int64_t)c.kv_heads * c.head_dim, q_row = (int64_t)c.heads * c.head_dim;
  if (n_tokens > 1 && (k_stride < row || v_stride < row || q_stride < q_row || q_out_stride < q_row)) return RF2_ERR_INVALID_ARG;
  if (k_stride % 8 != 0 || v_stride % 8 != 0 || q_stride % 8 != 0 || q_out_stride % 8 != 0) return RF2_ERR_INVALID_ARG;
  const int64_t most = (int64_t)1 << 36;                     // (times 2^20 tokens: far from what 64 bits count)
  if (n_tokens > 1 && (k_stride > most || v_stride > most || q_stride > most || q_out_stride > most)) return RF2_ERR_INVALID_ARG;
  for (const void* t : {q, k, v, (const void*)k_cache, (const void*)v_cache, (const void*)q_out})
    if (!rf2_aligned(t, 16)) return RF2_ERR_INVALID_ARG;
  if (!rf2_aligned(slots, 4) || !rf2_aligned(n_live, 4)) return RF2_ERR_INVALID_ARG;
  if (n_tokens > 0 && (!rf2_rope_pos_fits(rope, pos) || !rf2_rope_weight_fits(rope, wq) || !rf2_rope_weight_fits(rope, wk))) return RF2_ERR_INVALID_ARG;
  const unsigned windows = (unsigned)(n_tokens + TOKENS - 1) / TOKENS, run = (windows * (unsigned)c.kv_heads + 7) / 8;
  if (run >= 1u << 20) return RF2_ERR_UNSUPPORTED;           // (a grid has less than 2^32 threads, half of them for Q)
  if (const int rc = rf2_check_paged_device(plan)) return rc;
  if (n_tokens == 0) return RF2_OK;
  const rf2_rows q_rows{q, 0, n_tokens > 1 ? q_stride : q_row, c.head_dim}, out_rows{q_out, 0, n_tokens > 1 ? q_out_stride : q_row, c.head_dim};
  const RopeSide side{rope_rows(q_rows), rope_rows(out_rows), wq, rope_share(q_rows, c.heads, r, (uint32_t)n_tokens)};
  const StoreRopeArgs a{(const uint16_t*)k, (const uint16_t*)v, k_stride, v_stride, slots, n_tokens, __builtin_ctz((unsigned)c.page), c.kv_heads,
                        (int64_t)c.n_pages * c.page, windows, run, (uint16_t*)k_cache, (uint16_t*)v_cache, rope_args(rope), pos, wk,
                        r.norm == RF2_NORM_RMS, n_live, side};
  const dim3 grid(8 * run + rope_workgroups(side.share));
  const bool keep = (int64_t)n_tokens * q_row * 4 <= ROPE_KEEP;
  hipStream_t st = (hipStream_t)stream;
  return rope_for_types(r, [&](auto type, auto d, auto halves) {
    if (keep) store_rope_kernel<decltype(type), d(), halves(), true><<<grid, 256, 0, st>>>(a);
    else store_rope_kernel<decltype(type), d(), halves(), false><<<grid, 256, 0, st>>>(a);
  });
}
