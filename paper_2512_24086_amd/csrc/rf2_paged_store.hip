// Rows of K and V into the operand tiles of a paged cache (gfx950).
//
// HBM bound: every row is read once and written once.  A workgroup takes 32 tokens of one K/V head through LDS: rows are
// read whole, and left as the tiles want them: 16 bytes of a key's channels with neighbouring keys side by side (K), the keys
// of a channel side by side (V).  V goes out 16 bytes a lane where the tokens fill the eight keys of a storage group (0-3 and
// 8-11, or 4-7 and 12-15, of 16 slots), as those of a chunk do, eight bytes where they fill four keys in a row, else key by key.
// A group belongs to the workgroup of its first token, which reads up to 11 tokens more for it.
//
// 4,680 tokens of 40 heads of 128 channels: 192 MB in 37 us, 5.2 TB/s (33 to 34 us the kernel by itself; a large copy reaches 6.2).  Windows
// of 64 tokens take longer to fill a compute unit's LDS and gain nothing; stores that are not to be kept cost the lines that two
// windows complete (44 us).  48 single tokens of 8 heads: 6.7 us, of which 0.1 are its bytes: in each of 16
// workgroups V's lone keys go out two at a time, one pair behind the other.
#include "rf2_paged_store.h"

namespace {

template <int D>
__global__ void __launch_bounds__(256) store_kernel(const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, int64_t k_stride,
                                                    int64_t v_stride, const int32_t* __restrict__ slots, int n_tokens, int64_t n_slots,
                                                    int page_shift, int kv_heads, unsigned windows, unsigned run, uint16_t* __restrict__ k_cache,
                                                    uint16_t* __restrict__ v_cache) {
  __shared__ StoreLds<D, true, STORE_TOKENS> lds;
  store_rows(k, v, k_stride, v_stride, slots, n_tokens, n_slots, page_shift, kv_heads, windows, run, k_cache, v_cache, blockIdx.x, lds);
}

}  // namespace

extern "C" int rf2_paged_store(const rf2_paged_plan* plan, int32_t n_tokens, const void* k, int64_t k_stride, const void* v,
                               int64_t v_stride, const int32_t* slots, void* k_cache, void* v_cache, void* stream) {
  if (!plan || n_tokens < 0 || n_tokens > plan->cfg.max_tokens || !k_cache || !v_cache) return RF2_ERR_INVALID_ARG;
  if (n_tokens > 0 && (!k || !v || !slots)) return RF2_ERR_INVALID_ARG;
  const rf2_paged_config& c = plan->cfg;
  const int64_t row = (int64_t)c.kv_heads * c.head_dim;
  if (n_tokens > 1 && (k_stride < row || v_stride < row)) return RF2_ERR_INVALID_ARG;
  if (k_stride % 8 != 0 || v_stride % 8 != 0) return RF2_ERR_INVALID_ARG;
  if (!rf2_aligned(k, 16) || !rf2_aligned(v, 16) || !rf2_aligned(k_cache, 16) || !rf2_aligned(v_cache, 16) || !rf2_aligned(slots, 4))
    return RF2_ERR_INVALID_ARG;
  const unsigned windows = (unsigned)(n_tokens + STORE_TOKENS - 1) / STORE_TOKENS, run = (windows * (unsigned)c.kv_heads + 7) / 8;
  if (run >= 1u << 21) return RF2_ERR_UNSUPPORTED;         // (a grid has less than 2^32 threads)
  if (const int rc = rf2_check_paged_device(plan)) return rc;
  if (n_tokens == 0) return RF2_OK;
  const auto launch = [&](auto kernel) {
    kernel<<<dim3(8 * run), dim3(256), 0, (hipStream_t)stream>>>((const uint16_t*)k, (const uint16_t*)v, k_stride, v_stride, slots, n_tokens,
                                                               (int64_t)c.n_pages * c.page, __builtin_ctz((unsigned)c.page), c.kv_heads,
                                                               windows, run, (uint16_t*)k_cache, (uint16_t*)v_cache);
  };
  if (c.head_dim == 128) launch(store_kernel<128>);
  else launch(store_kernel<64>);
  RF2_LAUNCH_CHECK();
  return RF2_OK;
}
