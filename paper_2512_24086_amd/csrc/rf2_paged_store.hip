// Rows of K and V into the operand tiles of a paged cache (gfx950).
//
// HBM bound: every row is read once and written once.  A workgroup takes 32 tokens of one K/V head through LDS: rows are
// read whole, and left as the tiles want them: 16 bytes of a key's channels with neighbouring keys side by side (K), the keys
// of a channel side by side (V).  V goes out four keys at a time where four tokens fill an aligned group of four slots, as
// tokens of a chunk do, else key by key.
#include "rf2_paged.h"

namespace {

constexpr int TOKENS = 32;

// 16-bit values are moved, whatever they stand for.
template <int D>
__global__ void __launch_bounds__(256) store_kernel(const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, int64_t k_stride,
                                                    int64_t v_stride, const int32_t* __restrict__ slots, int n_tokens, int64_t n_slots,
                                                    int page_shift, int kv_heads, uint16_t* __restrict__ k_cache, uint16_t* __restrict__ v_cache) {
  constexpr int C = D / 8, PITCH = D + 8;                       // 16-byte chunks of a row; LDS rows are 16 bytes further apart
  __shared__ __attribute__((aligned(16))) uint16_t rows[2][TOKENS * PITCH];
  __shared__ int32_t slot_of[TOKENS];
  const int tid = (int)threadIdx.x, head = (int)blockIdx.y;
  const int64_t n0 = (int64_t)blockIdx.x * TOKENS;
  const int count = (int)min((int64_t)TOKENS, n_tokens - n0);
  if (tid < TOKENS) {
    const int slot = tid < count ? slots[n0 + tid] : -1;
    slot_of[tid] = slot >= 0 && slot < n_slots ? slot : -1;
  }
#pragma unroll
  for (int i = 0; i < TOKENS * C / 256; ++i) {
    const int x = i * 256 + tid, r = x / C, c = x % C;
    if (r < count) {
      const int64_t at = (int64_t)head * D + 8 * c;
      const uint4 a = *reinterpret_cast<const uint4*>(k + (n0 + r) * k_stride + at);
      const uint4 b = *reinterpret_cast<const uint4*>(v + (n0 + r) * v_stride + at);
      *reinterpret_cast<uint4*>(&rows[0][r * PITCH + 8 * c]) = a;
      *reinterpret_cast<uint4*>(&rows[1][r * PITCH + 8 * c]) = b;
    }
  }
  __syncthreads();
  // element of the tile that holds a slot, and the slot's place in it
  auto tile_of = [&](int slot) {
    const int page = slot >> page_shift, r = slot & ((1 << page_shift) - 1);
    return (((int64_t)page * kv_heads + head) * (1 << (page_shift - 5)) + (r >> 5)) * (32 * D);
  };
#pragma unroll
  for (int i = 0; i < TOKENS * C / 256; ++i) {
    const int x = i * 256 + tid, c = x / TOKENS, r = x % TOKENS, slot = slot_of[r];
    if (slot >= 0)
      *reinterpret_cast<uint4*>(k_cache + tile_of(slot) + (c * 32 + (slot & 31)) * 8) = *reinterpret_cast<const uint4*>(&rows[0][r * PITCH + 8 * c]);
  }
  // a wavefront has one token at a time, a lane one channel
  constexpr int AT_ONCE = 256 / D;
  const int ch = tid % D;
  for (int r = tid / D; r < count; r += AT_ONCE) {
    const int slot = __builtin_amdgcn_readfirstlane(slot_of[r]);
    if (slot < 0) continue;
    const int lead = r - (slot & 3);                            // the token that would lead this one's group of four
    bool four = lead >= 0 && lead + 3 < count;
    if (four)
#pragma unroll
      for (int e = 0; e < 4; ++e) four &= slot_of[lead + e] == (slot & ~3) + e;
    if (four && lead != r) continue;
    const int key = slot & 31;
    uint16_t* const to = v_cache + tile_of(slot) + ((key / 16 * 2 + key % 8 / 4) * D + ch) * 8 + key % 16 / 8 * 4 + key % 4;
    const uint16_t* const from = &rows[1][r * PITCH + ch];
    if (four) {
      const uint2 x = {from[0] | (uint32_t)from[PITCH] << 16, from[2 * PITCH] | (uint32_t)from[3 * PITCH] << 16};
      *reinterpret_cast<uint2*>(to) = x;
    } else {
      *to = from[0];
    }
  }
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
  if (const int rc = rf2_check_paged_device(plan)) return rc;
  if (n_tokens == 0) return RF2_OK;
  const dim3 grid((n_tokens + TOKENS - 1) / TOKENS, c.kv_heads);
  const auto launch = [&](auto kernel) {
    kernel<<<grid, dim3(256), 0, (hipStream_t)stream>>>((const uint16_t*)k, (const uint16_t*)v, k_stride, v_stride, slots, n_tokens,
                                                         (int64_t)c.n_pages * c.page, __builtin_ctz((unsigned)c.page), c.kv_heads,
                                                         (uint16_t*)k_cache, (uint16_t*)v_cache);
  };
  if (c.head_dim == 128) launch(store_kernel<128>);
  else launch(store_kernel<64>);
  RF2_LAUNCH_CHECK();
  return RF2_OK;
}
