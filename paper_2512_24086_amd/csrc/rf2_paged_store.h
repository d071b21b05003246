// Rows of K and V into the operand tiles of a paged cache: what a workgroup of 256 threads does (not installed).
#pragma once
#include "rf2_paged.h"

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int STORE_TOKENS = 32;

constexpr int MORE = 11;                                        // rows of V that groups of a workgroup's last tokens may need
template <int D, bool WITH_K, int TOKENS>
struct StoreLds {
  static constexpr int PITCH = D + 8;                           // rows are 16 bytes further apart
  __attribute__((aligned(16))) uint16_t k_rows[WITH_K ? TOKENS * PITCH : 8];
  __attribute__((aligned(16))) uint16_t v_rows[(TOKENS + MORE) * PITCH];
  int32_t slot_of[2 * MORE + TOKENS];
  int32_t todo[TOKENS + 1];                                     // tokens of V that lead a group, four keys, or none; how many
};

// A workgroup has TOKENS tokens of a K/V head, 64 at most.  16-bit values are moved, whatever they stand for.  K may be left out.
template <int D, bool WITH_K, int TOKENS>
__device__ __forceinline__ void store_rows(const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, int64_t k_stride, int64_t v_stride,
                                           const int32_t* __restrict__ slots, int n_tokens, int64_t n_slots, int page_shift, int kv_heads, unsigned windows,
                                           unsigned run, uint16_t* __restrict__ k_cache, uint16_t* __restrict__ v_cache, unsigned group,
                                           StoreLds<D, WITH_K, TOKENS>& lds) {
  constexpr int ROWS = TOKENS + MORE, C = D / 8, PITCH = StoreLds<D, WITH_K, TOKENS>::PITCH;      // 16-byte chunks of a row
  uint16_t *const k_rows = lds.k_rows, *const v_rows = lds.v_rows;
  int32_t *const slot_of = lds.slot_of, *const todo = lds.todo;
  // Workgroups with equal number % 8 share an XCD: each XCD gets a run of windows head by head, so that lines which two
  // windows write in parts are completed in its L2.
  const unsigned at = (group & 7) * run + (group >> 3);
  if (at >= windows * (unsigned)kv_heads) return;
  const int tid = (int)threadIdx.x, head = (int)(at / windows);
  const int64_t n0 = (int64_t)(at % windows) * TOKENS;
  const int count = (int)min((int64_t)TOKENS, n_tokens - n0), more = (int)min((int64_t)ROWS, n_tokens - n0);
  const int64_t column = (int64_t)head * D;
  // (rows are read once: marked as not to be kept, they leave the caches to what is written; 4,680 tokens of 40 heads 47.1 -> 36.0 us)
  u32x4 x[WITH_K ? TOKENS * C / 256 : 1], y[(ROWS * C + 255) / 256];
#pragma unroll
  for (int i = 0; i < TOKENS * C / 256 && WITH_K; ++i) {
    const int r = min((i * 256 + tid) / C, count - 1);
    x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(k + (n0 + r) * k_stride + column + tid % C * 8));
  }
#pragma unroll
  for (int i = 0; i < (ROWS * C + 255) / 256; ++i) {
    const int r = min((i * 256 + tid) / C, more - 1);
    y[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(v + (n0 + r) * v_stride + column + tid % C * 8));
  }
  if (tid < MORE + ROWS) {
    const int64_t n = n0 + tid - MORE;
    const int slot = n >= 0 && n < n_tokens ? slots[n] : -1;
    slot_of[tid] = slot >= 0 && slot < n_slots ? slot : -1;
  }
#pragma unroll
  for (int i = 0; i < TOKENS * C / 256 && WITH_K; ++i) {
    const int r = (i * 256 + tid) / C;
    if (r < count) *reinterpret_cast<u32x4*>(&k_rows[r * PITCH + tid % C * 8]) = x[i];
  }
#pragma unroll
  for (int i = 0; i < (ROWS * C + 255) / 256; ++i) {
    const int r = (i * 256 + tid) / C;
    if (r < more) *reinterpret_cast<u32x4*>(&v_rows[r * PITCH + tid % C * 8]) = y[i];
  }
  __syncthreads();
  if (tid < 64) {
    // What token tid does: 8, its slot begins a group that is complete; 4, four keys; 1, one; 0, another token does its part.
    int kind = 0;
    if (tid < count && slot_of[MORE + tid] >= 0) {
      const int slot = slot_of[MORE + tid], key = slot & 15, lead = tid - (key & 3);      // of its four keys
      const auto four = [&](int first, int from) {            // tokens first .. + 3 have slots from .. + 3
        bool yes = first >= -MORE && first + 3 < ROWS;
#pragma unroll
        for (int e = 0; e < 4; ++e) yes = yes && slot_of[MORE + first + e] == from + e;
        return yes;
      };
      kind = 1;
      if (four(lead, slot & ~3)) {
        const bool upper = key >= 8, group = four(upper ? lead - 8 : lead + 8, (slot & ~3) + (upper ? -8 : 8));
        kind = lead != tid ? 0 : group ? (upper ? 0 : 8) : 4;
      }
    }
    const uint64_t some = __builtin_amdgcn_ballot_w64(kind != 0);
    if (kind != 0) todo[__popcll(some & ((1ull << tid) - 1))] = tid | kind << 8;
    if (tid == 0) todo[TOKENS] = __popcll(some);
  }
  // element of the tile that holds a slot, and the slot's place in it
  auto tile_of = [&](int slot) {
    const int page = slot >> page_shift, r = slot & ((1 << page_shift) - 1);
    return (((int64_t)page * kv_heads + head) * (1 << (page_shift - 5)) + (r >> 5)) * (32 * D);
  };
#pragma unroll
  for (int i = 0; i < TOKENS * C / 256 && WITH_K; ++i) {
    const int z = i * 256 + tid, c = z / TOKENS, r = z % TOKENS, slot = slot_of[MORE + r];
    if (r < count && slot >= 0)
      *reinterpret_cast<uint4*>(k_cache + tile_of(slot) + (c * 32 + (slot & 31)) * 8) = *reinterpret_cast<const uint4*>(&k_rows[r * PITCH + 8 * c]);
  }
  __syncthreads();
  // a wavefront has one token of the list at a time, a lane one channel
  const int ch = tid % D, n_todo = todo[TOKENS];
  for (int i = tid / D; i < n_todo; i += 256 / D) {
    const int what = __builtin_amdgcn_readfirstlane(todo[i]), r = what & 255, slot = slot_of[MORE + r], key = slot & 31;
    uint16_t* const to = v_cache + tile_of(slot) + ((key / 16 * 2 + key % 8 / 4) * D + ch) * 8 + key % 16 / 8 * 4 + key % 4;
    const uint16_t* const from = &v_rows[r * PITCH + ch];
    const auto pair = [&](int e) { return from[e * PITCH] | (uint32_t)from[(e + 1) * PITCH] << 16; };
    if (what >> 8 == 8) *reinterpret_cast<uint4*>(to) = make_uint4(pair(0), pair(2), pair(8), pair(10));
    else if (what >> 8 == 4) *reinterpret_cast<uint2*>(to) = make_uint2(pair(0), pair(2));
    else *to = from[0];
  }
}

}  // namespace
