// New tokens of a paged cache, one launch: Q normalised and rotated, K too and into the cache's operand tiles, V into its own (gfx950).
//
// HBM bound, or by the launch where tokens are few: every row is read once and written once.  The first workgroups do V as rf2_paged_store does,
// the next K, the others Q as rf2_rope_apply does.  K goes from the registers in which it is rotated to its tiles: a wavefront has eight tokens, whose
// 16-byte chunks stand side by side there, and goes through a few heads with their cosines and sines.  (With K through LDS, head by head, as in
// rf2_paged_store, 62.8 us for 4,680 tokens of 40 heads where this way took 58.6.)  288 MB in 52.2 us are 5.5 TB/s; by themselves V takes 21, K 23,
// Q 20.  Stores of K and V stay in the caches, for the attention (past them 56.1).
#include "rf2_paged_store.h"
#include "rf2_rope.h"

namespace {

// Tokens of a workgroup of K, and of V.  V's read 11 rows more than they have, so 64 tokens are better than 32 where there are enough of them for all
// compute units, COMPUTE_UNITS (us in a graph, 32 and 64: 4,680 tokens of 40 heads 59.4, 57.2, 1,000 18.8, 17.6, 8,000 of 8 39.8, 38.4).  V of single
// tokens goes out key by key, one behind the other, so fewer are 32 to a workgroup (512 single tokens on 8 heads 8.7, 64: 12.4), or 8 as long as those are
// no more than compute units (32 and 8: 48 single tokens on 8 heads 6.2, 3.7, 200 7.1, 4.7, 48 on 40 heads 7.2, 4.7, a run of 200 on 8 4.3, 3.9; beyond:
// 256 single tokens on 40 heads 13.9, 16.4, a run of 500 on 8 5.8, 6.4).
constexpr int K_TOKENS = 32, COMPUTE_UNITS = 256;

struct StoreRopeArgs {
  const uint16_t *k, *v;
  int64_t k_stride, v_stride;
  const int32_t* slots;
  int n_tokens, page_shift, kv_heads;
  int64_t n_slots;
  int v_tokens;                      // of a workgroup, 8, 32 or 64
  unsigned windows, run;             // of V
  uint16_t *k_cache, *v_cache;
  RopeArgs rope;
  const int32_t* pos;
  const void* wk;
  int norm;
  int k_steps;                       // heads of a wavefront
  unsigned k_windows, k_workgroups;
  const int32_t* n_live;             // tokens that are not padding, or NULL
  RopeSide q;
};

template <class T, int D, bool HALVES, bool NORM>
__device__ __forceinline__ void store_k(const StoreRopeArgs& a, unsigned id) {
  constexpr int C = D / 8, SETS = C / 8, AHEAD = 2;              // sets of rows of a wavefront
  const unsigned group = id / a.k_windows, window = id - group * a.k_windows;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane % C, g = lane / C;
  const int at = (int)window * K_TOKENS + 8 * wave, h0 = (int)group * a.k_steps, end = min(a.kv_heads, h0 + a.k_steps);
  if (at >= a.n_tokens) return;
  // In large calls a wavefront's tokens begin with the first of the eight keys that share lines with token `at`, where that is a few tokens before:
  // within a run they are eight whose lines are theirs alone, at its ends 1 to 15 (4,680 tokens of 40 heads 57.1 -> 53.4 us, 1,000 16.9 -> 16.4, but 1,000
  // of 8 heads, which wait for the slots, 8.2 -> 9.3).
  int begin = at, last = min(at + 8, a.n_tokens);
  if (a.k_steps > 1) {
    const int near = a.slots[min(max(at - 8 + min(lane, 23), 0), a.n_tokens - 1)];                   // of the tokens from at - 8 to at + 15
    const auto early = [&](int i) {
      const int slot = __builtin_amdgcn_readlane(near, i), before = slot & 7;
      return slot >= 0 && before <= at + i - 8 && __builtin_amdgcn_readlane(near, i - before) == slot - before ? before : 0;
    };
    begin -= early(8);
    if (last < a.n_tokens) last -= early(16);
  }
  for (int first = begin; first < last; first += 8) {
    const uint16_t* from[SETS];
    u32x4 v[AHEAD][SETS];
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
      from[s] = a.k + min(first + 4 * s + g, last - 1) * a.k_stride + (int64_t)h0 * D + 8 * c;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) v[i][s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from[s] + min(i, end - 1 - h0) * D));
    }
    // the token whose rows a lane stores (below), and where
    const int mine = first + (SETS == 2 ? 4 * (c / 8) : 0) + g;
    const int slot = mine < last ? a.slots[mine] : -1;
    const bool store = slot >= 0 && slot < a.n_slots;
    const int page = slot >> a.page_shift, r = slot & ((1 << a.page_shift) - 1);
    const int64_t head = (int64_t)D << a.page_shift;               // elements of a head of a page
    uint16_t* to = a.k_cache + ((int64_t)page * a.kv_heads + h0) * head + (r >> 5) * (32 * D) + (c % 8 * 32 + (r & 31)) * 8;
    RopeArgs rope = a.rope;
    const void* wk = a.wk;
    asm volatile("" : "+s"(rope.table), "+s"(wk));                 // (what a second turn needs again is read again: in registers it costs wavefronts)
    float own[8], other[8], A[SETS][8], B[SETS][8];
    const RopeLane angles = rope_lane<D, HALVES>(rope, c);
    if constexpr (NORM) rope_weights<T>(rope, wk, c, own);
    if constexpr (NORM && HALVES) rope_weights<T>(rope, wk, c ^ (C / 2), other);
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
      const RopePlace place = rope_place(rope, angles, a.pos + (int64_t)min(first + 4 * s + g, last - 1) * a.rope.axes);
      rope_factors<D, HALVES, NORM>(angles, place, own, other, c, A[s], B[s]);
    }
    for (int h = h0; h < end; h += AHEAD)
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (h + i >= end) break;
        u32x4 z[SETS];
#pragma unroll
        for (int s = 0; s < SETS; ++s) {
          float x[8];
          T::unpack(v[i][s], x);
          v[i][s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from[s] + min(h + i + AHEAD, end - 1) * D - h0 * D));
          rope_row<D, HALVES, NORM>(a.rope, A[s], B[s], x);
          z[s] = T::pack(x);
        }
        if constexpr (SETS == 2) {
          // the upper chunks of four tokens against the lower ones of the next four: a store covers eight chunks of eight tokens
          u32x4 low, high;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t one = z[0][e], two = z[1][e];
            low[e] = (uint32_t)__builtin_amdgcn_update_dpp((int)one, (int)two, 0x128, 0xf, 0xc, false);      // row_ror:8 into lanes 8-15
            high[e] = (uint32_t)__builtin_amdgcn_update_dpp((int)two, (int)one, 0x128, 0xf, 0x3, false);     // and into lanes 0-7
          }
          if (store) {
            *reinterpret_cast<u32x4*>(to) = low;
            *reinterpret_cast<u32x4*>(to + 8 * 32 * 8) = high;
          }
        } else if (store) {
          *reinterpret_cast<u32x4*>(to) = z[0];
        }
        to += head;
      }
  }
}

template <class T, int D, bool HALVES, bool NORM, bool KEEP>
__global__ void __launch_bounds__(256) store_rope_kernel(StoreRopeArgs a) {
  __shared__ union {
    StoreLds<D, false, 8> few;
    StoreLds<D, false, 32> some;
    StoreLds<D, false, 64> many;
  } lds;
  unsigned id = blockIdx.x;
  if (id < 8 * a.run) {
    const auto rows = [&](auto& part) {
      store_rows(a.k, a.v, a.k_stride, a.v_stride, a.slots, a.n_tokens, a.n_slots, a.page_shift, a.kv_heads, a.windows, a.run, a.k_cache, a.v_cache, id, part);
    };
    a.v_tokens == 64 ? rows(lds.many) : a.v_tokens == 32 ? rows(lds.some) : rows(lds.few);
    return;
  }
  id -= 8 * a.run;
  if (id < a.k_workgroups) {
    store_k<T, D, HALVES, NORM>(a, id);
    return;
  }
  id -= a.k_workgroups;
  const uint32_t live = a.n_live ? (uint32_t)min(max(*a.n_live, 0), a.n_tokens) : (uint32_t)a.n_tokens;
  rope_apply_rows<T, D, HALVES, NORM, KEEP>(a.rope, RopeTokens{a.pos, 0, live, live}, a.q, id);
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
  const unsigned k_windows = (unsigned)(n_tokens + K_TOKENS - 1) / K_TOKENS;
  if ((k_windows * (unsigned)c.kv_heads + 7) / 8 >= 1u << 20) return RF2_ERR_UNSUPPORTED;   // (a grid has less than 2^32 threads, half of them for V and K)
  if (const int rc = rf2_check_paged_device(plan)) return rc;
  if (n_tokens == 0) return RF2_OK;
  const rf2_rows q_rows{q, 0, n_tokens > 1 ? q_stride : q_row, c.head_dim}, out_rows{q_out, 0, n_tokens > 1 ? q_out_stride : q_row, c.head_dim};
  const RopeSide side{rope_rows(q_rows), rope_rows(out_rows), wq, rope_share(q_rows, c.heads, r, (uint32_t)n_tokens)};
  // K's wavefronts take as many heads as leave 2,048 of them, eight (64 channels: five) at most (us, most heads 4, 8, 16: 4,680 tokens of 40 heads 53.5,
  // 52.3, 53.1, 20,000 of 32 207, 197, 199; 64 channels, HALVES, 4,680 of 40: 4 31.1, 5 30.6, 8 30.9)
  const int64_t k_work = (int64_t)((n_tokens + 7) / 8) * c.kv_heads;
  const int k_steps = (int)std::min<int64_t>(c.head_dim == 128 ? 8 : 5, std::max<int64_t>(1, k_work / 2048));
  const unsigned k_workgroups = k_windows * (unsigned)((c.kv_heads + k_steps - 1) / k_steps);
  const auto v_workgroups = [&](int tokens) { return (int64_t)((n_tokens + tokens - 1) / tokens) * c.kv_heads; };
  const int v_tokens = v_workgroups(8) <= COMPUTE_UNITS ? 8 : v_workgroups(64) < COMPUTE_UNITS ? 32 : 64;
  const unsigned windows = (unsigned)(n_tokens + v_tokens - 1) / v_tokens, run = (unsigned)((v_workgroups(v_tokens) + 7) / 8);
  const StoreRopeArgs a{(const uint16_t*)k, (const uint16_t*)v, k_stride, v_stride, slots, n_tokens, __builtin_ctz((unsigned)c.page), c.kv_heads,
                        (int64_t)c.n_pages * c.page, v_tokens, windows, run, (uint16_t*)k_cache, (uint16_t*)v_cache, rope_args(rope), pos, wk,
                        r.norm == RF2_NORM_RMS, k_steps, k_windows, k_workgroups, n_live, side};
  const dim3 grid(8 * run + k_workgroups + rope_workgroups(side.share));
  const bool keep = (int64_t)n_tokens * q_row * 4 <= ROPE_KEEP;
  hipStream_t st = (hipStream_t)stream;
  return rope_for_types(r, [&](auto type, auto d, auto halves) {
    const auto launch = [&](auto norm, auto kept) { store_rope_kernel<decltype(type), d(), halves(), norm(), kept()><<<grid, 256, 0, st>>>(a); };
    const auto with = [&](auto norm) { keep ? launch(norm, std::true_type()) : launch(norm, std::false_type()); };
    a.norm ? with(std::true_type()) : with(std::false_type());
  });
}
