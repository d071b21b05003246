// Window permutation and block means of a layer, Q and K normalised and rotated on the way (gfx950).
//
// HBM bound, like the permutation by itself: the same bytes are read and written, and a pass over Q and K before it is saved.  A workgroup takes
// a block of rows through two heads, a wavefront 64 / (d / 8) rows at a time, d / 8 lanes to a row.  Cosines and sines belong to a token, so both
// heads have them from one calculation, which is about as much work as a head's rows themselves (one head at a time: 75,600 tokens of 40 heads
// 826 us, two 806, three 807; rf2_permute by itself 790).  Small layers, which the latency of a block bounds, ask for the
// rows of the next turn before they work on this one (4,301 tokens of 12 heads 18.7 -> 15.6 us); elsewhere the registers that it takes cost
// wavefronts (64 channels, 32,760 tokens of 40 heads 191 -> 207).
#include "rf2_permute_rows.h"
#include "rf2_rope.h"

namespace {

struct PermuteRopeArgs {
  PermuteArgs p;
  RopeArgs rope;
  const int32_t* pos;
  int64_t pos_batch;
  const void *w[2], *w_text[2];      // of Q and K; of the tokens behind the grid's
  int video;                         // tokens of the grid
  int norm;
  uint32_t groups;                   // of heads
};

constexpr int HEADS = 2;

template <bool KEEP>
__device__ __forceinline__ rope_u32x4 ld_row(const u16* p) {
  if constexpr (KEEP) return *reinterpret_cast<const rope_u32x4*>(p);
  else return __builtin_nontemporal_load(reinterpret_cast<const rope_u32x4*>(p));
}
template <bool KEEP>
__device__ __forceinline__ void st_row(u16* p, const rope_u32x4& v) {
  if constexpr (KEEP) *reinterpret_cast<rope_u32x4*>(p) = v;
  else __builtin_nontemporal_store(v, reinterpret_cast<rope_u32x4*>(p));
}

template <int D>
struct rope_lds {
  float weights[2][D], sums[4][HEADS][D];        // weights of the grid's tokens, and of the text
};

// Rows of a block of Q (row by row) or K (operand parts, see rf2.h), HEADS heads from h0 on.
template <int D, bool IS_K, bool HALVES, bool NORM, int KEEP, bool RAGGED>
__device__ __forceinline__ void rope_rows_of(const PermuteRopeArgs& a, int rows, int n_blocks, int last_valid, int blk, int b, int h0,
                                           rope_lds<D>& lds) {
  constexpr int CH = D / 8, ROWS = 64 / CH;                 // rows of a wavefront
  const PermuteArgs& p = a.p;
  const u16* const x = reinterpret_cast<const u16*>(IS_K ? p.k : p.q) + (int64_t)b * p.st.batch * D;
  u16* const xp = reinterpret_cast<u16*>(IS_K ? p.kp : p.qp);
  float* const mean = IS_K ? p.kbar : p.qbar;
  const int heads = min(HEADS, p.heads - h0);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane % CH, g = lane / CH;
  const int half = rows / 2;
  const RopeLane angles = rope_lane<D, HALVES>(a.rope, c);
  if constexpr (NORM) {
    // (a row's lanes turn them into 32 bits, the first those of the grid, the next those of the text)
    if (threadIdx.x < 2 * CH) {
      float own[8];
      rope_weights<RopeBf16>(a.rope, threadIdx.x < CH || !a.w_text[IS_K] ? a.w[IS_K] : a.w_text[IS_K], threadIdx.x % CH, own);
#pragma unroll
      for (int e = 0; e < 8; ++e) lds.weights[threadIdx.x / CH][8 * (threadIdx.x % CH) + e] = own[e];
    }
    __syncthreads();
  }
  float sum[HEADS][8] = {};
  // Turns of ROWS rows, whose loads are asked for a turn ahead, their places two turns.
  const int turns = rows / (4 * ROWS);
  const auto row0 = [&](int turn) { return D == 128 ? 8 * wave + 32 * (turn / 2) + 4 * (turn % 2) : 8 * wave + 32 * turn; };
  const auto entry = [&](int turn) { return p.perm[blk * rows + row0(min(turn, turns - 1)) + g]; };
  rope_u32x4 v[HEADS], before[HEADS];
  RopePlace place;
  const auto ask = [&](int n) {
    const int at = RAGGED ? max(n, 0) : n;
    const u16* const from = x + (h0 * p.st.head + (int64_t)at * p.st.token) * D + 8 * c;
#pragma unroll
    for (int i = 0; i < HEADS; ++i) v[i] = ld_row<KEEP == 2>(from + min(i, heads - 1) * p.st.head * D);
    place = rope_place(a.rope, angles, a.pos + b * a.pos_batch + (int64_t)at * a.rope.axes);
    if constexpr (RAGGED) {
#pragma unroll
      for (int i = 0; i < HEADS; ++i)
        if (n < 0) v[i] = rope_u32x4{0, 0, 0, 0};
    }
  };
  constexpr bool AHEAD = KEEP == 2;
  int n = entry(0), next = entry(1);
  if constexpr (AHEAD) ask(n);
#pragma unroll 1
  for (int turn = 0; turn < turns; ++turn) {
    if constexpr (!AHEAD) ask(n);
    float A[8], B[8], own[8], other[8];
    if constexpr (NORM) {
      const float* const w = lds.weights[n >= a.video ? 1 : 0];
#pragma unroll
      for (int e = 0; e < 8; ++e) own[e] = w[8 * c + e];
      if constexpr (HALVES)
#pragma unroll
        for (int e = 0; e < 8; ++e) other[e] = w[8 * (c ^ (CH / 2)) + e];
    }
    rope_factors<D, HALVES, NORM>(angles, place, own, other, c, A, B);
    rope_u32x4 now[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) now[i] = v[i];
    const bool behind = n < 0;
    n = next;
    if constexpr (AHEAD) ask(n);
    next = entry(turn + 2);
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
      float y[8];
      RopeBf16::unpack(now[i], y);
      rope_row<D, HALVES, NORM>(a.rope, A, B, y);
      if constexpr (RAGGED) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = behind ? 0.f : y[e];      // rows behind the last are 0: not -0, and whatever the weights are
      }
      now[i] = RopeBf16::pack(y);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[i][e] += y[e];
    }
    const auto to = [&](int i) { return xp + ((int64_t)(b * p.heads + h0 + i) * n_blocks + blk) * rows * D; };
    const auto k_slot = [&](int r, int chunk) { return ((r % half) / 32 * CH + chunk) * 64 + r / half * 32 + r % 32; };
    if constexpr (IS_K && D == 128) {
      // K: the upper chunks of four rows against the lower ones of the next four: a store then covers eight rows of eight chunks, whole lines
      // of 128 bytes (half lines: 358 us for K of 75,600 tokens of 40 heads, whole ones 281).
      if (turn % 2 == 0) {
#pragma unroll
        for (int i = 0; i < HEADS; ++i) before[i] = now[i];
      } else {
        const int r = row0(turn - 1) + 4 * (c / 8) + g;
#pragma unroll
        for (int i = 0; i < HEADS; ++i)
          if (i < heads) {
            rope_u32x4 low, high;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t first = before[i][e], second = now[i][e];
              low[e] = (uint32_t)__builtin_amdgcn_update_dpp((int)first, (int)second, 0x128, 0xf, 0xc, false);      // row_ror:8 into lanes 8-15
              high[e] = (uint32_t)__builtin_amdgcn_update_dpp((int)second, (int)first, 0x128, 0xf, 0x3, false);     // and into lanes 0-7
            }
            st_row<KEEP >= 1>(to(i) + k_slot(r, c % 8) * 8, low);
            st_row<KEEP >= 1>(to(i) + k_slot(r, 8 + c % 8) * 8, high);
          }
      }
    } else {
      const int r = row0(turn) + g;
#pragma unroll
      for (int i = 0; i < HEADS; ++i)
        if (i < heads) st_row<KEEP >= 1>(to(i) + (IS_K ? k_slot(r, c) : r * CH + c) * 8, now[i]);
    }
  }
  if (mean == nullptr) return;
  // the wavefront's rows are added lane by lane, the wavefronts' sums in LDS: a fixed order
#pragma unroll
  for (int i = 0; i < HEADS; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (D == 64) sum[i][e] += rope_dpp<0x128>(sum[i][e]);
      sum[i][e] += __shfl_xor(sum[i][e], 16);
      sum[i][e] += __shfl_xor(sum[i][e], 32);
    }
  if (lane < CH) {
#pragma unroll
    for (int i = 0; i < HEADS; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) lds.sums[wave][i][8 * c + e] = sum[i][e];
  }
  __syncthreads();
  const int count = blk == n_blocks - 1 ? last_valid : rows;
  for (int i = threadIdx.x; i < heads * D; i += 256) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) s += lds.sums[w][i / D][i % D];
    mean[((int64_t)(b * p.heads + h0 + i / D) * n_blocks + blk) * D + i % D] = s / (float)count;
  }
}

template <int D, bool IS_K, bool HALVES, int KEEP>
__device__ __forceinline__ void rope_block(const PermuteRopeArgs& a, int rows, int n_blocks, int last_valid, int blk, int b, int h0, rope_lds<D>& lds) {
  const auto with = [&](auto norm) {
    // (a block with rows behind the last one has code of its own, which costs the others no registers)
    if (blk == n_blocks - 1 && last_valid < rows) rope_rows_of<D, IS_K, HALVES, norm(), KEEP, true>(a, rows, n_blocks, last_valid, blk, b, h0, lds);
    else rope_rows_of<D, IS_K, HALVES, norm(), KEEP, false>(a, rows, n_blocks, last_valid, blk, b, h0, lds);
  };
  a.norm ? with(std::true_type()) : with(std::false_type());
}

// First the Q blocks, then the K blocks, then V's parts, as in the permutation by itself.
template <int D, int BK, bool HALVES, int KEEP>
__global__ void __launch_bounds__(256) permute_rope_kernel(PermuteRopeArgs a, int q_rows) {
  __shared__ __attribute__((aligned(16))) union { rope_lds<D> rope; v_rows<D> tile; } lds;
  const PermuteArgs& p = a.p;
  uint32_t id = blockIdx.y * gridDim.x + blockIdx.x;
  if (id < p.q_wgs) {
    const uint32_t at = id / p.n_q, blk = id - at * p.n_q, b = at / a.groups, h0 = (at - b * a.groups) * HEADS;
    rope_block<D, false, HALVES, KEEP>(a, q_rows, p.n_q, p.last_q, blk, b, h0, lds.rope);
    return;
  }
  id -= p.q_wgs;
  if (id < p.k_wgs) {
    const uint32_t at = id / p.n_k, blk = id - at * p.n_k, b = at / a.groups, h0 = (at - b * a.groups) * HEADS;
    rope_block<D, true, HALVES, KEEP>(a, BK, p.n_k, p.last_k, blk, b, h0, lds.rope);
    return;
  }
  id -= p.k_wgs;
  const uint32_t parts = p.n_k * (BK / 64);
  if (id < p.v_wgs) permute_vtile_part<D, BK, KEEP>(p.v, p.vp, p.perm, p.n_k, p.heads, p.st, id % parts, id / parts, lds.tile);
}

// V's parts by themselves, for large layers: they have no use for the registers of the others (75,600 tokens of 40 heads: 250 us with eight
// wavefronts to a SIMD, 320 with four).
template <int D, int BK, int KEEP>
__global__ void __launch_bounds__(256) permute_v_kernel(PermuteArgs p) {
  __shared__ __attribute__((aligned(16))) v_rows<D> tile;
  const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x, parts = p.n_k * (BK / 64);
  if (id < p.v_wgs) permute_vtile_part<D, BK, KEEP>(p.v, p.vp, p.perm, p.n_k, p.heads, p.st, id % parts, id / parts, tile);
}

template <int D, int BK>
int launch(const rf2_plan* plan, PermuteRopeArgs a, bool halves, uint32_t q_wgs, uint32_t k_wgs, uint32_t v_wgs, hipStream_t st) {
  const auto grid = [](uint32_t n) {
    const uint32_t rows = (n + 65535u) / 65536u;
    return dim3((n + rows - 1) / rows, rows);
  };
  const int keep = rf2_permute_keep(plan, a.p.bh);
  const bool apart = keep == 0 && v_wgs > 0;
  a.p.q_wgs = q_wgs, a.p.k_wgs = k_wgs, a.p.v_wgs = v_wgs;
  if (apart) {
    permute_v_kernel<D, BK, 0><<<grid(v_wgs), 256, 0, st>>>(a.p);
    RF2_LAUNCH_CHECK();
    a.p.v_wgs = 0;
  }
  if (q_wgs + k_wgs + a.p.v_wgs == 0) return RF2_OK;
  const auto with = [&](auto kernel) { kernel<<<grid(q_wgs + k_wgs + a.p.v_wgs), 256, 0, st>>>(a, plan->cfg.block); };
  if (halves) {
    if (keep == 2) with(permute_rope_kernel<D, BK, true, 2>);
    else if (keep == 1) with(permute_rope_kernel<D, BK, true, 1>);
    else with(permute_rope_kernel<D, BK, true, 0>);
  } else {
    if (keep == 2) with(permute_rope_kernel<D, BK, false, 2>);
    else if (keep == 1) with(permute_rope_kernel<D, BK, false, 1>);
    else with(permute_rope_kernel<D, BK, false, 0>);
  }
  RF2_LAUNCH_CHECK();
  return RF2_OK;
}

template <int D, int BK>
int permute_rope(const rf2_plan* plan, const PermuteRopeArgs& a, bool halves, hipStream_t st) {
  const uint32_t both = (uint32_t)plan->cfg.batch * a.groups, q = a.p.n_q * both, k = a.p.n_k * both, v = a.p.n_k * a.p.bh * (BK / 64);
  if (!tensors_overlap(plan, a.p)) return launch<D, BK>(plan, a, halves, q, k, v, st);
  if (const int rc = launch<D, BK>(plan, a, halves, q, 0, 0, st)) return rc;
  if (const int rc = launch<D, BK>(plan, a, halves, 0, k, 0, st)) return rc;
  return launch<D, BK>(plan, a, halves, 0, 0, v, st);
}

}  // namespace

extern "C" int rf2_permute_rope(const rf2_plan* plan, const rf2_rope_plan* rope, const void* q, const void* k, const void* v, const int32_t* pos,
                                int64_t pos_batch, const void* wq, const void* wk, const void* wq_text, const void* wk_text, void* qp, void* kp,
                                void* vp, float* qbar, float* kbar, void* stream) {
  if (!plan || !rope || !q || !k || !v || !qp || !kp || !vp || pos_batch < 0 || pos_batch > (int64_t)1 << 32) return RF2_ERR_INVALID_ARG;
  if ((qbar == nullptr) != (kbar == nullptr)) return RF2_ERR_INVALID_ARG;
  const rf2_rope_config& r = rope->cfg;
  if (r.heads != plan->cfg.heads || r.kv_heads != plan->cfg.heads || r.head_dim != plan->cfg.head_dim || r.dtype != RF2_DTYPE_BF16 ||
      rope->device != plan->device)
    return RF2_ERR_INVALID_ARG;
  if (!rf2_rope_pos_fits(rope, pos) || !rf2_rope_weight_fits(rope, wq) || !rf2_rope_weight_fits(rope, wk)) return RF2_ERR_INVALID_ARG;
  if ((wq_text == nullptr) != (wk_text == nullptr)) return RF2_ERR_INVALID_ARG;
  if (wq_text && (!rf2_rope_weight_fits(rope, wq_text) || !rf2_rope_weight_fits(rope, wk_text))) return RF2_ERR_INVALID_ARG;
  for (const void* t : {q, k, v, (const void*)qp, (const void*)kp, (const void*)vp})
    if (!rf2_rope_aligned(t, 16)) return RF2_ERR_INVALID_ARG;
  if (!rf2_rope_aligned(qbar, 4) || !rf2_rope_aligned(kbar, 4)) return RF2_ERR_INVALID_ARG;
  if (const int rc = rf2_check_device(plan)) return rc;
  const rf2_info& in = plan->info;
  const PermuteRopeArgs a{{(const uint4*)q, (const uint4*)k, (const uint4*)v, (uint4*)qp, (uint4*)kp, (uint4*)vp, qbar, kbar, plan->d_perm,
                           (uint32_t)in.n_blocks, (uint32_t)in.n_blocks_k, (uint32_t)(plan->cfg.batch * plan->cfg.heads), 0, 0, 0,
                           in.last_block_valid, in.last_block_valid_k, plan->cfg.heads, rf2_qkv_strides(plan)},
                          rope_args(rope), pos, pos_batch, {wq, wk}, {wq_text, wk_text}, (int)(in.N - plan->cfg.text_tokens),
                          r.norm == RF2_NORM_RMS, (uint32_t)((plan->cfg.heads + HEADS - 1) / HEADS)};
  const bool halves = r.pairing == RF2_ROPE_HALVES;
  hipStream_t st = (hipStream_t)stream;
  if (plan->cfg.head_dim == 128) return in.block_k == 128 ? permute_rope<128, 128>(plan, a, halves, st) : permute_rope<128, 64>(plan, a, halves, st);
  return in.block_k == 128 ? permute_rope<64, 128>(plan, a, halves, st) : permute_rope<64, 64>(plan, a, halves, st);
}
