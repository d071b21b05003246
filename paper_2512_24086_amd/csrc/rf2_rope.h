// Norms of heads' rows and rotation by positions: the plan, and what the kernels that do it share (not installed).
#pragma once
#include <algorithm>
#include <type_traits>

#include "rf2_internal.h"

// Of each pair of channels, turns per unit of its axis' position, whole turns left out, in units of 2^-32 (rounded to the nearest) and what is
// left of them in units of 2^-64 (to the nearest too); and the axis.  A lane reads those of its pairs in a few wide loads.
struct rf2_rope_table {
  int32_t turns[64], rest[64];
  uint8_t axis[64];
};

struct rf2_rope_plan {
  rf2_rope_config cfg;
  rf2_rope_info info;
  int device;
  rf2_rope_table* d_table;  // device, two: the second one turns the other way
};

// The sums of the weights' gradients: so many workgroups for each of Q and K at most, head_dim numbers of 32 bits from each, and so many runs of
// them, in 64 bits.
constexpr int RF2_ROPE_PARTS = 8192, RF2_ROPE_RUNS = 128, RF2_ROPE_FEW = 512, RF2_ROPE_MANY = 2048;
struct RopeWorkspace {
  int64_t sums, runs;        // in bytes, of Q (side 0) or K
};
inline RopeWorkspace rope_workspace(int head_dim, int side) {
  const int64_t sums = (int64_t)RF2_ROPE_PARTS * head_dim * 4, runs = (int64_t)RF2_ROPE_RUNS * head_dim * 8;
  return {side * sums, 2 * sums + side * runs};
}
inline int64_t rf2_rope_workspace(int head_dim) { return rope_workspace(head_dim, 2).runs; }

inline bool rf2_rope_aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

inline int rf2_check_rope_device(const rf2_rope_plan* plan) {
  if (plan->device < 0) return rf2_note_hip_error(hipErrorNoDevice);
  int current = -1;
  const hipError_t e = hipGetDevice(&current);
  if (e != hipSuccess) return rf2_note_hip_error(e);
  return current == plan->device ? RF2_OK : RF2_ERR_INVALID_ARG;
}

// Whether weights go with a plan: all of those that a norm needs, aligned for loads of 16 bytes, and none without a norm.
inline bool rf2_rope_weight_fits(const rf2_rope_plan* plan, const void* w) {
  return plan->cfg.norm == RF2_NORM_RMS ? w && rf2_rope_aligned(w, 16) : !w;
}
inline bool rf2_rope_pos_fits(const rf2_rope_plan* plan, const int32_t* pos) {
  return plan->cfg.axes == 0 || (pos && rf2_rope_aligned(pos, 4));
}

namespace {

// What the kernels read of a plan.
struct RopeArgs {
  const rf2_rope_table* table;
  int axes, weights_f32;
  float eps;
};
inline RopeArgs rope_args(const rf2_rope_plan* p, bool inverse = false) {
  return {p->d_table + (inverse ? 1 : 0), p->cfg.axes, p->cfg.weight_dtype == RF2_DTYPE_F32, p->cfg.eps};
}

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t rope_u32x4;

// Eight channels of a row, 16 bytes, as 32-bit numbers and back (to the nearest, ties to even: off by half a step at most).
struct RopeBf16 {
  typedef __attribute__((ext_vector_type(2))) __bf16 x2;
  static __device__ __forceinline__ void unpack(const rope_u32x4& v, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ rope_u32x4 pack(const float (&x)[8]) {
    rope_u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x[2 * i], x[2 * i + 1]}, x2));
    return v;
  }
};
struct RopeF16 {
  typedef __attribute__((ext_vector_type(2))) _Float16 x2;
  static __device__ __forceinline__ void unpack(const rope_u32x4& v, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t both = v[i];              // (a bit cast of a vector's element takes its first one)
      const x2 two = __builtin_bit_cast(x2, both);
      x[2 * i] = (float)two.x;
      x[2 * i + 1] = (float)two.y;
    }
  }
  static __device__ __forceinline__ rope_u32x4 pack(const float (&x)[8]) {
    rope_u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x[2 * i], x[2 * i + 1]}, x2));
    return v;
  }
};

// CH = D / 8 neighbouring lanes hold a row, lane c of them channels 8c to 8c + 7.
template <int CTRL>
__device__ __forceinline__ float rope_dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
// Sum over the lanes of a row, in each of them (neighbours, pairs, quads, groups of eight mirrored).
template <int D>
__device__ __forceinline__ float rope_row_sum(float x) {
  x += rope_dpp<0xB1>(x);
  x += rope_dpp<0x4E>(x);
  x += rope_dpp<0x141>(x);
  if constexpr (D == 128) x += rope_dpp<0x140>(x);
  return x;
}
// The value of the lane that holds the channels d/2 away.
template <int D>
__device__ __forceinline__ float rope_other_half(float x) {
  if constexpr (D == 128) return rope_dpp<0x128>(x);
  else return rope_dpp<0x1B>(rope_dpp<0x141>(x));
}
// The eight channels that a lane's channels are paired with.
template <int D, bool HALVES>
__device__ __forceinline__ void rope_partners(const float (&x)[8], float (&y)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = HALVES ? rope_other_half<D>(x[e]) : x[e ^ 1];
}

// What a lane keeps of the frequencies: of its four pairs (HALVES: the lanes of a pair's two channels have the same eight pairs, of which each
// has four), turns per unit of position and where the position is among a token's.
struct RopeLane {
  int32_t turns[4], rest[4], axis[4];
};
template <int D, bool HALVES>
__device__ __forceinline__ RopeLane rope_lane(const RopeArgs& a, int c) {
  const int pair = HALVES ? 8 * c - (c >= D / 16 ? D / 2 - 4 : 0) : 4 * c;
  const int4 t = *reinterpret_cast<const int4*>(a.table->turns + pair), r = *reinterpret_cast<const int4*>(a.table->rest + pair);
  const uint32_t axes = *reinterpret_cast<const uint32_t*>(a.table->axis + pair);
  return {{t.x, t.y, t.z, t.w}, {r.x, r.y, r.z, r.w}, {(int)(axes & 255), (int)(axes >> 8 & 255), (int)(axes >> 16 & 255), (int)(axes >> 24)}};
}
struct RopePlace {
  int32_t at[4];
};
// A token's positions for a lane's pairs (without axes nothing turns, whatever is read).
__device__ __forceinline__ RopePlace rope_place(const RopeArgs& a, const RopeLane& lane, const int32_t* __restrict__ pos) {
  const int32_t* const from = a.axes > 0 ? pos : reinterpret_cast<const int32_t*>(a.table);
  return {{from[lane.axis[0]], from[lane.axis[1]], from[lane.axis[2]], from[lane.axis[3]]}};
}

// Cosine and signed sine for each of a lane's channels: channel c turns to x_c cs_c + x_partner sn_c.
// Position times frequency in whole numbers, of which the carries out of 32 bits are whole turns and fall away: what is left is the angle's
// fraction of a turn with a sign.  At any position it is off by 1.5 2^-32 of one at most: cut off below 2^-32, a frequency half of 2^-64 off, and half
// of 2^-64 more where it comes from a base of 1 or more (a smaller base has frequencies above 1, in 64 bits: (|ln f| + 2) f 2^-64 radians).  In 32 bits
// (2^-26 turns off at most) it goes to the hardware's sine and cosine (off by 1.3e-7 at most, measured over 2^20 angles; 3.5e-8 on average, where
// rounding to 32 bits alone is 1.5e-8).
template <int D, bool HALVES>
__device__ __forceinline__ void rope_angles(const RopeLane& lane, const RopePlace& place, int c, float (&cs)[8], float (&sn)[8]) {
  float co[4], si[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t high = (int64_t)((uint64_t)((uint32_t)place.at[i] * (uint32_t)lane.turns[i]) << 32);
    const int64_t turns = (int64_t)((uint64_t)((int64_t)place.at[i] * lane.rest[i]) + (uint64_t)high);
    const float part = (float)(int32_t)(turns >> 32) * 0x1p-32f;
    co[i] = __builtin_amdgcn_cosf(part), si[i] = __builtin_amdgcn_sinf(part);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (HALVES) {
      const bool upper = c >= D / 16;
      const float other_co = rope_other_half<D>(co[i]), other_si = rope_other_half<D>(si[i]);
      cs[i] = upper ? other_co : co[i];
      cs[4 + i] = upper ? co[i] : other_co;
      sn[i] = upper ? other_si : -si[i];
      sn[4 + i] = upper ? si[i] : -other_si;
    } else {
      cs[2 * i] = cs[2 * i + 1] = co[i];
      sn[2 * i] = -si[i];
      sn[2 * i + 1] = si[i];
    }
  }
}

// A lane's weights.
template <class T>
__device__ __forceinline__ void rope_weights(const RopeArgs& a, const void* __restrict__ w, int c, float (&x)[8]) {
  if (a.weights_f32) {
    const float4 u = reinterpret_cast<const float4*>(w)[2 * c], v = reinterpret_cast<const float4*>(w)[2 * c + 1];
    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
  } else {
    T::unpack(reinterpret_cast<const rope_u32x4*>(w)[c], x);
  }
}

// Weights and angles in one: channel c of a row x, normalised, becomes x_c A_c + x_partner B_c, A = w_c cos, B = -+ w_partner sin.
template <int D, bool HALVES, bool NORM>
__device__ __forceinline__ void rope_factors(const RopeLane& lane, const RopePlace& place, const float (&own)[8], const float (&other)[8], int c,
                                             float (&A)[8], float (&B)[8]) {
  rope_angles<D, HALVES>(lane, place, c, A, B);
  if constexpr (NORM) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      A[e] *= own[e];
      B[e] *= HALVES ? other[e] : own[e ^ 1];
    }
  }
}
template <class T, int D, bool HALVES, bool NORM>
__device__ __forceinline__ void rope_factors(const RopeArgs& a, const RopeLane& lane, const RopePlace& place, const void* __restrict__ w, int c,
                                             float (&A)[8], float (&B)[8]) {
  float own[8], other[8];
  if constexpr (NORM) rope_weights<T>(a, w, c, own);
  if constexpr (NORM && HALVES) rope_weights<T>(a, w, c ^ (D / 16), other);
  rope_factors<D, HALVES, NORM>(lane, place, own, other, c, A, B);
}

// x becomes x / sqrt(mean(x^2) + eps); returns the factor.  A row whose squares leave 32 bits is made smaller first, by a power of two (next to
// it eps is nothing).
template <int D>
__device__ __forceinline__ float rope_squares(const float (&x)[8]) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(x[e], x[e], s);
  return rope_row_sum<D>(s);
}
template <int D>
__device__ __forceinline__ float rope_normalise(const RopeArgs& a, float (&x)[8]) {
  float s = rope_squares<D>(x), eps = a.eps, less = 1.f;
  if (__builtin_amdgcn_ballot_w64(!(s < 0x1p120f)) != 0) {       // (the whole wavefront or none of it: a factor of 1 changes nothing)
    less = s < 0x1p120f ? 1.f : 0x1p-70f;
    eps = s < 0x1p120f ? eps : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= less;
    s = rope_squares<D>(x);
  }
  const float r = __builtin_amdgcn_rsqf(fmaf(s, 1.f / D, eps));
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= r;
  return r * less;
}

// A row's channels in 32 bits, normalised, weighted and rotated.
template <int D, bool HALVES, bool NORM>
__device__ __forceinline__ void rope_row(const RopeArgs& a, const float (&A)[8], const float (&B)[8], float (&x)[8]) {
  if constexpr (NORM) rope_normalise<D>(a, x);
  float y[8];
  rope_partners<D, HALVES>(x, y);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = fmaf(y[e], B[e], x[e] * A[e]);
}

// Rows of a tensor, in elements.
struct RopeRows {
  const uint16_t* at;
  int64_t batch, token, head;
};

// How wavefronts share rows: one takes 2^heads_log2 neighbouring heads (they divide all) of as many tokens as that leaves rows for, and goes on
// through the heads, `steps` times; `groups` of them have the same tokens.  Workgroups that start one after the other have neighbouring
// groups of the same four wavefronts' tokens, a tile, or neighbouring tiles.
struct RopeShare {
  int heads, heads_log2, steps, groups;
  uint32_t tiles, fast, inverse;     // fast: groups or tiles; inverse: (2^32 - 1) / fast
};
// Rows of Q or of K, in and out.
struct RopeSide {
  RopeRows x, z;
  const void* w;
  RopeShare share;
};
struct RopeUnit {
  uint32_t tile, group;
};
__device__ __forceinline__ RopeUnit rope_unit(const RopeShare& s, uint32_t id) {
  uint32_t slow = __umulhi(id, s.inverse), fast = id - slow * s.fast;      // id / fast, or one less (a division: 525 us in place of 512 for 75,600 tokens of 40 + 40 heads)
  if (fast >= s.fast) ++slow, fast -= s.fast;
  return s.fast == (uint32_t)s.groups ? RopeUnit{slow, fast} : RopeUnit{fast, slow};
}
// Tokens and their positions.
struct RopeTokens {
  const int32_t* pos;
  int64_t pos_batch;
  uint32_t tokens, total;    // of an element of the batch, of all
};
template <bool KEEP>
__device__ __forceinline__ rope_u32x4 rope_load(const uint16_t* p) {
  if constexpr (KEEP) return *reinterpret_cast<const rope_u32x4*>(p);
  else return __builtin_nontemporal_load(reinterpret_cast<const rope_u32x4*>(p));
}
template <bool KEEP>
__device__ __forceinline__ void rope_store(uint16_t* p, const rope_u32x4& v) {
  if constexpr (KEEP) *reinterpret_cast<rope_u32x4*>(p) = v;
  else __builtin_nontemporal_store(v, reinterpret_cast<rope_u32x4*>(p));
}

// Token m of all, as an element of the batch and a token of it.
struct RopeToken {
  uint32_t b, n;
};
__device__ __forceinline__ RopeToken rope_token(uint32_t m, uint32_t tokens, uint32_t total) {
  if (tokens == total) return {0, m};
  const uint32_t b = m / tokens;
  return {b, m - b * tokens};
}

// What workgroup `id` of 256 threads does of a side: a tile of tokens through a group of heads.
template <class T, int D, bool HALVES, bool NORM, bool KEEP>
__device__ __forceinline__ void rope_apply_rows(const RopeArgs& a, const RopeTokens& t, const RopeSide& s, uint32_t id) {
  constexpr int CH = D / 8, R = 64 / CH, U = 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane % CH, g = lane / CH;
  const RopeUnit unit = rope_unit(s.share, id);
  const int log2 = s.share.heads_log2, by_token = R >> log2;
  const uint32_t m = (unit.tile * 4 + wave) * by_token + (g >> log2);
  if (m >= t.total) return;
  const RopeToken token = rope_token(m, t.tokens, t.total);
  const int first = unit.group * s.share.steps, end = min(s.share.heads >> log2, first + s.share.steps);
  const int h = (first << log2) + (g & ((1 << log2) - 1));
  const uint16_t* from = s.x.at + token.b * s.x.batch + token.n * s.x.token + h * s.x.head + 8 * c;
  uint16_t* to = const_cast<uint16_t*>(s.z.at) + token.b * s.z.batch + token.n * s.z.token + h * s.z.head + 8 * c;
  const int64_t from_step = s.x.head << log2, to_step = s.z.head << log2;
  rope_u32x4 v[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (first + u < end) v[u] = rope_load<false>(from + u * from_step);
  const RopeLane angles = rope_lane<D, HALVES>(a, c);
  const RopePlace place = rope_place(a, angles, t.pos + token.b * t.pos_batch + (int64_t)token.n * a.axes);
  float A[8], B[8];
  rope_factors<T, D, HALVES, NORM>(a, angles, place, s.w, c, A, B);
  for (int step = first; step < end; step += U) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (step + u < end) {
        float x[8];
        T::unpack(v[u], x);
        rope_row<D, HALVES, NORM>(a, A, B, x);
        rope_store<KEEP>(to + u * to_step, T::pack(x));
      }
    from += U * from_step;
    to += U * to_step;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (step + U + u < end) v[u] = rope_load<false>(from + u * from_step);
  }
}

// ---- host -------------------------------------------------------------------------------------------------------

inline RopeRows rope_rows(const rf2_rows& r) { return {(const uint16_t*)r.at, r.batch, r.token, r.head}; }

// How many rows of a wavefront are neighbouring heads of a token (log2): where heads lie side by side, as many as divide all of them.
inline int rope_heads_log2(const rf2_rows& r, int heads, int rows) {
  if (r.head >= r.token) return 0;
  int log2 = 0;
  while (2 << log2 <= rows && heads % (2 << log2) == 0) ++log2;
  return log2;
}

// The share of each wavefront.  Angles are worked out once for all its steps (HALVES costs twice the exchange), loads of four steps are on their way
// together, and what is read at a time should lie close together.  Measured (us, steps of a wavefront):
//   heads side by side, 75,600 tokens x 40 + 40 heads      1: 641   2: 515   4 of 10: 511   5: 516   all: 541
//     64 channels, 32,760 tokens x 40 + 40                 4 of 5: 115   all: 109;   HALVES, 20,000 x 32 + 8   4 of 8: 75   all: 72
//   tokens side by side, 75,600 x 40 + 40                  1: 650   2: 496   3: 511   4: 518   8: 530   all: 582 (a copy of as much: 498)
//     HALVES, 32,760 x 40 + 40                             2: 254   4: 229   5: 221   8: 228   all: 245
//     4,096 x 12 + 12                                      2: 11.6  4: 9.5   8: 11.0;   1,000 x 40 + 40   2: 9.7   4: 8.1   all: 8.2
// With few rows a wavefront takes fewer, so that there are 2,048.
inline RopeShare rope_share(const rf2_rows& x, int heads, const rf2_rope_config& c, uint32_t tokens) {
  if (!x.at || tokens == 0) return {heads, 0, 1, 0, 0, 1, 0};
  const int rows = 512 / c.head_dim, log2 = rope_heads_log2(x, heads, rows), all_steps = heads >> log2;
  const int64_t wavefronts = (((int64_t)tokens << log2) + rows - 1) / rows, work = wavefronts * all_steps;
  const bool halves = c.pairing == RF2_ROPE_HALVES, along_tokens = x.token < x.head;
  const int most = along_tokens ? (halves ? 5 : work > 150000 ? 2 : 4) : halves ? 10 : 5;
  const int parts = (all_steps + most - 1) / most, even = along_tokens ? most : (all_steps + parts - 1) / parts;
  int steps = (int)std::min<int64_t>(std::min(even, all_steps), std::max<int64_t>(1, work / 2048));
  // (a grid has less than 2^32 threads: at most 2^22 tiles, and 2^23 workgroups of a side)
  while (steps < all_steps && (wavefronts + 3) / 4 * ((all_steps + steps - 1) / steps) >= (int64_t)1 << 22) steps = std::min(all_steps, 2 * steps);
  const int groups = (all_steps + steps - 1) / steps;
  const uint32_t tiles = (uint32_t)((wavefronts + 3) / 4), fast = along_tokens ? tiles : (uint32_t)groups;
  return {heads, log2, steps, groups, tiles, fast, UINT32_MAX / fast};
}
inline uint32_t rope_workgroups(const RopeShare& s) { return s.tiles * (uint32_t)s.groups; }

// Rows are read once and left to what reads them next.  Past the caches is the faster way (4,096 tokens, 10 + 10 heads, 42 MB: 7.5 us for 9.9,
// 134 MB: 23.2 for 25.1), but rows that the L2s hold are there for the next kernel (17 MB, with rf2_permute behind: 15.0 us for 13.1; 42 MB: 22.1 for
// 21.3).  So stores are kept up to 32 MiB, in bytes read and written.
constexpr int64_t ROPE_KEEP = (int64_t)32 << 20;

template <class F>
int rope_for_types(const rf2_rope_config& c, F f) {
  const auto pairing = [&](auto type, auto d) {
    if (c.pairing == RF2_ROPE_HALVES) f(type, d, std::true_type());
    else f(type, d, std::false_type());
  };
  const auto dim = [&](auto type) {
    if (c.head_dim == 128) pairing(type, std::integral_constant<int, 128>());
    else pairing(type, std::integral_constant<int, 64>());
  };
  if (c.dtype == RF2_DTYPE_F16) dim(RopeF16());
  else dim(RopeBf16());
  RF2_LAUNCH_CHECK();
  return RF2_OK;
}

}  // namespace
