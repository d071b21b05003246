// Norms of heads' rows and rotation by positions: the plan, and what the kernels that do it share (not installed).
#pragma once
#include <algorithm>
#include <type_traits>

#include "rf2_internal.h"

// A pair of channels: turns per unit of its axis' position.
struct rf2_rope_pair {
  double turns;
  int32_t axis, unused;
};

struct rf2_rope_plan {
  rf2_rope_config cfg;
  rf2_rope_info info;
  int device;
  rf2_rope_pair* d_pairs;  // device, 64 of them, and 64 that turn the other way
};

// The sums of the weights' gradients: so many workgroups for each of Q and K at most, head_dim numbers of 32 bits from each.
constexpr int RF2_ROPE_PARTS = 1024;
inline int64_t rf2_rope_workspace(int head_dim) { return (int64_t)2 * RF2_ROPE_PARTS * head_dim * 4; }

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
  const rf2_rope_pair* pairs;
  int axes, weights_f32;
  float eps;
};
inline RopeArgs rope_args(const rf2_rope_plan* p, bool inverse = false) {
  return {p->d_pairs + (inverse ? 64 : 0), p->cfg.axes, p->cfg.weight_dtype == RF2_DTYPE_F32, p->cfg.eps};
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

// Cosine and signed sine for each of a lane's channels: channel c turns to x_c cs_c + x_partner sn_c.
// The angle is taken in turns in 64 bits, less the nearest whole number, which leaves an error of 2^-22 turns at positions of 2^31 and
// frequencies of 1; sine and cosine of what is left are the hardware's, off by 1.3e-7 at most (measured over 2^20 angles: 3.5e-8 on average,
// where rounding to 32 bits alone is 1.5e-8).
template <int D, bool HALVES>
__device__ __forceinline__ void rope_angles(const RopeArgs& a, const int32_t* __restrict__ pos, int c, float (&cs)[8], float (&sn)[8]) {
#pragma clang fp contract(off)                  // (the kernels that share this are to give the same bits)
  constexpr int N = HALVES ? 8 : 4;
  int p[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < a.axes) p[i] = pos[i];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const rf2_rope_pair pair = a.pairs[HALVES ? (8 * c + i) % (D / 2) : 4 * c + i];
    const int at = pair.axis == 0 ? p[0] : pair.axis == 1 ? p[1] : pair.axis == 2 ? p[2] : p[3];
    const double turns = (double)at * pair.turns;
    const float part = (float)(turns - __builtin_rint(turns));
    const float co = __builtin_amdgcn_cosf(part), si = __builtin_amdgcn_sinf(part);
    if constexpr (HALVES) {
      cs[i] = co;
      sn[i] = c < D / 16 ? -si : si;
    } else {
      cs[2 * i] = cs[2 * i + 1] = co;
      sn[2 * i] = -si;
      sn[2 * i + 1] = si;
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
template <class T, int D, bool HALVES, bool NORM>
__device__ __forceinline__ void rope_factors(const RopeArgs& a, const int32_t* __restrict__ pos, const void* __restrict__ w, int c, float (&A)[8],
                                             float (&B)[8]) {
  if constexpr (NORM) {
    float own[8], other[8];
    rope_weights<T>(a, w, c, own);
    if constexpr (HALVES) rope_weights<T>(a, w, c ^ (D / 16), other);
    rope_angles<D, HALVES>(a, pos, c, A, B);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      A[e] *= own[e];
      B[e] *= HALVES ? other[e] : own[e ^ 1];
    }
  } else {
    rope_angles<D, HALVES>(a, pos, c, A, B);
  }
}

// x becomes x / sqrt(mean(x^2) + eps); returns the factor.  A row whose squares leave 32 bits is made smaller first, by a power of two (next to
// it eps is nothing).
template <int D>
__device__ __forceinline__ float rope_normalise(const RopeArgs& a, float (&x)[8]) {
  const auto squares = [&] {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x[e], x[e], s);
    return rope_row_sum<D>(s);
  };
  float s = squares(), r;
  if (s < 0x1p120f) {
    r = __builtin_amdgcn_rsqf(fmaf(s, 1.f / D, a.eps));
  } else {                                      // (all lanes of a row are here, or none)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= 0x1p-70f;
    r = __builtin_amdgcn_rsqf(squares() * (1.f / D));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= r;
    return r * 0x1p-70f;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= r;
  return r;
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

// Rows of Q or of K, in and out, and how wavefronts share them.
struct RopeSide {
  RopeRows x, z;                 // in, out
  const void* w;
  int heads, heads_log2;     // heads; log2 of the rows of a wavefront that are neighbouring heads
  int steps, groups;         // of heads a wavefront goes through, and wavefronts that share a token's heads
  uint32_t workgroups;
};

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

// What a workgroup of 256 threads does of a side: 4 * (64 / (d / 8)) rows at a time.
template <class T, int D, bool HALVES, bool NORM, bool KEEP>
__device__ __forceinline__ void rope_apply_rows(const RopeArgs& a, const RopeTokens& t, const RopeSide& s, uint32_t id) {
  constexpr int CH = D / 8, R = 64 / CH, U = 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane % CH, g = lane / CH;
  const int by_head = 1 << s.heads_log2, by_token = R >> s.heads_log2;
  const uint32_t tile = id / (uint32_t)s.groups, group = id - tile * (uint32_t)s.groups;
  const uint32_t m = (tile * 4 + wave) * by_token + (g >> s.heads_log2);
  if (m >= t.total) return;
  const RopeToken token = rope_token(m, t.tokens, t.total);
  int h = group * s.steps * by_head + (g & (by_head - 1));
  const int end = min(s.heads, (int)(group + 1) * s.steps * by_head);
  const uint16_t* from = s.x.at + token.b * s.x.batch + token.n * s.x.token + h * s.x.head + 8 * c;
  uint16_t* to = const_cast<uint16_t*>(s.z.at) + token.b * s.z.batch + token.n * s.z.token + h * s.z.head + 8 * c;
  const int64_t from_step = s.x.head * by_head, to_step = s.z.head * by_head;
  float A[8], B[8];
  bool first = true;
  while (h < end) {
    rope_u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h + u * by_head < end) v[u] = rope_load<KEEP>(from + u * from_step);
    if (first) {
      rope_factors<T, D, HALVES, NORM>(a, t.pos + token.b * t.pos_batch + (int64_t)token.n * a.axes, s.w, c, A, B);
      first = false;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h + u * by_head < end) {
        float x[8];
        T::unpack(v[u], x);
        rope_row<D, HALVES, NORM>(a, A, B, x);
        rope_store<KEEP>(to + u * to_step, T::pack(x));
      }
    h += U * by_head;
    from += U * from_step;
    to += U * to_step;
  }
}

// ---- host -------------------------------------------------------------------------------------------------------

inline RopeRows rope_rows(const rf2_rows& r) { return {(const uint16_t*)r.at, r.batch, r.token, r.head}; }

// How many rows of a wavefront are neighbouring heads of a token (log2): all where heads lie side by side and there are as many.
inline int rope_heads_log2(const rf2_rows& r, int heads, int rows) {
  if (r.head >= r.token) return 0;
  int log2 = 0;
  while (2 << log2 <= rows && 2 << log2 <= heads) ++log2;
  return log2;
}

// How the wavefronts of a launch share rows: `wavefronts` of tokens, `groups` of heads for each.
struct RopeShare {
  int heads_log2, steps, groups;
  uint32_t tiles;            // of four wavefronts' tokens
};
inline RopeShare rope_share(const rf2_rows& x, int heads, int head_dim, uint32_t tokens) {
  const int rows = 512 / head_dim, log2 = rope_heads_log2(x, heads, rows), by_head = 1 << log2, all_steps = (heads + by_head - 1) / by_head;
  const int64_t wavefronts = ((int64_t)tokens * by_head + rows - 1) / rows;
  const int steps = (int)std::min<int64_t>(all_steps, std::max<int64_t>(1, wavefronts * all_steps / 8192));
  return {log2, steps, (all_steps + steps - 1) / steps, (uint32_t)((wavefronts + 3) / 4)};
}
inline RopeSide rope_side(const rf2_rows& x, const rf2_rows& z, const void* w, int heads, int head_dim, uint32_t tokens) {
  const RopeShare s = rope_share(x, heads, head_dim, tokens);
  return {rope_rows(x), rope_rows(z), w, heads, s.heads_log2, s.steps, s.groups, x.at ? s.tiles * (uint32_t)s.groups : 0};
}

constexpr int64_t ROPE_KEEP = (int64_t)160 << 20;

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
