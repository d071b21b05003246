// Norms of heads' rows and rotation by positions: the plan, and what the kernels that do it share (not installed).
#pragma once
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

}  // namespace
