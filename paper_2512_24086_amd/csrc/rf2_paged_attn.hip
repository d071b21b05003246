// Attention of new tokens over a paged cache (gfx950).
//
// Rows.  The query heads that share a K/V head are rows side by side: row r of a sequence and K/V head h is token r / G,
// query head h G + r % G (G = heads / kv_heads), so a step of single tokens has G rows to a product and a chunk n G.  A
// workgroup owns a tile of these rows: 16 or 32 where a sequence has few (few_attn_kernel, bound by memory), 128 where it has
// many (many_attn_kernel, bound by the matrix cores).
//
// Parts.  A tile's keys are cut into parts of `units` units of 32 keys, counted from key 0 for all tiles of a sequence; the
// workgroups of one part of different tiles run at the same time and find each other's keys in the caches.  With
//     W = sum over sequences of tiles * units(length),   units >= max(least, W / aimed),
// a sequence that is cut (c = ceil(units(length) / units) >= 2) has c < 2 units(length) / units parts to a tile, all of them
// less than 2 W / units <= 2 aimed: the size of the workspace.  Few rows take the least such number; for many, and up to 64
// sequences, it is searched for (find_part).  The lengths are in device memory, so every workgroup works this out for itself
// and finds its own part: 2 to 4 us with up to 16 sequences, 5 with 64.  Above 256 sequences a launch before adds up what they have in
// common (survey_kernel).  The grid is the most there can be; workgroups without a part leave.
//
// Sums.  The sums of a tile that is cut go to the workspace in fp32; its first part lists its rows there (Joint), and a second
// launch, join_kernel, adds what is listed in the order of the parts: no atomics, the same bits each time.
//
// Products: S^T = K Q^T, O^T = V^T P^T, operands from the cache's tiles straight into registers, 1 KiB an instruction; P is what
// the accumulators of S^T hold: the cache's order of keys is theirs.  P is rounded to the type of V, half a step as V's own values
// are, for products of fp32 run at a sixteenth of the rate; O once, when it is whole.
//
// Softmax: a probability is exp2(q.k c - m), c = scale log2(e), with a reference m per row that is moved only when the sum
// of a unit's probabilities leaves the range that P's type carries: no maximum per unit, and O is hardly ever rescaled.  Sums are
// fp32, of unrounded P.
#include "rf2_paged_parts.h"

#include <cfloat>
#include <type_traits>

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

struct Bf16 {
  typedef bf16x8 x8;
  typedef bf16x4 x4;
  typedef bf16x2 x2;
  typedef __bf16 x1;
  // P = exp2(x - m): bf16 and fp32 carry 2^40 as well as 1
  static constexpr float RANGE = 1.0995e12f, HEAD = 0.f;
  static constexpr uint32_t EXPONENT = 0x7f80, MANTISSA = 0x7f;
  static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x4 mfma16(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  template <bool ACC>
  static __device__ __forceinline__ void qk(f32x16& s, const x8& a, const x8& b, bool first) {
    if constexpr (ACC) {
      if (first) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "a"(b));
      else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "a"(b));
    } else {
      if (first) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "v"(b));
      else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "v"(b));
    }
  }
};
struct F16 {
  typedef f16x8 x8;
  typedef f16x4 x4;
  typedef f16x2 x2;
  typedef _Float16 x1;
  // fp16 ends at 65,504 and loses its steps below 2^-14: the largest P stands at 2^8 when the reference is set (HEAD), may grow to
  // 2^15, and what is rounded away below 2^-25 is 2^-33 of it
  static constexpr float RANGE = 32768.f, HEAD = 8.f;
  static constexpr uint32_t EXPONENT = 0x7c00, MANTISSA = 0x3ff;
  static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x4 mfma16(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  template <bool ACC>
  static __device__ __forceinline__ void qk(f32x16& s, const x8& a, const x8& b, bool first) {
    if constexpr (ACC) {
      if (first) asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "a"(b));
      else asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "a"(b));
    } else {
      if (first) asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "v"(b));
      else asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "v"(b));
    }
  }
};

template <int ROWS, int D>
__device__ __forceinline__ float* part_sums(const Args& a, int place) { return a.parts + 8 * (a.most_joints + 1) + (int64_t)place * (ROWS * D); }
template <int ROWS, int D>
__device__ __forceinline__ float2* part_stats(const Args& a, int place) {
  return (float2*)(a.parts + 8 * (a.most_joints + 1) + (int64_t)a.places * (ROWS * D)) + (int64_t)place * ROWS;
}

// Where the sum of channel ch (a multiple of 2) of row r of a tile lies.  Few rows: row by row.  Many: as the accumulators of
// v_mfma_f32_32x32x16 have it, so that a wavefront stores 1 KiB at a time: four channels of 32 rows side by side.
template <int ROWS, int D>
__device__ __forceinline__ int part_at(int r, int ch) {
  return ROWS < RF2_PAGED_ROWS_MANY ? r * D + ch : (r / 32 * (D / 4) + ch / 4) * 128 + r % 32 * 4 + ch % 4;
}

// Keys that row r of a sequence sees.
__device__ __forceinline__ int limit_of(const Args& a, const Seq& s, int row) {
  return a.causal ? min(max(s.len - s.n_new + token_of(a, row) + 1, 0), s.len) : s.len;
}
// Units of a tile whose rows end before row `end`, and parts of it.
template <int ROWS>
__device__ __forceinline__ int tile_units(const Args& a, const Part& w) {
  return units_of(limit_of(a, w.s, min(w.s.n_new * a.group, (w.tile + 1) * ROWS) - 1));
}

__device__ __forceinline__ const unsigned char* uniform_ptr(const void* p) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (const unsigned char*)(((uint64_t)hi << 32) | lo);
}

// Place of 16-byte chunk `chunk` of row `row` among rows of CPR chunks in LDS: 16 lanes that move the same chunk of neighbouring
// rows, or the chunks of a row in turn, meet different banks.
template <int CPR>
__device__ __forceinline__ int row_slot(int row, int chunk) {
  return row * CPR + (chunk ^ (row / (16 / CPR) % CPR));
}

// What a wavefront of a part does.
struct Span {
  int n_rows, row0;               // rows of the sequence and K/V head; this wavefront's first
  int begin, end;                 // its units
  int free_units;                 // units that every row of it sees whole
  int kv_head;
  bool whole;                     // the tile has no other part
};
// Finds a wavefront's work: OWN rows of the ROWS of a tile from row `first` on, share kw of KW of the part's keys.
template <int ROWS, int OWN, int KW>
__device__ __forceinline__ bool enter(const Args& a, int first, int kw, Part& w, Span& p) {
  if (!find_part<ROWS>(a, blockIdx.x, w)) return false;
  p.n_rows = uniform(w.s.n_new * a.group);
  p.row0 = uniform(w.tile * ROWS + first);
  p.kv_head = uniform(w.head);
  if (p.row0 >= p.n_rows) return false;
  const int all = tile_units<ROWS>(a, w), u0 = w.chunk * w.units;
  if (w.place >= 0 && w.chunk == 0 && threadIdx.x < ROWS / JOINT<ROWS>) {
    const int row = w.tile * ROWS + JOINT<ROWS> * (int)threadIdx.x;
    if (row < p.n_rows)
      joints(a)[w.joint + threadIdx.x] = {all > w.units ? (all + w.units - 1) / w.units : 0, w.place, w.tiles, row, min(p.n_rows - row, JOINT<ROWS>),
                                          w.s.first, w.head, 0};
  }
  if (w.chunk > 0 && u0 >= all) return false;                // this tile ends before
  p.whole = all <= w.units;
  const int most = (limit_of(a, w.s, min(p.row0 + OWN, p.n_rows) - 1) + 31) >> 5;    // units that a row of this wavefront sees
  const int u1 = min(u0 + w.units, all), share = (u1 - u0 + KW - 1) / KW;
  p.begin = uniform(u0 + kw * share);
  p.end = uniform(min(min(p.begin + share, most), u1));
  p.free_units = uniform(limit_of(a, w.s, p.row0) >> 5);
  return true;
}

// Pages of the columns p to p1 - 1 of a row of the table that exist, in order, with their columns: a wavefront's own list in LDS.
// Unit x of the list is unit x % 2^unit_shift of page x / 2^unit_shift; units x0 to x1 - 1 are those from `begin` on and before `stop`.
template <int WINDOW>
__device__ __forceinline__ void list_pages(const Args& a, const int32_t* table, int2* pages, int p, int p1, int begin, int stop, int& x0, int& x1) {
  const int lane = (int)threadIdx.x & 63;
  int n = 0;
  const auto note = [&](int id, int column) __attribute__((always_inline)) {
    const bool there = column < p1 && (unsigned)id < (unsigned)a.n_pages;
    const uint64_t some = __builtin_amdgcn_ballot_w64(there);
    if (there) pages[n + __popcll(some & ((1ull << lane) - 1))] = make_int2(id, column);
    n += __popcll(some);
  };
  wave_fence();
  if (p1 - p <= 64) {                                        // (the usual length of a part: one request)
    note(table[min(p + lane, a.max_pages - 1)], p + lane);
  } else {
    int ids[WINDOW / 64];
#pragma unroll
    for (int i = 0; i < WINDOW / 64; ++i) ids[i] = table[min(p + 64 * i + lane, a.max_pages - 1)];
#pragma unroll
    for (int i = 0; i < WINDOW / 64; ++i) note(ids[i], p + 64 * i + lane);
  }
  wave_fence();
  const int per = 1 << a.unit_shift;
  x0 = n > 0 && uniform(pages[0].y) == begin >> a.unit_shift ? begin & (per - 1) : 0;
  x1 = n * per;
  if (n > 0 && uniform(pages[n - 1].y) == (stop - 1) >> a.unit_shift) x1 -= per - 1 - ((stop - 1) & (per - 1));
}

// Operands of a tile: buffer loads, the tile's address in scalar registers, a constant offset of the lane, and nothing past the
// tile; of no tile (`there` false) they are zeros that are not fetched.
template <int D>
__device__ __forceinline__ int64_t tile_at(const Args& a, int kv_head, int u, int page) {
  return (((int64_t)page * a.kv_heads + kv_head) * (1 << a.unit_shift) + (u & ((1 << a.unit_shift) - 1))) * (32 * D * 2);
}
template <int D>
__device__ __forceinline__ auto tile_buffer(const void* cache, int64_t at, bool there) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)uniform_ptr((const unsigned char*)cache + at), 0, uniform(there ? 32 * D * 2 : 0), 0x00020000);
}

// V behind the last token of the sequence: 0 times whatever is there has to be 0.  A lane's eight keys of an operand are 4 from
// the one that `left` keys are left of, and 4 from eight further.
template <class x8>
__device__ __forceinline__ x8 clear_behind(x8 v, int left) {
  u32x4 x = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int key = e / 2 * 8 + e % 2 * 2;
    x[e] &= (key < left ? 0xffffu : 0u) | (key + 1 < left ? 0xffff0000u : 0u);
  }
  return __builtin_bit_cast(x8, x);
}

// Values of V that are not finite, in units of which some row of a tile does not see all tokens: 0 times such a value is no 0, so they
// are taken out of V, and rows that see them get them by products of their own: the largest bf16 number where a value is +infinity
// or not a number, times the same where a row sees the key, is +infinity in fp32 and 0 elsewhere; the negative one likewise.
// (Two halves of a register at a time: an exponent of all ones carries into the sign's place.)
template <class T>
__device__ __forceinline__ uint32_t not_finite(uint32_t x) {
  constexpr uint32_t E = T::EXPONENT | T::EXPONENT << 16, ONE = (0x8000u - T::EXPONENT) | (0x8000u - T::EXPONENT) << 16;
  return ((x & E) + ONE) & 0x80008000u;
}
__device__ __forceinline__ uint32_t halves(uint32_t signs) { return (signs >> 15) * 0xffffu; }     // whole halves from their sign places
template <class T, class x8>
__device__ __forceinline__ uint32_t any_not_finite(const x8& v) {
  const u32x4 x = __builtin_bit_cast(u32x4, v);
  return not_finite<T>(x[0]) | not_finite<T>(x[1]) | not_finite<T>(x[2]) | not_finite<T>(x[3]);
}
// The places of those that count as +infinity (or as -infinity; what is not a number counts as both), as bf16 numbers.
template <class T, bool MINUS, class x8>
__device__ __forceinline__ bf16x8 infinities(const x8& v) {
  constexpr uint32_t M = T::MANTISSA | T::MANTISSA << 16;
  const u32x4 x = __builtin_bit_cast(u32x4, v);
  u32x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t nan = (x[e] & M) + (0x80008000u - 0x00010001u);        // (a mantissa above 0 carries into the sign's place)
    y[e] = halves(not_finite<T>(x[e]) & (nan | (MINUS ? x[e] : ~x[e]))) & (MINUS ? 0xff7fff7fu : 0x7f7f7f7fu);
  }
  return __builtin_bit_cast(bf16x8, y);
}
// Zeros in all their places.  (In the registers that hold v: as other values they would be copied around the branch.)
template <class T, class x8>
__device__ __forceinline__ void take_out(x8& v) {
  u32x4 x = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    uint32_t y = x[e];
    asm("v_and_b32 %0, %1, %0" : "+v"(y) : "v"(~halves(not_finite<T>(y))));
    x[e] = y;
  }
  v = __builtin_bit_cast(x8, x);
}
// The largest bf16 number for each of a lane's eight keys of an operand (4 in a row, and 4 from eight further) that is among the
// first `left`, else 0.
__device__ __forceinline__ bf16x8 seen(int left) {
  u32x4 x;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int key = e / 2 * 8 + e % 2 * 2;
    x[e] = (key < left ? 0x7f7fu : 0u) | (key + 1 < left ? 0x7f7f0000u : 0u);
  }
  return __builtin_bit_cast(bf16x8, x);
}

// 1 / l of a finished row; a row that sees no key yields zeros, one whose sum is not a number that.
__device__ __forceinline__ float weight_of(float l) { return l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l); }
__device__ __forceinline__ float lse_of(float m, float l) { return (m + __log2f(l)) * 0.6931471805599453f; }

// Many rows: two wavefronts of 64 rows each (two tiles of 32) walk a part's keys (v_mfma_f32_32x32x16).  64 rows, for each of
// K's and V's bytes from the caches serves two products, and what a wavefront holds (D = 128: O 128, Q 64, S and P of two units 96,
// operands of two units 128 registers) just fits into the 512 of a SIMD.  One wavefront to a SIMD has to hide everything by itself:
// a step does S of the next unit, O += V P of the one before and the softmax of the present one, operand by operand, a load into an
// operand's registers right behind the products that read it, two steps ahead for K and one for V.  At D = 64 half a step apart is
// enough and two wavefronts share a SIMD.
//
// Bound by the matrix cores, which hold the card at about 1.7 GHz here (power): 4,680 tokens over 32,760 keys, 40 heads, full, bf16,
// D = 128: 2,480 to 2,630 us by the card, 1,270 to 1,195 TFLOP/s, matrix cores busy in 70% of the cycles; a library product of 8192^3
// reaches 1,192.  D = 64, where there is as much softmax for half the products: 1,550 to 1,630 us, 1,010 to 960 TFLOP/s, 53%.  Five prompts (361 to 2,397 tokens, 32 heads on 8,
// causal): 117 to 122 us, 890 to 850 TFLOP/s; there 512 workgroups run in fewer than three rounds, of which the last leaves 12% of the places empty.
template <class T, int D>
__global__ void __launch_bounds__(128, D == 128 ? 1 : 2) many_attn_kernel(Args a) {
  constexpr int DS = D / 16, DT = D / 32, ROWS = RF2_PAGED_ROWS_MANY;
  constexpr int WINDOW = 512;      // columns of the table that a wavefront has listed at a time
  typedef typename T::x8 x8;
  const int wave = uniform((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63, l32 = lane & 31, lh = lane >> 5;
  Part w;
  Span sp;
  if (!enter<ROWS, 64, 1>(a, 64 * wave, 0, w, sp)) return;

  // this lane's rows: query column l32 of each tile (rows past the last stand for the last and are not written)
  auto row_of = [&](int q) __attribute__((always_inline)) { return sp.row0 + 32 * q + l32; };
  x8 qf[2][DS];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int r = min(row_of(q), sp.n_rows - 1), t = token_of(a, r), head = sp.kv_head * a.group + r - t * a.group;
    const typename T::x1* const from = (const typename T::x1*)a.q + (w.s.first + t) * a.q_stride + head * D + 8 * lh;
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) qf[q][ds] = *reinterpret_cast<const x8*>(from + 16 * ds);
  }
  f32x16 o[2][DT];
  float m[2], l[2];             // reference (in the exponent of 2), sum of the probabilities of this lane's keys
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    m[q] = -FLT_MAX;
    l[q] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[q][dt][i] = 0.f;
  }

  // Keys that the wavefront's rows see; in LDS, where they are hardly ever read.
  __shared__ int row_limits[2][64];
  int* const limits = row_limits[wave];
  limits[lane] = limit_of(a, w.s, min(sp.row0 + lane, sp.n_rows - 1));
  wave_fence();
  // Keys of unit u that a row does not see.
  auto mask = [&](f32x16& S, int q, int u) __attribute__((always_inline)) {
    const int left = limits[32 * q + l32] - 32 * u - 4 * lh;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (8 * (i / 4) + i % 4 >= left) S[i] = -INFINITY;
  };
  const uint32_t k_lane = (uint32_t)lane * 16, v_lane = (uint32_t)(lh * D + l32) * 16;
  auto k_load = [&](auto tile, int c) __attribute__((always_inline)) {
    return __builtin_bit_cast(x8, __builtin_amdgcn_raw_buffer_load_b128(tile, k_lane + c % 4 * 1024, c / 4 * 4096, 0));
  };
  auto v_load = [&](auto tile, int j) __attribute__((always_inline)) {
    return __builtin_bit_cast(x8, __builtin_amdgcn_raw_buffer_load_b128(tile, v_lane + j / 2 * 512, j % 2 * (2 * D * 16), 0));
  };
  auto operand_p = [](const uint32_t (&P)[8], int ks) __attribute__((always_inline)) {
    const u32x4 x = {P[4 * ks], P[4 * ks + 1], P[4 * ks + 2], P[4 * ks + 3]};
    return __builtin_bit_cast(x8, x);
  };
  // The reference of tile q moves to the largest exponent of S, if that is larger; returns what has been summed is to be scaled by.
  auto move_reference = [&](int q, const f32x16& S) __attribute__((always_inline)) {
    float top = S[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, S[i]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * a.scale_log2 - T::HEAD, -FLT_MAX);
    // (a row without a key so far has no sums but, at d = 64, infinities that the guard below gave it ahead of their unit: 0 times them
    // would not be a number)
    const float to = fmaxf(m[q], top), alpha = m[q] == -FLT_MAX ? 1.f : __builtin_amdgcn_exp2f(m[q] - to);
    m[q] = to;
    return alpha;
  };
  auto probabilities = [&](int q, const f32x16& S, uint32_t (&P)[8]) __attribute__((always_inline)) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(S[i], a.scale_log2, -m[q])), p1 = __builtin_amdgcn_exp2f(fmaf(S[i + 1], a.scale_log2, -m[q]));
      const typename T::x2 pk = {(typename T::x1)p0, (typename T::x1)p1};
      sum += p0 + p1;
      P[i / 2] = __builtin_bit_cast(uint32_t, pk);
    }
    return sum;
  };
  const int32_t* const table = a.table + (int64_t)uniform(w.seq) * a.max_pages;
  __shared__ int2 page_lists[2][WINDOW];
  int2* const pages = page_lists[wave];
  constexpr int NQ = DS, NP = 2 * DT, PAIRS = 16 / (NQ + NP);
  x8 kr[2][NQ], vr[2][NP];
  float last[2] = {};                      // sums of the latest unit, still to be added to l
  constexpr int NONE = 1 << 25;            // a unit that no sequence has
  // V of unit u, of which some row does not see all, without values that are not finite (see take_out).  The first row sees least; where all
  // rows are of one token (many heads share a K/V head), others can stand behind it.
  const bool unseen = uniform(limit_of(a, w.s, sp.row0) < w.s.len);
  auto guard = [&](x8 (&v)[NP], int u) __attribute__((always_inline)) {
    uint32_t any = 0;
#pragma unroll
    for (int j = 0; j < NP; ++j) any |= any_not_finite<T>(v[j]);
    if (__builtin_amdgcn_ballot_w64(any != 0) == 0ull) return;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      __builtin_amdgcn_sched_barrier(0);     // (one operand after the other: there are no registers for more)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const bf16x8 sees = seen(limits[32 * q + l32] - 32 * u - 16 * (j % 2) - 4 * lh);
        o[q][j / 2] = Bf16::mfma(infinities<T, false>(v[j]), sees, o[q][j / 2]);
        __builtin_amdgcn_sched_barrier(0);
        o[q][j / 2] = Bf16::mfma(infinities<T, true>(v[j]), sees, o[q][j / 2]);
        __builtin_amdgcn_sched_barrier(0);
      }
      take_out<T>(v[j]);
    }
  };
  // O of tile q times alpha.  In accumulation registers it is scaled where it is, through one vector register (left to the
  // compiler, the copies cost the registers of the loop); the wait states cover a product in flight and one that follows.
  auto rescale = [&](int q, float alpha) __attribute__((always_inline)) {
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float x = o[q][dt][i], t;
        asm volatile("v_accvgpr_read_b32 %1, %0\n\ts_nop 1\n\tv_mul_f32 %1, %1, %2\n\ts_nop 1\n\tv_accvgpr_write_b32 %0, %1"
                     : "+a"(x), "=&v"(t) : "v"(alpha));
        o[q][dt][i] = x;
      }
    asm volatile("s_nop 7" ::: "memory");
  };
  // Step: S of the next unit, O += V P of the one before, the softmax arithmetic of the present one, operand by operand.  The
  // operands' registers are loaded again as soon as both MFMAs that read them are issued: K at k_at, V at v_at.
  auto step = [&](auto odd, f32x16 (&Scur)[2], f32x16 (&Snext)[2], uint32_t (&Pprev)[2][8], uint32_t (&Pcur)[2][8], auto kb, auto vb,
                  int u, int u_next) __attribute__((always_inline)) {
    constexpr int B = decltype(odd)::value;
    __builtin_amdgcn_sched_barrier(0);
    float rs[2] = {}, e0[PAIRS], e1[PAIRS];
#pragma unroll
    for (int g = 0; g < NQ + NP; ++g) {
      const int j = g - NQ;
      if (g % 2 == 0) {                    // (one wait for two operands)
        if (g < NQ) asm volatile("" ::"v"(kr[B][g + 1]));
        else asm volatile("" ::"v"(vr[B][j + 1]));
      }
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        if (g < NQ) {
          T::template qk<true>(Snext[q], kr[B][g], qf[q][g], g == 0);
        } else {
          o[q][j / 2] = T::mfma(vr[B][j], operand_p(Pprev[q], j % 2), o[q][j / 2]);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (q == 0) {
#pragma unroll
          for (int p = 0; p < PAIRS; ++p) {
            const int x = g * PAIRS + p, tile = x / 8, i = 2 * (x % 8);
            e0[p] = __builtin_amdgcn_exp2f(fmaf(Scur[tile][i], a.scale_log2, -m[tile]));
            e1[p] = __builtin_amdgcn_exp2f(fmaf(Scur[tile][i + 1], a.scale_log2, -m[tile]));
            asm volatile("" : "+v"(e0[p]), "+v"(e1[p]));
          }
        } else {
          if (g < NQ) kr[B][g] = k_load(kb, g);
          else vr[B][j] = v_load(vb, j);
          asm volatile("" ::: "memory");   // (the load stays here)
#pragma unroll
          for (int p = 0; p < PAIRS; ++p) {
            const int x = g * PAIRS + p, tile = x / 8, i = 2 * (x % 8);
            const typename T::x2 pk = {(typename T::x1)e0[p], (typename T::x1)e1[p]};
            uint32_t word = __builtin_bit_cast(uint32_t, pk);
            rs[tile] = i == 0 ? e0[p] + e1[p] : rs[tile] + (e0[p] + e1[p]);
            asm volatile("" : "+v"(word), "+v"(rs[tile]));
            Pcur[tile][i / 2] = word;
            if (i == 0) {
              l[tile] += last[tile];
              asm volatile("" : "+v"(l[tile]));
            }
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    last[0] = rs[0];
    last[1] = rs[1];
    // One branch, hardly ever taken: the present unit is out of range, or rows do not see all of the next one.
    // (the limit is an integer select: as a float one it would be two branches, and the step twice)
    int bound = max(u, u_next) >= sp.free_units ? __builtin_bit_cast(int, -1.f) : __builtin_bit_cast(int, T::RANGE);
    asm volatile("" : "+s"(bound));
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(rs[0] + rs[1] <= __builtin_bit_cast(float, bound))) != 0ull, 0)) {
      if (__builtin_amdgcn_ballot_w64(!(rs[0] + rs[1] <= T::RANGE)) != 0ull)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float alpha = move_reference(q, Scur[q]);
          l[q] *= alpha;
          rescale(q, alpha);
          last[q] = probabilities(q, Scur[q], Pcur[q]);
        }
      if (u_next >= sp.free_units) mask(Snext[0], 0, u_next), mask(Snext[1], 1, u_next);
      if (unseen && u >= sp.free_units && u != NONE) guard(vr[1 - B], u);
    }
  };
  // Units x0 to x1 - 1 of the list (behind unit `lead` of page `lead_page`, where there is one).
  auto walk = [&](int x0, int x1, int lead, int lead_page, bool begins) __attribute__((always_inline)) {
    // Units s to s + 3 and where they lie in either cache; past the last one none.
    int us[4], x = x0;
    int64_t at[4];
    int2 entry = pages[max(min(x, x1 - 1), 0) >> a.unit_shift];       // of unit x, read a step before it is used
    auto following = [&](int i) __attribute__((always_inline)) {
      const int u = (uniform(entry.y) << a.unit_shift) + (x & ((1 << a.unit_shift) - 1));
      at[i] = tile_at<D>(a, sp.kv_head, u, uniform(entry.x));
      us[i] = x < x1 ? u : NONE;
      ++x;
      entry = pages[max(min(x, x1 - 1), 0) >> a.unit_shift];
    };
    auto shift = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 3; ++i) us[i] = us[i + 1], at[i] = at[i + 1];
    };
    auto k_of = [&](int i) __attribute__((always_inline)) { return tile_buffer<D>(a.k_cache, at[i], us[i] != NONE); };
    auto v_of = [&](int i) __attribute__((always_inline)) { return tile_buffer<D>(a.v_cache, at[i], us[i] != NONE); };
    if (lead >= 0) us[0] = lead, at[0] = tile_at<D>(a, sp.kv_head, lead, lead_page);
    else following(0);
    following(1);
    following(2);
    if constexpr (D == 128) {
      x8 k0[NQ];
#pragma unroll
      for (int c = 0; c < NQ; ++c) k0[c] = k_load(k_of(0), c);
#pragma unroll
      for (int c = 0; c < NQ; ++c) kr[0][c] = k_load(k_of(1), c);
      asm volatile("" ::: "memory");
#pragma unroll
      for (int c = 0; c < NQ; ++c) kr[1][c] = k_load(k_of(2), c);
      asm volatile("" ::: "memory");
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        vr[1][j] = v_load(v_of(0), j);
#pragma unroll
        for (int e = 0; e < 8; ++e) vr[0][j][e] = (typename T::x1)0.f;     // step 0 has no unit before it: it adds 0 x 0
      }
      f32x16 Sa[2], Sb[2];
      uint32_t Pa[2][8], Pb[2][8];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
#pragma unroll
        for (int ds = 0; ds < DS; ++ds) {
          T::template qk<true>(Sa[q], k0[ds], qf[q][ds], ds == 0);
        }
        asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 1" : "+v"(Sa[q]));
        if (us[0] >= sp.free_units) mask(Sa[q], q, us[0]);
        if (begins) (void)move_reference(q, Sa[q]);
#pragma unroll
        for (int e = 0; e < 8; ++e) Pb[q][e] = 0u;
#pragma unroll
        for (int i = 0; i < 16; ++i) Sb[q][i] = 0.f;
      }
      if (lead >= 0)
#pragma unroll
        for (int j = 0; j < NP; ++j) vr[1][j] = clear_behind(vr[1][j], w.s.len - 32 * lead - 16 * (j % 2) - 4 * lh);
      // (arrived before the loop, whose waits would else be those of its first round)
#pragma unroll
      for (int c = 0; c < NQ; ++c) asm volatile("" : "+v"(kr[0][c]));
      // Steps in pairs: behind an odd number of units comes one of which no row sees anything.
      do {
        following(3);
        step(std::integral_constant<int, 0>{}, Sa, Sb, Pb, Pa, k_of(3), v_of(1), us[0], us[1]);
        shift();
        following(3);
        step(std::integral_constant<int, 1>{}, Sb, Sa, Pa, Pb, k_of(3), v_of(1), us[0], us[1]);
        shift();
      } while (us[0] != NONE);
      // last product
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        l[q] += last[q];
        last[q] = 0.f;
#pragma unroll
        for (int j = 0; j < NP; ++j) o[q][j / 2] = T::mfma(vr[0][j], operand_p(Pb[q], j % 2), o[q][j / 2]);
      }
    } else {
      // The two tiles of rows half a step apart, so that one S and one P of each are enough (two wavefronts per SIMD).
      x8 k0[NQ];
#pragma unroll
      for (int c = 0; c < NQ; ++c) k0[c] = k_load(k_of(0), c);
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int j = 0; j < NQ; ++j) {
          kr[1 - i][j] = k_load(k_of(i + 1), j);
          asm volatile("" ::: "memory");
          vr[i][j] = v_load(v_of(i), j);
          asm volatile("" ::: "memory");
        }
      }
      f32x16 S[2];
      uint32_t P[2][8];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
#pragma unroll
        for (int ds = 0; ds < DS; ++ds) T::template qk<false>(S[q], k0[ds], qf[q][ds], ds == 0);
        asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 1" : "+v"(S[q]));
        if (us[0] >= sp.free_units) mask(S[q], q, us[0]);
        if (begins) (void)move_reference(q, S[q]);
#pragma unroll
        for (int e = 0; e < 8; ++e) P[q][e] = 0u;
      }
      if (lead >= 0)
#pragma unroll
        for (int j = 0; j < NP; ++j) vr[0][j] = clear_behind(vr[0][j], w.s.len - 32 * lead - 16 * (j % 2) - 4 * lh);
      // Probabilities of a tile whose unit was out of range, or is the first of a list: O and l have all earlier units.
      auto redo = [&](int q) __attribute__((always_inline)) {
        const float alpha = move_reference(q, S[q]);
        l[q] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[q][dt][i] *= alpha;
        last[q] = probabilities(q, S[q], P[q]);
      };
      if (unseen && us[0] >= sp.free_units) guard(vr[0], us[0]);
      redo(0);
      // Half of a step for tile Q: S of the next unit and O += V P of the present one, in turn, around the softmax arithmetic of the
      // other tile X (the present unit of tile 1 in the first half, the next one of tile 0 in the second).  In the second half the
      // operands' registers are loaded again.
      auto half = [&](auto tile, auto odd, auto kb, auto vb, int u_next) __attribute__((always_inline)) {
        constexpr int Q = decltype(tile)::value, X = 1 - Q, ODD = decltype(odd)::value;
        __builtin_amdgcn_sched_barrier(0);
        float rs = 0.f, e[2][2];
        // sum and packing of pair p, a slot behind its exponentials: no instruction waits for the one before it
        auto finish_pair = [&](int p) __attribute__((always_inline)) {
          const typename T::x2 pk = {(typename T::x1)e[p & 1][0], (typename T::x1)e[p & 1][1]};
          uint32_t word = __builtin_bit_cast(uint32_t, pk);
          rs = p == 0 ? e[0][0] + e[0][1] : rs + (e[p & 1][0] + e[p & 1][1]);
          asm volatile("" : "+v"(word), "+v"(rs));
          P[X][p] = word;
        };
#pragma unroll
        for (int g = 0; g < NQ + NP; ++g) {
          const int j = g / 2;
          if (g % 2 == 0) T::template qk<false>(S[Q], kr[1 - ODD][j], qf[Q][j], j == 0);
          else o[Q][j / 2] = T::mfma(vr[ODD][j], operand_p(P[Q], j % 2), o[Q][j / 2]);
          __builtin_amdgcn_sched_barrier(0);
          if constexpr (Q == 1) {
            if (g % 2 == 0) kr[1 - ODD][j] = k_load(kb, j);
            else vr[ODD][j] = v_load(vb, j);
            asm volatile("" ::: "memory");
          }
          if (g > 0) finish_pair(g - 1);
          if (g == 0) {
            l[Q] += last[Q];
            asm volatile("" : "+v"(l[Q]));
          }
          e[g & 1][0] = __builtin_amdgcn_exp2f(fmaf(S[X][2 * g], a.scale_log2, -m[X]));
          e[g & 1][1] = __builtin_amdgcn_exp2f(fmaf(S[X][2 * g + 1], a.scale_log2, -m[X]));
          asm volatile("" : "+v"(e[g & 1][0]), "+v"(e[g & 1][1]));
          if (g == 7) finish_pair(7);
          __builtin_amdgcn_sched_barrier(0);
        }
        last[X] = rs;
        // One branch, hardly ever taken, as above.
        int bound = u_next >= sp.free_units ? __builtin_bit_cast(int, -1.f) : __builtin_bit_cast(int, T::RANGE);
        asm volatile("" : "+s"(bound));
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(rs <= __builtin_bit_cast(float, bound))) != 0ull, 0)) {
          if (__builtin_amdgcn_ballot_w64(!(rs <= T::RANGE)) != 0ull) redo(X);
          if (u_next >= sp.free_units) mask(S[Q], Q, u_next);
          if (Q == 1 && unseen && u_next >= sp.free_units && u_next != NONE) guard(vr[1 - ODD], u_next);
        }
      };
      constexpr std::integral_constant<int, 0> zero{};
      constexpr std::integral_constant<int, 1> one{};
      do {
        following(3);
        half(zero, zero, k_of(3), v_of(2), us[1]);
        half(one, zero, k_of(3), v_of(2), us[1]);
        shift();
        following(3);
        half(zero, one, k_of(3), v_of(2), us[1]);
        half(one, one, k_of(3), v_of(2), us[1]);
        shift();
      } while (us[0] != NONE);
      last[0] = last[1] = 0.f;               // (of no unit)
    }
  };
  // The last unit of a sequence can have keys behind its last token, whose V has to be cleared: it goes first, so that no step
  // has to look for it.
  int stop = sp.end, lead = -1, lead_page = 0;
  if (sp.begin < sp.end && 32 * sp.end > w.s.len) {
    stop = sp.end - 1;
    lead_page = uniform(table[stop >> a.unit_shift]);
    lead = (unsigned)lead_page < (unsigned)a.n_pages ? stop : -1;
  }
  bool begins = true;
  for (int p = sp.begin >> a.unit_shift, p1 = (stop + (1 << a.unit_shift) - 1) >> a.unit_shift; p < p1 || lead >= 0; p += WINDOW) {
    int x0, x1;
    list_pages<WINDOW>(a, table, pages, p, min(p + WINDOW, p1), sp.begin, stop, x0, x1);
    if (x0 < x1 || lead >= 0) {
      walk(x0, x1, lead, lead_page, begins);
      begins = false;
      lead = -1;
    }
  }

  // Results leave as whole rows, through LDS (8 or 16 bytes a lane at a stride of a row keep the address unit of a compute unit busy
  // for 64 cycles an instruction); sums of a part as the registers have them (see part_at).
  __shared__ uint4 out_rows[2][32 * (D / 8)];
  uint4* const staged = out_rows[wave];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    // sums of the two lane halves, which have different keys of a row
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[q]), __float_as_uint(l[q]), false, false);
    l[q] = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    const int first = sp.row0 + 32 * q;        // of the tile's rows
    if (!sp.whole) {
      if (row_of(q) < sp.n_rows) {
        const int r = row_of(q) - w.tile * ROWS;
#pragma unroll
        for (int x = 0; x < 4 * DT; ++x)
          *reinterpret_cast<float4*>(part_sums<ROWS, D>(a, w.place) + part_at<ROWS, D>(r, 8 * x + 4 * lh)) =
              make_float4(o[q][x / 4][4 * (x % 4)], o[q][x / 4][4 * (x % 4) + 1], o[q][x / 4][4 * (x % 4) + 2], o[q][x / 4][4 * (x % 4) + 3]);
        if (lh == 0) part_stats<ROWS, D>(a, w.place)[r] = make_float2(m[q], l[q]);
      }
      continue;
    }
    const float f = weight_of(l[q]);
    wave_fence();
#pragma unroll
    for (int x = 0; x < 4 * DT; ++x) {
      typename T::x4 pk;
#pragma unroll
      for (int e = 0; e < 4; ++e) pk[e] = (typename T::x1)(o[q][x / 4][4 * (x % 4) + e] * f);
      reinterpret_cast<typename T::x4*>(&staged[row_slot<D / 8>(l32, x)])[lh] = pk;
    }
    wave_fence();
    if (a.lse != nullptr && lh == 0 && row_of(q) < sp.n_rows) {
      const int t = token_of(a, row_of(q));
      a.lse[(int64_t)(w.s.first + t) * a.heads + (sp.kv_head - t) * a.group + row_of(q)] = lse_of(m[q], l[q]);
    }
    constexpr int CPR = D / 8, STEP = 64 / CPR;      // 16-byte chunks of a row, rows that the wavefront moves at a time
#pragma unroll
    for (int i = 0; i < 32 / STEP; ++i) {
      const int r = lane / CPR + i * STEP, row = first + r, t = token_of(a, row);
      const uint4 piece = staged[row_slot<CPR>(r, lane % CPR)];
      if (row < sp.n_rows)
        *reinterpret_cast<uint4*>((typename T::x1*)a.o + ((int64_t)(w.s.first + t) * a.heads + (sp.kv_head - t) * a.group + row) * D + lane % CPR * 8) = piece;
    }
  }
}

// Few rows: QT tiles of 16, whose keys four wavefronts share (v_mfma_f32_16x16x32).  A product of 16 keys takes the keys of a unit
// that S^T's accumulators then hold as V^T's storage groups have them: rows 4 i + e of the first are keys 0-3, 4-7, 16-19, 20-23, those
// of the second eight more, and a lane's eight probabilities are the eight keys of storage group lane / 16.
//
// Bound by memory: operands of two units are on their way (each is asked for as soon as the one two before has been read).
// 64 single tokens over 0.79 GB of keys and values: 131 us, 6.0 TB/s; four over 0.58 GB, 21,000 to 61,000 keys each: 105 us, 5.6 TB/s
// (a kernel that only reads reaches 6.5, one that copies 6.2); 64 at 64 channels over 0.39 GB: 70 us, 5.6 TB/s.  One token over 200 keys
// takes 5.8 us, of which 0.1 are its bytes.
template <class T, int D, int QT>
__global__ void __launch_bounds__(256, D == 64 && QT == 1 ? 3 : 2) few_attn_kernel(Args a) {
  constexpr int KW = 4, CS = D / 32, CT = D / 16, ROWS = 16 * QT;
  constexpr int WINDOW = 256;      // columns of the table that a wavefront has listed at a time
  typedef typename T::x8 x8;
  const int kw = uniform((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4;
  Part w;
  Span sp;
  if (!enter<ROWS, ROWS, KW>(a, 0, kw, w, sp)) return;

  auto row_of = [&](int q) __attribute__((always_inline)) { return sp.row0 + 16 * q + l16; };
  x8 qf[QT][CS];
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    const int r = min(row_of(q), sp.n_rows - 1), t = token_of(a, r), head = sp.kv_head * a.group + r - t * a.group;
    const typename T::x1* const from = (const typename T::x1*)a.q + (w.s.first + t) * a.q_stride + head * D + 8 * lq;
#pragma unroll
    for (int cs = 0; cs < CS; ++cs) qf[q][cs] = *reinterpret_cast<const x8*>(from + 32 * cs);
  }
  const bool unseen = uniform(limit_of(a, w.s, sp.row0) < w.s.len);   // some row does not see all tokens (the first sees least)
  f32x4 o[QT][CT];
  float m[QT], l[QT];
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    m[q] = -FLT_MAX;
    l[q] = 0.f;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) o[q][ct] = (f32x4)0.f;
  }
  const int key0 = (lq & 1) * 4 + (lq >> 1) * 16;                     // first of this lane's keys of a unit (the other four: 8 further)
  int limit[QT];                                                      // keys that a row sees, less that
#pragma unroll
  for (int q = 0; q < QT; ++q) limit[q] = limit_of(a, w.s, min(row_of(q), sp.n_rows - 1)) - key0;
  const uint32_t k_lane = (uint32_t)(lq * 512 + ((l16 & 7) + (l16 >> 3) * 16) * 16), v_lane = (uint32_t)(lq * D + l16) * 16;
  // Tiles are read once, or a few times at the same time, and then not for long: the loads are marked as not to be kept (64 single
  // tokens over 0.79 GB of keys and values 149.7 -> 137.4 us).
  constexpr int ONCE = 2;
  auto k_load = [&](auto tile, int t, int cs) __attribute__((always_inline)) {
    return __builtin_bit_cast(x8, __builtin_amdgcn_raw_buffer_load_b128(tile, k_lane + t * 128 + cs % 2 * 2048, cs / 2 * 4096, ONCE));
  };
  auto v_load = [&](auto tile, int ct) __attribute__((always_inline)) {
    return __builtin_bit_cast(x8, __builtin_amdgcn_raw_buffer_load_b128(tile, v_lane + ct * 256, 0, ONCE));
  };
  const int32_t* const table = a.table + (int64_t)uniform(w.seq) * a.max_pages;
  __shared__ int2 page_lists[KW][WINDOW];
  int2* const pages = page_lists[kw];
  constexpr int AHEAD = QT == 2 && D == 128 ? 1 : 2;      // units that are asked for ahead: what registers there are for
  x8 kr[AHEAD][2][CS], vr[AHEAD][CT];
  int us[AHEAD];
  for (int p = sp.begin >> a.unit_shift, p1 = (sp.end + (1 << a.unit_shift) - 1) >> a.unit_shift; sp.begin < sp.end && p < p1; p += WINDOW) {
    int x0, x1;
    list_pages<WINDOW>(a, table, pages, p, min(p + WINDOW, p1), sp.begin, sp.end, x0, x1);
    if (x0 >= x1) continue;
    int64_t at[AHEAD];
    auto place = [&](int x, int& u, int64_t& at) __attribute__((always_inline)) {
      const int2 entry = pages[min(x, x1 - 1) >> a.unit_shift];
      u = (uniform(entry.y) << a.unit_shift) + (x & ((1 << a.unit_shift) - 1));
      at = tile_at<D>(a, sp.kv_head, u, uniform(entry.x));
    };
    // unit x, whose place is held in us and at
    auto fetch_k = [&](auto slot, int x) __attribute__((always_inline)) {
      constexpr int B = decltype(slot)::value;
      const auto kb = tile_buffer<D>(a.k_cache, at[B], x < x1);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) kr[B][t][cs] = k_load(kb, t, cs);
      asm volatile("" ::: "memory");
    };
    auto fetch_v = [&](auto slot, int x) __attribute__((always_inline)) {
      constexpr int B = decltype(slot)::value;
      const auto vb = tile_buffer<D>(a.v_cache, at[B], x < x1);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) vr[B][ct] = v_load(vb, ct);
      asm volatile("" ::: "memory");
    };
    auto unit = [&](auto slot, int x) __attribute__((always_inline)) {
      constexpr int B = decltype(slot)::value;
      const int u = us[B];
      place(x + AHEAD, us[B], at[B]);
      f32x4 S[QT][2];
#pragma unroll
      for (int q = 0; q < QT; ++q)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          S[q][t] = (f32x4)0.f;
#pragma unroll
          for (int cs = 0; cs < CS; ++cs) S[q][t] = T::mfma16(kr[B][t][cs], qf[q][cs], S[q][t]);
        }
      fetch_k(slot, x + AHEAD);
      x8 P[QT];
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        if (u >= sp.free_units) {                            // keys that a row does not see
          const int left = limit[q] - 32 * u;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (8 * (i / 4) + i % 4 >= left) S[q][i / 4][i % 4] = -INFINITY;
        }
        float sum;
        auto probabilities = [&]() __attribute__((always_inline)) {
          sum = 0.f;
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(S[q][i / 4][i % 4], a.scale_log2, -m[q]));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(S[q][i / 4][i % 4 + 1], a.scale_log2, -m[q]));
            P[q][i] = (typename T::x1)p0;
            P[q][i + 1] = (typename T::x1)p1;
            sum += p0 + p1;
          }
        };
        probabilities();
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum <= T::RANGE)) != 0ull, 0)) {
          // Out of range, or the first unit with a key: the reference moves to the largest exponent, what is there is rescaled.
          float top = S[q][0][0];
#pragma unroll
          for (int i = 1; i < 8; ++i) top = fmaxf(top, S[q][i / 4][i % 4]);
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          top = fmaxf(top * a.scale_log2 - T::HEAD, -FLT_MAX);
          const float to = fmaxf(m[q], top), alpha = __builtin_amdgcn_exp2f(m[q] - to);
          m[q] = to;
          l[q] *= alpha;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) o[q][ct] *= alpha;
          probabilities();
        }
        l[q] += sum;
      }
      if (32 * u + 32 > w.s.len)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) vr[B][ct] = clear_behind(vr[B][ct], w.s.len - 32 * u - key0);
      uint32_t any = 0;
      if (unseen && u >= sp.free_units)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) any |= any_not_finite<T>(vr[B][ct]);
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(any != 0) != 0ull, 0)) {
        // values of V that are not finite, where a row does not see all (see take_out); one operand after the other
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int q = 0; q < QT; ++q) {
            int left = limit[q] - 32 * u;
            asm volatile("" : "+v"(left));                     // (worked out anew each time)
            const bf16x8 sees = seen(left);
            o[q][ct] = Bf16::mfma16(infinities<T, false>(vr[B][ct]), sees, o[q][ct]);
            o[q][ct] = Bf16::mfma16(infinities<T, true>(vr[B][ct]), sees, o[q][ct]);
          }
          take_out<T>(vr[B][ct]);
        }
      }
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int q = 0; q < QT; ++q) o[q][ct] = T::mfma16(vr[B][ct], P[q], o[q][ct]);
      fetch_v(slot, x + AHEAD);
    };
    constexpr std::integral_constant<int, 0> zero{};
    constexpr std::integral_constant<int, AHEAD - 1> one{};
    place(x0, us[0], at[0]);
    fetch_k(zero, x0);
    fetch_v(zero, x0);
    if constexpr (AHEAD == 2) {
      place(x0 + 1, us[1], at[1]);
      fetch_k(one, x0 + 1);
      fetch_v(one, x0 + 1);
    }
    for (int x = x0;; x += 2) {
      unit(zero, x);
      if (x + 1 >= x1) break;
      unit(one, x + 1);
      if (x + 2 >= x1) break;
    }
  }

  // Sums of the lanes with different keys of a row; then of the wavefronts, each of which finishes a quarter of the channels.
  constexpr int OWN = CT / KW;
  __shared__ float4 tiles[KW][QT][CT][64];
  __shared__ float2 stats[KW][QT][16];
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    l[q] += __shfl_xor(l[q], 16);
    l[q] += __shfl_xor(l[q], 32);
    if (lq == 0) stats[kw][q][l16] = make_float2(m[q], l[q]);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) tiles[kw][q][ct][lane] = make_float4(o[q][ct][0], o[q][ct][1], o[q][ct][2], o[q][ct][3]);
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    float2 st[KW];
    float top = -FLT_MAX, sum = 0.f;
#pragma unroll
    for (int k = 0; k < KW; ++k) st[k] = stats[k][q][l16], top = fmaxf(top, st[k].x);
    f32x4 mine[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) mine[i] = (f32x4)0.f;
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      const float weight = __builtin_amdgcn_exp2f(st[k].x - top);
      sum = fmaf(st[k].y, weight, sum);
#pragma unroll
      for (int i = 0; i < OWN; ++i) {
        const float4 x = tiles[k][q][kw * OWN + i][lane];
        mine[i][0] = fmaf(x.x, weight, mine[i][0]);
        mine[i][1] = fmaf(x.y, weight, mine[i][1]);
        mine[i][2] = fmaf(x.z, weight, mine[i][2]);
        mine[i][3] = fmaf(x.w, weight, mine[i][3]);
      }
    }
    if (row_of(q) >= sp.n_rows) continue;
    const int t = token_of(a, row_of(q));
    const int64_t out_row = (int64_t)(w.s.first + t) * a.heads + (sp.kv_head - t) * a.group + row_of(q);
    const float f = weight_of(sum);
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      const int ch = 16 * (kw * OWN + i) + 4 * lq;
      if (sp.whole) {
        typename T::x4 pk;
#pragma unroll
        for (int e = 0; e < 4; ++e) pk[e] = (typename T::x1)(mine[i][e] * f);
        *reinterpret_cast<typename T::x4*>((typename T::x1*)a.o + out_row * D + ch) = pk;
      } else {
        *reinterpret_cast<float4*>(part_sums<ROWS, D>(a, w.place) + (16 * q + l16) * D + ch) = make_float4(mine[i][0], mine[i][1], mine[i][2], mine[i][3]);
      }
    }
    if (kw == 0 && lq == 0) {
      if (!sp.whole) part_stats<ROWS, D>(a, w.place)[16 * q + l16] = make_float2(top, sum);
      else if (a.lse != nullptr) a.lse[out_row] = lse_of(top, sum);
    }
  }
}

// Adds the parts of the tiles that are cut: 4 to 7 us, with nothing listed too, most of it the launch.  A workgroup takes a joint at a
// time: 8 rows with 32 lanes each, or, of few rows, two whose parts 4 times 32 lanes share, or one with 8 times.
template <class T, int D, int ROWS>
__global__ void __launch_bounds__(256) join_kernel(Args a) {
  constexpr int E = D / 32, DEEP = 8;              // channels of a lane; parts asked for at a time
  typedef __attribute__((ext_vector_type(E))) float fE;
  typedef __attribute__((ext_vector_type(E))) typename T::x1 tE;
  __shared__ fE sums[8][32];
  __shared__ float2 totals[8];
  // Of many rows, neighbouring lanes take neighbouring rows: their sums lie side by side.
  constexpr bool MANY = ROWS >= RF2_PAGED_ROWS_MANY;
  const int half = MANY ? (int)threadIdx.x & 7 : (int)threadIdx.x >> 5, lane = MANY ? (int)threadIdx.x >> 3 : (int)threadIdx.x & 31;
  // (the first joint is asked for beside their number: there is memory for it either way)
  const int count = *joints_count(a);
  Joint j = joints(a)[blockIdx.x];
  for (int task = (int)blockIdx.x; task < count; task += (int)gridDim.x) {
    if (task != (int)blockIdx.x) j = joints(a)[task];
    if (j.parts == 0) continue;
    const int share = MANY ? 0 : j.n_rows > 1 ? 2 : 3, every = 1 << share, r = half >> share;
    const bool there = r < j.n_rows;
    fE acc = (fE)0.f;
    float top = -FLT_MAX, sum = 0.f;
    auto take = [&](float at, float total, const fE& x) __attribute__((always_inline)) {
      const float weight = __builtin_amdgcn_exp2f(at - top);
      sum = fmaf(total, weight, sum);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(x[e], weight, acc[e]);
    };
    auto reach = [&](float at) __attribute__((always_inline)) {
      const float to = fmaxf(top, at), alpha = __builtin_amdgcn_exp2f(top - to);
      top = to;
      sum *= alpha;
      acc *= alpha;
    };
    for (int p0 = half & (every - 1); there && p0 < j.parts; p0 += every * DEEP) {
      float2 st[DEEP];
      fE x[DEEP];
#pragma unroll
      for (int i = 0; i < DEEP; ++i) {
        const int p = p0 + i * every, place = j.place + min(p, j.parts - 1) * j.step, row = j.row % ROWS + r;
        st[i] = part_stats<ROWS, D>(a, place)[row];
        x[i] = *reinterpret_cast<const fE*>(part_sums<ROWS, D>(a, place) + part_at<ROWS, D>(row, lane * E));
        if (p >= j.parts) st[i] = make_float2(-FLT_MAX, 0.f), x[i] = (fE)0.f;
      }
      float most = st[0].x;
#pragma unroll
      for (int i = 1; i < DEEP; ++i) most = fmaxf(most, st[i].x);
      reach(most);
#pragma unroll
      for (int i = 0; i < DEEP; ++i) take(st[i].x, st[i].y, x[i]);
    }
    if (share > 0) {                               // (the same for the whole workgroup)
      sums[half][lane] = acc;
      if (lane == 0) totals[half] = make_float2(top, sum);
      __syncthreads();
      if ((half & (every - 1)) == 0)
        for (int k = 1; k < every; ++k) {
          reach(totals[half + k].x);
          take(totals[half + k].x, totals[half + k].y, sums[half + k][lane]);
        }
      __syncthreads();
    }
    if (!there || (half & (every - 1)) != 0) continue;
    const float f = weight_of(sum);
    const int row = j.row + r;
    const int t = token_of(a, row);
    const int64_t out = (int64_t)(j.first + t) * a.heads + (j.head - t) * a.group + row;
    tE pk;
#pragma unroll
    for (int e = 0; e < E; ++e) pk[e] = (typename T::x1)(acc[e] * f);
    *reinterpret_cast<tE*>((typename T::x1*)a.o + out * D + lane * E) = pk;
    if (a.lse != nullptr && lane == 0) a.lse[out] = lse_of(top, sum);
  }
}

template <class T, int D, int ROWS, class Kernel>
int launch(const rf2_paged_plan* plan, Args a, Kernel kernel, int threads, hipStream_t st) {
  const rf2_paged_config& c = plan->cfg;
  const Sizes size = size_launch<ROWS>(c, a);
  // With a launch for the sums 4,096 sequences of 200 keys take 694 us, 2,040 without; 1,024 of 500 343 and 404; 512 of 700 233 and 245; 256 of
  // 1,000 170 and 171; 128 of them 88.4 and 87.4.
  a.survey = a.n_seqs > RF2_PAGED_SURVEY ? (int4*)((char*)a.parts + rf2_paged_parts_bytes(c)) : nullptr;
  if (a.survey) {
    survey_kernel<ROWS><<<dim3(1), dim3(1024), 0, st>>>(a);
    RF2_LAUNCH_CHECK();
  }
  kernel<<<dim3((unsigned)size.grid), dim3(threads), 0, st>>>(a);
  RF2_LAUNCH_CHECK();
  if (size.can_be_cut) {
    // (with at most 1,024 workgroups 16 mixed sequences take 27.4 us, with 512 28.7, with 256 31.4; where nothing is listed it is the same)
    const int64_t joints = std::min((int64_t)a.most_joints, size.joints);
    join_kernel<T, D, ROWS><<<dim3((unsigned)std::min(joints, (int64_t)1024)), dim3(256), 0, st>>>(a);
    RF2_LAUNCH_CHECK();
  }
  return RF2_OK;
}

template <class T, int D>
int dispatch(const rf2_paged_plan* plan, const Args& a, hipStream_t st) {
  switch (tile_rows(a)) {
    case 16: return launch<T, D, 16>(plan, a, few_attn_kernel<T, D, 1>, 256, st);
    case 32: return launch<T, D, 32>(plan, a, few_attn_kernel<T, D, 2>, 256, st);
    default: return launch<T, D, RF2_PAGED_ROWS_MANY>(plan, a, many_attn_kernel<T, D>, 128, st);
  }
}

}  // namespace

extern "C" int rf2_paged_attn(const rf2_paged_plan* plan, int32_t n_seqs, int32_t n_tokens, const void* q, int64_t q_stride,
                              const void* k_cache, const void* v_cache, const int32_t* block_table, const int32_t* seq_len,
                              const int32_t* cu_new, void* workspace, void* o, float* lse, void* stream) {
  if (!plan || n_seqs < 0 || n_seqs > plan->cfg.max_seqs || n_tokens < 0 || n_tokens > plan->cfg.max_tokens) return RF2_ERR_INVALID_ARG;
  if (!k_cache || !v_cache || !workspace) return RF2_ERR_INVALID_ARG;
  if (n_tokens > 0 && (!q || !o)) return RF2_ERR_INVALID_ARG;
  if (n_seqs > 0 && (!block_table || !seq_len || !cu_new)) return RF2_ERR_INVALID_ARG;
  const rf2_paged_config& c = plan->cfg;
  if (q_stride % 8 != 0 || (n_tokens > 1 && q_stride < (int64_t)c.heads * c.head_dim)) return RF2_ERR_INVALID_ARG;
  for (const void* p : {q, k_cache, v_cache, (const void*)workspace, (const void*)o})
    if (!rf2_aligned(p, 16)) return RF2_ERR_INVALID_ARG;
  for (const void* p : {(const void*)block_table, (const void*)seq_len, (const void*)cu_new, (const void*)lse})
    if (!rf2_aligned(p, 4)) return RF2_ERR_INVALID_ARG;
  if (const int rc = rf2_check_paged_device(plan)) return rc;
  if (n_seqs == 0 || n_tokens == 0) return RF2_OK;
  Args a{};
  a.q = q, a.k_cache = k_cache, a.v_cache = v_cache;
  a.table = block_table, a.seq_len = seq_len, a.cu_new = cu_new;
  a.parts = (float*)workspace, a.o = o, a.lse = lse;
  a.q_stride = q_stride;
  a.n_seqs = n_seqs, a.n_tokens = n_tokens, a.heads = c.heads, a.kv_heads = c.kv_heads, a.group = c.heads / c.kv_heads;
  uint32_t k = 0;
  while ((1 << k) < a.group) ++k;
  a.group_shift = 29 + k;
  a.group_magic = (uint32_t)((((uint64_t)1 << a.group_shift) + a.group - 1) / a.group);
  a.unit_shift = __builtin_ctz((unsigned)c.page) - 5;
  a.n_pages = c.n_pages, a.max_pages = c.max_pages, a.causal = c.causal;
  a.scale_log2 = plan->scale_log2;
  const bool bf16 = c.dtype == RF2_DTYPE_BF16;
  hipStream_t st = (hipStream_t)stream;
  if (c.head_dim == 128) return bf16 ? dispatch<Bf16, 128>(plan, a, st) : dispatch<F16, 128>(plan, a, st);
  return bf16 ? dispatch<Bf16, 64>(plan, a, st) : dispatch<F16, 64>(plan, a, st);
}
