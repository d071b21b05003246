// Attention of new tokens over a paged cache (gfx950).
//
// Rows.  The query heads that share a K/V head are rows side by side: row r of a sequence and K/V head h is token r / G,
// query head h G + r % G (G = heads / kv_heads), so a step of single tokens has G rows to a product and a chunk n G.  A
// workgroup owns a tile of these rows.
//
// Parts.  A tile's keys are cut into parts of `units` units of 32 keys, counted from key 0 for all tiles of a sequence; the
// workgroups of one part of different tiles run at the same time and find each other's keys in the caches.  With
//     W = sum over sequences of tiles * units(length),   units = max(least, ceil(W / aimed)),
// a sequence that is cut (c = ceil(units(length) / units) >= 2) has c < 2 units(length) / units parts to a tile, all of them
// less than 2 W / units <= 2 aimed: the size of the workspace.  The lengths are in device memory, so every workgroup works
// this out for itself and finds its own part; the grid is the most there can be.
//
// Products as in rf2_attn.hip: S^T = K Q^T, O^T = V^T P^T (v_mfma_f32_32x32x16), operands from the cache's tiles straight
// into registers, P the accumulators of S^T.
//
// Softmax: a probability is exp2(q.k c - m), c = scale log2(e), with a reference m per row that is moved only when the sum
// of a unit's probabilities leaves the range that P's type carries (as in rf2_attn.hip).  Sums are fp32, of unrounded P.
#include "rf2_paged.h"

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
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

struct Bf16 {
  typedef bf16x8 x8;
  typedef bf16x4 x4;
  typedef bf16x2 x2;
  typedef __bf16 x1;
  // P = exp2(x - m): bf16 and fp32 carry 2^40 as well as 1
  static constexpr float RANGE = 1.0995e12f, HEAD = 0.f;
  static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
struct F16 {
  typedef f16x8 x8;
  typedef f16x4 x4;
  typedef f16x2 x2;
  typedef _Float16 x1;
  // fp16 ends at 65,504 and loses its steps below 2^-14: the largest P stands at 2^8 when the reference is set (HEAD), may grow to
  // 2^15, and what is rounded away below 2^-25 is 2^-33 of it
  static constexpr float RANGE = 32768.f, HEAD = 8.f;
  static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

struct Args {
  const void *q, *k_cache, *v_cache;
  const int32_t *table, *seq_len, *cu_new;
  float* parts;
  void* o;
  float* lse;
  int64_t q_stride;
  int n_seqs, n_tokens, heads, kv_heads, group, unit_shift, n_pages, max_pages, causal, aimed, least;
  float scale_log2;
};

// A sequence of the call.
struct Seq {
  int first, n_new, len;      // rows of q and o; tokens cached
};
__device__ __forceinline__ Seq seq_of(const Args& a, int s) {
  const int first = min(max(a.cu_new[s], 0), a.n_tokens), end = min(max(a.cu_new[s + 1], first), a.n_tokens);
  return {first, end - first, min(max(a.seq_len[s], 0), a.max_pages << (a.unit_shift + 5))};
}
__device__ __forceinline__ int units_of(int keys) { return max((keys + 31) >> 5, 1); }

// What a workgroup works on: a part of a tile of rows.
struct Part {
  int seq, head, tile, chunk;     // chunk: number of the part
  int tiles, chunks, units;       // of the sequence; units of a part
  Seq s;
  int64_t place;                  // of the sequence's first part of K/V head 0 among those of the sequences that are cut
};

__device__ __forceinline__ int64_t wave_sum_before(int64_t& x) {      // inclusive sum in x, returns the exclusive one
  const int lane = (int)threadIdx.x & 63;
  const int64_t mine = x;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t other = __shfl_up(x, d);
    x += lane >= d ? other : 0;
  }
  return x - mine;
}

// Finds part number `block` of the launch (CUT: tile number `block` of the sequences that are cut).  ROWS: of a tile.
// Every wavefront does it for itself, 64 sequences at a time.
template <int ROWS, bool CUT>
__device__ __forceinline__ bool find_part(const Args& a, unsigned block, Part& w) {
  const int lane = (int)threadIdx.x & 63;
  int64_t work = 0;
  Seq s{0, 0, 0};
  for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
    if (s0 + lane < a.n_seqs) {
      s = seq_of(a, s0 + lane);
      work += (int64_t)((s.n_new * a.group + ROWS - 1) / ROWS) * units_of(s.len);
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) work += __shfl_xor(work, d);
  // (no sequence has more than 2^19 units)
  const int units = (int)min(max((work + a.aimed - 1) / a.aimed, (int64_t)a.least), (int64_t)1 << 20);
  // Workgroups with equal number % 8 share an XCD and its L2.  Where the K/V heads can be dealt to the XCDs evenly, they are.
  const bool dealt = a.kv_heads % 8 == 0;
  const int heads = dealt ? a.kv_heads / 8 : a.kv_heads;
  int64_t at = dealt ? block >> 3 : block;
  at /= heads;                                       // parts before this one, one head's counted
  int64_t items_before = 0, place = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
    const bool there = s0 + lane < a.n_seqs;
    if (a.n_seqs > 64) s = there ? seq_of(a, s0 + lane) : Seq{0, 0, 0};
    const int tiles = there ? (s.n_new * a.group + ROWS - 1) / ROWS : 0;
    const int chunks = (units_of(s.len) + units - 1) / units;
    const int64_t cut = chunks > 1 ? (int64_t)tiles * chunks : 0;
    int64_t sum = CUT ? (chunks > 1 ? tiles : 0) : (int64_t)tiles * chunks, cut_sum = cut;
    const int64_t before = items_before + wave_sum_before(sum), cut_before = place + wave_sum_before(cut_sum);
    sum += items_before;
    const uint64_t past = __builtin_amdgcn_ballot_w64(sum <= at);
    if (past != ~0ull) {                             // (a lane's sum only grows: the first lane that is beyond)
      const int l = __builtin_ctzll(~past);
      const auto pick = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
      const auto pick64 = [&](int64_t x) { return (int64_t)((uint64_t)(uint32_t)pick((int)(x >> 32)) << 32 | (uint32_t)pick((int)x)); };
      w.seq = s0 + l;
      w.s = {pick(s.first), pick(s.n_new), pick(s.len)};
      w.tiles = pick(tiles);
      w.chunks = pick(chunks);
      w.units = units;
      w.place = pick64(cut_before) * a.kv_heads;
      const int64_t each = CUT ? w.tiles : (int64_t)w.tiles * w.chunks;
      const int64_t rest = (dealt ? (int64_t)(block >> 3) : (int64_t)block) - pick64(before) * heads;
      const int hh = (int)(rest / each), x = (int)(rest % each);
      w.head = dealt ? hh * 8 + (int)(block & 7) : hh;
      w.chunk = CUT ? 0 : x / w.tiles;
      w.tile = w.tiles - 1 - (CUT ? x : x % w.tiles);      // (under a causal mask the last tile is the longest: it goes first)
      return true;
    }
    items_before = __shfl(sum, 63);
    place += __shfl(cut_sum, 63);
  }
  return false;
}

// Keys that row r of a sequence sees.
__device__ __forceinline__ int limit_of(const Args& a, const Seq& s, int row) {
  return a.causal ? min(max(s.len - s.n_new + row / a.group + 1, 0), s.len) : s.len;
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

// The units of a wavefront that lie in pages, in order.  64 entries of the table are held, one to a lane, and 64 more are on
// their way.
struct Pages {
  const int32_t* row;
  int end, shift, n_pages, last;      // last: of the row
  int base, ids, next_ids;
  uint64_t there;
  __device__ __forceinline__ int load(int from) const { return row[min(from + ((int)threadIdx.x & 63), last)]; }
  __device__ __forceinline__ void begin(int u) {
    base = u >> shift;
    ids = load(base);
    next_ids = load(base + 64);
    there = __builtin_amdgcn_ballot_w64((unsigned)ids < (unsigned)n_pages);
  }
  // The first unit at or after u that lies in a page, or `end`.
  __device__ __forceinline__ int seek(int u) {
    while (u < end) {
      const int at = (u >> shift) - base;
      if (at >= 64) {
        base += 64;
        ids = next_ids;
        next_ids = load(base + 64);
        there = __builtin_amdgcn_ballot_w64((unsigned)ids < (unsigned)n_pages);
        continue;
      }
      const uint64_t rest = there >> at;
      if (rest & 1) return u;
      u = (base + (rest == 0 ? 64 : at + __builtin_ctzll(rest))) << shift;
    }
    return end;
  }
  __device__ __forceinline__ int page(int u) const { return __builtin_amdgcn_readlane(ids, (u >> shift) - base); }
};

// QT: tiles of 32 rows to a wavefront; RW wavefronts with rows of their own, times KW that share a part's keys.
template <class T, int D, int QT, int RW, int KW>
__global__ void __launch_bounds__(64 * RW * KW, QT == 1 ? 2 : 1) paged_attn_kernel(Args a) {
  constexpr int DS = D / 16, DT = D / 32, ROWS = 32 * QT * RW;
  typedef typename T::x8 x8;
  Part w;
  if (!find_part<ROWS, false>(a, blockIdx.x, w)) return;
  const int lane = (int)threadIdx.x & 63, l32 = lane & 31, lh = lane >> 5;
  const int wave = RW * KW > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0, rw = wave / KW, kw = wave % KW;
  const int n_rows = w.s.n_new * a.group, row0 = w.tile * ROWS + rw * 32 * QT;
  static_assert(RW == 1 || KW == 1, "a wavefront without rows leaves here");
  if (row0 >= n_rows) return;
  const int all = tile_units<ROWS>(a, w), u0 = w.chunk * w.units;
  if (w.chunk > 0 && u0 >= all) return;                      // this tile ends before
  const bool whole = all <= w.units;                         // its only part: no other has to be added
  const int last_row = min(row0 + 32 * QT, n_rows) - 1;
  const int most = (limit_of(a, w.s, last_row) + 31) >> 5;    // units that a row of this wavefront sees
  const int share = (min(u0 + w.units, all) - u0 + KW - 1) / KW;
  const int begin = u0 + kw * share, end = min(min(begin + share, most), min(u0 + w.units, all));
  const int free_units = limit_of(a, w.s, row0) >> 5;         // units that every row sees whole

  // this lane's rows: query column l32 of each tile (rows past the last stand for the last and are not written)
  int row[QT], limit[QT];
  int64_t out_row[QT];
  x8 qf[QT][DS];
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    row[q] = row0 + 32 * q + l32;
    const int r = min(row[q], n_rows - 1), t = r / a.group, head = w.head * a.group + r % a.group;
    limit[q] = limit_of(a, w.s, r);
    out_row[q] = (int64_t)(w.s.first + t) * a.heads + head;
    const typename T::x1* const from = (const typename T::x1*)a.q + (w.s.first + t) * a.q_stride + head * D + 8 * lh;
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) qf[q][ds] = *reinterpret_cast<const x8*>(from + 16 * ds);
  }

  f32x16 o[QT][DT];
  float m[QT], l[QT];           // reference (in the exponent of 2), sum of the probabilities of this lane's keys
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    m[q] = -FLT_MAX;
    l[q] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[q][dt][i] = 0.f;
  }

  Pages pages{a.table + (int64_t)w.seq * a.max_pages, end, a.unit_shift, a.n_pages, a.max_pages - 1};
  const uint32_t k_lane = (uint32_t)lane * 16, v_lane = (uint32_t)(lh * D + l32) * 16;
  x8 kr[2][DS], vr[2 * DT];
  auto tile_at = [&](const void* cache, int u, int page) {
    const int64_t tile = ((int64_t)page * a.kv_heads + w.head) * (1 << a.unit_shift) + (u & ((1 << a.unit_shift) - 1));
    return uniform_ptr((const unsigned char*)cache + tile * (32 * D * 2));
  };
  auto load = [&](auto odd, int u, int page) {
    const unsigned char* const kb = tile_at(a.k_cache, u, page);
#pragma unroll
    for (int c = 0; c < DS; ++c) kr[decltype(odd)::value][c] = *reinterpret_cast<const x8*>(kb + c * 1024 + k_lane);
  };
  auto load_v = [&](int u, int page) {
    const unsigned char* const vb = tile_at(a.v_cache, u, page);
#pragma unroll
    for (int j = 0; j < 2 * DT; ++j) vr[j] = *reinterpret_cast<const x8*>(vb + j % 2 * (2 * D * 16) + j / 2 * 512 + v_lane);
  };
  // Unit u, whose operands are in registers B.
  auto unit = [&](auto odd, int u) {
    constexpr int B = decltype(odd)::value;
    f32x16 S[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) {
#pragma unroll
      for (int i = 0; i < 16; ++i) S[q][i] = 0.f;
#pragma unroll
      for (int ds = 0; ds < DS; ++ds) S[q] = T::mfma(kr[B][ds], qf[q][ds], S[q]);
    }
    if (u >= free_units) {                                   // keys that a row does not see
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        const int left = limit[q] - 32 * u - 4 * lh;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (8 * (i / 4) + i % 4 >= left) S[q][i] = -INFINITY;
      }
    }
    if (32 * u + 32 > w.s.len) {                             // V behind the last token: 0 times whatever is there has to be 0
#pragma unroll
      for (int j = 0; j < 2 * DT; ++j) {
        const int left = w.s.len - 32 * u - 16 * (j % 2) - 4 * lh;
        u32x4 x = __builtin_bit_cast(u32x4, vr[j]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = e / 2 * 8 + e % 2 * 2;
          x[e] &= (key < left ? 0xffffu : 0u) | (key + 1 < left ? 0xffff0000u : 0u);
        }
        vr[j] = __builtin_bit_cast(x8, x);
      }
    }
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      uint32_t P[8];
      float sum;
      auto probabilities = [&] {
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(S[q][i], a.scale_log2, -m[q]));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(S[q][i + 1], a.scale_log2, -m[q]));
          const typename T::x2 pk = {(typename T::x1)p0, (typename T::x1)p1};
          sum += p0 + p1;
          P[i / 2] = __builtin_bit_cast(uint32_t, pk);
        }
      };
      probabilities();
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum <= T::RANGE)) != 0ull, 0)) {
        // Out of range, or the first unit with a key: the reference moves to the largest exponent, what is there is rescaled.
        float top = S[q][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, S[q][i]);
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * a.scale_log2 - T::HEAD, -FLT_MAX);
        const float to = fmaxf(m[q], top), alpha = __builtin_amdgcn_exp2f(m[q] - to);
        m[q] = to;
        l[q] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[q][dt][i] *= alpha;
        probabilities();
      }
      l[q] += sum;
#pragma unroll
      for (int j = 0; j < 2 * DT; ++j) {
        const u32x4 p = {P[4 * (j % 2)], P[4 * (j % 2) + 1], P[4 * (j % 2) + 2], P[4 * (j % 2) + 3]};
        o[q][j / 2] = T::mfma(vr[j], __builtin_bit_cast(x8, p), o[q][j / 2]);
      }
    }
  };
  if (begin < end) {
    pages.begin(begin);
    int u = pages.seek(begin);
    if (u < end) {
      int page = pages.page(u);
      load(std::integral_constant<int, 0>{}, u, page);
      while (true) {
        // (past the last unit it is fetched again: no branch stands between a load and its use)
        const int u1 = pages.seek(u + 1), page1 = u1 < end ? pages.page(u1) : page;
        load_v(u, page);
        load(std::integral_constant<int, 1>{}, u1 < end ? u1 : u, page1);
        unit(std::integral_constant<int, 0>{}, u);
        if (u1 >= end) break;
        u = pages.seek(u1 + 1);
        page = u < end ? pages.page(u) : page1;
        load_v(u1, page1);
        load(std::integral_constant<int, 0>{}, u < end ? u : u1, page);
        unit(std::integral_constant<int, 1>{}, u1);
        if (u >= end) break;
      }
    }
  }

  // sums of the two lane halves, which have different keys of a row
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[q]), __float_as_uint(l[q]), false, false);
    l[q] = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
  // Wavefronts that share the keys: each finishes the channels of one tile of O (those beyond DT none).
  if constexpr (KW > 1) {
    static_assert(QT == 1 && KW >= DT, "a tile to a wavefront");
    __shared__ float4 tiles[KW][DT][4][64];
    __shared__ float2 stats[KW][32];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      if (dt != kw)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          tiles[kw][dt][g][lane] = make_float4(o[0][dt][4 * g], o[0][dt][4 * g + 1], o[0][dt][4 * g + 2], o[0][dt][4 * g + 3]);
    if (lh == 0) stats[kw][l32] = make_float2(m[0], l[0]);
    __syncthreads();
    float top = m[0], sum = 0.f;
#pragma unroll
    for (int k = 0; k < KW; ++k) top = fmaxf(top, stats[k][l32].x);
    const float own = __builtin_amdgcn_exp2f(m[0] - top);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      if (dt == kw)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[0][dt][i] *= own;
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      const float2 st = stats[k][l32];
      const float weight = __builtin_amdgcn_exp2f(st.x - top);
      sum = fmaf(st.y, weight, sum);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        if (dt == kw && k != kw)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const float4 x = tiles[k][dt][g][lane];
            o[0][dt][4 * g] = fmaf(x.x, weight, o[0][dt][4 * g]);
            o[0][dt][4 * g + 1] = fmaf(x.y, weight, o[0][dt][4 * g + 1]);
            o[0][dt][4 * g + 2] = fmaf(x.z, weight, o[0][dt][4 * g + 2]);
            o[0][dt][4 * g + 3] = fmaf(x.w, weight, o[0][dt][4 * g + 3]);
          }
    }
    m[0] = top;
    l[0] = sum;
  }
  const int64_t place = w.place + ((int64_t)w.head * w.chunks + w.chunk) * w.tiles + w.tile;
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    if (row[q] >= n_rows) continue;
    const float f = whole ? (l[q] > 0.f ? 1.0f / l[q] : (l[q] == 0.f ? 0.f : l[q])) : 1.0f;     // a row that sees no key yields zeros
    const int r = row[q] - w.tile * ROWS;
    float* const part = a.parts + place * (ROWS * (D + 2));
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      if (KW > 1 && dt != kw) continue;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int ch = 32 * dt + 8 * g + 4 * lh;
        if (whole) {
          typename T::x4 pk;
#pragma unroll
          for (int e = 0; e < 4; ++e) pk[e] = (typename T::x1)(o[q][dt][4 * g + e] * f);
          *reinterpret_cast<typename T::x4*>((typename T::x1*)a.o + out_row[q] * D + ch) = pk;
        } else {
          *reinterpret_cast<float4*>(part + r * D + ch) = make_float4(o[q][dt][4 * g], o[q][dt][4 * g + 1], o[q][dt][4 * g + 2], o[q][dt][4 * g + 3]);
        }
      }
    }
    if (lh == 0 && kw == 0) {
      if (!whole) *reinterpret_cast<float2*>(part + ROWS * D + 2 * r) = make_float2(m[q], l[q]);
      else if (a.lse != nullptr) a.lse[out_row[q]] = (m[q] + __log2f(l[q])) * 0.6931471805599453f;
    }
  }
}

// Adds the parts of the tiles that are cut: 8 rows of a tile to a workgroup, 32 lanes to a row.
template <class T, int D, int ROWS>
__global__ void __launch_bounds__(256) join_kernel(Args a) {
  Part w;
  if (!find_part<ROWS, true>(a, blockIdx.x, w)) return;
  const int parts = (tile_units<ROWS>(a, w) + w.units - 1) / w.units;
  if (parts < 2) return;
  constexpr int E = D / 32;                        // channels of a lane
  typedef __attribute__((ext_vector_type(E))) float fE;
  typedef __attribute__((ext_vector_type(E))) typename T::x1 tE;
  const int r = (int)blockIdx.y * 8 + ((int)threadIdx.x >> 5), row = w.tile * ROWS + r, ch = ((int)threadIdx.x & 31) * E;
  if (row >= w.s.n_new * a.group) return;
  const float* const from = a.parts + (w.place + (int64_t)w.head * w.chunks * w.tiles + w.tile) * (ROWS * (D + 2));
  const int64_t step = (int64_t)w.tiles * (ROWS * (D + 2));
  float top = -FLT_MAX;
  for (int p = 0; p < parts; ++p) top = fmaxf(top, from[p * step + ROWS * D + 2 * r]);
  float sum = 0.f;
  fE acc = (fE)0.f;
#pragma unroll 4
  for (int p = 0; p < parts; ++p) {
    const float2 st = *reinterpret_cast<const float2*>(from + p * step + ROWS * D + 2 * r);
    const float weight = __builtin_amdgcn_exp2f(st.x - top);
    const fE x = *reinterpret_cast<const fE*>(from + p * step + r * D + ch);
    sum = fmaf(st.y, weight, sum);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(x[e], weight, acc[e]);
  }
  const float f = sum > 0.f ? 1.0f / sum : (sum == 0.f ? 0.f : sum);
  const int t = row / a.group;
  const int64_t out = (int64_t)(w.s.first + t) * a.heads + w.head * a.group + row % a.group;
  tE pk;
#pragma unroll
  for (int e = 0; e < E; ++e) pk[e] = (typename T::x1)(acc[e] * f);
  *reinterpret_cast<tE*>((typename T::x1*)a.o + out * D + ch) = pk;
  if (a.lse != nullptr && ch == 0) a.lse[out] = (top + __log2f(sum)) * 0.6931471805599453f;
}

template <class T, int D, int QT, int RW, int KW>
int launch(const rf2_paged_plan* plan, Args a, hipStream_t st) {
  constexpr int ROWS = 32 * QT * RW;
  const rf2_paged_config& c = plan->cfg;
  a.aimed = rf2_paged_parts_per_head(c.kv_heads);
  a.least = KW > 1 ? 16 : 8;
  // tiles there can be: a sequence has at most one that is not full
  const int64_t rows = (int64_t)a.n_tokens * a.group;
  const int64_t tiles = std::min(rows / ROWS + std::min(a.n_seqs, a.n_tokens), (int64_t)a.n_tokens * ((a.group + ROWS - 1) / ROWS));
  const bool can_be_cut = (int64_t)c.max_pages * c.page > 32 * a.least;
  const int64_t grid = (tiles + (can_be_cut ? a.aimed : 0)) * c.kv_heads;
  if (grid * 64 * RW * KW >= (int64_t)1 << 32) return RF2_ERR_UNSUPPORTED;
  paged_attn_kernel<T, D, QT, RW, KW><<<dim3((unsigned)grid), dim3(64 * RW * KW), 0, st>>>(a);
  RF2_LAUNCH_CHECK();
  if (can_be_cut) {
    // (of tiles that are cut there are at most as many as parts are aimed at)
    const unsigned some = (unsigned)(std::min(tiles, (int64_t)a.aimed) * c.kv_heads);
    const unsigned rows_of_tile = (unsigned)std::min((int64_t)ROWS, rows);
    join_kernel<T, D, ROWS><<<dim3(some, (rows_of_tile + 7) / 8), dim3(256), 0, st>>>(a);
    RF2_LAUNCH_CHECK();
  }
  return RF2_OK;
}

template <class T, int D>
int dispatch(const rf2_paged_plan* plan, const Args& a, hipStream_t st) {
  // Up to 64 rows a sequence on average: one tile of 32 rows, four wavefronts share its keys.  More: two wavefronts of 64 rows.
  if ((int64_t)a.n_tokens * a.group <= 64 * (int64_t)a.n_seqs) return launch<T, D, 1, 1, 4>(plan, a, st);
  return launch<T, D, 2, 2, 1>(plan, a, st);
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
  a.unit_shift = __builtin_ctz((unsigned)c.page) - 5;
  a.n_pages = c.n_pages, a.max_pages = c.max_pages, a.causal = c.causal;
  a.scale_log2 = plan->scale_log2;
  const bool bf16 = c.dtype == RF2_DTYPE_BF16;
  hipStream_t st = (hipStream_t)stream;
  if (c.head_dim == 128) return bf16 ? dispatch<Bf16, 128>(plan, a, st) : dispatch<F16, 128>(plan, a, st);
  return bf16 ? dispatch<Bf16, 64>(plan, a, st) : dispatch<F16, 64>(plan, a, st);
}
