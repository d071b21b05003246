// Which part of an attention launch a workgroup has (rf2_paged_attn.hip): found by every wavefront from the sequences' lengths, which
// are in device memory.  Apart from the kernels so that the tests can run it on the host too.
#pragma once
#include "rf2_paged.h"
#include "rf2_paged_wave.h"

namespace {

struct Args {
  const void *q, *k_cache, *v_cache;
  const int32_t *table, *seq_len, *cu_new;
  float* parts;
  int4* survey;                           // see survey_kernel; nullptr: there is none
  void* o;
  float* lse;
  int64_t q_stride;
  int n_seqs, n_tokens, heads, kv_heads, group, unit_shift, n_pages, max_pages, causal, aimed, least, places, most_joints, at_once;
  uint32_t group_magic, group_shift;      // see token_of
  float scale_log2;
};

// Token of a row: row / group, for rows below 2^29, as (row * ceil(2^(29 + k) / group)) >> (29 + k) with 2^k >= group: the factor is
// too large by less than 2^k / 2^(29 + k) of a row.
__device__ __forceinline__ int token_of(const Args& a, int row) { return (int)((uint64_t)(uint32_t)row * a.group_magic >> a.group_shift); }

// A sequence of the call.
struct Seq {
  int first, n_new, len;      // rows of q and o; tokens cached
};
__device__ __forceinline__ Seq seq_of(const Args& a, int s) {
  const int first = min(max(a.cu_new[s], 0), a.n_tokens), end = min(max(a.cu_new[s + 1], first), a.n_tokens);
  return {first, end - first, min(max(a.seq_len[s], 0), a.max_pages << (a.unit_shift + 5))};
}
// A value that is the same in every lane, which the compiler cannot always see (it then lives in a scalar register).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int units_of(int keys) { return max((keys + 31) >> 5, 1); }

// What a workgroup works on: a part of a tile of rows.
struct Part {
  int seq, head, tile, chunk;     // chunk: number of the part
  int tiles, units;               // of the sequence; units of a part of it
  Seq s;
  int place, joint;               // of the part among those of the sequences that are cut, of the tile's first rows; -1: it is not cut
};

// What is to be added up, a few rows of a tile that is cut at a time: written by the workgroup of the tile's first part, in the
// workspace behind their number.
struct Joint {
  int parts, place, step;         // parts of the tile (0: the tile has one and is done); place of the first, places to the next
  int row, n_rows;                // first row of the sequence's, how many
  int first, head;                // the sequence's first token, K/V head
  int pad;
};
__device__ __forceinline__ int* joints_count(const Args& a) { return (int*)a.parts; }
__device__ __forceinline__ Joint* joints(const Args& a) { return (Joint*)a.parts + 1; }
// Rows of a joint: a workgroup of join_kernel has 32 lanes for each, 128 or 256 where there are few rows.
template <int ROWS>
constexpr int JOINT = ROWS < RF2_PAGED_ROWS_MANY ? 2 : 8;

// A sequence's share of the parts, and what the ones before it have (of one K/V head).
struct Share {
  unsigned items, places, joints, chunks;
};
template <int ROWS>
__device__ __forceinline__ int tiles_of(const Args& a, const Seq& s) { return (int)((unsigned)(s.n_new * a.group + ROWS - 1) / (unsigned)ROWS); }
template <int ROWS>
__device__ __forceinline__ unsigned joints_of(const Args& a, const Seq& s) { return (unsigned)(s.n_new * a.group + JOINT<ROWS> - 1) / JOINT<ROWS>; }

// Units of a part, of so many units of all tiles.  (Rounded up by more than the sums are off; no sequence has more than 2^19 units.)
__device__ __forceinline__ int parts_of(const Args& a, float work) { return max((int)fminf(work * 1.0001f / (float)a.aimed, 1048576.f) + 1, a.least); }

// Part number `mine` of the launch's (on this XCD, where K/V heads are dealt to them), which is one of sequence `seq`.
template <int ROWS>
__device__ __forceinline__ bool settle(const Args& a, unsigned block, unsigned mine, unsigned heads, int seq, const Seq& s, const Share& before, Part& w) {
  w.seq = seq;
  w.s = s;
  w.tiles = tiles_of<ROWS>(a, s);
  const unsigned n = before.chunks, each = w.tiles * n;
  w.units = (int)((unsigned)(units_of(s.len) + n - 1) / n);          // (all parts alike, but for the last)
  const unsigned rest = mine - before.items * heads, hh = rest / each, x = rest % each;
  w.head = (int)(heads < (unsigned)a.kv_heads ? hh * 8 + (block & 7) : hh);
  w.chunk = (int)(x / (unsigned)w.tiles);
  w.tile = w.tiles - 1 - (int)(x % (unsigned)w.tiles);               // (under a causal mask the last tile is the longest: it goes first)
  w.place = w.joint = -1;
  // Only what is cut has places in the workspace, less of them than there are; tiles that are whole can be any number.
  if (n > 1) {
    w.place = (int)((before.places * a.kv_heads + w.head * each) + x);
    w.joint = (int)(before.joints * a.kv_heads + w.head * joints_of<ROWS>(a, s)) + w.tile * (ROWS / JOINT<ROWS>);
    if (w.place >= a.places || w.joint + ROWS / JOINT<ROWS> > a.most_joints) return false;
  }
  return w.head < a.kv_heads;
}

// Finds part number `block` of the launch.  ROWS: of a tile.  Every wavefront does it for itself, 64 sequences at a time.
template <int ROWS>
__device__ __forceinline__ bool find_part(const Args& a, unsigned block, Part& w) {
  const int lane = (int)threadIdx.x & 63;
  // Workgroups with equal number % 8 share an XCD and its L2.  Where the K/V heads can be dealt to the XCDs evenly, they are.
  const bool dealt = a.kv_heads % 8 == 0;
  const unsigned heads = dealt ? a.kv_heads / 8 : a.kv_heads, mine = dealt ? block >> 3 : block, at = mine / heads;
  if (a.survey) {
    // The last sequence with no more than `at` items before it, of 64 at equal distances and then of those from there on.
    const int n = a.survey[0].x, step = (n + 63) >> 6;
    const auto last = [&](int i, int end) __attribute__((always_inline)) {
      return __popcll(__builtin_amdgcn_ballot_w64(i < end && (unsigned)a.survey[1 + min(i, a.n_seqs - 1)].x <= at)) - 1;
    };
    if (n == 0) return false;
    const int from = uniform(last(lane * step, n)) * step, seq = from + uniform(last(from + lane, min(from + step, n)));
    const int4 r = a.survey[1 + seq];
    const Seq s = seq_of(a, seq);
    if (at >= (unsigned)r.x + tiles_of<ROWS>(a, s) * (unsigned)r.w) return false;
    return settle<ROWS>(a, block, mine, heads, seq, s, {(unsigned)r.x, (unsigned)r.y, (unsigned)r.z, (unsigned)r.w}, w);
  }
  Seq s{0, 0, 0};
  int tiles = 0;
  const auto look = [&](int at) __attribute__((always_inline)) {
    s = at < a.n_seqs ? seq_of(a, at) : Seq{0, 0, 0};
    tiles = tiles_of<ROWS>(a, s);
  };
  float work = 0.f, tokens = 0.f;
  for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
    look(s0 + lane);
    work += (float)tiles * (float)units_of(s.len);
    tokens += (float)s.n_new;
  }
  work = wave_total(work);
  tokens = wave_total(tokens);
  // Rows that overlap, which no table of this library has, can be more than the grid and the workspace are made for: nothing is done.
  // (Sums up to 2^24 are exact, n_tokens is at most 2^20.)
  const int n_seqs = uniform(tokens <= (float)a.n_tokens) ? a.n_seqs : 0;
  int units = parts_of(a, work);
  if (ROWS == RF2_PAGED_ROWS_MANY && a.n_seqs <= 64) {
    // How many parts there are and how they fill the chip's places (for at_once workgroups) counts.  Lane i holds what a launch takes
    // with i + 1 64ths of the parts that are aimed at: rounds of parts of mean length, and what the longest has more, in units; START
    // more a round for first loads and last stores, three times that for each chip full of parts whose sums are written and joined.
    // (As many parts as are aimed at, without a search: one prompt of 100 tokens behind 32,000 at 32 heads on 8 87 us, 74 with it; 16
    // chunks of 32 behind 4,000 96 and 76; 700 tokens beside 15 single ones, D = 64, 24.4 and 27.4: the search itself takes one.
    // START 4: 12 prompts 90 us for 83.6; 16: the same.)
    constexpr float START = 8.f;
    const int mine = max((int)fminf(work * 1.0001f * 64.f / ((float)a.aimed * (float)(lane + 1)), 1048576.f) + 1, a.least);
    const float per = 1.f / (float)mine, my_tiles = (float)tiles, my_units = (float)units_of(s.len);
    const float longest = fminf(-wave_least(tiles > 0 ? -my_units : 0.f), (float)mine);
    float items = 0.f, cut = 0.f;
    for (int i0 = 0; i0 < a.n_seqs; i0 += 4) {       // (lanes without a sequence have no tiles)
#pragma unroll
      for (int i = i0; i < i0 + 4; ++i) {
        const float n = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_tiles), i));
        const float c = ceilf(__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_units), i)) * per);
        items = fmaf(n, c, items);
        cut = fmaf(c > 1.f ? n : 0.f, c, cut);
      }
    }
    const float share = (float)a.kv_heads / (float)a.at_once, mean = work / fmaxf(items, 1.f);
    const float cost = ceilf(items * share) * (mean + START) + 3.f * START * cut * share + (longest - mean);
    const float best = wave_least(cost);
    const uint64_t those = __builtin_amdgcn_ballot_w64(cost <= best);
    units = __builtin_amdgcn_readlane(mine, those == 0 ? 63 : __builtin_ctzll(those));
  }
  unsigned before = 0, places = 0, joined = 0;       // of the sequences before, one head's
  bool found = false, looked = false;                // (looked: the part's sequence is behind us; workgroup 0 goes on for the sums)
  for (int s0 = 0; s0 < n_seqs; s0 += 64) {
    if (a.n_seqs > 64) look(s0 + lane);
    const unsigned chunks = (unsigned)(units_of(s.len) + units - 1) / (unsigned)units;
    const unsigned items = tiles * chunks, cut = chunks > 1 ? items : 0, joint = chunks > 1 ? joints_of<ROWS>(a, s) : 0;
    const unsigned sum = before + wave_sums(items), cut_sum = places + wave_sums(cut), joint_sum = joined + wave_sums(joint);
    const uint64_t past = __builtin_amdgcn_ballot_w64(sum <= at);
    if (!looked && past != ~0ull) {                  // (a lane's sum only grows: the first lane that is beyond)
      looked = true;
      const int l = __builtin_ctzll(~past);
      const auto pick = [&](int x) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(x, l); };
      found = settle<ROWS>(a, block, mine, heads, s0 + l, {pick(s.first), pick(s.n_new), pick(s.len)},
                           {(unsigned)pick((int)(sum - items)), (unsigned)pick((int)(cut_sum - cut)), (unsigned)pick((int)(joint_sum - joint)),
                            (unsigned)pick((int)chunks)}, w);
      if (block != 0) return found;
    }
    before = (unsigned)__builtin_amdgcn_readlane((int)sum, 63);
    places = (unsigned)__builtin_amdgcn_readlane((int)cut_sum, 63);
    joined = (unsigned)__builtin_amdgcn_readlane((int)joint_sum, 63);
  }
  if (block == 0 && threadIdx.x == 0) *joints_count(a) = (int)min(joined * (unsigned)a.kv_heads, (unsigned)a.most_joints);
  return found;
}

// Where a launch has many sequences, what every workgroup would add up is added up once: entry 1 + s is sequence s's Share, entry 0 how many
// sequences there are (none, where rows overlap).  Every thread has a run of sequences.
template <int ROWS>
__global__ void __launch_bounds__(1024) survey_kernel(Args a) {
  __shared__ float sums[2][16];
  __shared__ uint32_t ends[3][16];
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const int run = (a.n_seqs + 1023) >> 10, s0 = min((int)threadIdx.x * run, a.n_seqs), s1 = min(s0 + run, a.n_seqs);
  float work = 0.f, tokens = 0.f;
  for (int i = s0; i < s1; ++i) {
    const Seq s = seq_of(a, i);
    work += (float)tiles_of<ROWS>(a, s) * (float)units_of(s.len);
    tokens += (float)s.n_new;
  }
  work = wave_total(work);
  tokens = wave_total(tokens);
  if (lane == 0) sums[0][wave] = work, sums[1][wave] = tokens;
  __syncthreads();
  work = tokens = 0.f;
  for (int i = 0; i < 16; ++i) work += sums[0][i], tokens += sums[1][i];
  const bool fine = tokens <= (float)a.n_tokens;
  const int units = parts_of(a, work);
  Share mine{0, 0, 0, 0};
  const auto add = [&](const Seq& s) {
    const unsigned chunks = (unsigned)(units_of(s.len) + units - 1) / (unsigned)units, items = tiles_of<ROWS>(a, s) * chunks;
    mine.items += items;
    if (chunks > 1) mine.places += items, mine.joints += joints_of<ROWS>(a, s);
    return chunks;
  };
  for (int i = s0; i < s1; ++i) add(seq_of(a, i));
  const uint32_t all[3] = {wave_sums(mine.items), wave_sums(mine.places), wave_sums(mine.joints)};
  if (lane == 63)
    for (int k = 0; k < 3; ++k) ends[k][wave] = all[k];
  __syncthreads();
  mine = {all[0] - mine.items, all[1] - mine.places, all[2] - mine.joints, 0};
  uint32_t joined = 0;
  for (int i = 0; i < 16; ++i) {
    if (i < wave) mine.items += ends[0][i], mine.places += ends[1][i], mine.joints += ends[2][i];
    joined += ends[2][i];
  }
  for (int i = s0; i < s1; ++i) {
    const Share before = mine;
    const unsigned chunks = add(seq_of(a, i));
    a.survey[1 + i] = make_int4((int)before.items, (int)before.places, (int)before.joints, (int)chunks);
  }
  if (threadIdx.x == 0) {
    a.survey[0] = make_int4(fine ? a.n_seqs : 0, 0, 0, 0);
    *joints_count(a) = fine ? (int)min(joined * (unsigned)a.kv_heads, (unsigned)a.most_joints) : 0;
  }
}

// Rows of a launch's tiles (host).  Up to 32 rows a sequence on average: four wavefronts share the keys of one or two tiles of 16.  More: two wavefronts of 64 rows.
// (16 sequences of 4,000 keys, 8 K/V heads, 48 rows each: 83.7 us as two tiles of 32, 62.1 as one of 128; 128 rows: 131 and 78.6.)
// (16 rows as a tile of 16 or one of 32: 64 single tokens 130.3 and 132.5 us, 16 chunks of 4 tokens behind 4,000 53.5 and 54.9.)
// Rows of padding count, for the lengths are not known here: 64 single tokens among 8,064 rows take 169 us.
inline int tile_rows(const Args& a) {
  const int64_t rows = (int64_t)a.n_tokens * a.group;
  return rows <= 16 * (int64_t)a.n_seqs ? 16 : rows <= 32 * (int64_t)a.n_seqs ? 32 : RF2_PAGED_ROWS_MANY;
}

// How large a launch is, with what of it the workgroups have to know in `a` (host).
struct Sizes {
  int64_t grid, joints;           // workgroups; joints that there can be
  bool can_be_cut;                // else no sequence is long enough
};
template <int ROWS>
Sizes size_launch(const rf2_paged_config& c, Args& a) {
  a.aimed = rf2_paged_parts_per_head(c.kv_heads);
  // No sequence is cut below 16 units (a single token of 2,000 keys 13.1 us, 16.2 with 32), and 8 (with 16 a chunk of 700
  // tokens and 15 single ones take 3% longer; with 4 as long).
  a.least = ROWS < RF2_PAGED_ROWS_MANY ? 16 : 8;
  a.at_once = ROWS < RF2_PAGED_ROWS_MANY || c.head_dim == 128 ? 512 : 1024;      // (of few rows nothing is searched for)
  a.places = 2 * a.aimed * c.kv_heads;
  a.most_joints = a.aimed * c.kv_heads * RF2_PAGED_JOINTS;
  static_assert(ROWS / JOINT<ROWS> <= RF2_PAGED_JOINTS, "the workspace has room for so many to a tile");
  // tiles there can be: a sequence has at most one that is not full
  const int64_t rows = (int64_t)a.n_tokens * a.group, some = std::min(a.n_seqs, a.n_tokens);
  const int64_t tiles = std::min(rows / ROWS + some, (int64_t)a.n_tokens * ((a.group + ROWS - 1) / ROWS));
  const bool can_be_cut = (int64_t)c.max_pages * c.page > 32 * a.least;
  // (2^20 tokens of 512 heads and 4,096 sequences are less than 2^30 threads)
  return {(tiles + (can_be_cut ? a.aimed : 0)) * c.kv_heads, (rows / JOINT<ROWS> + some) * c.kv_heads, can_be_cut};
}

}  // namespace
