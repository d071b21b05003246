// Pages and slots of a paged cache from the lengths of its sequences, and the way back of pages (gfx950).
//
// With P tokens to a page, sequence s needs need_s = ceil((len_s + new_s) / P) - ceil(len_s / P) new pages; the sums
// cu_s of new_r and base_s of need_r over r < s say which rows and which entries of the stack are its own, so pages are
// dealt without atomics and the same call always gives the same tables.
#include "rf2_paged.h"
#include "rf2_paged_wave.h"

namespace {

// wave_sums for values of up to 2^40 (20 bits at a time: no part overflows).
__device__ __forceinline__ int64_t wave_sums64(int64_t x) {
  return ((int64_t)wave_sums((uint32_t)(x >> 20)) << 20) + wave_sums((uint32_t)x & 0xfffffu);
}

// What the wavefronts of a workgroup tell each other: two sums and flags.
struct Across {
  int64_t a[16], b[16];
  int flags[16];
};
// Sums over the workgroup of what the threads before this one have, in a and b; of all, in all_a and all_b; flags of all.
template <int NT>
__device__ __forceinline__ void block_sums(Across& m, int64_t& a, int64_t& b, int64_t& all_a, int64_t& all_b, int& flags) {
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const int64_t sum_a = wave_sums64(a), sum_b = wave_sums64(b);
  int set = 0;
#pragma unroll
  for (int bit = 1; bit <= RF2_PAGED_POOL_FULL; bit *= 2) set |= __builtin_amdgcn_ballot_w64((flags & bit) != 0) != 0 ? bit : 0;
  if (lane == 63) m.a[wave] = sum_a, m.b[wave] = sum_b, m.flags[wave] = set;
  __syncthreads();
  int64_t before_a = 0, before_b = 0;
  all_a = all_b = 0;
  flags = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    before_a += w < wave ? m.a[w] : 0;
    before_b += w < wave ? m.b[w] : 0;
    all_a += m.a[w];
    all_b += m.b[w];
    flags |= m.flags[w];
  }
  a = before_a + sum_a - a;
  b = before_b + sum_b - b;
}

struct AppendArgs {
  const int32_t *seq_len, *new_len, *free_pages, *n_free;
  int32_t *table, *seq_len_out, *n_free_out, *cu_new, *slots, *status;
  int n_seqs, n_tokens, page_shift, max_pages, n_pages;
};

// What the workgroup knows of the sequences: in LDS, 48 KiB.
struct Lengths {
  int32_t cu[RF2_PAGED_MAX_SEQS + 1];   // rows before a sequence
  int32_t base[RF2_PAGED_MAX_SEQS];     // new pages before it
  int32_t old[RF2_PAGED_MAX_SEQS];      // its tokens so far
  Across across;
};

__device__ __forceinline__ int pages_of(int64_t tokens, int shift) { return (int)((tokens + (1 << shift) - 1) >> shift); }

// Slots of the tokens `first`, `first` + step, ... and the table entries of the pages that begin with one of them.
__device__ __forceinline__ void deal_slots(const AppendArgs& a, const Lengths& m, int n_free, bool fine, int first, int end, int step) {
  const int P1 = (1 << a.page_shift) - 1, total = m.cu[a.n_seqs];
  for (int i = first; i < end; i += step) {
    int slot = -1;
    if (fine && i < total) {
      int lo = 0, hi = a.n_seqs;                    // the last sequence that begins at or before i (it is the one that is not empty)
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (m.cu[mid] <= i) lo = mid; else hi = mid;
      }
      const int old = m.old[lo], pos = old + i - m.cu[lo], at = pos >> a.page_shift, have = pages_of(old, a.page_shift);
      const int64_t entry = (int64_t)lo * a.max_pages + at;
      int page;
      if (at < have) {
        page = a.table[entry];
      } else {
        page = a.free_pages[n_free - 1 - (m.base[lo] + at - have)];
        if ((pos & P1) == 0) a.table[entry] = page;
      }
      if ((unsigned)page < (unsigned)a.n_pages) slot = (page << a.page_shift) + (pos & P1);
    }
    a.slots[i] = slot;
  }
}

constexpr int SLOT_THREADS = 1024, SLOTS_OF_GROUP = 2 * SLOT_THREADS;

// Sums, checks, lengths; with `slots` the slots too, by one workgroup or SLOTS_OF_GROUP by each: all do the sums, the first writes
// what is not a slot.  Every thread has a run of sequences.  Bound by its latency: 2.8 us for 24 single tokens (a launch takes about 3).
template <int NT>
__global__ void __launch_bounds__(NT) append_kernel(AppendArgs a, bool slots) {
  __shared__ Lengths m;
  const int run = (a.n_seqs + NT - 1) / NT, s0 = min((int)threadIdx.x * run, a.n_seqs), s1 = min(s0 + run, a.n_seqs);
  const int64_t cap = (int64_t)a.max_pages << a.page_shift;
  const int n_free = a.n_free[0];
  const bool writes = blockIdx.x == 0;
  int bad = n_free < 0 || n_free > a.n_pages ? RF2_PAGED_BAD_LENGTH : 0;
  int64_t cu = 0, base = 0;
  for (int s = s0; s < s1; ++s) {
    const int old = a.seq_len[s], more = a.new_len[s];
    m.old[s] = old;
    if (more < 0 || old < 0 || old > cap) { bad |= RF2_PAGED_BAD_LENGTH; continue; }
    if ((int64_t)old + more > cap) bad |= RF2_PAGED_SEQ_FULL;
    cu += more;
    base += pages_of((int64_t)old + more, a.page_shift) - pages_of(old, a.page_shift);
  }
  int64_t all_tokens, all_pages;
  int status = bad;
  block_sums<NT>(m.across, cu, base, all_tokens, all_pages, status);
  if (all_tokens > a.n_tokens) status |= RF2_PAGED_TOKENS_FULL;
  if (all_pages > n_free) status |= RF2_PAGED_POOL_FULL;
  const bool fine = status == 0;
  for (int s = s0; s < s1; ++s) {
    const int old = m.old[s], more = fine ? a.new_len[s] : 0;
    m.cu[s] = fine ? (int)cu : 0;
    m.base[s] = (int)base;
    if (writes) a.cu_new[s] = m.cu[s], a.seq_len_out[s] = old + more;
    if (fine) {
      cu += more;
      base += pages_of((int64_t)old + more, a.page_shift) - pages_of(old, a.page_shift);
    }
  }
  if (threadIdx.x == 0) {
    m.cu[a.n_seqs] = fine ? (int)all_tokens : 0;
    if (writes) {
      a.cu_new[a.n_seqs] = m.cu[a.n_seqs];
      a.n_free_out[0] = fine ? n_free - (int)all_pages : n_free;
      a.status[0] = status;
    }
  }
  if (!slots) return;
  __syncthreads();
  const int first = (int)blockIdx.x * SLOTS_OF_GROUP;
  deal_slots(a, m, n_free, fine, first + (int)threadIdx.x, gridDim.x == 1 ? a.n_tokens : min(first + SLOTS_OF_GROUP, a.n_tokens), NT);
}

// Slots where there are many and outputs lie over inputs, so that these have to be read before: every workgroup repeats the sums, from
// what append_kernel left.
__global__ void __launch_bounds__(SLOT_THREADS) slots_kernel(AppendArgs a) {
  constexpr int NT = SLOT_THREADS;
  __shared__ Lengths m;
  const int run = (a.n_seqs + NT - 1) / NT, s0 = min((int)threadIdx.x * run, a.n_seqs), s1 = min(s0 + run, a.n_seqs);
  const int n_free = a.n_free_out[0];
  const bool fine = a.status[0] == 0;
  int64_t base = 0, none = 0, all_pages = 0, no_sum;
  if (fine) {
    for (int s = s0; s < s1; ++s) {
      const int now = a.seq_len_out[s], old = now - a.new_len[s];
      m.old[s] = old;
      m.cu[s] = a.cu_new[s];
      base += pages_of(now, a.page_shift) - pages_of(old, a.page_shift);
    }
    if (threadIdx.x == 0) m.cu[a.n_seqs] = a.cu_new[a.n_seqs];
    int flags = 0;
    block_sums<NT>(m.across, base, none, all_pages, no_sum, flags);
    for (int s = s0; s < s1; ++s) {
      m.base[s] = (int)base;
      base += pages_of(a.seq_len_out[s], a.page_shift) - pages_of(m.old[s], a.page_shift);
    }
  } else if (threadIdx.x == 0) {
    m.cu[a.n_seqs] = 0;
  }
  __syncthreads();
  const int first = (int)blockIdx.x * SLOTS_OF_GROUP;
  deal_slots(a, m, n_free + (int)all_pages, fine, first + (int)threadIdx.x, min(first + SLOTS_OF_GROUP, a.n_tokens), NT);
}

struct ReleaseArgs {
  const uint8_t* done;
  const int32_t *seq_len, *table, *n_free;
  int32_t *free_pages, *seq_len_out, *n_free_out, *status;
  int n_seqs, page_shift, max_pages, n_pages;
};

// One workgroup.  The columns of all sequences that give back stand in one row of `all` entries, of which a round takes
// NT * DEEP, a wavefront 64 * DEEP side by side; what is a page among them goes to the next places of the stack.  Bound by what one
// compute unit issues to find each entry's place: 29,000 entries of 264 sequences, a fifth of them holes, 18.3 us.
template <int NT>
__global__ void __launch_bounds__(NT) release_kernel(ReleaseArgs a) {
  constexpr int DEEP = 8, WAVES = NT / 64, OF_WAVE = 64 * DEEP;
  __shared__ Across across;
  __shared__ int32_t first[RF2_PAGED_MAX_SEQS + 1];    // entries before a sequence that gives some back
  __shared__ uint16_t which[RF2_PAGED_MAX_SEQS];       // its row of the table
  __shared__ int32_t found[2][WAVES];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int run = (a.n_seqs + NT - 1) / NT, s0 = min((int)threadIdx.x * run, a.n_seqs), s1 = min(s0 + run, a.n_seqs);
  const int64_t cap = (int64_t)a.max_pages << a.page_shift;
  const int n_free = a.n_free[0];
  int flags = n_free < 0 || n_free > a.n_pages ? RF2_PAGED_BAD_LENGTH : 0;
  int64_t before = 0, rows = 0, all64, all_rows;
  for (int s = s0; s < s1; ++s) {
    const int len = a.seq_len[s];
    if (len < 0 || len > cap) flags |= RF2_PAGED_BAD_LENGTH;
    else if (a.done[s] && len > 0) before += pages_of(len, a.page_shift), rows += 1;
  }
  block_sums<NT>(across, before, rows, all64, all_rows, flags);
  int status = flags;
  const int all = status ? 0 : (int)all64, n_rows = (int)all_rows;
  if (!status) {
    for (int s = s0; s < s1; ++s) {
      const int len = a.seq_len[s];
      if (!a.done[s] || len == 0) continue;
      first[rows] = (int)before;
      which[rows] = (uint16_t)s;
      before += pages_of(len, a.page_shift);
      rows += 1;
    }
    if (threadIdx.x == 0) first[n_rows] = all;
  }
  __syncthreads();
  // Entries of a round that begin at `at` for this wavefront.  Its place among the sequences only moves on.  Where the 64
  // sequences from there on begin stands in its lanes, so that a step from one to the next is a step of the scalar unit.
  int place = 0;
  auto look = [&](int at, int (&entry)[DEEP]) __attribute__((always_inline)) {
    int begins = 0, cells = 0, held = 0;             // of sequence place + lane, what an entry is from its cell; of how many this is known
    auto hold = [&]() __attribute__((always_inline)) {
      begins = first[min(place + lane, n_rows)];
      cells = which[min(place + lane, max(n_rows - 1, 0))] * a.max_pages - begins;      // (a table has at most 2^30 cells)
      held = min(64, n_rows - place);
    };
    if (at < all) {
      while (true) {                                 // (64 sequences' ends at a time)
        const int next = place + 1 + lane;
        const int passed = __popcll(__builtin_amdgcn_ballot_w64(next < n_rows && first[min(next, n_rows)] <= at));
        place += passed;
        if (passed < 64) break;
      }
      hold();
    }
    int k = 0;                                       // the sequence looked at is number place + k
#pragma unroll
    for (int j = 0; j < DEEP; ++j) {
      const int from = at + 64 * j, i = from + lane;
      entry[j] = -1;
      if (from >= all) continue;
      int cell = 0;                                  // of entry i in the table
      bool more;
      do {                                           // sequences that begin before the end of the 64 entries
        const int begin = __builtin_amdgcn_readlane(begins, k), to = __builtin_amdgcn_readlane(cells, k);
        cell = i >= begin ? i + to : cell;
        int next = k + 1;
        if (next == held && place + held < n_rows) {
          place += k;                                // (the last one stays: entries of it may follow)
          hold();
          k = 0, next = 1;
        }
        more = next < held && __builtin_amdgcn_readlane(begins, next & 63) < from + 64;
        if (more) k = next;
      } while (more);
      if (i < all) entry[j] = a.table[cell];
    }
    place += k;
  };
  // How many pages stand before the wavefront's entries in the round, and how many there are in all.
  int turn = 0;
  auto count = [&](const int (&entry)[DEEP], int& ahead) __attribute__((always_inline)) {
    int mine = 0;
#pragma unroll
    for (int j = 0; j < DEEP; ++j) mine += __popcll(__builtin_amdgcn_ballot_w64((unsigned)entry[j] < (unsigned)a.n_pages));
    if (lane == 0) found[turn][wave] = mine;
    __syncthreads();
    int sum = 0;
    ahead = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      ahead += w < wave ? found[turn][w] : 0;
      sum += found[turn][w];
    }
    turn ^= 1;                                       // (the next round writes elsewhere: one barrier a round is enough)
    return sum;
  };
  int entry[DEEP], ahead;
  // Only where every entry as a page would be too many is it counted first.
  if (!status && (int64_t)all + n_free > a.n_pages) {
    int64_t pages = 0;
    for (int at = 0; at < all; at += NT * DEEP) {
      look(at + wave * OF_WAVE, entry);
      pages += count(entry, ahead);
    }
    if (pages + n_free > a.n_pages) status |= RF2_PAGED_POOL_FULL;
    place = 0;
  }
  int top = n_free;
  if (!status && all > 0) {
    look(wave * OF_WAVE, entry);
    for (int at = 0; at < all; at += NT * DEEP) {
      int next[DEEP];
      look(at + NT * DEEP + wave * OF_WAVE, next);   // on their way while this round is counted
      const int sum = count(entry, ahead);
      int to = top + ahead;
#pragma unroll
      for (int j = 0; j < DEEP; ++j) {
        const bool page = (unsigned)entry[j] < (unsigned)a.n_pages;
        const uint64_t pages = __builtin_amdgcn_ballot_w64(page);
        if (page) a.free_pages[__builtin_amdgcn_mbcnt_hi((uint32_t)(pages >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)pages, (uint32_t)to))] = entry[j];
        to += __popcll(pages);
        entry[j] = next[j];
      }
      top += sum;
    }
  }
  for (int s = s0; s < s1; ++s) a.seq_len_out[s] = !status && a.done[s] ? 0 : a.seq_len[s];
  if (threadIdx.x == 0) {
    a.n_free_out[0] = top;
    a.status[0] = status;
  }
}

int page_shift(const rf2_paged_plan* plan) { return __builtin_ctz((unsigned)plan->cfg.page); }

}  // namespace

extern "C" int rf2_paged_append(const rf2_paged_plan* plan, int32_t n_seqs, int32_t n_tokens, const int32_t* seq_len,
                                const int32_t* new_len, const int32_t* free_pages, const int32_t* n_free, int32_t* block_table,
                                int32_t* seq_len_out, int32_t* n_free_out, int32_t* cu_new, int32_t* slots, int32_t* status,
                                void* stream) {
  if (!plan || n_seqs < 0 || n_seqs > plan->cfg.max_seqs || n_tokens < 0 || n_tokens > plan->cfg.max_tokens) return RF2_ERR_INVALID_ARG;
  if (!free_pages || !n_free || !n_free_out || !cu_new || !status || (n_tokens > 0 && !slots)) return RF2_ERR_INVALID_ARG;
  if (n_seqs > 0 && (!seq_len || !new_len || !block_table || !seq_len_out)) return RF2_ERR_INVALID_ARG;
  for (const void* p : {(const void*)seq_len, (const void*)new_len, (const void*)free_pages, (const void*)n_free, (const void*)block_table,
                        (const void*)seq_len_out, (const void*)n_free_out, (const void*)cu_new, (const void*)slots, (const void*)status})
    if (!rf2_aligned(p, 4)) return RF2_ERR_INVALID_ARG;
  if (const int rc = rf2_check_paged_device(plan)) return rc;
  const AppendArgs a{seq_len, new_len, free_pages, n_free, block_table, seq_len_out, n_free_out, cu_new, slots, status,
                     n_seqs, n_tokens, page_shift(plan), plan->cfg.max_pages, plan->cfg.n_pages};
  // Fewer threads meet sooner (in a graph, 24 single tokens 3.0 us with 256, 3.7 with 1,024; 1,000 of them 7.3 and 5.4).  More slots than a
  // workgroup's go to several, each of which repeats the sums (81,936 tokens of 256 sequences 5.6 us, 8.4 in two launches), unless outputs
  // lie over inputs: then one deals up to 4,096 (5.3 us, 7.2 in two launches; 8,192 7.3 and 6.9), and more are left to a second launch.
  const bool few = n_tokens <= 512 && n_seqs <= 512, over = seq_len_out == seq_len || n_free_out == n_free, two = over && n_tokens > 4096;
  const unsigned groups = std::max(1, (n_tokens + SLOTS_OF_GROUP - 1) / SLOTS_OF_GROUP);
  if (few) append_kernel<256><<<dim3(1), dim3(256), 0, (hipStream_t)stream>>>(a, true);
  else append_kernel<SLOT_THREADS><<<dim3(over ? 1 : groups), dim3(SLOT_THREADS), 0, (hipStream_t)stream>>>(a, !two);
  RF2_LAUNCH_CHECK();
  if (two) {
    slots_kernel<<<dim3(groups), dim3(SLOT_THREADS), 0, (hipStream_t)stream>>>(a);
    RF2_LAUNCH_CHECK();
  }
  return RF2_OK;
}

extern "C" int rf2_paged_release(const rf2_paged_plan* plan, int32_t n_seqs, const uint8_t* done, const int32_t* seq_len,
                                 const int32_t* block_table, int32_t* free_pages, const int32_t* n_free, int32_t* seq_len_out,
                                 int32_t* n_free_out, int32_t* status, void* stream) {
  if (!plan || n_seqs < 0 || n_seqs > plan->cfg.max_seqs) return RF2_ERR_INVALID_ARG;
  if (!free_pages || !n_free || !n_free_out || !status) return RF2_ERR_INVALID_ARG;
  if (n_seqs > 0 && (!done || !seq_len || !block_table || !seq_len_out)) return RF2_ERR_INVALID_ARG;
  for (const void* p : {(const void*)seq_len, (const void*)block_table, (const void*)free_pages, (const void*)n_free,
                        (const void*)seq_len_out, (const void*)n_free_out, (const void*)status})
    if (!rf2_aligned(p, 4)) return RF2_ERR_INVALID_ARG;
  if (const int rc = rf2_check_paged_device(plan)) return rc;
  const ReleaseArgs a{done, seq_len, block_table, n_free, free_pages, seq_len_out, n_free_out, status, n_seqs, page_shift(plan),
                      plan->cfg.max_pages, plan->cfg.n_pages};
  // Two rounds of the smaller workgroup at most (in a graph, 3 sequences of 32 give back in 4.1 us with 256 threads, 5.4 with 1,024; all of
  // 64 with 4,300 pages in 9.1 and 6.7).
  if ((int64_t)n_seqs * plan->cfg.max_pages <= 4096) release_kernel<256><<<dim3(1), dim3(256), 0, (hipStream_t)stream>>>(a);
  else release_kernel<1024><<<dim3(1), dim3(1024), 0, (hipStream_t)stream>>>(a);
  RF2_LAUNCH_CHECK();
  return RF2_OK;
}
