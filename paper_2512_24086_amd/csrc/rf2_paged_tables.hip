// Pages and slots of a paged cache from the lengths of its sequences, and the way back of pages (gfx950).
//
// With P tokens to a page, sequence s needs need_s = ceil((len_s + new_s) / P) - ceil(len_s / P) new pages; the sums
// cu_s of new_r and base_s of need_r over r < s say which rows and which entries of the stack are its own, so pages are
// dealt without atomics and the same call always gives the same tables.
#include "rf2_paged.h"

namespace {

constexpr int NT = 1024, WAVES = NT / 64;

// Sum over the workgroup of what the threads before this one have; `total`: of all.
__device__ __forceinline__ int64_t block_scan(int64_t mine, int64_t* across, int64_t& total) {
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  int64_t sum = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t other = __shfl_up(sum, d);
    sum += lane >= d ? other : 0;
  }
  if (lane == 63) across[wave] = sum;
  __syncthreads();
  int64_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    before += w < wave ? across[w] : 0;
    total += across[w];
  }
  __syncthreads();
  return before + sum - mine;
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
  int64_t across[WAVES];
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

// One workgroup: sums, checks, lengths; with `slots` the slots too.  Every thread has a run of sequences.
__global__ void __launch_bounds__(NT) append_kernel(AppendArgs a, bool slots) {
  __shared__ Lengths m;
  const int run = (a.n_seqs + NT - 1) / NT, s0 = min((int)threadIdx.x * run, a.n_seqs), s1 = min(s0 + run, a.n_seqs);
  const int64_t cap = (int64_t)a.max_pages << a.page_shift;
  const int n_free = a.n_free[0];
  int bad = n_free < 0 || n_free > a.n_pages ? RF2_PAGED_BAD_LENGTH : 0;
  int64_t tokens = 0, pages = 0;
  for (int s = s0; s < s1; ++s) {
    const int old = a.seq_len[s], more = a.new_len[s];
    m.old[s] = old;
    if (more < 0 || old < 0 || old > cap) { bad |= RF2_PAGED_BAD_LENGTH; continue; }
    if ((int64_t)old + more > cap) bad |= RF2_PAGED_SEQ_FULL;
    tokens += more;
    pages += pages_of((int64_t)old + more, a.page_shift) - pages_of(old, a.page_shift);
  }
  int64_t all_tokens, all_pages;
  int64_t cu = block_scan(tokens, m.across, all_tokens), base = block_scan(pages, m.across, all_pages);
  if (all_tokens > a.n_tokens) bad |= RF2_PAGED_TOKENS_FULL;
  if (all_pages > n_free) bad |= RF2_PAGED_POOL_FULL;
  int status = 0;
#pragma unroll
  for (int bit = 1; bit <= RF2_PAGED_POOL_FULL; bit *= 2) status |= __syncthreads_or(bad & bit) ? bit : 0;
  const bool fine = status == 0;
  for (int s = s0; s < s1; ++s) {
    const int old = m.old[s], more = fine ? a.new_len[s] : 0;
    m.cu[s] = a.cu_new[s] = fine ? (int)cu : 0;
    m.base[s] = (int)base;
    a.seq_len_out[s] = old + more;
    if (fine) {
      cu += more;
      base += pages_of((int64_t)old + more, a.page_shift) - pages_of(old, a.page_shift);
    }
  }
  if (threadIdx.x == 0) {
    m.cu[a.n_seqs] = a.cu_new[a.n_seqs] = fine ? (int)all_tokens : 0;
    a.n_free_out[0] = fine ? n_free - (int)all_pages : n_free;
    a.status[0] = status;
  }
  if (!slots) return;
  __syncthreads();
  deal_slots(a, m, n_free, fine, (int)threadIdx.x, a.n_tokens, NT);
}

constexpr int SLOTS_OF_GROUP = 2 * NT;

// Slots where there are many: every workgroup repeats the sums (from what append_kernel left, which may lie over its inputs).
__global__ void __launch_bounds__(NT) slots_kernel(AppendArgs a) {
  __shared__ Lengths m;
  const int run = (a.n_seqs + NT - 1) / NT, s0 = min((int)threadIdx.x * run, a.n_seqs), s1 = min(s0 + run, a.n_seqs);
  const bool fine = a.status[0] == 0;
  int64_t pages = 0, all_pages = 0;
  if (fine) {
    for (int s = s0; s < s1; ++s) {
      const int now = a.seq_len_out[s], old = now - a.new_len[s];
      m.old[s] = old;
      m.cu[s] = a.cu_new[s];
      pages += pages_of(now, a.page_shift) - pages_of(old, a.page_shift);
    }
    if (threadIdx.x == 0) m.cu[a.n_seqs] = a.cu_new[a.n_seqs];
    int64_t base = block_scan(pages, m.across, all_pages);
    for (int s = s0; s < s1; ++s) {
      m.base[s] = (int)base;
      base += pages_of(a.seq_len_out[s], a.page_shift) - pages_of(m.old[s], a.page_shift);
    }
  } else if (threadIdx.x == 0) {
    m.cu[a.n_seqs] = 0;
  }
  __syncthreads();
  const int first = (int)blockIdx.x * SLOTS_OF_GROUP;
  deal_slots(a, m, a.n_free_out[0] + (int)all_pages, fine, first + (int)threadIdx.x, min(first + SLOTS_OF_GROUP, a.n_tokens), NT);
}

struct ReleaseArgs {
  const uint8_t* done;
  const int32_t *seq_len, *table, *n_free;
  int32_t *free_pages, *seq_len_out, *n_free_out, *status;
  int n_seqs, page_shift, max_pages, n_pages;
};

// One workgroup.  The columns of all finished sequences stand in one row of `all` entries, of which a round takes NT * DEEP;
// what is a page among them goes to the next places of the stack.
__global__ void __launch_bounds__(NT) release_kernel(ReleaseArgs a) {
  constexpr int DEEP = 4;
  __shared__ int64_t across[WAVES];
  __shared__ int32_t first[RF2_PAGED_MAX_SEQS + 1];    // entries before a sequence
  __shared__ int32_t found[DEEP][WAVES];
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const int run = (a.n_seqs + NT - 1) / NT, s0 = min((int)threadIdx.x * run, a.n_seqs), s1 = min(s0 + run, a.n_seqs);
  const int64_t cap = (int64_t)a.max_pages << a.page_shift;
  const int n_free = a.n_free[0];
  int bad = n_free < 0 || n_free > a.n_pages ? 1 : 0;
  int64_t mine = 0, all64;
  for (int s = s0; s < s1; ++s) {
    const int len = a.seq_len[s];
    if (len < 0 || len > cap) bad = 1;
    else if (a.done[s]) mine += pages_of(len, a.page_shift);
  }
  int64_t before = block_scan(mine, across, all64);
  int status = __syncthreads_or(bad) ? RF2_PAGED_BAD_LENGTH : 0;
  if (all64 > INT32_MAX) status |= RF2_PAGED_POOL_FULL;     // (more than any pool has)
  const int all = status ? 0 : (int)all64;
  if (!status) {
    for (int s = s0; s < s1; ++s) {
      first[s] = (int)before;
      before += a.done[s] ? pages_of(a.seq_len[s], a.page_shift) : 0;
    }
    if (threadIdx.x == 0) first[a.n_seqs] = all;
  }
  __syncthreads();
  // pages among the entries of a round, in order: what stands before a thread's entry of row j, and how many there are
  int entry[DEEP], rank[DEEP];
  auto round = [&](int at) {
#pragma unroll
    for (int j = 0; j < DEEP; ++j) {
      const int i = at + j * NT + (int)threadIdx.x;
      entry[j] = -1;
      if (i < all) {
        int lo = 0, hi = a.n_seqs;
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (first[mid] <= i) lo = mid; else hi = mid;
        }
        entry[j] = a.table[(int64_t)lo * a.max_pages + (i - first[lo])];
      }
    }
#pragma unroll
    for (int j = 0; j < DEEP; ++j) {
      const uint64_t pages = __builtin_amdgcn_ballot_w64((unsigned)entry[j] < (unsigned)a.n_pages);
      rank[j] = __popcll(pages & ((1ull << lane) - 1));
      if (lane == 0) found[j][wave] = __popcll(pages);
    }
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int j = 0; j < DEEP; ++j)
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        rank[j] += w == wave ? sum : 0;
        sum += found[j][w];
      }
    __syncthreads();
    return sum;
  };
  // Only where every entry as a page would be too many is it counted first.
  int64_t pages = all;
  if (!status && pages + n_free > a.n_pages) {
    pages = 0;
    for (int at = 0; at < all; at += NT * DEEP) pages += round(at);
    if (pages + n_free > a.n_pages) status |= RF2_PAGED_POOL_FULL;
  }
  int top = n_free;
  if (!status)
    for (int at = 0; at < all; at += NT * DEEP) {
      const int sum = round(at);
#pragma unroll
      for (int j = 0; j < DEEP; ++j)
        if ((unsigned)entry[j] < (unsigned)a.n_pages) a.free_pages[top + rank[j]] = entry[j];
      top += sum;
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
  // One workgroup deals this many slots in about the time of another launch.
  const bool together = n_tokens <= 4 * NT;
  append_kernel<<<dim3(1), dim3(NT), 0, (hipStream_t)stream>>>(a, together);
  RF2_LAUNCH_CHECK();
  if (!together) {
    slots_kernel<<<dim3((n_tokens + SLOTS_OF_GROUP - 1) / SLOTS_OF_GROUP), dim3(NT), 0, (hipStream_t)stream>>>(a);
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
  release_kernel<<<dim3(1), dim3(NT), 0, (hipStream_t)stream>>>(
      ReleaseArgs{done, seq_len, block_table, n_free, free_pages, seq_len_out, n_free_out, status, n_seqs, page_shift(plan),
                  plan->cfg.max_pages, plan->cfg.n_pages});
  RF2_LAUNCH_CHECK();
  return RF2_OK;
}
