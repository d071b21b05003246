// The search for a workgroup's part of a paged attention launch, run on the host: the header that the kernels include, with 64 lanes
// to a wavefront that take turns.  A lane runs until it hands a value to the others; then the next one does, and when it is
// the first one's turn again every lane has handed its own over (tests/test_paged_parts_host.py compiles and loads this).
#define __HIP_PLATFORM_AMD__
#include <hip/hip_runtime.h>

#include <setjmp.h>
#include <ucontext.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <memory>
#include <vector>

namespace lanes {

constexpr int MOST = 1024, STACK = 96 * 1024;
struct Lane {
  ucontext_t context;
  jmp_buf at;
  std::unique_ptr<char[]> stack;
  bool begun = false;
  int steps = 0;
};
std::vector<Lane> all(MOST);
jmp_buf home;
int count, current;
uint32_t told[2][MOST];
const std::function<void()>* job;

void resume(int i) {
  current = i;
  Lane& l = all[i];
  if (l.begun) _longjmp(l.at, 1);
  l.begun = true;
  setcontext(&l.context);
}
void body() {
  for (;;) {
    (*job)();
    Lane& l = all[current];
    if (l.steps != all[0].steps) std::puts("lanes parted"), std::abort();
    if (_setjmp(l.at) == 0) {
      if (current + 1 == count) _longjmp(home, 1);
      resume(current + 1);
    }
  }
}
// Hands x over; returns what all lanes have.
const uint32_t* meet(uint32_t x) {
  const int me = current;
  Lane& l = all[me];
  uint32_t* const row = told[l.steps++ & 1];
  row[me] = x;
  if (_setjmp(l.at) == 0) resume((me + 1) % count);
  return row;
}
const uint32_t* wave(uint32_t x) {
  const int first = current & ~63;
  return meet(x) + first;
}
void run(int n, const std::function<void()>& f) {
  count = n;
  job = &f;
  for (int i = 0; i < n; ++i) {
    Lane& l = all[i];
    l.steps = 0;
    if (l.stack) continue;
    l.stack.reset(new char[STACK]);
    getcontext(&l.context);
    l.context.uc_stack.ss_sp = l.stack.get();
    l.context.uc_stack.ss_size = STACK;
    l.context.uc_link = nullptr;
    makecontext(&l.context, body, 0);
  }
  if (_setjmp(home) == 0) resume(0);
}

uint32_t readlane(uint32_t x, int from) { return wave(x)[from]; }
uint64_t ballot(bool x) {
  const uint32_t* const v = wave(x);
  uint64_t bits = 0;
  for (int i = 0; i < 64; ++i) bits |= (uint64_t)(v[i] != 0) << i;
  return bits;
}
// row_shr:1 to 15, row_bcast:15 and row_bcast:31, all banks; a lane without a source has 0, or `old`
int update_dpp(int old, int x, int ctrl, int rows, bool zero) {
  const uint32_t* const v = wave((uint32_t)x);
  const int lane = current & 63, row = lane / 16;
  if (!(rows >> row & 1)) return old;
  int from = -1;
  if (ctrl > 0x110 && ctrl < 0x120) from = lane % 16 >= ctrl - 0x110 ? lane - (ctrl - 0x110) : -1;
  else if (ctrl == 0x142) from = row > 0 ? row * 16 - 1 : -1;
  else if (ctrl == 0x143) from = row > 1 ? 31 : -1;
  else std::abort();
  return from >= 0 ? (int)v[from] : zero ? 0 : old;
}

}  // namespace lanes

#undef __device__
#undef __global__
#undef __shared__
#undef __forceinline__
#undef __launch_bounds__
#define __device__
#define __global__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __popcll __builtin_popcountll
#define __syncthreads() (void)lanes::meet(0)
#define __builtin_amdgcn_readfirstlane(x) ((int)lanes::readlane((uint32_t)(x), 0))
#define __builtin_amdgcn_readlane(x, l) ((int)lanes::readlane((uint32_t)(x), l))
#define __builtin_amdgcn_ballot_w64(x) lanes::ballot(x)
#define __builtin_amdgcn_update_dpp(old, x, ctrl, rows, banks, zero) lanes::update_dpp(old, x, ctrl, rows, zero)
#define __builtin_amdgcn_fence(...)
#define __builtin_amdgcn_wave_barrier()
struct ThreadIdx {
  struct X {
    operator unsigned() const { return (unsigned)lanes::current; }
  } x;
};
static ThreadIdx thread_idx;
#define threadIdx thread_idx
using std::max;
using std::min;

#include "rf2_paged_parts.h"

namespace {

// What a workgroup makes of its number: 1, seq, head, tile, chunk, tiles, units, place, joint; or 0.
template <int ROWS>
int run(const rf2_paged_config& c, Args a, int32_t* found, int64_t room) {
  const Sizes size = size_launch<ROWS>(c, a);
  if (size.grid > room) return -1;
  if (a.survey) lanes::run(1024, [&] { survey_kernel<ROWS>(a); });
  for (int64_t block = 0; block < size.grid; ++block)
    lanes::run(64, [&] {
      Part w{};
      const bool yes = find_part<ROWS>(a, (unsigned)block, w);
      const int32_t mine[9] = {yes, w.seq, w.head, w.tile, w.chunk, w.tiles, w.units, w.place, w.joint};
      if (lanes::current == 0) std::copy(mine, mine + 9, found + 9 * block);
    });
  return (int)size.grid;
}

}  // namespace

// Returns the workgroups of the launch; `about`: rows of a tile, joints that are listed, joints and places that the workspace has.
extern "C" int paged_parts(const rf2_paged_config* cfg, int n_seqs, int n_tokens, const int32_t* seq_len, const int32_t* cu_new, int32_t* found,
                           int64_t room, int32_t* about) {
  const rf2_paged_config& c = *cfg;
  int32_t listed = -1;
  std::vector<int4> survey(n_seqs + 1);
  Args a{};
  a.seq_len = seq_len, a.cu_new = cu_new;
  a.parts = (float*)&listed;
  a.survey = n_seqs > RF2_PAGED_SURVEY ? survey.data() : nullptr;
  a.n_seqs = n_seqs, a.n_tokens = n_tokens, a.heads = c.heads, a.kv_heads = c.kv_heads, a.group = c.heads / c.kv_heads;
  a.unit_shift = __builtin_ctz((unsigned)c.page) - 5;
  a.max_pages = c.max_pages;
  const int rows = tile_rows(a), grid = rows == 16 ? run<16>(c, a, found, room) : rows == 32 ? run<32>(c, a, found, room)
                                                                                            : run<RF2_PAGED_ROWS_MANY>(c, a, found, room);
  const int aimed = rf2_paged_parts_per_head(c.kv_heads) * c.kv_heads;
  about[0] = rows, about[1] = listed, about[2] = aimed * RF2_PAGED_JOINTS, about[3] = 2 * aimed;
  return grid;
}
