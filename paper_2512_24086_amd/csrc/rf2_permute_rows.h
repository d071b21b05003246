// What the permutations of Q, K and V share: streams past or through the caches, V's operand parts, overlapping tensors (not installed).
#pragma once
#include "rf2_internal.h"

// KEEP of a layer of `bh` heads in all (rf2_permute.hip)
int rf2_permute_keep(const rf2_plan* plan, int64_t bh);

namespace {

typedef unsigned short u16;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

// KEEP 0: every row is read and written past the caches, 1: stores are kept there, 2: loads too
template <bool KEEP>
__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
  const u32x4* const from = reinterpret_cast<const u32x4*>(p);
  const u32x4 v = KEEP ? *from : __builtin_nontemporal_load(from);
  return make_uint4(v.x, v.y, v.z, v.w);
}
template <bool KEEP>
__device__ __forceinline__ void st_stream(uint4* p, uint4 v) {
  const u32x4 w = {v.x, v.y, v.z, v.w};
  if constexpr (KEEP) *reinterpret_cast<u32x4*>(p) = w;
  else __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p));
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Position inside a 16-key group of the key-major V tile -> key offset (see rf2.h).
__device__ __forceinline__ int rho(int r) { return (r & 3) | ((r & 4) << 1) | ((r & 8) >> 1); }

// One workgroup gathers the 64 permuted rows of V that make up one operand part into LDS and writes
// the part [8][D][8] of the attention kernel's second product (16 KiB or 8 KiB, contiguous).
// Storage position s of a key inside its block: each 16-key group is listed in the order
// 0-3, 8-11, 4-7, 12-15.  With KH = BLK/2, position s goes to part (s % KH) / 32, chunk
// g = (s / KH)*4 + (s % 32) / 8, element s % 8; the 16-byte chunk (part, g, ch) holds
// channel ch of those 8 keys.  A part thus holds the block rows 32*part .. 32*part+31 and
// KH + 32*part .. KH + 32*part + 31 (the reordering stays inside a 16-key group).
template <int D>
using v_rows = u16[64 * (D + 2)];
template <int D, int BLK, int KEEP>
__device__ __forceinline__ void permute_vtile_part(
    const uint4* __restrict__ v, uint4* __restrict__ vp, const int32_t* __restrict__ perm, int n_blocks, int heads,
    const rf2_strides& st, int block_part, int bh, v_rows<D>& tile) {
  constexpr int CH = D / 8;
  constexpr int RG = 256 / CH;
  constexpr int PITCH = D + 2;       // u16 elements per LDS row: odd number of dwords
  constexpr int PB = BLK / 64, KH = BLK / 2;
  const int blk = block_part / PB, part = block_part % PB;
  const uint4* __restrict__ src = v + ((bh / heads) * st.batch + (bh % heads) * st.head) * CH;
  const int c = threadIdx.x % CH, rg = threadIdx.x / CH;
#pragma unroll
  for (int lr = rg; lr < 64; lr += RG) {                      // local row -> block row
    const int r = (lr / 32) * KH + part * 32 + lr % 32;
    const int n = perm[blk * BLK + r];
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (n >= 0) x = ld_stream<KEEP == 2>(&src[(size_t)n * st.token * CH + c]);
    uint32_t* row = reinterpret_cast<uint32_t*>(tile + lr * PITCH + c * 8);  // 4-byte aligned: PITCH, c*8 even
    row[0] = x.x; row[1] = x.y; row[2] = x.z; row[3] = x.w;
  }
  __syncthreads();
  uint4* __restrict__ dst = vp + (((size_t)bh * n_blocks + blk) * PB + part) * D * 8;
  for (int o = threadIdx.x; o < D * 8; o += 256) {
    const int g = o / D, ch = o % D;   // consecutive lanes -> consecutive channels: contiguous 16-byte stores
    const int sbase = (g / 4) * 32 + (g % 4) * 8;             // first local storage position of this chunk
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int s0 = sbase + 2 * e, s1 = s0 + 1;
      const int k0 = (s0 & ~15) + rho(s0 & 15), k1 = (s1 & ~15) + rho(s1 & 15);
      w[e] = (uint32_t)tile[k0 * PITCH + ch] | ((uint32_t)tile[k1 * PITCH + ch] << 16);
    }
    st_stream<KEEP >= 1>(&dst[o], make_uint4(w[0], w[1], w[2], w[3]));
  }
}

// Q and K blocks of a launch, and its V parts.
struct PermuteArgs {
  const uint4 *q, *k, *v;
  uint4 *qp, *kp, *vp;
  float *qbar, *kbar;
  const int32_t* perm;
  uint32_t n_q, n_k, bh;            // Q and K blocks of a head, heads of all batches
  uint32_t q_wgs, k_wgs, v_wgs;     // workgroups of the launch for each tensor
  int last_q, last_k, heads;
  rf2_strides st;
};
// Whether what is written for one of the three tensors shares memory with what is read or written for another: a caller
// may lay kp over q, and vp over k or q, to save a buffer.
bool tensors_overlap(const rf2_plan* plan, const PermuteArgs& a) {
  const rf2_info& in = plan->info;
  const uint64_t row = (uint64_t)a.bh * plan->cfg.head_dim * 2;
  struct Range { const void* at; uint64_t bytes; int tensor; bool written; };
  const Range r[] = {{a.q, row * in.N, 0, false}, {a.k, row * in.N, 1, false}, {a.v, row * in.N, 2, false},
                     {a.qp, row * in.N_pad, 0, true}, {a.kp, row * in.N_pad_k, 1, true}, {a.vp, row * in.N_pad_k, 2, true},
                     {a.qbar, a.qbar ? row * 2 * a.n_q : 0, 0, true}, {a.kbar, a.kbar ? row * 2 * a.n_k : 0, 1, true}};
  for (const Range& x : r)
    for (const Range& y : r)
      if (x.written && x.tensor != y.tensor && (uint64_t)x.at < (uint64_t)y.at + y.bytes &&
          (uint64_t)y.at < (uint64_t)x.at + x.bytes)
        return true;
  return false;
}

}  // namespace
