// Norms of heads' rows and rotation by positions, Q and K in one launch, and their gradients (gfx950).
//
// HBM bound: each row is read once and written once.  d / 8 neighbouring lanes hold a row, 16 bytes each.  Cosines and sines belong to a
// token, not to a head: a wavefront takes a few tokens, works their angles out once and goes through the heads, 64 / (d / 8) rows at a
// time.  Those are consecutive tokens of a head where tokens lie side by side, consecutive heads of a token where heads do.  75,600 tokens of
// 40 + 40 heads: 3.1 GB in 497 us, 6.2 TB/s (a large copy reaches 6.2); the vector unit is 77 % busy beside it.  48 tokens: 2.8 us in a graph, 8.0 with
// the host's part of a call.
#include "rf2_rope.h"

namespace {

struct ApplyArgs {
  RopeArgs rope;
  RopeTokens tokens;
  RopeSide side[2];
};

template <class T, int D, bool HALVES, bool NORM, bool KEEP>
__global__ void __launch_bounds__(256) apply_kernel(ApplyArgs a) {
  const uint32_t of_q = a.side[0].share.tiles * (uint32_t)a.side[0].share.groups;
  const bool second = blockIdx.x >= of_q;
  rope_apply_rows<T, D, HALVES, NORM, KEEP>(a.rope, a.tokens, a.side[second ? 1 : 0], blockIdx.x - (second ? of_q : 0));
}

// ---- gradients --------------------------------------------------------------------------------------------------

struct BackSide {
  RopeRows x, dz, dx;
  const void* w;
  float* sums;               // of the workgroups, [workgroups][d]; the gradient itself where there is one workgroup
  RopeShare share;
  uint32_t workgroups;
};
struct BackArgs {
  RopeArgs rope;
  RopeTokens tokens;
  BackSide side[2];
};

// With g = R(-phi) dz and x^ = x r:  dx = r (g w - x^ mean(g w x^)),  dw = sum over rows of g x^.  Sums of dw: a token's heads in 32 bits, a
// lane's tokens in 64, then the rows of the workgroup in order, in 64 too.  A lane's sum and a workgroup's are handed on in 32 bits
// (2^-24 of each, no more than a sum of a token's heads may be off).
//
// HBM bound: x and dz are read once, dx is written once.  Loads of a token's next two heads are asked for before those in hand are worked on.  Large
// calls take 8,192 workgroups for each of Q and K, many more than are resident, which reads faster than few that go round (32,760 tokens of
// 40 + 40 heads: 1,024 354 us, 4,096 336, 8,192 323, and 10 for their sums; sums by elements, read and written alike, take 312).  Smaller ones,
// up to 2,048 units, take 512 at most, whose sums one launch adds up.
template <class T, int D, bool HALVES, bool KEEP>
__global__ void __launch_bounds__(256, 4) backward_kernel(BackArgs a) {
  constexpr int CH = D / 8, R = 64 / CH, U = 2;
  __shared__ float part[4 * R][D + 4];
  const bool second = blockIdx.x >= a.side[0].workgroups;
  const BackSide& s = a.side[second ? 1 : 0];
  const uint32_t id = blockIdx.x - (second ? a.side[0].workgroups : 0);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane % CH, g = lane / CH;
  const int log2 = s.share.heads_log2, by_token = R >> log2;
  const int64_t x_step = s.x.head << log2, dz_step = s.dz.head << log2, dx_step = s.dx.head << log2;
  float w[8];
  rope_weights<T>(a.rope, s.w, c, w);
  const RopeLane angles = rope_lane<D, HALVES>(a.rope, c);
  double total[8] = {};
  for (uint32_t i = id; i < s.share.tiles * (uint32_t)s.share.groups; i += s.workgroups) {
    const RopeUnit unit = rope_unit(s.share, i);
    const uint32_t m = (unit.tile * 4 + wave) * by_token + (g >> log2);
    const int first = unit.group * s.share.steps, end = m < a.tokens.total ? min(s.share.heads >> log2, first + s.share.steps) : 0;
    const int h = (first << log2) + (g & ((1 << log2) - 1));
    const RopeToken t = rope_token(min(m, a.tokens.total - 1), a.tokens.tokens, a.tokens.total);
    const uint16_t* x_at = s.x.at + t.b * s.x.batch + t.n * s.x.token + h * s.x.head + 8 * c;
    const uint16_t* dz_at = s.dz.at + t.b * s.dz.batch + t.n * s.dz.token + h * s.dz.head + 8 * c;
    uint16_t* dx_at = const_cast<uint16_t*>(s.dx.at) + t.b * s.dx.batch + t.n * s.dx.token + h * s.dx.head + 8 * c;
    rope_u32x4 vx[U], vz[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (first + u < end) {
        vx[u] = rope_load<KEEP>(x_at + u * x_step);
        vz[u] = rope_load<KEEP>(dz_at + u * dz_step);
      }
    float cs[8], sn[8], sum[8] = {};
    rope_angles<D, HALVES>(angles, rope_place(a.rope, angles, a.tokens.pos + t.b * a.tokens.pos_batch + (int64_t)t.n * a.rope.axes), c, cs, sn);
    for (int step = first; step < end; step += U) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (step + u < end) {
          float x[8], z[8], y[8];
          T::unpack(vx[u], x);
          T::unpack(vz[u], z);
          const float r = rope_normalise<D>(a.rope, x);
          rope_partners<D, HALVES>(z, y);
          float m = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            z[e] = fmaf(z[e], cs[e], -y[e] * sn[e]);
            sum[e] = fmaf(z[e], x[e], sum[e]);
            z[e] *= w[e];
            m = fmaf(z[e], x[e], m);
          }
          m = rope_row_sum<D>(m) * (1.f / D);
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = r * fmaf(-x[e], m, z[e]);
          rope_store<KEEP>(dx_at + u * dx_step, T::pack(z));
        }
      x_at += U * x_step;
      dz_at += U * dz_step;
      dx_at += U * dx_step;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (step + U + u < end) {
          vx[u] = rope_load<KEEP>(x_at + u * x_step);
          vz[u] = rope_load<KEEP>(dz_at + u * dz_step);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) total[e] += (double)sum[e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) part[wave * R + g][8 * c + e] = (float)total[e];
  __syncthreads();
  if (threadIdx.x < D) {
    double sum = 0;
#pragma unroll
    for (int i = 0; i < 4 * R; ++i) sum += (double)part[i][threadIdx.x];
    s.sums[(size_t)id * D + threadIdx.x] = (float)sum;
  }
}

// The workgroups' sums to one, in 64 bits and a fixed order.  Latency of loads and launches is all it costs.  Up to 512 lines, or runs of many, are added
// up by workgroups of 8 channels each, 128 lines at a time (join_kernel); more lines go to runs of 64 first (runs_kernel): 8,192 lines 9.3
// us, without 23, and 25 in one launch whose last workgroup ends it (counting up in one place for all XCDs is slow).
template <class IN, class OUT>
struct JoinSide {
  const IN* in;              // [lines][d]
  OUT* out;                  // [groups][d]
  uint32_t lines, groups;
};
template <class IN, class OUT>
struct JoinArgs {
  JoinSide<IN, OUT> side[2];
};

template <int D>
__global__ void __launch_bounds__(256) runs_kernel(JoinArgs<float, double> a) {
  constexpr int LANES = D / 4, SLICES = 256 / LANES, U = 64 / SLICES;
  __shared__ double part[SLICES][D];
  const bool second = blockIdx.x >= a.side[0].groups;
  const JoinSide<float, double>& s = a.side[second ? 1 : 0];
  const uint32_t group = blockIdx.x - (second ? a.side[0].groups : 0);
  const int slice = threadIdx.x / LANES, c = threadIdx.x % LANES * 4;
  float4 x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t line = group * 64 + u * SLICES + slice;
    x[u] = line < s.lines ? *reinterpret_cast<const float4*>(s.in + (size_t)line * D + c) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  double sum[4] = {};
#pragma unroll
  for (int u = 0; u < U; ++u) sum[0] += x[u].x, sum[1] += x[u].y, sum[2] += x[u].z, sum[3] += x[u].w;
#pragma unroll
  for (int e = 0; e < 4; ++e) part[slice][c + e] = sum[e];
  __syncthreads();
  if (threadIdx.x < D) {
    double total = 0;
#pragma unroll
    for (int i = 0; i < SLICES; ++i) total += part[i][threadIdx.x];
    s.out[(size_t)group * D + threadIdx.x] = total;
  }
}

template <int D, class IN>
__global__ void __launch_bounds__(1024) join_kernel(JoinArgs<IN, float> a) {
  __shared__ double part[128][8];
  const JoinSide<IN, float>& s = a.side[blockIdx.x / (D / 8)];
  if (s.out == nullptr) return;
  const int ch = blockIdx.x % (D / 8) * 8 + threadIdx.x % 8, slice = threadIdx.x / 8;
  double sum = 0;
#pragma unroll 4
  for (uint32_t i = slice; i < s.lines; i += 128) sum += (double)s.in[(size_t)i * D + ch];
  part[slice][threadIdx.x % 8] = sum;
  __syncthreads();
#pragma unroll
  for (int half = 64; half >= 1; half /= 2) {
    if (slice < half) part[slice][threadIdx.x % 8] += part[slice + half][threadIdx.x % 8];
    __syncthreads();
  }
  if (slice == 0) s.out[ch] = (float)part[0][threadIdx.x];
}
template <class IN>
int launch_join(int d, const JoinArgs<IN, float>& a, hipStream_t st) {
  if (!a.side[0].out && !a.side[1].out) return RF2_OK;
  if (d == 128) join_kernel<128, IN><<<2 * 128 / 8, 1024, 0, st>>>(a);
  else join_kernel<64, IN><<<2 * 64 / 8, 1024, 0, st>>>(a);
  RF2_LAUNCH_CHECK();
  return RF2_OK;
}

// ---- host -------------------------------------------------------------------------------------------------------

// Whether rows can be read (strides of whole 16 bytes), and whether no two of them share memory, so that they can be written.
bool readable(const rf2_rows& r) {
  return rf2_rope_aligned(r.at, 16) && r.batch >= 0 && r.token >= 0 && r.head >= 0 && r.batch % 8 == 0 && r.token % 8 == 0 && r.head % 8 == 0;
}
bool writable(const rf2_rows& r, int32_t batch, int32_t tokens, int32_t heads, int d) {
  if (!readable(r)) return false;
  struct Axis { int64_t stride; int64_t n; } ax[3] = {{r.batch, batch}, {r.token, tokens}, {r.head, heads}};
  std::sort(ax, ax + 3, [](const Axis& x, const Axis& y) { return x.stride < y.stride; });
  int64_t extent = d;                       // of what lies within a step of the next axis
  for (const Axis& x : ax) {
    if (x.n <= 1) continue;
    if (x.stride < extent) return false;
    if (x.stride > ((int64_t)1 << 60) / x.n) return false;
    extent = x.stride * (x.n - 1) + extent;
  }
  return true;
}
// The last element of rows that are read is within what 64 bits count.
bool in_range(const rf2_rows& r, int32_t batch, int32_t tokens, int32_t heads) {
  const int64_t most = (int64_t)1 << 58;
  return r.batch <= most / batch && r.token <= most / tokens && r.head <= most / heads;
}

template <bool B>
using flag = std::integral_constant<bool, B>;

// Rows of Q and K, in and out: all of a side or nothing.  Strides of axes of one say nothing.
int check_rows(const rf2_rope_plan* plan, int32_t batch, int32_t n_tokens, rf2_rows* const (&rows)[2][3], int n) {
  for (int i = 0; i < 2; ++i) {
    const int32_t heads = i == 0 ? plan->cfg.heads : plan->cfg.kv_heads;
    for (int j = 0; j < n; ++j) {
      if (batch == 1) rows[i][j]->batch = 0;
      if (n_tokens == 1) rows[i][j]->token = rows[i][j]->batch;
      if (heads == 1) rows[i][j]->head = 0;
      if ((rows[i][j]->at == nullptr) != (rows[i][n - 1]->at == nullptr)) return RF2_ERR_INVALID_ARG;
      if (rows[i][j]->at && (!readable(*rows[i][j]) || !in_range(*rows[i][j], batch, n_tokens, heads))) return RF2_ERR_INVALID_ARG;
      // (the only token has its heads side by side, whatever its stride is)
      if (rows[i][j]->at && batch == 1 && n_tokens == 1) rows[i][j]->token = rows[i][j]->head * heads;
    }
    const rf2_rows& out = *rows[i][n - 1];
    if (out.at && !writable(out, batch, n_tokens, heads, plan->cfg.head_dim)) return RF2_ERR_INVALID_ARG;
  }
  return rows[0][0]->at || rows[1][0]->at ? RF2_OK : RF2_ERR_INVALID_ARG;
}

int check_tokens(int32_t batch, int32_t n_tokens, int64_t pos_batch) {
  if (batch < 0 || n_tokens < 0 || pos_batch < 0) return RF2_ERR_INVALID_ARG;
  if ((int64_t)batch * n_tokens > (int64_t)1 << 24) return RF2_ERR_UNSUPPORTED;
  return pos_batch <= (int64_t)1 << 32 ? RF2_OK : RF2_ERR_INVALID_ARG;
}

int launch_apply(const rf2_rope_plan* plan, int32_t batch, int32_t n_tokens, const rf2_rows& q, const rf2_rows& k, const int32_t* pos, int64_t pos_batch,
                 const void* wq, const void* wk, const rf2_rows& q_out, const rf2_rows& k_out, bool norm, bool inverse, hipStream_t st) {
  const rf2_rope_config& c = plan->cfg;
  ApplyArgs a{rope_args(plan, inverse), {pos, pos_batch, (uint32_t)n_tokens, (uint32_t)batch * (uint32_t)n_tokens}, {}};
  int64_t bytes = 0;
  for (int i = 0; i < 2; ++i) {
    const rf2_rows& x = i == 0 ? q : k;
    const int heads = i == 0 ? c.heads : c.kv_heads;
    a.side[i] = {rope_rows(x), rope_rows(i == 0 ? q_out : k_out), i == 0 ? wq : wk, rope_share(x, heads, c, a.tokens.total)};
    if (x.at) bytes += (int64_t)a.tokens.total * heads * c.head_dim * 4;
  }
  const dim3 grid(rope_workgroups(a.side[0].share) + rope_workgroups(a.side[1].share));
  return rope_for_types(c, [&](auto type, auto d, auto halves) {
    const auto launch = [&](auto with_norm, auto keep) {
      apply_kernel<decltype(type), d(), halves(), with_norm(), keep()><<<grid, 256, 0, st>>>(a);
    };
    const auto with = [&](auto keep) { norm ? launch(flag<true>(), keep) : launch(flag<false>(), keep); };
    bytes <= ROPE_KEEP ? with(flag<true>()) : with(flag<false>());
  });
}

}  // namespace

extern "C" int rf2_rope_apply(const rf2_rope_plan* plan, int32_t batch, int32_t n_tokens, const rf2_rope_tensors* rows, const int32_t* pos,
                              int64_t pos_batch, const void* wq, const void* wk, void* stream) {
  if (!plan || !rows) return RF2_ERR_INVALID_ARG;
  rf2_rope_tensors t = *rows;
  if (const int rc = check_tokens(batch, n_tokens, pos_batch)) return rc;
  if (batch == 0 || n_tokens == 0) return rf2_check_rope_device(plan);     // (an empty tensor may have no address)
  rf2_rows* const sides[2][3] = {{&t.q, &t.q_out}, {&t.k, &t.k_out}};
  if (const int rc = check_rows(plan, batch, n_tokens, sides, 2)) return rc;
  if (!rf2_rope_pos_fits(plan, pos)) return RF2_ERR_INVALID_ARG;
  if ((t.q.at && !rf2_rope_weight_fits(plan, wq)) || (t.k.at && !rf2_rope_weight_fits(plan, wk))) return RF2_ERR_INVALID_ARG;
  if (const int rc = rf2_check_rope_device(plan)) return rc;
  return launch_apply(plan, batch, n_tokens, t.q, t.k, pos, pos_batch, wq, wk, t.q_out, t.k_out, plan->cfg.norm == RF2_NORM_RMS, false,
                      (hipStream_t)stream);
}

extern "C" int rf2_rope_backward(const rf2_rope_plan* plan, int32_t batch, int32_t n_tokens, const rf2_rope_gradients* rows, const int32_t* pos,
                                 int64_t pos_batch, const void* wq, const void* wk, float* dwq, float* dwk, void* workspace, void* stream) {
  if (!plan || !rows) return RF2_ERR_INVALID_ARG;
  rf2_rope_gradients t = *rows;
  if (const int rc = check_tokens(batch, n_tokens, pos_batch)) return rc;
  const rf2_rope_config& c = plan->cfg;
  const bool norm = c.norm == RF2_NORM_RMS, nothing = batch == 0 || n_tokens == 0;
  // without a norm the rows themselves are not read
  rf2_rows* const sides[2][3] = {{norm ? &t.q : &t.dq_out, &t.dq_out, &t.dq}, {norm ? &t.k : &t.dk_out, &t.dk_out, &t.dk}};
  if (!nothing) {
    if (const int rc = check_rows(plan, batch, n_tokens, sides, 3)) return rc;
    if (!rf2_rope_pos_fits(plan, pos)) return RF2_ERR_INVALID_ARG;
  }
  // Sides with rows; sums over no rows, of a side that is left out too, are zeros.
  const bool have[2] = {!nothing && t.dq.at != nullptr, !nothing && t.dk.at != nullptr};
  float* const dw[2] = {dwq, dwk};
  for (int i = 0; i < 2; ++i) {
    if (have[i] && !rf2_rope_weight_fits(plan, i == 0 ? wq : wk)) return RF2_ERR_INVALID_ARG;
    if (norm ? (have[i] && !dw[i]) || !rf2_rope_aligned(dw[i], 4) : dw[i] != nullptr) return RF2_ERR_INVALID_ARG;
  }
  if (norm && (!workspace || !rf2_rope_aligned(workspace, 16))) return RF2_ERR_INVALID_ARG;
  if (const int rc = rf2_check_rope_device(plan)) return rc;
  const hipStream_t st = (hipStream_t)stream;
  if (!norm) {
    if (nothing) return RF2_OK;
    return launch_apply(plan, batch, n_tokens, t.dq_out, t.dk_out, pos, pos_batch, nullptr, nullptr, t.dq, t.dk, false, true, st);
  }

  BackArgs a{rope_args(plan, false), {pos, pos_batch, (uint32_t)n_tokens, (uint32_t)batch * (uint32_t)n_tokens}, {}};
  JoinArgs<float, double> runs{};
  JoinArgs<double, float> join_runs{};
  JoinArgs<float, float> join{};
  int64_t bytes = 0;
  for (int i = 0; i < 2; ++i) {
    const RopeWorkspace ws = rope_workspace(c.head_dim, i);
    float* const sums = (float*)((char*)workspace + ws.sums);
    if (!have[i]) {
      if (dw[i]) join.side[i] = {sums, dw[i], 0, 1};
      continue;
    }
    BackSide& s = a.side[i];
    s.x = rope_rows(i == 0 ? t.q : t.k);
    s.dz = rope_rows(i == 0 ? t.dq_out : t.dk_out);
    s.dx = rope_rows(i == 0 ? t.dq : t.dk);
    s.w = i == 0 ? wq : wk;
    const int heads = i == 0 ? c.heads : c.kv_heads;
    s.share = rope_share(i == 0 ? t.q : t.k, heads, c, a.tokens.total);
    const uint32_t units = rope_workgroups(s.share);
    s.workgroups = std::min<uint32_t>(units, units > RF2_ROPE_MANY ? RF2_ROPE_PARTS : RF2_ROPE_FEW);
    s.sums = s.workgroups == 1 ? dw[i] : sums;
    if (s.workgroups > RF2_ROPE_FEW) {
      const uint32_t n = (s.workgroups + 63) / 64;
      double* const at = (double*)((char*)workspace + ws.runs);
      runs.side[i] = {sums, at, s.workgroups, n};
      join_runs.side[i] = {at, dw[i], n, 1};
    } else if (s.workgroups != 1) {
      join.side[i] = {sums, dw[i], s.workgroups, 1};
    }
    bytes += (int64_t)a.tokens.total * heads * c.head_dim * 6;
  }
  const dim3 grid(a.side[0].workgroups + a.side[1].workgroups);
  if (!nothing) {
    const int rc = rope_for_types(c, [&](auto type, auto d, auto halves) {
      if (bytes <= ROPE_KEEP) backward_kernel<decltype(type), d(), halves(), true><<<grid, 256, 0, st>>>(a);
      else backward_kernel<decltype(type), d(), halves(), false><<<grid, 256, 0, st>>>(a);
    });
    if (rc) return rc;
  }
  if (const uint32_t groups = runs.side[0].groups + runs.side[1].groups) {
    if (c.head_dim == 128) runs_kernel<128><<<groups, 256, 0, st>>>(runs);
    else runs_kernel<64><<<groups, 256, 0, st>>>(runs);
    RF2_LAUNCH_CHECK();
    if (const int rc = launch_join(c.head_dim, join_runs, st)) return rc;
  }
  return launch_join(c.head_dim, join, st);
}
