// The residual norm's C entry points, its rules of launch, and the join of the
// parameters' partial sums.
#include <algorithm>

#include "fno_host.h"
#include "fno_rownorm.h"

namespace fno {
namespace {

struct JoinArgs {
  const float* part;
  void* out[RS_COUNT];  // of each slot
  int gate_slot;        // the slot summed by gate row, -1: none
  int gate_dtype;
  int64_t units, units_per_gate, gate_rows;
  int C, sums;
};

constexpr int kJoinCols = 16, kJoinRows = 64;

// One job: kJoinCols columns of one sum (of one gate row's).  Doubles: a sum of
// up to 2^31 partial sums.
__global__ __launch_bounds__(kJoinCols* kJoinRows) void row_join_kernel(JoinArgs a) {
  __shared__ double red[kJoinRows][kJoinCols + 1];
  const int col = threadIdx.x % kJoinCols, lane = threadIdx.x / kJoinCols;
  const int64_t blocks = (a.C + kJoinCols - 1) / kJoinCols;
  const int64_t plain = a.sums - (a.gate_slot >= 0 ? 1 : 0);
  const int64_t jobs = blocks * (plain + (a.gate_slot >= 0 ? a.gate_rows : 0));
  for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
    const int64_t what = job / blocks;
    const int c = (int)(job - what * blocks) * kJoinCols + col;
    int slot = (int)what;
    int64_t first = 0, count = a.units, gate = 0;
    if (what >= plain) {
      slot = a.gate_slot;
      gate = what - plain;
      first = gate * a.units_per_gate;
      count = a.units_per_gate;
    } else if (a.gate_slot >= 0 && slot >= a.gate_slot) {
      ++slot;
    }
    double s = 0.0;
    if (c < a.C) {
      const float* p = a.part + (first * a.sums + slot) * a.C + c;
      const int64_t step = (int64_t)a.sums * a.C;
#pragma unroll 4
      for (int64_t i = lane; i < count; i += kJoinRows) s += (double)p[i * step];
    }
    __syncthreads();
    red[lane][col] = s;
    __syncthreads();
#pragma unroll
    for (int d = kJoinRows / 2; d > 0; d >>= 1) {
      if (lane < d) red[lane][col] += red[lane + d][col];
      __syncthreads();
    }
    if (lane == 0 && c < a.C) {
      const float v = (float)red[0][col];
      const int64_t at = gate * a.C + c;
      if (slot != a.gate_slot || a.gate_dtype == FNO_DTYPE_F32)
        static_cast<float*>(a.out[slot])[at] = v;
      else if (a.gate_dtype == FNO_DTYPE_F16)
        static_cast<_Float16*>(a.out[slot])[at] = (_Float16)v;
      else
        static_cast<__bf16*>(a.out[slot])[at] = (__bf16)v;
    }
  }
}

// --------------------------------------------------------------------------
// Host side
// --------------------------------------------------------------------------
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool ok16(const void* p) { return p && ((uintptr_t)p & 15u) == 0; }
inline bool null_or16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

fno_status check_desc(const fno_residual_norm_desc* d) {
  if (!d) return FNO_ERR_INVALID_ARGUMENT;
  if (d->dtype < FNO_DTYPE_F32 || d->dtype > FNO_DTYPE_BF16) return FNO_ERR_INVALID_ARGUMENT;
  if (d->norm != FNO_ROW_NORM_LAYER && d->norm != FNO_ROW_NORM_RMS) return FNO_ERR_INVALID_ARGUMENT;
  if (d->gate_dtype != FNO_DTYPE_F32 && d->gate_dtype != d->dtype) return FNO_ERR_INVALID_ARGUMENT;
  if (!(d->eps >= 0.0f && d->eps <= 3.4e38f)) return FNO_ERR_INVALID_ARGUMENT;
  if (d->rows < 1 || d->rows > ((int64_t)1 << 40) || d->channels < 1 || d->channels > 16384 ||
      d->rows > ((int64_t)1 << 42) / d->channels)
    return FNO_ERR_INVALID_ARGUMENT;
  if (d->gate_rows < 0 || d->gate_rows > d->rows || (d->gate_rows && d->rows % d->gate_rows))
    return FNO_ERR_INVALID_ARGUMENT;
  return FNO_OK;
}

struct RowPlan {
  RowNormArgs a;
  int team, vecs;
  int64_t units;
};

// A row's team: the fewest threads that hold it, a vector each, then two and four.
void team_of(int nvec, int* team, int* vecs) {
#define FNO_ROW(T_, V_) {T_, V_},
  static const int kTeams[][2] = {FNO_ROW_TEAMS(FNO_ROW)};
#undef FNO_ROW
  for (const auto& t : kTeams) {
    *team = t[0];
    *vecs = t[1];
    if (nvec <= t[0] * t[1]) return;
  }
}

constexpr int64_t kChain = 128;

// Whether teams take whole gate rows, many to a unit, instead of units a gate row
// (or a part of it) each.  Backward: units of their own each leave a row of partial
// sums, which past the data cost more than a gate row's rows one behind the other
// (about 1.5 us each).  Gates of 2, 8, 32 and 128 rows meet there at about 4096
// values of the gate for each of its rows: 64 channels, 8192 gates of 32 rows 263 us
// so, 52 by whole gate rows (data 49), 1024 gates 41 and 45; 4096 channels, 1024
// gates of 8 rows 1619 and 104.  Forward: nothing is summed, only teams without a
// row are lost (64 channels, 32 teams: 32768 gates of 8 rows 82 and 25 us).
bool by_run(const fno_residual_norm_desc& d, int64_t per_gate, int64_t slots, bool bwd) {
  if (!d.gate_rows || per_gate == 1) return d.gate_rows != 0;
  return per_gate <= kChain && d.gate_rows * d.channels >= 4096 * per_gate &&
         (bwd || per_gate * 4 <= slots);
}

RowPlan plan_of(const fno_residual_norm_desc& d, bool bwd) {
  RowPlan p{};
  RowNormArgs& a = p.a;
  const int V = d.dtype == FNO_DTYPE_F32 ? 4 : 8;
  a.rows = d.rows;
  a.C = (int)d.channels;
  a.nvec = (int)cdiv(a.C, V);
  a.layer = d.norm == FNO_ROW_NORM_LAYER;
  a.gate_f32 = d.gate_dtype == FNO_DTYPE_F32;
  a.eps = d.eps;
  int e = 0;
  while ((1 << e) < a.C) ++e;
  a.shrink = 1.0f / (float)(1 << e);
  a.per_channel = (float)((double)(1 << e) / a.C);
  a.inv_c = (float)(1.0 / a.C);
  const int64_t per_gate = d.gate_rows ? d.rows / d.gate_rows : d.rows;
  team_of(a.nvec, &p.team, &p.vecs);
  const int64_t slots = row_threads(p.team) / p.team;
  const int64_t fill = p.team <= 64 ? (bwd ? 1024 : 2048) : 131072 / p.team * (bwd ? 1 : 2);
  // A unit is rows of one gate row's share, in the backward at most kChain for a
  // thread (its chain of additions).
  a.by_run = by_run(d, per_gate, slots, bwd);
  a.run = a.by_run ? (int)per_gate : 1;
  const int64_t runs = a.by_run ? d.gate_rows : per_gate, spans = d.rows / a.run / runs;
  a.units_per_gate = std::max(std::min(cdiv(fill, spans), cdiv(runs, slots)),
                              bwd ? cdiv(runs, kChain / a.run * slots) : 1);
  a.runs_per_unit = cdiv(runs, a.units_per_gate);
  a.units_per_gate = cdiv(runs, a.runs_per_unit);
  a.span = runs * a.run;
  a.per_unit = a.runs_per_unit * a.run;
  p.units = a.units_per_gate * spans;
  return p;
}

constexpr int64_t kMaxGrid = (int64_t)1 << 20;
// Work-groups of a launch: their threads (up to 1024) stay below 2^32.
constexpr int64_t kMaxUnits = ((int64_t)1 << 22) - 1;
bool too_many(const fno_residual_norm_desc& d, const RowPlan& p) {
  return p.units > kMaxUnits || (d.gate_rows > kMaxUnits && d.gate_rows != d.rows);
}

fno_status set_params(RowNormArgs* a, const fno_residual_norm_desc& d,
                      const fno_residual_norm_params* q, bool post, bool pre) {
  if (!q) return FNO_ERR_INVALID_ARGUMENT;
  if (!null_or16(q->post_w) || !null_or16(q->post_b) || !null_or16(q->gate) ||
      !null_or16(q->scale) || !null_or16(q->pre_w) || !null_or16(q->pre_b))
    return FNO_ERR_INVALID_ARGUMENT;
  if (!post && (q->post_w || q->post_b || q->gate || q->scale)) return FNO_ERR_INVALID_ARGUMENT;
  if (!pre && (q->pre_w || q->pre_b)) return FNO_ERR_INVALID_ARGUMENT;
  if (post && (q->gate != nullptr) != (d.gate_rows > 0)) return FNO_ERR_INVALID_ARGUMENT;
  a->post_w = q->post_w;
  a->post_b = q->post_b;
  a->gate = q->gate;
  a->scale = q->scale;
  a->pre_w = q->pre_w;
  a->pre_b = q->pre_b;
  return FNO_OK;
}

struct RowLaunch {
  RowPlan p;
  int dtype;
  bool post, pre;
  JoinArgs join;
  hipStream_t stream;
};

RowLaunchSize size_of(const RowLaunch& L) {
  const int V = L.dtype == FNO_DTYPE_F32 ? 4 : 8, C = L.p.a.C;
  return RowLaunchSize{L.p.team, L.p.vecs, C % V == 0 ? ROW_WHOLE : C > V ? ROW_TAIL : ROW_SHORT,
                       (unsigned)L.p.units};
}

hipError_t launch_fwd(void* ctx) {
  const RowLaunch& L = *static_cast<RowLaunch*>(ctx);
  return launch_row_norm_fwd(L.p.a, L.dtype, size_of(L), L.stream);
}

hipError_t launch_bwd(void* ctx) {
  const RowLaunch& L = *static_cast<RowLaunch*>(ctx);
  const auto launch = L.dtype == FNO_DTYPE_F32   ? launch_row_norm_bwd_f32
                      : L.dtype == FNO_DTYPE_F16 ? launch_row_norm_bwd_f16
                                                 : launch_row_norm_bwd_bf16;
  const hipError_t e = launch(L.p.a, L.post, L.pre, size_of(L), L.stream);
  if (e != hipSuccess || !L.p.a.sums) return e;
  const int64_t jobs = cdiv(L.p.a.C, kJoinCols) *
                       (L.p.a.sums - (L.join.gate_slot >= 0) +
                        (L.join.gate_slot >= 0 ? L.join.gate_rows : 0));
  row_join_kernel<<<dim3((unsigned)std::min(jobs, kMaxGrid)), dim3(kJoinCols * kJoinRows), 0, L.stream>>>(L.join);
  return hipGetLastError();
}

// Bytes of the backward's partial sums.
int64_t ws_bytes(const fno_residual_norm_desc& d, const RowPlan& p) {
  const int64_t sums = RS_COUNT - (d.gate_rows == 0 || p.a.by_run ? 1 : 0);
  return std::max<int64_t>(256, cdiv(p.units * sums * p.a.C * 4, 256) * 256);
}

}  // namespace
}  // namespace fno

using namespace fno;

extern "C" fno_status fno_residual_norm_workspace_size(const fno_residual_norm_desc* d,
                                                       size_t* bytes) {
  const fno_status st = check_desc(d);
  if (st != FNO_OK) return st;
  if (!bytes) return FNO_ERR_INVALID_ARGUMENT;
  const RowPlan p = plan_of(*d, true);
  if (too_many(*d, p)) return FNO_ERR_UNSUPPORTED;
  *bytes = (size_t)ws_bytes(*d, p);
  return FNO_OK;
}

extern "C" fno_status fno_residual_norm_fwd(const fno_residual_norm_desc* d,
                                            const fno_residual_norm_params* params, const void* x,
                                            const void* u, void* y, void* h, hipStream_t stream) {
  fno_status st = check_desc(d);
  if (st != FNO_OK) return st;
  if (!ok16(x) || !null_or16(u) || !null_or16(y) || !null_or16(h)) return FNO_ERR_INVALID_ARGUMENT;
  if ((u != nullptr) != (y != nullptr) || (!u && !h) || (y && y == h)) return FNO_ERR_INVALID_ARGUMENT;
  RowLaunch L{plan_of(*d, false), d->dtype, u != nullptr, h != nullptr, {}, stream};
  st = set_params(&L.p.a, *d, params, L.post, L.pre);
  if (st != FNO_OK) return st;
  if (too_many(*d, L.p)) return FNO_ERR_UNSUPPORTED;
  L.p.a.x = x;
  L.p.a.u = u;
  L.p.a.y = y;
  L.p.a.h = h;
  const hipError_t e = timed_launch("residual_norm_fwd", stream, launch_fwd, &L);
  return e == hipSuccess ? FNO_OK : report_hip_error(e, "residual_norm_fwd");
}

extern "C" fno_status fno_residual_norm_bwd(const fno_residual_norm_desc* d,
                                            const fno_residual_norm_params* params, const void* x,
                                            const void* u, const void* y, const void* g_y,
                                            const void* g_h, void* g_x, void* g_u,
                                            const fno_residual_norm_grads* grads, void* ws,
                                            size_t ws_len, hipStream_t stream) {
  fno_status st = check_desc(d);
  if (st != FNO_OK) return st;
  const bool post = u != nullptr, pre = g_h != nullptr;
  if (!grads || !null_or16(x) || !null_or16(u) || !null_or16(y) || !null_or16(g_y) ||
      !null_or16(g_h) || !ok16(g_x) || !null_or16(g_u))
    return FNO_ERR_INVALID_ARGUMENT;
  if (!null_or16(grads->post_w) || !null_or16(grads->post_b) || !null_or16(grads->gate) ||
      !null_or16(grads->scale) || !null_or16(grads->pre_w) || !null_or16(grads->pre_b))
    return FNO_ERR_INVALID_ARGUMENT;
  if ((!g_y && !g_h) || (!post && !pre) || post != (g_u != nullptr) || g_x == g_u)
    return FNO_ERR_INVALID_ARGUMENT;
  if (!post && (y || !x || grads->post_w || grads->post_b || grads->gate || grads->scale))
    return FNO_ERR_INVALID_ARGUMENT;
  if (post && ((pre && !y) || (grads->scale && !x) || (grads->gate && !d->gate_rows)))
    return FNO_ERR_INVALID_ARGUMENT;
  if (!pre && (grads->pre_w || grads->pre_b)) return FNO_ERR_INVALID_ARGUMENT;
  RowLaunch L{plan_of(*d, true), d->dtype, post, pre, {}, stream};
  st = set_params(&L.p.a, *d, params, post, pre);
  if (st != FNO_OK) return st;
  if (too_many(*d, L.p)) return FNO_ERR_UNSUPPORTED;
  const bool row_gate = L.p.a.by_run;
  RowNormArgs& a = L.p.a;
  void* const out[RS_COUNT] = {grads->post_w, grads->post_b, row_gate ? nullptr : grads->gate,
                               grads->scale, grads->pre_w, grads->pre_b};
  L.join.gate_slot = -1;
  for (int i = 0; i < RS_COUNT; ++i) {
    a.slot[i] = out[i] ? a.sums : -1;
    if (!out[i]) continue;
    if (i == RS_GATE) L.join.gate_slot = a.sums;
    L.join.out[a.sums++] = out[i];
  }
  if (a.sums) {
    if (ws_len < (size_t)ws_bytes(*d, L.p)) return FNO_ERR_WORKSPACE_TOO_SMALL;
    if (!ok16(ws)) return FNO_ERR_INVALID_ARGUMENT;
  }
  if (any_twice({g_x, g_u, grads->post_w, grads->post_b, grads->gate, grads->scale, grads->pre_w,
                 grads->pre_b}))
    return FNO_ERR_INVALID_ARGUMENT;
  a.part = static_cast<float*>(ws);
  a.g_gate = row_gate ? grads->gate : nullptr;
  a.x = x;
  a.u = u;
  a.y_in = post ? y : x;
  a.g_y = g_y;
  a.g_h = g_h;
  a.g_x = g_x;
  a.g_u = g_u;
  L.join.part = a.part;
  L.join.gate_dtype = d->gate_dtype;
  L.join.units = L.p.units;
  L.join.units_per_gate = a.units_per_gate;
  L.join.gate_rows = d->gate_rows;
  L.join.C = a.C;
  L.join.sums = a.sums;
  const hipError_t e = timed_launch("residual_norm_bwd", stream, launch_bwd, &L);
  return e == hipSuccess ? FNO_OK : report_hip_error(e, "residual_norm_bwd");
}
