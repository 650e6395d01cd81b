// Residual norm, forward: y = scale x + gate (post_w norm(u) + post_b) and h =
// pre_w norm(y) + pre_b, a row held by a team of threads from its loads to its
// stores, the next row's loads under way.  Bound by memory: 32 x 128^2 rows of 64,
// fp16, four tensors, 46 us (5.8 TB/s; 72 with a division for each row's gate and no
// row ahead).
#include "fno_rownorm.h"

namespace fno {
namespace {

template <typename T, int TEAM, int VPT, int MODE>
__global__ __launch_bounds__(row_threads(TEAM)) void row_norm_fwd_kernel(RowNormArgs a) {
  constexpr int V = kRowVec<T>, SLOTS = row_threads(TEAM) / TEAM;
  constexpr bool KEPT = !row_lean(TEAM);
  const RowPlace<T, TEAM, VPT> at(a);
  const Param<KEPT, VPT, V> post_w(a.post_w, 1.0f, at.vec, a.C), post_b(a.post_b, 0.0f, at.vec, a.C);
  const Param<KEPT, VPT, V> scale(a.scale, 1.0f, at.vec, a.C);
  const Param<KEPT, VPT, V> pre_w(a.pre_w, 1.0f, at.vec, a.C), pre_b(a.pre_b, 0.0f, at.vec, a.C);
  Team<TEAM> team;
  RowStat st[1];
  UnitRows<SLOTS> at_row(a, (int)threadIdx.x / TEAM);
  float gate[VPT][V];
  if (a.u && !a.by_run) load_gate<T, VPT, MODE>(gate, a, at_row.span, at.vec, at.valid);
  RawRow<T, VPT, MODE> nx, nu;
  auto fetch = [&](int64_t row) {
    nx.load(a.x, row * a.C, at.vec, at.valid, a.C);
    if (a.u) nu.load(a.u, row * a.C, at.vec, at.valid, a.C);
  };
  if (KEPT && at_row.row < at_row.end) fetch(at_row.row);
  for (; at_row.row < at_row.end; at_row.advance(a)) {
    const int64_t start = at_row.row * a.C, next = at_row.next(a);
    if (!KEPT) fetch(at_row.row);
    float y[1][VPT][V], u[1][VPT][V];
    nx.widen(y[0]);
    if (a.u) nu.widen(u[0]);
    if (KEPT && next < at_row.end) fetch(next);
    if (a.u) {
      if (a.by_run && at_row.starts(a)) load_gate<T, VPT, MODE>(gate, a, at_row.gate, at.vec, at.valid);
      row_stats<1, VPT, V, TEAM>(team, u, at.valid, a, st);
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        float w[V], b[V], c[V];
        post_w.get(w, i, at.vec, a.C);
        post_b.get(b, i, at.vec, a.C);
        scale.get(c, i, at.vec, a.C);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float n = __builtin_fmaf((u[0][i][j] - st[0].mean) * st[0].r, w[j], b[j]);
          y[0][i][j] = __builtin_fmaf(gate[i][j], n, y[0][i][j] * c[j]);
        }
      }
      store_row<T, VPT, MODE>(a.y, start, at.vec, at.valid, a.C, y[0]);
    }
    if (a.h) {
      row_stats<1, VPT, V, TEAM>(team, y, at.valid, a, st);
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        float w[V], b[V];
        pre_w.get(w, i, at.vec, a.C);
        pre_b.get(b, i, at.vec, a.C);
#pragma unroll
        for (int j = 0; j < V; ++j)
          y[0][i][j] = __builtin_fmaf((y[0][i][j] - st[0].mean) * st[0].r, w[j], b[j]);
      }
      store_row<T, VPT, MODE>(a.h, start, at.vec, at.valid, a.C, y[0]);
    }
  }
}

template <typename T, int MODE>
hipError_t launch_mode(const RowNormArgs& a, const RowLaunchSize& l, hipStream_t s) {
#define FNO_ROW(T_, V_)                                                                        \
  if (l.team == T_ && l.vecs == V_) {                                                          \
    if constexpr (T_ * V_ * kRowVec<T> <= 16384) /* the longest row */ \
      row_norm_fwd_kernel<T, T_, V_, MODE><<<dim3(l.grid), dim3(row_threads(T_)), 0, s>>>(a); \
    return hipGetLastError();                                                                  \
  }
  if constexpr (MODE == ROW_SHORT) {  // one vector
    FNO_ROW(4, 1)
  } else {
    FNO_ROW_TEAMS(FNO_ROW)
  }
#undef FNO_ROW
  return hipErrorInvalidValue;
}
template <typename T>
hipError_t launch_of(const RowNormArgs& a, const RowLaunchSize& l, hipStream_t s) {
  if (l.mode == ROW_WHOLE) return launch_mode<T, ROW_WHOLE>(a, l, s);
  return l.mode == ROW_TAIL ? launch_mode<T, ROW_TAIL>(a, l, s) : launch_mode<T, ROW_SHORT>(a, l, s);
}

}  // namespace

hipError_t launch_row_norm_fwd(const RowNormArgs& a, int dtype, const RowLaunchSize& l, hipStream_t s) {
  if (dtype == FNO_DTYPE_F32) return launch_of<float>(a, l, s);
  return dtype == FNO_DTYPE_F16 ? launch_of<_Float16>(a, l, s) : launch_of<__bf16>(a, l, s);
}

}  // namespace fno
