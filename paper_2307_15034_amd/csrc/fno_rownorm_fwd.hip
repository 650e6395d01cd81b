// Residual norm, forward: y = scale x + gate (post_w norm(u) + post_b) and h =
// pre_w norm(y) + pre_b, a row held by a team of threads from its loads to its
// stores.
#include "fno_rownorm.h"

namespace fno {
namespace {

template <typename T, int TEAM, int VPT>
__global__ __launch_bounds__(row_threads(TEAM)) void row_norm_fwd_kernel(RowNormArgs a) {
  constexpr int V = kRowVec<T>, SLOTS = row_threads(TEAM) / TEAM;
  const RowPlace<T, TEAM, VPT> at(a);
  float post_w[VPT][V], post_b[VPT][V], scale[VPT][V], pre_w[VPT][V], pre_b[VPT][V];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    load_param<V>(post_w[i], a.post_w, at.vec[i], a.C, 1.0f);
    load_param<V>(post_b[i], a.post_b, at.vec[i], a.C, 0.0f);
    load_param<V>(scale[i], a.scale, at.vec[i], a.C, 1.0f);
    load_param<V>(pre_w[i], a.pre_w, at.vec[i], a.C, 1.0f);
    load_param<V>(pre_b[i], a.pre_b, at.vec[i], a.C, 0.0f);
  }
  Team<TEAM> team;
  RowStat st[1];
  for (int64_t row = (int64_t)blockIdx.x * SLOTS + threadIdx.x / TEAM; row < a.rows;
       row += (int64_t)gridDim.x * SLOTS) {
    const int64_t start = row * a.C;
    float y[1][VPT][V];
    load_row<T, VPT>(y[0], a.x, start, at.vec, at.valid, a.C);
    if (a.u) {
      float u[1][VPT][V], gate[VPT][V];
      load_row<T, VPT>(u[0], a.u, start, at.vec, at.valid, a.C);
      load_gate<T, VPT>(gate, a, row, at.vec, at.valid);
      row_stats<1, VPT, V, TEAM>(team, u, at.valid, a, st);
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float n = __builtin_fmaf((u[0][i][j] - st[0].mean) * st[0].r, post_w[i][j], post_b[i][j]);
          y[0][i][j] = __builtin_fmaf(gate[i][j], n, y[0][i][j] * scale[i][j]);
        }
      store_row<T, VPT>(a.y, start, at.vec, at.valid, a.C, y[0]);
    }
    if (a.h) {
      row_stats<1, VPT, V, TEAM>(team, y, at.valid, a, st);
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j)
          y[0][i][j] = __builtin_fmaf((y[0][i][j] - st[0].mean) * st[0].r, pre_w[i][j], pre_b[i][j]);
      store_row<T, VPT>(a.h, start, at.vec, at.valid, a.C, y[0]);
    }
  }
}

template <typename T>
hipError_t launch_of(const RowNormArgs& a, int team, int vecs, unsigned grid, hipStream_t s) {
#define FNO_ROW(T_, V_)                                                                   \
  if (team == T_ && vecs == V_) {                                                         \
    row_norm_fwd_kernel<T, T_, V_><<<dim3(grid), dim3(row_threads(T_)), 0, s>>>(a);       \
    return hipGetLastError();                                                             \
  }
  FNO_ROW(4, 1)
  FNO_ROW(8, 1)
  FNO_ROW(16, 1)
  FNO_ROW(32, 1)
  FNO_ROW(64, 1)
  FNO_ROW(64, 2)
  FNO_ROW(256, 1)
  FNO_ROW(256, 2)
  FNO_ROW(512, 2)
  FNO_ROW(1024, 2)
  FNO_ROW(1024, 4)
#undef FNO_ROW
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_row_norm_fwd(const RowNormArgs& a, int dtype, int team, int vecs, unsigned grid,
                               hipStream_t s) {
  if (dtype == FNO_DTYPE_F32) return launch_of<float>(a, team, vecs, grid, s);
  if (dtype == FNO_DTYPE_F16) return launch_of<_Float16>(a, team, vecs, grid, s);
  return launch_of<__bf16>(a, team, vecs, grid, s);
}

}  // namespace fno
