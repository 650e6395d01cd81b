// Residual norm, backward.  With xh the normalised row, r = 1 / sqrt(var + eps)
// and t = w g the gradient of xh, a norm's gradient is
//     r (t - mean(t) - xh mean(t xh))     (LAYER; without mean(t): RMS).
// Both rows' statistics are formed again from the rows, which a team of threads
// holds whole; the parameters' sums stay in registers over a unit's rows and
// leave as one partial row a unit.  Bound by memory, as long as the next row is on
// its way while one is worked on: 32 x 128^2 rows of 64, fp16, seven tensors, 103 us
// (4.6 TB/s), 8192 rows of 4096, bf16, six tensors, 98 (4.1); without the row ahead,
// its loads in branches, 163 and 180.
#pragma once

#include "fno_rownorm.h"

namespace fno {
namespace {

template <int VPT, int V, int TEAM>
__device__ __forceinline__ void norm_grad(Team<TEAM>& team, const float (&t)[VPT][V],
                                          const float (&xh)[VPT][V], const RowNormArgs& a, float r,
                                          float (&out)[VPT][V]) {
  float s[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      s[0] += t[i][j];
      s[1] = __builtin_fmaf(t[i][j], xh[i][j], s[1]);
    }
  team.template sum<2>(s);
  const float m = a.layer ? s[0] * a.inv_c : 0.0f, q = s[1] * a.inv_c;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) out[i][j] = r * __builtin_fmaf(-xh[i][j], q, t[i][j] - m);
}

// Adds a sum over the work-group's teams and writes it to `part`.
template <int TEAM, int VPT, int V>
__device__ __forceinline__ void write_sums(const RowNormArgs& a, int which, float (&v)[VPT][V],
                                           const int (&vec)[VPT], float* lds) {
  const int slot = a.slot[which];
  if (slot < 0) return;
  float* out = a.part + ((int64_t)blockIdx.x * a.sums + slot) * a.C;
  if constexpr (TEAM > 64) {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (vec[i] * V + j < a.C) out[vec[i] * V + j] = v[i][j];
  } else {
    constexpr int WAVES = row_threads(TEAM) / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int d = TEAM; d < 64; d *= 2) v[i][j] += __shfl_xor(v[i][j], d);
    __syncthreads();
    if (lane < TEAM) {
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) lds[wave * (TEAM * VPT * V) + vec[i] * V + j] = v[i][j];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.C; c += row_threads(TEAM)) {
      float s = lds[c];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) s += lds[w * (TEAM * VPT * V) + c];
      out[c] = s;
    }
  }
}

template <typename T, int TEAM, int VPT, int MODE, bool POST, bool PRE>
__global__ __launch_bounds__(row_threads(TEAM)) void row_norm_bwd_kernel(RowNormArgs a) {
  constexpr int V = kRowVec<T>, SLOTS = row_threads(TEAM) / TEAM;
  constexpr int K = (POST ? 1 : 0) + (PRE ? 1 : 0);  // rows with statistics
  __shared__ float lds[TEAM > 64 ? 1 : row_threads(TEAM) / 64 * TEAM * VPT * V];
  constexpr bool KEPT = !row_lean(TEAM);
  const RowPlace<T, TEAM, VPT> at(a);
  const Param<KEPT && POST, VPT, V> post_w(a.post_w, 1.0f, at.vec, a.C), post_b(a.post_b, 0.0f, at.vec, a.C);
  const Param<KEPT && POST, VPT, V> scale(a.scale, 1.0f, at.vec, a.C);
  const Param<KEPT && PRE, VPT, V> pre_w(a.pre_w, 1.0f, at.vec, a.C);
  float sums[RS_COUNT][VPT][V];
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int q = 0; q < RS_COUNT; ++q)
#pragma unroll
      for (int j = 0; j < V; ++j) sums[q][i][j] = 0.0f;
  Team<TEAM> team;
  UnitRows<SLOTS> at_row(a, (int)threadIdx.x / TEAM);
  float gate[VPT][V];
  if (POST && !a.by_run) load_gate<T, VPT, MODE>(gate, a, at_row.span, at.vec, at.valid);
  const bool with_x = POST && a.slot[RS_SCALE] >= 0;
  RawRow<T, VPT, MODE> ru, ry, rh, rg, rx;
  auto fetch = [&](int64_t row) {
    const int64_t start = row * a.C;
    if constexpr (POST) ru.load(a.u, start, at.vec, at.valid, a.C);
    if constexpr (PRE) {
      ry.load(a.y_in, start, at.vec, at.valid, a.C);
      rh.load(a.g_h, start, at.vec, at.valid, a.C);
    }
    if (a.g_y) rg.load(a.g_y, start, at.vec, at.valid, a.C);
    if (with_x) rx.load(a.x, start, at.vec, at.valid, a.C);
  };
  if (KEPT && at_row.row < at_row.end) fetch(at_row.row);
  for (; at_row.row < at_row.end; at_row.advance(a)) {
    const int64_t start = at_row.row * a.C, next = at_row.next(a);
    if (!KEPT) fetch(at_row.row);
    float v[K][VPT][V], G[VPT][V], t[VPT][V], xh[VPT][V], x[VPT][V];
    RowStat st[K];
    if constexpr (POST) ru.widen(v[0]);
    if constexpr (PRE) {
      ry.widen(v[K - 1]);
      rh.widen(t);
    }
    if (a.g_y) {
      rg.widen(G);
    } else {
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) G[i][j] = 0.0f;
    }
    if (with_x) rx.widen(x);
    if (KEPT && next < at_row.end) fetch(next);
    row_stats<K, VPT, V, TEAM>(team, v, at.valid, a, st);
    if constexpr (PRE) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        float w[V];
        pre_w.get(w, i, at.vec, a.C);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          xh[i][j] = (v[K - 1][i][j] - st[K - 1].mean) * st[K - 1].r;
          sums[RS_PRE_W][i][j] = __builtin_fmaf(t[i][j], xh[i][j], sums[RS_PRE_W][i][j]);
          sums[RS_PRE_B][i][j] += t[i][j];
          t[i][j] *= w[j];
        }
      }
      float d[VPT][V];
      norm_grad<VPT, V, TEAM>(team, t, xh, a, st[K - 1].r, d);
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) G[i][j] += d[i][j];
    }
    if constexpr (POST) {
      if (with_x) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j)
            sums[RS_SCALE][i][j] = __builtin_fmaf(G[i][j], x[i][j], sums[RS_SCALE][i][j]);
      }
      if (a.by_run && at_row.starts(a)) {
        load_gate<T, VPT, MODE>(gate, a, at_row.gate, at.vec, at.valid);
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j) sums[RS_GATE][i][j] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        float w[V], b[V];
        post_w.get(w, i, at.vec, a.C);
        post_b.get(b, i, at.vec, a.C);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          xh[i][j] = (v[0][i][j] - st[0].mean) * st[0].r;
          sums[RS_GATE][i][j] += G[i][j] * __builtin_fmaf(xh[i][j], w[j], b[j]);
        }
      }
      if (a.g_gate && at_row.ends()) {
        const int64_t to = at_row.gate * a.C;
        if (a.gate_f32) {
#pragma unroll
          for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int q = 0; q < V / 4; ++q) {
              RowVec<float> r;
#pragma unroll
              for (int j = 0; j < 4; ++j) r.e[j] = sums[RS_GATE][i][4 * q + j];
              if (at.valid[i] > 4 * q)
                store_row_vec<float, ROW_TAIL>(static_cast<float*>(a.g_gate) + to, at.vec[i] * (V / 4) + q, a.C, r);
            }
        } else {
          store_row<T, VPT, MODE>(a.g_gate, to, at.vec, at.valid, a.C, sums[RS_GATE]);
        }
      }
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        float w[V], c[V];
        post_w.get(w, i, at.vec, a.C);
        scale.get(c, i, at.vec, a.C);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          t[i][j] = G[i][j] * gate[i][j];
          G[i][j] *= c[j];
          sums[RS_POST_W][i][j] = __builtin_fmaf(t[i][j], xh[i][j], sums[RS_POST_W][i][j]);
          sums[RS_POST_B][i][j] += t[i][j];
          t[i][j] *= w[j];
        }
      }
      float d[VPT][V];
      norm_grad<VPT, V, TEAM>(team, t, xh, a, st[0].r, d);
      store_row<T, VPT, MODE>(a.g_u, start, at.vec, at.valid, a.C, d);
    }
    store_row<T, VPT, MODE>(a.g_x, start, at.vec, at.valid, a.C, G);
  }
  if (a.sums) {
    if constexpr (POST) {
      write_sums<TEAM, VPT, V>(a, RS_POST_W, sums[RS_POST_W], at.vec, lds);
      write_sums<TEAM, VPT, V>(a, RS_POST_B, sums[RS_POST_B], at.vec, lds);
      write_sums<TEAM, VPT, V>(a, RS_GATE, sums[RS_GATE], at.vec, lds);
      write_sums<TEAM, VPT, V>(a, RS_SCALE, sums[RS_SCALE], at.vec, lds);
    }
    if constexpr (PRE) {
      write_sums<TEAM, VPT, V>(a, RS_PRE_W, sums[RS_PRE_W], at.vec, lds);
      write_sums<TEAM, VPT, V>(a, RS_PRE_B, sums[RS_PRE_B], at.vec, lds);
    }
  }
}

template <typename T, bool POST, bool PRE, int MODE>
hipError_t launch_mode(const RowNormArgs& a, const RowLaunchSize& l, hipStream_t s) {
#define FNO_ROW(T_, V_)                                                                        \
  if (l.team == T_ && l.vecs == V_) {                                                          \
    if constexpr (T_ * V_ * kRowVec<T> <= 16384) /* the longest row */ \
      row_norm_bwd_kernel<T, T_, V_, MODE, POST, PRE><<<dim3(l.grid), dim3(row_threads(T_)), 0, s>>>(a); \
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
template <typename T, bool POST, bool PRE>
hipError_t launch_of(const RowNormArgs& a, const RowLaunchSize& l, hipStream_t s) {
  if (l.mode == ROW_WHOLE) return launch_mode<T, POST, PRE, ROW_WHOLE>(a, l, s);
  return l.mode == ROW_TAIL ? launch_mode<T, POST, PRE, ROW_TAIL>(a, l, s)
                            : launch_mode<T, POST, PRE, ROW_SHORT>(a, l, s);
}
template <typename T>
hipError_t launch_form(const RowNormArgs& a, bool post, bool pre, const RowLaunchSize& l, hipStream_t s) {
  if (post && pre) return launch_of<T, true, true>(a, l, s);
  return post ? launch_of<T, true, false>(a, l, s) : launch_of<T, false, true>(a, l, s);
}

}  // namespace
}  // namespace fno
