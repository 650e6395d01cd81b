// What the kernels of the residual norm share: teams of threads that hold a
// row, the rows' vectors and statistics, and the launches by type.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/fno_spectral_conv.h"

namespace fno {

// The sums of a backward's rows, in the order of the workspace.
enum RowSum { RS_POST_W, RS_POST_B, RS_GATE, RS_SCALE, RS_PRE_W, RS_PRE_B, RS_COUNT };

struct RowNormArgs {
  const void *x, *u, *y_in, *g_y, *g_h;
  void *y, *h, *g_x, *g_u;
  const float *post_w, *post_b, *scale, *pre_w, *pre_b;
  const void* gate;
  void* g_gate;         // with `by_run`: written by the gate row's own team
  float* part;          // [units][sums][C]
  int64_t rows;
  int64_t span;         // rows that units share: those of a gate row, or all with `by_run`
  int64_t per_unit, units_per_gate;  // of a span
  int64_t runs_per_unit;             // gate rows of a unit, with `by_run`
  int run;              // rows in sequence that a team takes: a gate row's with `by_run`, else 1
  int by_run;           // a team takes whole gate rows, of which a unit has many
  int C, nvec;
  int layer;            // FNO_ROW_NORM_LAYER
  int gate_f32;         // the gate is fp32 (else of the rows' type)
  int slot[RS_COUNT];   // where a sum stands in `part`, -1: not wanted
  int sums;
  float eps;
  float shrink, per_channel;  // 2^-p >= 1 / C, and 2^p / C
  float inv_c;
};

// Threads of a team (a row's) and the vectors that each holds.  Teams of up to a
// wave share work-groups of 256, larger ones are a work-group each.
constexpr int row_threads(int team) { return team <= 64 ? 256 : team; }
// Work-groups of 1024 threads have 128 registers a thread: parameters are read
// again for each row there, and no row is loaded ahead.
constexpr bool row_lean(int team) { return team >= 1024; }
#define FNO_ROW_TEAMS(DO) \
  DO(4, 1) DO(8, 1) DO(16, 1) DO(32, 1) DO(64, 1) DO(128, 1) DO(256, 1) DO(512, 1) DO(1024, 1) \
  DO(1024, 2) DO(1024, 4)

struct RowLaunchSize {
  int team, vecs, mode;  // mode: RowMode
  unsigned grid;
};
hipError_t launch_row_norm_fwd(const RowNormArgs& a, int dtype, const RowLaunchSize& l, hipStream_t s);
// The backward's kernels, by type (one source each: they are many).
hipError_t launch_row_norm_bwd_f32(const RowNormArgs& a, bool post, bool pre, const RowLaunchSize& l,
                                   hipStream_t s);
hipError_t launch_row_norm_bwd_f16(const RowNormArgs& a, bool post, bool pre, const RowLaunchSize& l,
                                   hipStream_t s);
hipError_t launch_row_norm_bwd_bf16(const RowNormArgs& a, bool post, bool pre, const RowLaunchSize& l,
                                    hipStream_t s);

// --------------------------------------------------------------------------
// Device code
// --------------------------------------------------------------------------
template <typename T>
constexpr int kRowVec = 16 / (int)sizeof(T);

template <typename T>
struct RowVec {
  T e[kRowVec<T>];
};

// How a row's vectors lie: all whole, the last one short, or the row shorter than
// a vector.
enum RowMode { ROW_WHOLE, ROW_TAIL, ROW_SHORT };

// Vector v (of the row's values from v V on) of a row of C values at `row`; zeros
// behind the row's end.  Rows start at any element.  A short last vector is read
// as the row's last V values and shifted, so that loads need no branch: they are
// issued a row ahead, and a branch would wait for them.
template <typename T, int MODE>
__device__ __forceinline__ RowVec<T> load_row_vec(const T* row, int v, int C, int valid) {
  constexpr int V = kRowVec<T>;
  RowVec<T> r;
  if constexpr (MODE == ROW_WHOLE) {
#pragma unroll
    for (int j = 0; j < V; ++j) r.e[j] = (T)0.0f;
    if (valid) __builtin_memcpy(&r, __builtin_assume_aligned(row + v * V, sizeof(T)), sizeof(r));
  } else if constexpr (MODE == ROW_TAIL) {
    const int at = v * V < C - V ? v * V : C - V;
    const int cut = (V - valid) * (int)sizeof(T) * 8;  // bits in front of the vector's own
    struct {
      uint64_t lo, hi;
    } w;
    __builtin_memcpy(&w, __builtin_assume_aligned(row + at, sizeof(T)), sizeof(w));
    const int s = cut & 63;
    const uint64_t up = (w.hi << 1) << (63 - s);
    const uint64_t lo = cut >= 64 ? w.hi >> s : (w.lo >> s) | up, hi = cut >= 64 ? 0 : w.hi >> s;
    w.lo = cut >= 128 ? 0 : lo;
    w.hi = hi;
    __builtin_memcpy(&r, &w, sizeof(r));
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      r.e[j] = (T)0.0f;
      if (v * V + j < C) r.e[j] = row[v * V + j];
    }
  }
  return r;
}
template <typename T, int MODE>
__device__ __forceinline__ void store_row_vec(T* row, int v, int C, const RowVec<T>& r) {
  constexpr int V = kRowVec<T>;
  if (MODE == ROW_WHOLE || (v + 1) * V <= C) {
    __builtin_memcpy(__builtin_assume_aligned(row + v * V, sizeof(T)), &r, sizeof(r));
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (v * V + j < C) row[v * V + j] = r.e[j];
  }
}
// The same of fp32 parameters (V values from channel v V on); `other` where
// there are none, zeros behind the row's end (what is multiplied by them there
// leaves no trace in the row's sums).
template <int V>
__device__ __forceinline__ void load_param(float (&out)[V], const float* p, int v, int C,
                                           float other) {
  if (p && (v + 1) * V <= C) {
    __builtin_memcpy(out, __builtin_assume_aligned(p + v * V, 4), sizeof(out));
    return;
  }
#pragma unroll
  for (int j = 0; j < V; ++j) out[j] = v * V + j < C ? (p ? p[v * V + j] : other) : 0.0f;
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// Sums over N consecutive lanes (a power of two up to 64), in all of them.  Lane
// permutations of the vector unit: each step adds the neighbour at distance 1, 2,
// then mirrors (equal lanes by then) of 8 and 16, then rows and halves swapped.
template <int N>
__device__ __forceinline__ float lane_sum(float v) {
  if constexpr (N >= 2) v += dpp<0xB1>(v);
  if constexpr (N >= 4) v += dpp<0x4E>(v);
  if constexpr (N >= 8) v += dpp<0x141>(v);
  if constexpr (N >= 16) v += dpp<0x140>(v);
  if constexpr (N >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v),
                                                    __builtin_bit_cast(unsigned, v), false, false);
    v = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
  }
  if constexpr (N >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v),
                                                    __builtin_bit_cast(unsigned, v), false, false);
    v = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
  }
  return v;
}

// Sums over a team.  A team of several waves is a whole work-group, all of whose
// threads call with the same number of values; two buffers taken in turn need
// one barrier a call.
template <int TEAM>
struct Team {
  int turn = 0;
  template <int K>
  __device__ __forceinline__ void sum(float (&v)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lane_sum<(TEAM < 64 ? TEAM : 64)>(v[k]);
    if constexpr (TEAM > 64) {
      constexpr int W = TEAM / 64;
      __shared__ float red[2][4][W];
      const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
      if (lane == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) red[turn][k][wave] = v[k];
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = lane_sum<W>(red[turn][k][lane & (W - 1)]);
      turn ^= 1;
    }
  }
};

struct RowStat {
  float mean, r;
};

// Means and 1 / sqrt(var + eps) of K rows at once (v[k]: a thread's values,
// `valid` of each vector's are the row's).  The mean is of values scaled by a
// power of two, whose sum stays within fp32; the squares are of distances from
// it.  Where their sum leaves what fp32 holds exactly enough (rows larger
// than 2^60 or so, or as small as eps = 0 would need), they are formed again at
// another power of two.
template <int K, int VPT, int V, int TEAM>
__device__ __forceinline__ void row_stats(Team<TEAM>& team, const float (&v)[K][VPT][V],
                                          const int (&valid)[VPT], const RowNormArgs& a,
                                          RowStat (&st)[K]) {
  float s[K];
#pragma unroll
  for (int k = 0; k < K; ++k) s[k] = 0.0f;
  if (a.layer) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) s[k] = __builtin_fmaf(v[k][i][j], a.shrink, s[k]);
    team.template sum<K>(s);
  }
#pragma unroll
  for (int k = 0; k < K; ++k) st[k].mean = s[k] * a.per_channel;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    s[k] = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float d = j < valid[i] ? v[k][i][j] - st[k].mean : 0.0f;
        s[k] = __builtin_fmaf(d, d, s[k]);
      }
  }
  team.template sum<K>(s);
  bool odd = false;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    st[k].r = __builtin_amdgcn_rsqf(__builtin_fmaf(s[k], a.inv_c, a.eps));
    odd |= !(s[k] < 0x1p120f) || (s[k] < 0x1p-70f && a.eps < 0x1p-90f);
  }
  if (odd) {  // the same for all threads of the team
    float q[2 * K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      q[2 * k] = q[2 * k + 1] = 0.0f;
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float d = j < valid[i] ? v[k][i][j] - st[k].mean : 0.0f;
          const float lo = d * 0x1p-72f, hi = d * 0x1p72f;
          q[2 * k] = __builtin_fmaf(lo, lo, q[2 * k]);
          q[2 * k + 1] = __builtin_fmaf(hi, hi, q[2 * k + 1]);
        }
    }
    team.template sum<2 * K>(q);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!(s[k] < 0x1p120f)) {
        const float big = q[2 * k] * a.inv_c;
        st[k].r = big < 0x1p127f
                      ? __builtin_amdgcn_rsqf(__builtin_fmaf(a.eps, 0x1p-144f, big)) * 0x1p-72f
                      : __builtin_nanf("");  // a value that is not finite
      }
      if (s[k] < 0x1p-70f && a.eps < 0x1p-90f)
        st[k].r = __builtin_amdgcn_rsqf(__builtin_fmaf(q[2 * k + 1], a.inv_c, a.eps * 0x1p72f * 0x1p72f)) * 0x1p72f;
    }
  }
}

// Everything of a thread that does not change from row to row.
template <typename T, int TEAM, int VPT>
struct RowPlace {
  int vec[VPT], valid[VPT];
  __device__ __forceinline__ explicit RowPlace(const RowNormArgs& a) {
    constexpr int V = kRowVec<T>;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      vec[i] = (int)(threadIdx.x % TEAM) + i * TEAM;
      const int left = a.C - vec[i] * V;
      valid[i] = left < 0 ? 0 : left > V ? V : left;
    }
  }
};

// A thread's vectors of a row as they are in memory.
template <typename T, int VPT, int MODE>
struct RawRow {
  RowVec<T> v[VPT];
  __device__ __forceinline__ void load(const void* base, int64_t at, const int (&vec)[VPT],
                                       const int (&valid)[VPT], int C) {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      v[i] = load_row_vec<T, MODE>(static_cast<const T*>(base) + at, vec[i], C, valid[i]);
  }
  __device__ __forceinline__ void widen(float (&out)[VPT][kRowVec<T>]) const {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < kRowVec<T>; ++j) out[i][j] = (float)v[i].e[j];
  }
};

template <typename T, int VPT, int MODE>
__device__ __forceinline__ void store_row(void* base, int64_t at, const int (&vec)[VPT],
                                          const int (&valid)[VPT], int C,
                                          const float (&v)[VPT][kRowVec<T>]) {
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    if (valid[i] > 0) {
      RowVec<T> r;
#pragma unroll
      for (int j = 0; j < kRowVec<T>; ++j) r.e[j] = (T)v[i][j];
      store_row_vec<T, MODE>(static_cast<T*>(base) + at, vec[i], C, r);
    }
}
// A row of the gate (ones without it).
template <typename T, int VPT, int MODE>
__device__ __forceinline__ void load_gate(float (&out)[VPT][kRowVec<T>], const RowNormArgs& a,
                                          int64_t gate_row, const int (&vec)[VPT],
                                          const int (&valid)[VPT]) {
  constexpr int V = kRowVec<T>;
  if (!a.gate) {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) out[i][j] = 1.0f;
    return;
  }
  const int64_t at = gate_row * a.C;
  if (a.gate_f32) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) load_param<V>(out[i], static_cast<const float*>(a.gate) + at, vec[i], a.C, 0.0f);
  } else {
    RawRow<T, VPT, MODE> r;
    r.load(a.gate, at, vec, valid, a.C);
    r.widen(out);
  }
}

// A parameter's values for a thread, kept over the rows, or read where they are used.
template <bool KEPT, int VPT, int V>
struct Param {
  float kept[KEPT ? VPT : 1][V];
  const float* from;
  float other;
  __device__ __forceinline__ Param(const float* p, float none, const int (&vec)[VPT], int C)
      : from(p), other(none) {
    if constexpr (KEPT) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) load_param<V>(kept[i], p, vec[i], C, none);
    }
  }
  __device__ __forceinline__ void get(float (&out)[V], int i, const int (&vec)[VPT], int C) const {
    if constexpr (KEPT) {
#pragma unroll
      for (int j = 0; j < V; ++j) out[j] = kept[i][j];
    } else {
      load_param<V>(out, from, vec[i], C, other);
    }
  }
};

// The rows of a unit, a piece of one span, as the team of one of SLOTS slots goes
// through them: a run of rows, then the run SLOTS runs on.
template <int SLOTS>
struct UnitRows {
  int64_t span, end;
  int64_t row, gate;  // (gate: with `by_run`)
  int left;           // rows of the run from this one on, the same for all teams
  __device__ __forceinline__ UnitRows(const RowNormArgs& a, int slot) {
    span = (int64_t)blockIdx.x / a.units_per_gate;
    const int64_t first = span * a.span + ((int64_t)blockIdx.x - span * a.units_per_gate) * a.per_unit;
    const int64_t last = (span + 1) * a.span;
    end = first + a.per_unit < last ? first + a.per_unit : last;
    row = first + (int64_t)slot * a.run;
    gate = (int64_t)blockIdx.x * a.runs_per_unit + slot;
    left = a.run;
  }
  __device__ __forceinline__ bool starts(const RowNormArgs& a) const { return left == a.run; }
  __device__ __forceinline__ bool ends() const { return left == 1; }
  __device__ __forceinline__ int64_t next(const RowNormArgs& a) const {
    return row + (left > 1 ? 1 : (int64_t)(SLOTS - 1) * a.run + 1);
  }
  __device__ __forceinline__ void advance(const RowNormArgs& a) {
    row = next(a);
    if (left > 1) {
      --left;
    } else {
      left = a.run;
      gate += SLOTS;
    }
  }
};

}  // namespace fno
