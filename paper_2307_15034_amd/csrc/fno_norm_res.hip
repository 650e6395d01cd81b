// Group norm with each group held by one work-group: its values go from memory
// into registers once, all loads in flight together, and from there both
// through the sums and into the results.  Nothing is read twice, and a call is
// one launch (the backward of several samples adds one that joins the
// parameter gradients).  Groups of at most 16384 elements: a thread holds 32
// elements of each tensor in work-groups of 256, 16 in those of 1024 (half as many
// where they come one by one).  That fills the registers: the channels-last
// backward of 1024 threads keeps 24 to 88 bytes a lane in scratch in 16 of its
// bodies (64 samples of 2048 x 8, fp16: 14.8 us, their forward 10.4).
//
// channels first:  a plane of the group belongs to a team of waves (planes to
//                  teams in turn, where there are more planes than waves);
// channels last:   a thread keeps to one piece of W channels of the group's
//                  part of a row and takes it from every so many-th row.
//
// Bound by latency at the sizes that fit (2 x 64^2 x 16, fp16, four groups:
// 7.9 us on the device, eight work-groups in one chain of load, sum, result;
// a call 15.4 us through the two passes, 12.3 so, 10.2 since calls are leaner).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "fno_norm.h"

namespace fno {
namespace {

constexpr int kSmall = 256, kLarge = 1024;  // work-groups' threads

// Elements of a tensor that a thread holds, in pieces of W.
__host__ __device__ constexpr int each_of(int threads, int W) {
  return threads == kLarge ? (W == 1 ? 8 : 16) : (W == 1 ? 16 : 32);
}

// The sum over a work-group's THREADS threads, for all of them; `red` holds
// one entry per wave.
template <int THREADS>
__device__ __forceinline__ Sums block_sums(Sums v, Sums* red) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = add(v, Sums{__shfl_xor(v.s, d), __shfl_xor(v.q, d)});
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) v = add(v, red[w]);
  return v;
}

template <typename T, int W, int ACT>
__device__ __forceinline__ Vec<T, W> forward_vec(const Vec<T, W>& x, const Vec<T, W>& r, bool res, const Line* l, int step) {
  float y[W];
#pragma unroll
  for (int j = 0; j < W; ++j) y[j] = act_any<T>(on_line(l[j * step], x.e[j]), ACT);
  if (res)
#pragma unroll
    for (int j = 0; j < W; ++j) y[j] += (float)r.e[j];
  Vec<T, W> o;
#pragma unroll
  for (int j = 0; j < W; ++j) o.e[j] = (T)y[j];
  return o;
}

// --------------------------------------------------------------------------
// Channels first
// --------------------------------------------------------------------------
// How a work-group of WAVES waves shares the Cg planes of a group: teams of
// `tw` waves, team t taking planes t, t + teams, ...; lane `lane` of a team's
// `lanes` takes vectors lane, lane + lanes, ... of a plane, `per` at most.
struct Share {
  int teams, lanes, team, lane, per;
};
__host__ __device__ inline int team_waves(int Cg, int waves) {
  int tw = 1;
  while (tw * 2 * Cg <= waves) tw *= 2;
  return tw;
}
template <int WAVES>
__device__ __forceinline__ Share share_of(const NormArgs& a, int vec) {
  const int tw = team_waves(a.Cg, WAVES), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  Share s;
  s.teams = WAVES / tw;
  s.lanes = tw * 64;
  s.team = wave / tw;
  s.lane = (int)threadIdx.x - s.team * s.lanes;
  s.per = ((int)a.P / vec + s.lanes - 1) / s.lanes;
  return s;
}

// f(k, plane, vector, first of the plane) for a thread's pieces k < K of the
// group: piece k is vector `vector` of plane `plane` (there is none where plane
// >= Cg or vector >= vectors of a plane).
template <int K, typename F>
__device__ __forceinline__ void over_pieces(const Share& s, F f) {
  int plane = s.team, i = 0;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    f(k, plane, s.lane + i * s.lanes, i == 0);
    if (++i >= s.per) {
      i = 0;
      plane += s.teams;
    }
  }
}

template <typename T, int ACT, int THREADS>
__global__ __launch_bounds__(THREADS) void res_first_fwd_kernel(NormArgs a) {
  constexpr int V = kVec<T>, K = each_of(THREADS, V) / V;
  __shared__ Sums red[THREADS / 64];
  for (int64_t bg = blockIdx.x; bg < a.B * a.G; bg += gridDim.x) {
    const Share s = share_of<THREADS / 64>(a, V);
    const int P = (int)a.P, nv = P / V, rest = P - nv * V, c0 = (int)(bg % a.G) * a.Cg;
    const int64_t at = bg * a.Cg * a.P;
    const T* x = static_cast<const T*>(a.x) + at;
    const T* r = a.res ? static_cast<const T*>(a.res) + at : nullptr;
    T* out = static_cast<T*>(a.out) + at;
    Vec<T, V> xv[K], rv[K];
    T xt[K], rt[K];  // a plane's last elements, one per lane
    over_pieces<K>(s, [&](int k, int c, int v, bool start) {
      const bool in = c < a.Cg && v < nv, last = c < a.Cg && start && s.lane < rest;
      const uint32_t e = in ? (uint32_t)(c * P + v * V) : 0u;
      const uint32_t e1 = last ? (uint32_t)(c * P + nv * V + s.lane) : 0u;
      if (nv) xv[k] = load_vec<T, V>(x + e);
      if (nv && r) rv[k] = load_vec<T, V>(r + e);
      if (rest) xt[k] = x[e1];
      if (rest && r) rt[k] = r[e1];
    });
    Sums t{0.0, 0.0}, t1{0.0, 0.0};
    over_pieces<K>(s, [&](int k, int c, int v, bool start) {
      if (c < a.Cg && v < nv)
#pragma unroll
        for (int j = 0; j < V; ++j) add_value(j & 1 ? &t1 : &t, (float)xv[k].e[j]);
      if (c < a.Cg && start && s.lane < rest) add_value(&t, (float)xt[k]);
    });
    const Stat st = stat_of(a, block_sums<THREADS>(add(t, t1), red));
    if (a.stats && threadIdx.x == 0) {
      a.stats[2 * bg] = st.mean;
      a.stats[2 * bg + 1] = st.rstd;
    }
    over_pieces<K>(s, [&](int k, int c, int v, bool start) {
      if (c >= a.Cg) return;
      const Line l = line_of(a, st, c0 + c);
      if (v < nv) store_vec<T, V>(out + (uint32_t)(c * P + v * V), forward_vec<T, V, ACT>(xv[k], rv[k], r != nullptr, &l, 0));
      if (start && s.lane < rest) {
        float y = act_any<T>(on_line(l, xt[k]), ACT);
        if (r) y += (float)rt[k];
        out[(uint32_t)(c * P + nv * V + s.lane)] = (T)y;
      }
    });
    __syncthreads();
  }
}

// The parameter gradients of a channel from one sample: into the result where
// there is only one sample.
__device__ __forceinline__ void put_channel(const NormArgs& a, int64_t b, int c, const Sums& t) {
  if (a.B == 1) {
    if (a.gbeta) a.gbeta[c] = (float)t.s;
    if (a.ggamma) a.ggamma[c] = (float)t.q;
  } else {
    a.chan[b * a.C + c] = t;
  }
}

template <typename T, int ACT, int THREADS>
__global__ __launch_bounds__(THREADS) void res_first_bwd_kernel(NormArgs a) {
  constexpr int V = kVec<T>, K = each_of(THREADS, V) / V, WAVES = THREADS / 64;
  __shared__ Sums red[WAVES];
  __shared__ float2 part[WAVES * K];  // by wave and its planes in turn
  for (int64_t bg = blockIdx.x; bg < a.B * a.G; bg += gridDim.x) {
    const Share s = share_of<WAVES>(a, V);
    const int P = (int)a.P, nv = P / V, rest = P - nv * V, c0 = (int)(bg % a.G) * a.Cg;
    const int64_t at = bg * a.Cg * a.P;
    const T* x = static_cast<const T*>(a.x) + at;
    const T* g = static_cast<const T*>(a.gout) + at;
    T* out = static_cast<T*>(a.out) + at;
    Vec<T, V> xv[K], gv[K];
    T xt[K], gt[K];
    over_pieces<K>(s, [&](int k, int c, int v, bool start) {
      const bool in = c < a.Cg && v < nv, last = c < a.Cg && start && s.lane < rest;
      const uint32_t e = in ? (uint32_t)(c * P + v * V) : 0u;
      const uint32_t e1 = last ? (uint32_t)(c * P + nv * V + s.lane) : 0u;
      if (nv) {
        xv[k] = load_vec<T, V>(x + e);
        gv[k] = load_vec<T, V>(g + e);
      }
      if (rest) {
        xt[k] = x[e1];
        gt[k] = g[e1];
      }
    });
    float h[K][V], ht[K], sh = 0.0f, sq = 0.0f;
    over_pieces<K>(s, [&](int k, int c, int v, bool start) {
      if (c >= a.Cg) return;  // the same for the wave's lanes
      if (start) sh = sq = 0.0f;
      const Coef q = bwd_coef<T>(a, bg, c0 + c);
      float d;
      if (v < nv)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          bwd_terms<ACT>(q, xv[k].e[j], gv[k].e[j], &h[k][j], &d);
          sh += h[k][j];
          sq = __builtin_fmaf(h[k][j], d, sq);
        }
      if (start && s.lane < rest) {
        bwd_terms<ACT>(q, xt[k], gt[k], &ht[k], &d);
        sh += ht[k];
        sq = __builtin_fmaf(ht[k], d, sq);
      }
      // the plane's last piece: its sums over the wave
      const int turn = (c - s.team) / s.teams, done = k - turn * s.per + 1;
      if (done < s.per) return;
      const float2 m = bwd_sums(q, ACT, sh, sq);
      const Sums w = team_sum<64>(Sums{m.x, m.y});
      if ((threadIdx.x & 63) == 0) part[((int)threadIdx.x >> 6) * K + turn] = make_float2((float)w.s, (float)w.q);
    });
    __syncthreads();
    // channel c: the waves of its team, at its turn
    Sums t{0.0, 0.0};
    for (int c = threadIdx.x; c < a.Cg; c += THREADS) {
      const int tw = s.lanes / 64, w0 = c % s.teams * tw, turn = c / s.teams;
      Sums v{0.0, 0.0};
      for (int w = 0; w < tw; ++w) v = add(v, Sums{part[(w0 + w) * K + turn].x, part[(w0 + w) * K + turn].y});
      put_channel(a, bg / a.G, c0 + c, v);
      const double ga = a.gamma ? (double)a.gamma[c0 + c] : 1.0;
      t = add(t, Sums{ga * v.s, ga * v.q});
    }
    const Means m = means_of(a, block_sums<THREADS>(t, red));
    over_pieces<K>(s, [&](int k, int c, int v, bool start) {
      if (c >= a.Cg) return;
      const Coef q = bwd_coef<T>(a, bg, c0 + c);
      const Gx gk = gx_coef(q, m);
      if (v < nv) {
        Vec<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.e[j] = (T)bwd_gx(gk, h[k][j], distance(q, xv[k].e[j]));
        store_vec<T, V>(out + (uint32_t)(c * P + v * V), o);
      }
      if (start && s.lane < rest)
        out[(uint32_t)(c * P + nv * V + s.lane)] = (T)bwd_gx(gk, ht[k], distance(q, xt[k]));
    });
    __syncthreads();
  }
}

// --------------------------------------------------------------------------
// Channels last
// --------------------------------------------------------------------------
// The group's part of a row is S = Cg / W pieces of W channels; A threads (a
// multiple of S) take piece t mod S of rows t / S, t / S + A / S, ...
struct Rows {
  int64_t at;  // the element of the sample's first row where the piece starts
  int row, step, c;
  bool on;
};
template <int THREADS, int W>
__device__ __forceinline__ Rows rows_of(const NormArgs& a, int64_t bg) {
  const int S = a.Cg / W, n = THREADS / S, t = (int)threadIdx.x, g = (int)(bg % a.G);
  Rows r;
  r.on = t < n * S;
  r.row = t / S;
  r.step = n;
  r.c = g * a.Cg + (t - r.row * S) * W;
  r.at = bg / a.G * a.R + r.c;
  return r;
}

template <typename T, int W, int ACT, int THREADS>
__global__ __launch_bounds__(THREADS) void res_last_fwd_kernel(NormArgs a) {
  constexpr int K = each_of(THREADS, W) / W;
  __shared__ Sums red[THREADS / 64];
  for (int64_t bg = blockIdx.x; bg < a.B * a.G; bg += gridDim.x) {
    const Rows w = rows_of<THREADS, W>(a, bg);
    const T* x = static_cast<const T*>(a.x) + w.at;
    const T* r = a.res ? static_cast<const T*>(a.res) + w.at : nullptr;
    T* out = static_cast<T*>(a.out) + w.at;
    Vec<T, W> xv[K], rv[K];
    const int P = (int)a.P;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int row = w.row + k * w.step;
      const int64_t e = w.on && row < P ? (int64_t)row * a.C : 0;
      xv[k] = load_vec<T, W>(x + e);
      if (r) rv[k] = load_vec<T, W>(r + e);
    }
    Sums t{0.0, 0.0}, t1{0.0, 0.0};
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (w.on && w.row + k * w.step < P)
#pragma unroll
        for (int j = 0; j < W; ++j) add_value((k * W + j) & 1 ? &t1 : &t, (float)xv[k].e[j]);
    const Stat st = stat_of(a, block_sums<THREADS>(add(t, t1), red));
    if (a.stats && threadIdx.x == 0) {
      a.stats[2 * bg] = st.mean;
      a.stats[2 * bg + 1] = st.rstd;
    }
    if (w.on) {
      Line l[W];
#pragma unroll
      for (int j = 0; j < W; ++j) l[j] = line_of(a, st, w.c + j);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int row = w.row + k * w.step;
        if (row < P) store_vec<T, W>(out + (int64_t)row * a.C, forward_vec<T, W, ACT>(xv[k], rv[k], r != nullptr, l, 1));
      }
    }
    __syncthreads();
  }
}

template <typename T, int W, int ACT, int THREADS>
__global__ __launch_bounds__(THREADS) void res_last_bwd_kernel(NormArgs a) {
  constexpr int K = each_of(THREADS, W) / W;
  extern __shared__ __align__(16) unsigned char smem[];
  float2* lds = reinterpret_cast<float2*>(smem);             // [THREADS][W]
  Sums* ch = reinterpret_cast<Sums*>(lds + (size_t)THREADS * W);  // [Cg]
  __shared__ Sums red[THREADS / 64];
  for (int64_t bg = blockIdx.x; bg < a.B * a.G; bg += gridDim.x) {
    const Rows w = rows_of<THREADS, W>(a, bg);
    const T* x = static_cast<const T*>(a.x) + w.at;
    const T* g = static_cast<const T*>(a.gout) + w.at;
    T* out = static_cast<T*>(a.out) + w.at;
    Vec<T, W> xv[K], gv[K];
    const int P = (int)a.P;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int row = w.row + k * w.step;
      const int64_t e = w.on && row < P ? (int64_t)row * a.C : 0;
      xv[k] = load_vec<T, W>(x + e);
      gv[k] = load_vec<T, W>(g + e);
    }
    Coef q[W];
    float h[K][W], sh[W], sq[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      q[j] = bwd_coef<T>(a, bg, w.c + j);
      sh[j] = sq[j] = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (w.on && w.row + k * w.step < P)
#pragma unroll
        for (int j = 0; j < W; ++j) {
          float d;
          bwd_terms<ACT>(q[j], xv[k].e[j], gv[k].e[j], &h[k][j], &d);
          sh[j] += h[k][j];
          sq[j] = __builtin_fmaf(h[k][j], d, sq[j]);
        }
#pragma unroll
    for (int j = 0; j < W; ++j) lds[threadIdx.x * W + j] = bwd_sums(q[j], ACT, sh[j], sq[j]);
    __syncthreads();
    // entry [t][j] is channel (t mod S) W + j of the group
    group_sums<THREADS>(a.Cg, w.step,
                        [&](int c, int i) { const float2 t = lds[i * a.Cg + c]; return Sums{t.x, t.y}; },
                        [&](int c, const Sums& t) {
                          const int cc = (int)(bg % a.G) * a.Cg + c;
                          put_channel(a, bg / a.G, cc, t);
                          const double ga = a.gamma ? (double)a.gamma[cc] : 1.0;
                          ch[c] = Sums{ga * t.s, ga * t.q};
                        });
    __syncthreads();
    Sums t{0.0, 0.0};
    for (int c = threadIdx.x; c < a.Cg; c += THREADS) t = add(t, ch[c]);
    const Means m = means_of(a, block_sums<THREADS>(t, red));
    if (w.on) {
      Gx gk[W];
#pragma unroll
      for (int j = 0; j < W; ++j) gk[j] = gx_coef(q[j], m);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int row = w.row + k * w.step;
        if (row >= P) continue;
        Vec<T, W> o;
#pragma unroll
        for (int j = 0; j < W; ++j) o.e[j] = (T)bwd_gx(gk[j], h[k][j], distance(q[j], xv[k].e[j]));
        store_vec<T, W>(out + (int64_t)row * a.C, o);
      }
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(NT) void res_param_kernel(NormArgs a) { param_grads(a, (int)blockIdx.x); }

// --------------------------------------------------------------------------
// Host side
// --------------------------------------------------------------------------
int vec_of(int dtype) { return dtype == FNO_DTYPE_F32 ? 4 : 8; }

// Whether a work-group of `threads` holds a group of planes.
bool first_fits(const NormArgs& a, int vec, int threads) {
  const int each = each_of(threads, vec);
  if (a.P > threads * each || a.Cg > threads * each) return false;
  const int tw = team_waves(a.Cg, threads / 64), teams = threads / 64 / tw;
  const int64_t per = std::max<int64_t>(1, (a.P / vec + tw * 64 - 1) / (tw * 64));
  return per * ((a.Cg + teams - 1) / teams) <= each / vec;
}

// The widest piece that divides the group's part of a row (aligned rows not needed).
int piece_of(const NormArgs& a, int dtype) {
  const int V = vec_of(dtype);
  return a.Cg % V == 0 ? V : V == 8 && a.Cg % 4 == 0 ? 4 : 1;
}
// The backward's LDS of a call: sums by thread and by channel.
size_t last_bwd_lds(const NormArgs& a, int W, int threads) {
  return (size_t)threads * W * sizeof(float2) + (size_t)a.Cg * sizeof(Sums);
}
// Beside it the waves' sums of the two joins; 160 KiB in all (which one or two
// rows of 6120 channels to a group pass, with pieces of eight).
constexpr size_t kLdsMax = 160 * 1024;
bool last_fits(const NormArgs& a, int W, int threads, bool bwd) {
  const int S = a.Cg / W;
  if (S > threads || a.P > (int64_t)(threads / S) * (each_of(threads, W) / W)) return false;
  return !bwd || last_bwd_lds(a, W, threads) + 2 * (threads / 64) * sizeof(Sums) <= kLdsMax;
}

template <typename T, int ACT, int THREADS>
void launch_first(const NormArgs& a, bool bwd, unsigned grid, hipStream_t s) {
  if (bwd) hipLaunchKernelGGL((res_first_bwd_kernel<T, ACT, THREADS>), dim3(grid), dim3(THREADS), 0, s, a);
  else hipLaunchKernelGGL((res_first_fwd_kernel<T, ACT, THREADS>), dim3(grid), dim3(THREADS), 0, s, a);
}
template <typename T, int W, int ACT, int THREADS>
hipError_t launch_last(const NormArgs& a, bool bwd, unsigned grid, hipStream_t s) {
  if (!bwd) {
    hipLaunchKernelGGL((res_last_fwd_kernel<T, W, ACT, THREADS>), dim3(grid), dim3(THREADS), 0, s, a);
    return hipSuccess;
  }
  const size_t lds = last_bwd_lds(a, W, THREADS);
  auto k = res_last_bwd_kernel<T, W, ACT, THREADS>;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k, dim3(grid), dim3(THREADS), lds, s, a);
  return hipSuccess;
}

template <typename T, int ACT>
hipError_t launch_act(const NormArgs& a, int dtype, bool first, bool bwd, unsigned grid, hipStream_t s) {
  constexpr int V = kVec<T>;
  if (first) {
    if (first_fits(a, V, kSmall)) launch_first<T, ACT, kSmall>(a, bwd, grid, s);
    else launch_first<T, ACT, kLarge>(a, bwd, grid, s);
    return hipSuccess;
  }
  const int W = piece_of(a, dtype);
  const bool small = last_fits(a, W, kSmall, bwd);
  if (W == V)
    return small ? launch_last<T, V, ACT, kSmall>(a, bwd, grid, s) : launch_last<T, V, ACT, kLarge>(a, bwd, grid, s);
  if (V == 8 && W == 4)
    return small ? launch_last<T, 4, ACT, kSmall>(a, bwd, grid, s) : launch_last<T, 4, ACT, kLarge>(a, bwd, grid, s);
  return small ? launch_last<T, 1, ACT, kSmall>(a, bwd, grid, s) : launch_last<T, 1, ACT, kLarge>(a, bwd, grid, s);
}

template <typename T>
hipError_t launch_type(const NormArgs& a, int dtype, bool first, bool bwd, unsigned grid, hipStream_t s) {
  switch (a.act) {
    case FNO_NORM_ACT_GELU: return launch_act<T, FNO_NORM_ACT_GELU>(a, dtype, first, bwd, grid, s);
    case FNO_NORM_ACT_SILU: return launch_act<T, FNO_NORM_ACT_SILU>(a, dtype, first, bwd, grid, s);
    default: return launch_act<T, FNO_NORM_ACT_NONE>(a, dtype, first, bwd, grid, s);
  }
}

}  // namespace

bool norm_resident_fits(const NormArgs& a, int dtype, bool first, bool bwd) {
  if (first) return first_fits(a, vec_of(dtype), kLarge);
  return last_fits(a, piece_of(a, dtype), kLarge, bwd);
}

hipError_t norm_resident_launch(const NormArgs& a0, int dtype, bool first, bool bwd, hipStream_t s) {
  NormArgs a = a0;
  a.nc = 1;
  const unsigned grid = (unsigned)std::min<int64_t>(a.B * a.G, 1 << 20);
  hipError_t e = dtype == FNO_DTYPE_F32   ? launch_type<float>(a, dtype, first, bwd, grid, s)
                 : dtype == FNO_DTYPE_F16 ? launch_type<_Float16>(a, dtype, first, bwd, grid, s)
                                          : launch_type<__bf16>(a, dtype, first, bwd, grid, s);
  if (e != hipSuccess) return e;
  if (bwd && a.B > 1 && (a.ggamma || a.gbeta))
    hipLaunchKernelGGL(res_param_kernel, dim3((unsigned)a.C), dim3(NT), 0, s, a);
  return hipGetLastError();
}

}  // namespace fno
