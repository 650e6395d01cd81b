// Group norm with an activation (and the block's residual), forward and
// backward, in either layout.
//
//   xh = (x - mu) r,  r = 1 / sqrt(var + eps),  z = gamma xh + beta,
//   out = act(z) (+ residual)
//   h = g_out act'(z),  g_beta = sum h,  g_gamma = sum h xh,
//   gx = r (gamma h - a - xh d),  a, d = the group's means of gamma h, gamma h xh
//
// Both directions read a group's sums before its first result, so they run in
// two passes: the first leaves partial sums (a pair of doubles for each group
// and work-group, in a fixed place, so that every order is fixed), the second
// joins its group's and streams the tensors again.
//
// Every thread keeps to the same channels from its first vector to its last,
// with their coefficients and sums in registers:
//   channels last, "flat":  a sample is one run of 16-byte vectors whose
//     channels repeat after L = C / gcd(C, vector) vectors; A = the multiple of
//     L threads that fit take vectors t, t + A, t + 2 A, ...  No channel
//     count costs alignment: rows of 20 channels are as good as rows of 64;
//   channels last, "wide" (L beyond a work-group):  a thread takes one vector
//     of channels (one channel where C is no multiple of a vector) down the rows;
//   channels first:  a team of threads takes one plane or a segment of it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <numeric>

#include "../../include/fno_spectral_conv.h"
#include "fno_act.h"
#include "fno_host.h"

namespace fno {
namespace {

constexpr int NT = 256;  // threads of a work-group

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t rup(int64_t a, int64_t b) { return cdiv(a, b) * b; }

struct Sums {  // of x and x^2, or of h and h xh
  double s, q;
};

template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);
template <typename T, int W = kVec<T>>
struct Vec {
  T e[W];
};
// W consecutive elements at any element address, in one access.
template <typename T, int W>
__device__ __forceinline__ Vec<T, W> load_vec(const T* p) {
  Vec<T, W> v;
  __builtin_memcpy(&v, __builtin_assume_aligned(p, sizeof(T)), sizeof(v));
  return v;
}
template <typename T, int W>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, W>& v) {
  __builtin_memcpy(__builtin_assume_aligned(p, sizeof(T)), &v, sizeof(v));
}

// --------------------------------------------------------------------------
// Activations
// --------------------------------------------------------------------------
// Half of erfc(|z| / sqrt 2) by Abramowitz & Stegun 7.1.26 (absolute error at
// most 0.75e-7), and exp(-z^2 / 2).
__device__ __forceinline__ float half_erfc(float z, float* e) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(z), 0.23164189f, 1.0f));
  float p = __builtin_fmaf(t, 0.5307027145f, -0.7265760135f);
  p = __builtin_fmaf(t, p, 0.7107068705f);
  p = __builtin_fmaf(t, p, -0.142248368f);
  p = __builtin_fmaf(t, p, 0.127414796f);
  *e = __builtin_amdgcn_exp2f(z * (z * -0.72134752044448f));
  return p * t * *e;
}
// z Phi(z) = max(z, 0) - |z| erfc(|z| / sqrt 2) / 2.
__device__ __forceinline__ float gelu_of(float z) {
  float e;
  const float h = half_erfc(z, &e);
  return __builtin_fmaf(-__builtin_fabsf(z), h, __builtin_fmaxf(z, 0.0f));
}
// Phi(z) + z phi(z), Phi = 1/2 + sign(z) (1/2 - erfc / 2).
__device__ __forceinline__ float gelu_grad_of(float z) {
  float e;
  const float h = half_erfc(z, &e);
  const float phi = 0.5f + __builtin_copysignf(0.5f - h, z);
  return __builtin_fmaf(z * 0.39894228040143268f, e, phi);
}

template <int ACT>
__device__ __forceinline__ float act_f(float z) {
  return ACT == FNO_NORM_ACT_GELU ? gelu_of(z) : ACT == FNO_NORM_ACT_SILU ? silu_f(z) : z;
}
template <int ACT>
__device__ __forceinline__ float act_grad_f(float z) {
  return ACT == FNO_NORM_ACT_GELU ? gelu_grad_of(z) : ACT == FNO_NORM_ACT_SILU ? silu_grad_f(z) : 1.0f;
}

// --------------------------------------------------------------------------
// Arguments
// --------------------------------------------------------------------------
struct NormArgs {
  const void *x, *res, *gout;
  const float *gamma, *beta;
  void* out;             // out or gx
  const float* stats_in; // backward: [B][G][2]
  float* stats;          // forward: [B][G][2] or null
  Sums* part;            // [B][G][n]: the first pass's sums of each group
  Sums* joined;          // [B][G], where `collapse`
  Sums* chan;            // [B][C][nc]: the backward's sums of each channel
  float *ggamma, *gbeta;
  int64_t B, P, R;       // R = P C elements of a sample
  int C, G, Cg;
  int n, nc;             // entries of a group in part, of a channel in chan
  int collapse;          // part is joined by a launch of its own
  int act;
  float eps;
  // flat: L, A as above; vectors of a chunk (a multiple of A) and chunks of a
  // sample, in the first and in the second pass
  int L, A, n1, n2;
  int64_t v1, v2;
  // wide: rows of a chunk, column blocks, chunks (n1)
  // first: elements of a segment, segments of a plane (n1)
  int64_t rows;
  int cols;
  // this launch's work items and the work-groups that share them (further
  // ones, one per channel, form the parameter gradients)
  int64_t u0, u1;
  int main;
};

// A group's statistics from its sums.
struct Stat {
  float mean, rstd;
};
__device__ __forceinline__ Stat stat_of(const NormArgs& a, const Sums& t) {
  const double m = (double)a.P * a.Cg;
  const double mean = t.s / m, var = __builtin_fmax(t.q / m - mean * mean, 0.0);
  // a value that is not finite makes the sum of squares so
  const bool ok = t.q <= 1.7976931348623157e308;
  const float nan = __builtin_nanf("");
  return Stat{ok ? (float)mean : nan, ok ? (float)(1.0 / sqrt(var + (double)a.eps)) : nan};
}

__device__ __forceinline__ Sums add(const Sums& a, const Sums& b) { return Sums{a.s + b.s, a.q + b.q}; }

// Sums over the TEAM consecutive threads of a team (a power of two; a whole
// work-group for 256), for all of them.
template <int TEAM>
__device__ __forceinline__ Sums team_sum(Sums v) {
#pragma unroll
  for (int d = (TEAM < 64 ? TEAM : 64) / 2; d > 0; d >>= 1)
    v = add(v, Sums{__shfl_xor(v.s, d), __shfl_xor(v.q, d)});
  if (TEAM > 64) {
    __shared__ Sums red[NT / 64];
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = add(add(red[0], red[1]), add(red[2], red[3]));
  }
  return v;
}

// For each of `groups` groups the sum of its `n` entries entry(g, i), handed
// to put(g, sum) by one thread; all threads of the work-group take part.
template <typename Entry, typename Put>
__device__ __forceinline__ void group_sums(int groups, int n, Entry entry, Put put) {
  __shared__ Sums red[NT / 64];
  if (groups > NT / 64) {
    // a power of two of threads (at most a wave) per group
    int sub = 1;
    while (sub < 64 && sub * 2 * groups <= NT) sub *= 2;
    const int s = threadIdx.x & (sub - 1);
    for (int g0 = 0; g0 < groups; g0 += NT / sub) {
      const int g = g0 + (int)threadIdx.x / sub;
      Sums v{0.0, 0.0};
      if (g < groups)
        for (int i = s; i < n; i += sub) v = add(v, entry(g, i));
      for (int d = sub / 2; d > 0; d >>= 1) v = add(v, Sums{__shfl_xor(v.s, d), __shfl_xor(v.q, d)});
      if (g < groups && s == 0) put(g, v);
    }
    return;
  }
  for (int g = 0; g < groups; ++g) {
    Sums v{0.0, 0.0};
    for (int i = threadIdx.x; i < n; i += NT) v = add(v, entry(g, i));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = add(v, Sums{__shfl_xor(v.s, d), __shfl_xor(v.q, d)});
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) put(g, add(add(red[0], red[1]), add(red[2], red[3])));
  }
}

// x and x^2 added in double: nothing cancels however far a group's mean or a
// few of its values lie from the rest, and the unit's double additions run at
// the rate of float ones.
__device__ __forceinline__ void add_value(Sums* t, float x) {
  const double d = (double)x;
  t->s += d;
  t->q = __builtin_fma(d, d, t->q);
}

// --------------------------------------------------------------------------
// Channels last, flat
// --------------------------------------------------------------------------
// A chunk of a sample, `size` vectors from `base` on (an element of the
// sample), and this thread's vectors of it: threadIdx, threadIdx + A, ...:
// `count` full ones, then perhaps the sample's last, partial one (`tail`).
struct Mine {
  int64_t base;
  int count;
  bool tail;
};
__device__ __forceinline__ Mine my_vectors(const NormArgs& a, int64_t chunk, int64_t size, int vec) {
  const int64_t full = a.R / vec, lo = chunk * size;
  Mine m{lo * vec, 0, false};
  if ((int)threadIdx.x >= a.A) return m;
  const int here = (int)(lo + size < full ? size : full > lo ? full - lo : 0);
  if ((int)threadIdx.x < here) m.count = (here - (int)threadIdx.x + a.A - 1) / a.A;
  const int next = (int)threadIdx.x + m.count * a.A;
  m.tail = a.R % vec != 0 && lo + next == full && next < size;
  return m;
}
// The element of the chunk where this thread's vector k starts (past its last:
// its last).  Chunks hold less than 2^31 elements.
__device__ __forceinline__ uint32_t my_at(const NormArgs& a, const Mine& m, int k, int vec) {
  return (uint32_t)(((int)threadIdx.x + (k < m.count ? k : m.count - 1) * a.A) * vec);
}

// The channel of element j of thread t's vectors.
__device__ __forceinline__ int my_channel(const NormArgs& a, int j, int vec) {
  return (vec * ((int)threadIdx.x % a.L) + j) % a.C;
}

// UNI: a vector's channels are of one group (and C is a multiple of a vector).
template <typename T, bool UNI>
__device__ __forceinline__ void flat_stats(const NormArgs& a, int64_t unit, Sums* lds) {  // [A][E]
  constexpr int V = kVec<T>, UN = 8, E = UNI ? 1 : V;
  const int64_t b = unit / a.n1, chunk = unit - b * a.n1;
  const Mine m = my_vectors(a, chunk, a.v1, V);
  const T* x = static_cast<const T*>(a.x) + b * a.R + m.base;
  Sums acc[E];
#pragma unroll
  for (int j = 0; j < E; ++j) acc[j] = Sums{0.0, 0.0};
  for (int k = 0; k < m.count; k += UN) {
    Vec<T, V> v[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u)
      v[u] = load_vec<T, V>(x + my_at(a, m, k + u, V));
#pragma unroll
    for (int u = 0; u < UN; ++u)
      if (k + u < m.count)
#pragma unroll
        for (int j = 0; j < V; ++j) add_value(&acc[UNI ? 0 : j], (float)v[u].e[j]);
  }
  if ((int)threadIdx.x < a.A) {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      if (m.tail) {
        const int64_t at = ((int)threadIdx.x + m.count * a.A) * V;
        for (int i = UNI ? 0 : j; i < (UNI ? V : j + 1); ++i)
          if (m.base + at + i < a.R) add_value(&acc[j], (float)x[at + i]);
      }
      lds[threadIdx.x * E + j] = acc[j];
    }
  }
  __syncthreads();
  const int C = UNI ? a.C / V : a.C, Cg = UNI ? a.Cg / V : a.Cg, per = a.A * E / C * Cg;
  group_sums(a.G, per, [&](int g, int i) { const int r = i / Cg; return lds[r * C + g * Cg + (i - r * Cg)]; },
             [&](int g, const Sums& t) { a.part[(b * a.G + g) * a.n + chunk] = t; });
}
template <typename T, bool UNI>
__global__ __launch_bounds__(NT) void flat_stats_kernel(NormArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  for (int64_t u = a.u0 + blockIdx.x; u < a.u1; u += gridDim.x) {
    flat_stats<T, UNI>(a, u, reinterpret_cast<Sums*>(smem));
    __syncthreads();
  }
}

// Each of a sample's groups joined, f(group, sum) into LDS.
template <typename V2, typename F>
__device__ __forceinline__ void load_groups(const NormArgs& a, int64_t b, V2* lds, F f) {
  const Sums* p = a.collapse ? a.joined + b * a.G : a.part + b * a.G * a.n;
  const int n = a.collapse ? 1 : a.n;
  group_sums(a.G, n, [&](int g, int i) { return p[(int64_t)g * n + i]; },
             [&](int g, const Sums& t) { lds[g] = f(g, t); });
  __syncthreads();
}

// z = (x - mu) k + beta, k = r gamma.  (Not x k + (beta - mu k): where a
// group's spread is nothing beside its mean, that has mu k 2^-24 of error.)
struct Line {
  float mu, k, be;
};
__device__ __forceinline__ Line line_of(const NormArgs& a, const Stat& st, int c) {
  return Line{st.mean, a.gamma ? st.rstd * a.gamma[c] : st.rstd, a.beta ? a.beta[c] : 0.0f};
}
__device__ __forceinline__ float on_line(const Line& l, float x) {
  return __builtin_fmaf(x - l.mu, l.k, l.be);
}

__device__ __forceinline__ void write_stat(const NormArgs& a, int64_t bg, const Stat& st) {
  a.stats[2 * bg] = st.mean;
  a.stats[2 * bg + 1] = st.rstd;
}

template <typename T, int ACT, bool UNI>
__device__ __forceinline__ void flat_fwd(const NormArgs& a, int64_t unit, Stat* lds) {  // [G]
  constexpr int V = kVec<T>, UN = 4;
  const int64_t b = unit / a.n2, chunk = unit - b * a.n2;
  load_groups(a, b, lds, [&](int g, const Sums& t) {
    const Stat st = stat_of(a, t);
    if (chunk == 0 && a.stats) write_stat(a, b * a.G + g, st);
    return st;
  });
  const bool res = a.res != nullptr;
  const Mine m = my_vectors(a, chunk, a.v2, V);
  const T* x = static_cast<const T*>(a.x) + b * a.R + m.base;
  const T* r = res ? static_cast<const T*>(a.res) + b * a.R + m.base : nullptr;
  T* out = static_cast<T*>(a.out) + b * a.R + m.base;
  if (!m.count && !m.tail) return;
  Line l[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int c = my_channel(a, j, V);
    l[j] = line_of(a, lds[c / a.Cg], c);
    if (UNI && j) l[j].mu = l[0].mu;
  }
  for (int k = 0; k < m.count; k += UN) {
    Vec<T, V> v[UN], rv[UN];
    uint32_t at[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      at[u] = my_at(a, m, k + u, V);
      v[u] = load_vec<T, V>(x + at[u]);
    }
    if (res)
#pragma unroll
      for (int u = 0; u < UN; ++u) rv[u] = load_vec<T, V>(r + at[u]);
#pragma unroll
    for (int u = 0; u < UN; ++u)
      if (k + u < m.count) {
        float y[V];
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = act_f<ACT>(on_line(l[j], (float)v[u].e[j]));
        if (res)
#pragma unroll
          for (int j = 0; j < V; ++j) y[j] += (float)rv[u].e[j];
        Vec<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.e[j] = (T)y[j];
        store_vec<T, V>(out + at[u], o);
      }
  }
  if (m.tail) {
    const int64_t at = ((int)threadIdx.x + m.count * a.A) * V;
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (m.base + at + j < a.R) {
        float y = act_f<ACT>(on_line(l[j], (float)x[at + j]));
        if (res) y += (float)r[at + j];
        out[at + j] = (T)y;
      }
  }
}
template <typename T, int ACT, bool UNI>
__global__ __launch_bounds__(NT) void flat_fwd_kernel(NormArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  for (int64_t u = a.u0 + blockIdx.x; u < a.u1; u += gridDim.x) {
    flat_fwd<T, ACT, UNI>(a, u, reinterpret_cast<Stat*>(smem));
    __syncthreads();
  }
}

// What the backward needs of a channel: xh = (x - mu) rs, z = xh ga + be.
struct Coef {
  float mu, rs, ga, be;
};
__device__ __forceinline__ Coef bwd_coef(const NormArgs& a, int64_t b, int c) {
  const float* st = a.stats_in + 2 * (b * a.G + c / a.Cg);
  return Coef{st[0], st[1], a.gamma ? a.gamma[c] : 1.0f, a.beta ? a.beta[c] : 0.0f};
}
// (Both passes form h alike: in a group whose values hardly differ gx is the
// small difference of large terms, and would show any difference of the two.)
template <int ACT>
__device__ __forceinline__ void bwd_terms(const Coef& k, float x, float g, float* h, float* xh) {
  *xh = (x - k.mu) * k.rs;
  *h = g * act_grad_f<ACT>(__builtin_fmaf(*xh, k.ga, k.be));
}
// A sum of h where the statistics are not finite: not a number (h itself may
// be finite there).
__device__ __forceinline__ float poisoned(const Coef& k, float s) { return __builtin_fmaf(0.0f, k.rs, s); }
// gx = rs (ga h - a - xh d).
struct Means {
  float a, d;
};
__device__ __forceinline__ float bwd_gx(const Coef& k, const Means& m, float h, float xh) {
  return k.rs * __builtin_fmaf(k.ga, h, __builtin_fmaf(xh, -m.d, -m.a));
}
__device__ __forceinline__ Means means_of(const NormArgs& a, const Sums& t) {
  const double m = (double)a.P * a.Cg;
  return Means{(float)(t.s / m), (float)(t.q / m)};
}

// lds [A][V]: by thread and element; ch [C]: gamma times the channel's sums.
template <typename T, int ACT, bool UNI>
__device__ __forceinline__ void flat_sums(const NormArgs& a, int64_t unit, float2* lds, Sums* ch) {
  constexpr int V = kVec<T>, UN = 2;
  const int64_t b = unit / a.n1, chunk = unit - b * a.n1;
  const Mine m = my_vectors(a, chunk, a.v1, V);
  const T* x = static_cast<const T*>(a.x) + b * a.R + m.base;
  const T* g = static_cast<const T*>(a.gout) + b * a.R + m.base;
  if ((int)threadIdx.x < a.A) {
    Coef k[V];
    float s[V], q[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      k[j] = bwd_coef(a, b, my_channel(a, j, V));
      if (UNI && j) {
        k[j].mu = k[0].mu;
        k[j].rs = k[0].rs;
      }
      s[j] = q[j] = 0.0f;
    }
    for (int i = 0; i < m.count; i += UN) {
      Vec<T, V> xv[UN], gv[UN];
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        const uint32_t at = my_at(a, m, i + u, V);
        xv[u] = load_vec<T, V>(x + at);
        gv[u] = load_vec<T, V>(g + at);
      }
#pragma unroll
      for (int u = 0; u < UN; ++u)
        if (i + u < m.count)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            float h, xh;
            bwd_terms<ACT>(k[j], (float)xv[u].e[j], (float)gv[u].e[j], &h, &xh);
            s[j] += h;
            q[j] = __builtin_fmaf(h, xh, q[j]);
          }
    }
    if (m.tail) {
      const int64_t at = ((int)threadIdx.x + m.count * a.A) * V;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (m.base + at + j < a.R) {
          float h, xh;
          bwd_terms<ACT>(k[j], (float)x[at + j], (float)g[at + j], &h, &xh);
          s[j] += h;
          q[j] = __builtin_fmaf(h, xh, q[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) lds[threadIdx.x * V + j] = make_float2(poisoned(k[j], s[j]), q[j]);
  }
  __syncthreads();
  // element f = V t + j of the threads is channel f mod C's
  group_sums(a.C, a.A * V / a.C,
             [&](int c, int i) { const float2 t = lds[i * a.C + c]; return Sums{t.x, t.y}; },
             [&](int c, const Sums& t) {
               a.chan[(b * a.C + c) * a.nc + chunk] = t;
               const double ga = a.gamma ? (double)a.gamma[c] : 1.0;
               ch[c] = Sums{ga * t.s, ga * t.q};
             });
  __syncthreads();
  group_sums(a.G, a.Cg, [&](int gr, int i) { return ch[gr * a.Cg + i]; },
             [&](int gr, const Sums& t) { a.part[(b * a.G + gr) * a.n + chunk] = t; });
}
template <typename T, int ACT, bool UNI>
__global__ __launch_bounds__(NT) void flat_sums_kernel(NormArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  float2* lds = reinterpret_cast<float2*>(smem);
  for (int64_t u = a.u0 + blockIdx.x; u < a.u1; u += gridDim.x) {
    flat_sums<T, ACT, UNI>(a, u, lds, reinterpret_cast<Sums*>(lds + (size_t)NT * kVec<T>));
    __syncthreads();
  }
}

// One channel's parameter gradients: the sum over samples and chunks.
__device__ __forceinline__ void param_grads(const NormArgs& a, int c) {
  Sums v{0.0, 0.0};
  for (int64_t i = threadIdx.x; i < a.B * a.nc; i += NT) {
    const int64_t b = i / a.nc;
    v = add(v, a.chan[(b * a.C + c) * a.nc + (i - b * a.nc)]);
  }
  v = team_sum<NT>(v);
  if (threadIdx.x == 0) {
    if (a.gbeta) a.gbeta[c] = (float)v.s;
    if (a.ggamma) a.ggamma[c] = (float)v.q;
  }
}

template <typename T, int ACT, bool UNI>
__device__ __forceinline__ void flat_bwd(const NormArgs& a, int64_t unit, Means* lds) {  // [G]
  constexpr int V = kVec<T>, UN = 2;
  const int64_t b = unit / a.n2, chunk = unit - b * a.n2;
  load_groups(a, b, lds, [&](int, const Sums& t) { return means_of(a, t); });
  const Mine m = my_vectors(a, chunk, a.v2, V);
  const T* x = static_cast<const T*>(a.x) + b * a.R + m.base;
  const T* g = static_cast<const T*>(a.gout) + b * a.R + m.base;
  T* out = static_cast<T*>(a.out) + b * a.R + m.base;
  if (!m.count && !m.tail) return;
  Coef k[V];
  Means mn[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int c = my_channel(a, j, V);
    k[j] = bwd_coef(a, b, c);
    mn[j] = lds[c / a.Cg];
    if (UNI && j) {
      k[j].mu = k[0].mu;
      k[j].rs = k[0].rs;
      mn[j] = mn[0];
    }
  }
  for (int i = 0; i < m.count; i += UN) {
    Vec<T, V> xv[UN], gv[UN];
    uint32_t at[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      at[u] = my_at(a, m, i + u, V);
      xv[u] = load_vec<T, V>(x + at[u]);
      gv[u] = load_vec<T, V>(g + at[u]);
    }
#pragma unroll
    for (int u = 0; u < UN; ++u)
      if (i + u < m.count) {
        Vec<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float h, xh;
          bwd_terms<ACT>(k[j], (float)xv[u].e[j], (float)gv[u].e[j], &h, &xh);
          o.e[j] = (T)bwd_gx(k[j], mn[j], h, xh);
        }
        store_vec<T, V>(out + at[u], o);
      }
  }
  if (m.tail) {
    const int64_t at = ((int)threadIdx.x + m.count * a.A) * V;
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (m.base + at + j < a.R) {
        float h, xh;
        bwd_terms<ACT>(k[j], (float)x[at + j], (float)g[at + j], &h, &xh);
        out[at + j] = (T)bwd_gx(k[j], mn[j], h, xh);
      }
  }
}

template <typename T, int ACT, bool UNI>
__global__ __launch_bounds__(NT) void flat_bwd_kernel(NormArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  if ((int)blockIdx.x >= a.main) return param_grads(a, (int)blockIdx.x - a.main);
  for (int64_t u = a.u0 + blockIdx.x; u < a.u1; u += a.main) {
    flat_bwd<T, ACT, UNI>(a, u, reinterpret_cast<Means*>(smem));
    __syncthreads();
  }
}

// Each group's entries joined: one wave per group.
__global__ __launch_bounds__(NT) void join_kernel(NormArgs a) {
  const int lane = threadIdx.x & 63;
  for (int64_t g = a.u0 + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); g < a.u1; g += (int64_t)gridDim.x * 4) {
    Sums v{0.0, 0.0};
    for (int i = lane; i < a.n; i += 64) v = add(v, a.part[g * a.n + i]);
    v = team_sum<64>(v);
    if (lane == 0) a.joined[g] = v;
  }
}

// --------------------------------------------------------------------------
// Channels last, wide: a thread takes W channels down the rows of a chunk
// --------------------------------------------------------------------------
struct Wide {
  int64_t b, chunk, at, rows;  // at: the element of the first row's channel c
  int c;                       // first channel (past the last: no work)
};
template <int W>
__device__ __forceinline__ Wide my_wide(const NormArgs& a, int64_t unit) {
  Wide w;
  const int64_t q = unit / a.cols;
  w.c = ((int)(unit - q * a.cols) * NT + (int)threadIdx.x) * W;
  w.b = q / a.n1;
  w.chunk = q - w.b * a.n1;
  const int64_t row = w.chunk * a.rows;
  w.at = (w.b * a.P + row) * a.C + w.c;
  w.rows = w.c >= a.C ? 0 : row + a.rows < a.P ? a.rows : a.P - row;
  return w;
}

__device__ __forceinline__ float act_any(float z, int act) {
  return act == FNO_NORM_ACT_GELU ? gelu_of(z) : act == FNO_NORM_ACT_SILU ? silu_f(z) : z;
}
__device__ __forceinline__ float act_grad_any(float z, int act) {
  return act == FNO_NORM_ACT_GELU ? gelu_grad_of(z) : act == FNO_NORM_ACT_SILU ? silu_grad_f(z) : 1.0f;
}

// f(row, vector of x, vector of the second tensor) for the thread's rows,
// four rows' loads in flight.
template <typename T, int W, typename F>
__device__ __forceinline__ void over_rows(const NormArgs& a, const Wide& w, const T* x, const T* y, F f) {
  constexpr int UN = 4;
  for (int64_t i = 0; i < w.rows; i += UN) {
    Vec<T, W> xv[UN], yv[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int64_t at = w.at + (i + u < w.rows ? i + u : w.rows - 1) * a.C;
      xv[u] = load_vec<T, W>(x + at);
      if (y) yv[u] = load_vec<T, W>(y + at);
    }
#pragma unroll
    for (int u = 0; u < UN; ++u)
      if (i + u < w.rows) f(i + u, xv[u], yv[u]);
  }
}

template <typename T, int W>
__global__ __launch_bounds__(NT) void wide_stats_kernel(NormArgs a) {
  for (int64_t u = a.u0 + blockIdx.x; u < a.u1; u += gridDim.x) {
    const Wide w = my_wide<W>(a, u);
    Sums acc[W];
#pragma unroll
    for (int j = 0; j < W; ++j) acc[j] = Sums{0.0, 0.0};
    over_rows<T, W>(a, w, static_cast<const T*>(a.x), (const T*)nullptr,
                    [&](int64_t, const Vec<T, W>& v, const Vec<T, W>&) {
#pragma unroll
                      for (int j = 0; j < W; ++j) add_value(&acc[j], (float)v.e[j]);
                    });
    if (w.rows)
#pragma unroll
      for (int j = 0; j < W; ++j)
        a.part[(w.b * a.C + w.c + j) * a.n1 + w.chunk] = acc[j];
  }
}

template <typename T, int W>
__global__ __launch_bounds__(NT) void wide_fwd_kernel(NormArgs a) {
  for (int64_t u = a.u0 + blockIdx.x; u < a.u1; u += gridDim.x) {
    const Wide w = my_wide<W>(a, u);
    if (!w.rows) continue;
    Line l[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const int64_t bg = w.b * a.G + (w.c + j) / a.Cg;
      const Stat st = stat_of(a, a.joined[bg]);
      l[j] = line_of(a, st, w.c + j);
      if (a.stats && w.chunk == 0 && (w.c + j) % a.Cg == 0) write_stat(a, bg, st);
    }
    T* out = static_cast<T*>(a.out) + w.at;
    over_rows<T, W>(a, w, static_cast<const T*>(a.x), static_cast<const T*>(a.res),
                    [&](int64_t i, const Vec<T, W>& v, const Vec<T, W>& r) {
                      Vec<T, W> o;
#pragma unroll
                      for (int j = 0; j < W; ++j) {
                        float y = act_any(on_line(l[j], (float)v.e[j]), a.act);
                        if (a.res) y += (float)r.e[j];
                        o.e[j] = (T)y;
                      }
                      store_vec<T, W>(out + i * a.C, o);
                    });
  }
}

template <typename T, int W>
__global__ __launch_bounds__(NT) void wide_sums_kernel(NormArgs a) {
  for (int64_t u = a.u0 + blockIdx.x; u < a.u1; u += gridDim.x) {
    const Wide w = my_wide<W>(a, u);
    if (!w.rows) continue;
    Coef k[W];
    float s[W], q[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      k[j] = bwd_coef(a, w.b, w.c + j);
      s[j] = q[j] = 0.0f;
    }
    over_rows<T, W>(a, w, static_cast<const T*>(a.x), static_cast<const T*>(a.gout),
                    [&](int64_t, const Vec<T, W>& x, const Vec<T, W>& g) {
#pragma unroll
                      for (int j = 0; j < W; ++j) {
                        const float xh = ((float)x.e[j] - k[j].mu) * k[j].rs;
                        const float h = (float)g.e[j] *
                                        act_grad_any(__builtin_fmaf(xh, k[j].ga, k[j].be), a.act);
                        s[j] += h;
                        q[j] = __builtin_fmaf(h, xh, q[j]);
                      }
                    });
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const int64_t at = (w.b * a.C + w.c + j) * a.n1 + w.chunk;
      const double sj = poisoned(k[j], s[j]);
      a.chan[at] = Sums{sj, q[j]};
      a.part[at] = Sums{(double)k[j].ga * sj, (double)k[j].ga * q[j]};
    }
  }
}

template <typename T, int W>
__global__ __launch_bounds__(NT) void wide_bwd_kernel(NormArgs a) {
  if ((int)blockIdx.x >= a.main) return param_grads(a, (int)blockIdx.x - a.main);
  for (int64_t u = a.u0 + blockIdx.x; u < a.u1; u += a.main) {
    const Wide w = my_wide<W>(a, u);
    if (!w.rows) continue;
    Coef k[W];
    Means mn[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      k[j] = bwd_coef(a, w.b, w.c + j);
      mn[j] = means_of(a, a.joined[w.b * a.G + (w.c + j) / a.Cg]);
    }
    T* out = static_cast<T*>(a.out) + w.at;
    over_rows<T, W>(a, w, static_cast<const T*>(a.x), static_cast<const T*>(a.gout),
                    [&](int64_t i, const Vec<T, W>& x, const Vec<T, W>& g) {
                      Vec<T, W> o;
#pragma unroll
                      for (int j = 0; j < W; ++j) {
                        const float xh = ((float)x.e[j] - k[j].mu) * k[j].rs;
                        const float h = (float)g.e[j] *
                                        act_grad_any(__builtin_fmaf(xh, k[j].ga, k[j].be), a.act);
                        o.e[j] = (T)bwd_gx(k[j], mn[j], h, xh);
                      }
                      store_vec<T, W>(out + i * a.C, o);
                    });
  }
}

// --------------------------------------------------------------------------
// Channels first: a team of TEAM threads takes a segment of a plane
// --------------------------------------------------------------------------
struct Seg {
  int64_t bc, at, bg;  // plane, the segment's first element, group
  int c, seg;
  int len;             // elements
};
__device__ __forceinline__ Seg seg_of(const NormArgs& a, int64_t unit) {
  Seg s;
  s.bc = unit / a.n1;
  s.seg = (int)(unit - s.bc * a.n1);
  s.bg = s.bc / a.Cg;
  const int64_t b = s.bc / a.C;
  s.c = (int)(s.bc - b * a.C);
  const int64_t p = s.seg * a.rows;
  s.at = s.bc * a.P + p;
  s.len = (int)(p + a.rows < a.P ? a.rows : a.P - p);
  return s;
}

// f(element, vector of x, vector of y) for this thread's full vectors of a
// segment, UN of them in flight, then f1(element) for at most one element of
// its last partial vector.
template <typename T, int TEAM, int UN, typename F, typename F1>
__device__ __forceinline__ void over_segment(const T* x, const T* y, int len, F f, F1 f1) {
  constexpr int V = kVec<T>;
  const int lane = threadIdx.x & (TEAM - 1), full = len / V;
  for (int i = lane; i < full; i += TEAM * UN) {
    Vec<T, V> xv[UN], yv[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int at = (i + u * TEAM < full ? i + u * TEAM : i) * V;
      xv[u] = load_vec<T, V>(x + at);
      if (y) yv[u] = load_vec<T, V>(y + at);
    }
#pragma unroll
    for (int u = 0; u < UN; ++u)
      if (i + u * TEAM < full) f((i + u * TEAM) * V, xv[u], yv[u]);
  }
  if (lane < len - full * V) f1(full * V + lane);
}

template <int TEAM>
__device__ __forceinline__ int64_t first_unit(const NormArgs& a) {
  return a.u0 + (int64_t)blockIdx.x * (NT / TEAM) + (int)threadIdx.x / TEAM;
}

template <typename T, int TEAM>
__global__ __launch_bounds__(NT) void first_stats_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  for (int64_t u = first_unit<TEAM>(a); u < a.u1; u += (int64_t)gridDim.x * (NT / TEAM)) {
    const Seg s = seg_of(a, u);
    const T* x = static_cast<const T*>(a.x) + s.at;
    Sums t{0.0, 0.0}, t1{0.0, 0.0};
    over_segment<T, TEAM, 4>(
        x, (const T*)nullptr, s.len,
        [&](int, const Vec<T, V>& v, const Vec<T, V>&) {
#pragma unroll
          for (int j = 0; j < V; ++j) add_value(j & 1 ? &t1 : &t, (float)v.e[j]);
        },
        [&](int e) { add_value(&t, (float)x[e]); });
    t = team_sum<TEAM>(add(t, t1));
    if ((threadIdx.x & (TEAM - 1)) == 0) a.part[u] = t;
  }
}

// The sums of the group of a segment.
template <int TEAM>
__device__ __forceinline__ Sums group_of(const NormArgs& a, int64_t bg) {
  if (a.collapse) return a.joined[bg];
  Sums v{0.0, 0.0};
  for (int i = threadIdx.x & (TEAM - 1); i < a.n; i += TEAM) v = add(v, a.part[bg * a.n + i]);
  return team_sum<TEAM>(v);
}

template <typename T, int TEAM, int ACT>
__global__ __launch_bounds__(NT) void first_fwd_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  for (int64_t u = first_unit<TEAM>(a); u < a.u1; u += (int64_t)gridDim.x * (NT / TEAM)) {
    const Seg s = seg_of(a, u);
    const Stat st = stat_of(a, group_of<TEAM>(a, s.bg));
    if (a.stats && s.seg == 0 && s.c % a.Cg == 0 && (threadIdx.x & (TEAM - 1)) == 0) write_stat(a, s.bg, st);
    const Line l = line_of(a, st, s.c);
    const T* x = static_cast<const T*>(a.x) + s.at;
    const T* r = a.res ? static_cast<const T*>(a.res) + s.at : nullptr;
    T* out = static_cast<T*>(a.out) + s.at;
    over_segment<T, TEAM, 4>(
        x, r, s.len,
        [&](int e, const Vec<T, V>& v, const Vec<T, V>& rv) {
          float y[V];
#pragma unroll
          for (int j = 0; j < V; ++j) y[j] = act_f<ACT>(on_line(l, (float)v.e[j]));
          if (r)
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] += (float)rv.e[j];
          Vec<T, V> o;
#pragma unroll
          for (int j = 0; j < V; ++j) o.e[j] = (T)y[j];
          store_vec<T, V>(out + e, o);
        },
        [&](int e) {
          float y = act_f<ACT>(on_line(l, (float)x[e]));
          if (r) y += (float)r[e];
          out[e] = (T)y;
        });
  }
}

template <typename T, int TEAM, int ACT>
__global__ __launch_bounds__(NT) void first_sums_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  for (int64_t u = first_unit<TEAM>(a); u < a.u1; u += (int64_t)gridDim.x * (NT / TEAM)) {
    const Seg s = seg_of(a, u);
    const Coef k = bwd_coef(a, s.bc / a.C, s.c);
    const T* x = static_cast<const T*>(a.x) + s.at;
    const T* g = static_cast<const T*>(a.gout) + s.at;
    float sh = 0.0f, sx = 0.0f;
    auto one = [&](float xv, float gv) {
      float h, xh;
      bwd_terms<ACT>(k, xv, gv, &h, &xh);
      sh += h;
      sx = __builtin_fmaf(h, xh, sx);
    };
    over_segment<T, TEAM, 2>(
        x, g, s.len,
        [&](int, const Vec<T, V>& xv, const Vec<T, V>& gv) {
#pragma unroll
          for (int j = 0; j < V; ++j) one((float)xv.e[j], (float)gv.e[j]);
        },
        [&](int e) { one((float)x[e], (float)g[e]); });
    const Sums t = team_sum<TEAM>(Sums{poisoned(k, sh), sx});
    if ((threadIdx.x & (TEAM - 1)) == 0) {
      a.chan[u] = t;
      a.part[u] = Sums{(double)k.ga * t.s, (double)k.ga * t.q};
    }
  }
}

template <typename T, int TEAM, int ACT>
__global__ __launch_bounds__(NT) void first_bwd_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  if ((int)blockIdx.x >= a.main) return param_grads(a, (int)blockIdx.x - a.main);
  for (int64_t u = first_unit<TEAM>(a); u < a.u1; u += (int64_t)a.main * (NT / TEAM)) {
    const Seg s = seg_of(a, u);
    const Coef k = bwd_coef(a, s.bc / a.C, s.c);
    const Means mn = means_of(a, group_of<TEAM>(a, s.bg));
    const T* x = static_cast<const T*>(a.x) + s.at;
    const T* g = static_cast<const T*>(a.gout) + s.at;
    T* out = static_cast<T*>(a.out) + s.at;
    auto one = [&](float xv, float gv) {
      float h, xh;
      bwd_terms<ACT>(k, xv, gv, &h, &xh);
      return bwd_gx(k, mn, h, xh);
    };
    over_segment<T, TEAM, 2>(
        x, g, s.len,
        [&](int e, const Vec<T, V>& xv, const Vec<T, V>& gv) {
          Vec<T, V> o;
#pragma unroll
          for (int j = 0; j < V; ++j) o.e[j] = (T)one((float)xv.e[j], (float)gv.e[j]);
          store_vec<T, V>(out + e, o);
        },
        [&](int e) { out[e] = (T)one((float)x[e], (float)g[e]); });
  }
}

// --------------------------------------------------------------------------
// Host side
// --------------------------------------------------------------------------
inline bool ok16(const void* p) { return p && ((uintptr_t)p & 15u) == 0; }
inline bool null_or16(const void* p) { return !p || ((uintptr_t)p & 15u) == 0; }

fno_status check_desc(const fno_norm_desc* d) {
  if (!d) return FNO_ERR_INVALID_ARGUMENT;
  if (d->dtype < FNO_DTYPE_F32 || d->dtype > FNO_DTYPE_BF16) return FNO_ERR_INVALID_ARGUMENT;
  if (d->layout != FNO_LAYOUT_CHANNELS_FIRST && d->layout != FNO_LAYOUT_CHANNELS_LAST)
    return FNO_ERR_INVALID_ARGUMENT;
  if (d->activation < FNO_NORM_ACT_NONE || d->activation > FNO_NORM_ACT_SILU)
    return FNO_ERR_INVALID_ARGUMENT;
  if (!(d->eps >= 0.0f && d->eps <= 3.4e38f)) return FNO_ERR_INVALID_ARGUMENT;
  if (d->batch < 1 || d->points < 1 || d->channels < 1 || d->channels > 65536 || d->groups < 1 ||
      d->groups > d->channels || d->channels % d->groups)
    return FNO_ERR_INVALID_ARGUMENT;
  if (d->batch > ((int64_t)1 << 38) / d->points ||
      d->batch * d->points > ((int64_t)1 << 38) / d->channels)
    return FNO_ERR_INVALID_ARGUMENT;
  return FNO_OK;
}

enum Route { FLAT, WIDE, FIRST };
constexpr int kFill = 2048;        // work-groups that fill the chip (eight per compute unit)
constexpr int kMaxGrid = 1 << 20;  // work-groups of a launch; more work is looped over

struct NormPlan {
  NormArgs a;  // sizes only
  Route route;
  int vec;     // elements of a vector (wide: of a thread)
  bool uni;    // flat: a vector's channels are of one group
  int team;    // first
  int64_t units1, units2;  // work items of the passes
};

NormPlan plan_of(const fno_norm_desc& d) {
  NormPlan p{};
  NormArgs& a = p.a;
  const int V = d.dtype == FNO_DTYPE_F32 ? 4 : 8;
  a.B = d.batch;
  a.P = d.points;
  a.C = (int)d.channels;
  a.G = (int)d.groups;
  a.Cg = a.C / a.G;
  a.R = a.P * a.C;
  a.act = d.activation;
  a.eps = d.eps;
  p.vec = V;
  if (d.layout == FNO_LAYOUT_CHANNELS_FIRST) {
    // a wave per plane up to 16 vectors a lane, else work-groups on segments
    // of at least four vectors a thread, enough of them to fill the chip
    p.route = FIRST;
    p.team = a.P <= 64 * V * 16 ? 64 : NT;
    a.n1 = 1;
    if (p.team == NT)
      a.n1 = (int)std::max<int64_t>({1, std::min(cdiv(2 * kFill, a.B * a.C), cdiv(a.P, NT * V * 4)), cdiv(a.P, (int64_t)1 << 30)});
    a.rows = rup(cdiv(a.P, a.n1), (int64_t)NT * V);
    a.n1 = (int)cdiv(a.P, a.rows);
    a.n = a.Cg * a.n1;
    a.nc = a.n1;
    a.collapse = a.n > (p.team == NT ? 1024 : 256);
    p.units1 = p.units2 = a.B * a.C * a.n1;
    return p;
  }
  const int64_t L = a.C / std::gcd(a.C, V);
  if (L <= NT) {
    p.route = FLAT;
    a.L = (int)L;
    a.A = (int)(NT / L * L);
    p.uni = a.C % V == 0 && a.Cg % V == 0;
    const int64_t nv = cdiv(a.R, V), room = std::max<int64_t>(1, nv / ((int64_t)a.A * 4));
    const int64_t want = std::max<int64_t>(std::max<int64_t>(1, kFill / a.B), cdiv(nv, (int64_t)1 << 26));
    a.v1 = a.v2 = rup(cdiv(nv, std::min(want, room)), a.A);  // room: four vectors a thread
    a.n1 = a.n2 = (int)cdiv(nv, a.v1);
    a.n = a.nc = a.n1;
    a.collapse = (int64_t)a.n * a.G > 2048;
    p.units1 = a.B * a.n1;
    p.units2 = a.B * a.n2;
    return p;
  }
  p.route = WIDE;
  p.vec = a.C % V == 0 ? V : 1;
  a.cols = (int)cdiv(a.C, (int64_t)NT * p.vec);
  const int64_t want = std::max<int64_t>(1, kFill / (a.B * a.cols));
  a.rows = cdiv(a.P, std::min(want, std::max<int64_t>(1, a.P / 8)));
  a.n1 = (int)cdiv(a.P, a.rows);
  a.n = a.Cg * a.n1;
  a.nc = a.n1;
  a.collapse = 1;
  p.units1 = p.units2 = a.B * a.n1 * a.cols;
  return p;
}

// Workspace: the groups' partial and joined sums, the channels' sums.
struct WsLayout {
  int64_t joined, chan, bytes;
};
WsLayout ws_of(const NormPlan& p, bool bwd) {
  const NormArgs& a = p.a;
  WsLayout w;
  w.joined = rup(a.B * a.G * a.n * (int64_t)sizeof(Sums), 256);
  w.chan = w.joined + rup(a.B * a.G * (int64_t)sizeof(Sums), 256);
  w.bytes = w.chan + (bwd ? rup(a.B * a.C * a.nc * (int64_t)sizeof(Sums), 256) : 0);
  return w;
}

struct NormLaunch {
  NormPlan p;
  int dt;
  hipStream_t s;
};

unsigned grid_of(int64_t units) { return (unsigned)std::min<int64_t>(units, kMaxGrid); }

void launch_join(NormLaunch& L) {
  NormArgs& a = L.p.a;
  if (!a.collapse) return;
  a.u0 = 0;
  a.u1 = a.B * a.G;
  hipLaunchKernelGGL(join_kernel, dim3(grid_of(cdiv(a.u1, 4))), dim3(NT), 0, L.s, a);
}

template <typename T>
void launch_stats(NormLaunch& L) {
  NormArgs& a = L.p.a;
  a.u0 = 0;
  a.u1 = L.p.units1;
  if (L.p.route == FLAT) {
    const size_t lds = (size_t)a.A * (L.p.uni ? 1 : kVec<T>) * sizeof(Sums);
    auto k = L.p.uni ? flat_stats_kernel<T, true> : flat_stats_kernel<T, false>;
    hipLaunchKernelGGL(k, dim3(grid_of(a.u1)), dim3(NT), lds, L.s, a);
  } else if (L.p.route == WIDE) {
    auto k = L.p.vec == 1 ? wide_stats_kernel<T, 1> : wide_stats_kernel<T, kVec<T>>;
    hipLaunchKernelGGL(k, dim3(grid_of(a.u1)), dim3(NT), 0, L.s, a);
  } else {
    auto k = L.p.team == 64 ? first_stats_kernel<T, 64> : first_stats_kernel<T, NT>;
    hipLaunchKernelGGL(k, dim3(grid_of(cdiv(a.u1, NT / L.p.team))), dim3(NT), 0, L.s, a);
  }
}

template <typename T, int ACT>
void launch_fwd_t(NormLaunch& L) {
  NormArgs& a = L.p.a;
  launch_stats<T>(L);
  launch_join(L);
  a.u0 = 0;
  a.u1 = L.p.units2;
  if (L.p.route == FLAT) {
    auto k = L.p.uni ? flat_fwd_kernel<T, ACT, true> : flat_fwd_kernel<T, ACT, false>;
    hipLaunchKernelGGL(k, dim3(grid_of(a.u1)), dim3(NT), a.G * sizeof(Stat), L.s, a);
  } else if (L.p.route == WIDE) {
    auto k = L.p.vec == 1 ? wide_fwd_kernel<T, 1> : wide_fwd_kernel<T, kVec<T>>;
    hipLaunchKernelGGL(k, dim3(grid_of(a.u1)), dim3(NT), 0, L.s, a);
  } else {
    auto k = L.p.team == 64 ? first_fwd_kernel<T, 64, ACT> : first_fwd_kernel<T, NT, ACT>;
    hipLaunchKernelGGL(k, dim3(grid_of(cdiv(a.u1, NT / L.p.team))), dim3(NT), 0, L.s, a);
  }
}

template <typename T, int ACT>
void launch_bwd_t(NormLaunch& L) {
  NormArgs& a = L.p.a;
  const int extra = a.ggamma || a.gbeta ? a.C : 0;
  a.u0 = 0;
  a.u1 = L.p.units1;
  if (L.p.route == FLAT) {
    const size_t lds = (size_t)NT * kVec<T> * sizeof(float2) + a.C * sizeof(Sums);
    auto k1 = L.p.uni ? flat_sums_kernel<T, ACT, true> : flat_sums_kernel<T, ACT, false>;
    hipLaunchKernelGGL(k1, dim3(grid_of(a.u1)), dim3(NT), lds, L.s, a);
    launch_join(L);
    a.u0 = 0;
    a.u1 = L.p.units2;
    a.main = (int)grid_of(a.u1);
    auto k2 = L.p.uni ? flat_bwd_kernel<T, ACT, true> : flat_bwd_kernel<T, ACT, false>;
    hipLaunchKernelGGL(k2, dim3(a.main + extra), dim3(NT), a.G * sizeof(Stat), L.s, a);
  } else if (L.p.route == WIDE) {
    auto k1 = L.p.vec == 1 ? wide_sums_kernel<T, 1> : wide_sums_kernel<T, kVec<T>>;
    hipLaunchKernelGGL(k1, dim3(grid_of(a.u1)), dim3(NT), 0, L.s, a);
    launch_join(L);
    a.u0 = 0;
    a.u1 = L.p.units2;
    a.main = (int)grid_of(a.u1);
    auto k2 = L.p.vec == 1 ? wide_bwd_kernel<T, 1> : wide_bwd_kernel<T, kVec<T>>;
    hipLaunchKernelGGL(k2, dim3(a.main + extra), dim3(NT), 0, L.s, a);
  } else {
    const int64_t per = NT / L.p.team;
    auto k1 = L.p.team == 64 ? first_sums_kernel<T, 64, ACT> : first_sums_kernel<T, NT, ACT>;
    hipLaunchKernelGGL(k1, dim3(grid_of(cdiv(a.u1, per))), dim3(NT), 0, L.s, a);
    launch_join(L);
    a.u0 = 0;
    a.u1 = L.p.units2;
    a.main = (int)grid_of(cdiv(a.u1, per));
    auto k2 = L.p.team == 64 ? first_bwd_kernel<T, 64, ACT> : first_bwd_kernel<T, NT, ACT>;
    hipLaunchKernelGGL(k2, dim3(a.main + extra), dim3(NT), 0, L.s, a);
  }
}

template <typename T>
hipError_t by_act(NormLaunch& L, bool bwd) {
  switch (L.p.a.act) {
    case FNO_NORM_ACT_GELU:
      bwd ? launch_bwd_t<T, FNO_NORM_ACT_GELU>(L) : launch_fwd_t<T, FNO_NORM_ACT_GELU>(L);
      break;
    case FNO_NORM_ACT_SILU:
      bwd ? launch_bwd_t<T, FNO_NORM_ACT_SILU>(L) : launch_fwd_t<T, FNO_NORM_ACT_SILU>(L);
      break;
    default:
      bwd ? launch_bwd_t<T, FNO_NORM_ACT_NONE>(L) : launch_fwd_t<T, FNO_NORM_ACT_NONE>(L);
  }
  return hipGetLastError();
}

hipError_t by_type(NormLaunch& L, bool bwd) {
  return L.dt == FNO_DTYPE_F32   ? by_act<float>(L, bwd)
         : L.dt == FNO_DTYPE_F16 ? by_act<_Float16>(L, bwd)
                                 : by_act<__bf16>(L, bwd);
}
hipError_t launch_fwd(void* ctx) { return by_type(*static_cast<NormLaunch*>(ctx), false); }
hipError_t launch_bwd(void* ctx) { return by_type(*static_cast<NormLaunch*>(ctx), true); }

void set_ws(NormArgs* a, const WsLayout& w, void* ws) {
  char* p = static_cast<char*>(ws);
  a->part = reinterpret_cast<Sums*>(p);
  a->joined = reinterpret_cast<Sums*>(p + w.joined);
  a->chan = reinterpret_cast<Sums*>(p + w.chan);
}

}  // namespace
}  // namespace fno

using namespace fno;

extern "C" fno_status fno_group_norm_act_workspace_size(const fno_norm_desc* d, fno_op op,
                                                        size_t* bytes) {
  const fno_status st = check_desc(d);
  if (st != FNO_OK) return st;
  if (!bytes || (op != FNO_OP_FWD && op != FNO_OP_BWD)) return FNO_ERR_INVALID_ARGUMENT;
  *bytes = (size_t)ws_of(plan_of(*d), op == FNO_OP_BWD).bytes;
  return FNO_OK;
}

extern "C" fno_status fno_group_norm_act_fwd(const fno_norm_desc* d, const void* x,
                                             const float* gamma, const float* beta,
                                             const void* residual, void* out, float* stats,
                                             void* ws, size_t ws_len, hipStream_t stream) {
  const fno_status st = check_desc(d);
  if (st != FNO_OK) return st;
  if (!ok16(x) || !ok16(out) || !null_or16(gamma) || !null_or16(beta) || !null_or16(residual) ||
      !null_or16(stats))
    return FNO_ERR_INVALID_ARGUMENT;
  NormLaunch L{plan_of(*d), d->dtype, stream};
  const WsLayout w = ws_of(L.p, false);
  if (ws_len < (size_t)w.bytes) return FNO_ERR_WORKSPACE_TOO_SMALL;
  if (!ok16(ws)) return FNO_ERR_INVALID_ARGUMENT;
  NormArgs& a = L.p.a;
  set_ws(&a, w, ws);
  a.x = x;
  a.gamma = gamma;
  a.beta = beta;
  a.res = residual;
  a.out = out;
  a.stats = stats;
  const hipError_t e = timed_launch("group_norm_act_fwd", stream, launch_fwd, &L);
  return e == hipSuccess ? FNO_OK : report_hip_error(e, "group_norm_act_fwd");
}

extern "C" fno_status fno_group_norm_act_bwd(const fno_norm_desc* d, const void* x,
                                             const float* gamma, const float* beta,
                                             const float* stats, const void* g_out, void* gx,
                                             float* g_gamma, float* g_beta, void* ws,
                                             size_t ws_len, hipStream_t stream) {
  const fno_status st = check_desc(d);
  if (st != FNO_OK) return st;
  if (!ok16(x) || !ok16(g_out) || !ok16(gx) || !ok16(stats) || !null_or16(gamma) ||
      !null_or16(beta) || !null_or16(g_gamma) || !null_or16(g_beta))
    return FNO_ERR_INVALID_ARGUMENT;
  NormLaunch L{plan_of(*d), d->dtype, stream};
  const WsLayout w = ws_of(L.p, true);
  if (ws_len < (size_t)w.bytes) return FNO_ERR_WORKSPACE_TOO_SMALL;
  if (!ok16(ws)) return FNO_ERR_INVALID_ARGUMENT;
  NormArgs& a = L.p.a;
  set_ws(&a, w, ws);
  a.x = x;
  a.gamma = gamma;
  a.beta = beta;
  a.stats_in = stats;
  a.gout = g_out;
  a.out = gx;
  a.ggamma = g_gamma;
  a.gbeta = g_beta;
  const hipError_t e = timed_launch("group_norm_act_bwd", stream, launch_bwd, &L);
  return e == hipSuccess ? FNO_OK : report_hip_error(e, "group_norm_act_bwd");
}
