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
// joins its group's and streams the tensors again.  The second pass takes the
// work items in the opposite order, so that what the first read last is still
// in the memory-side cache, and reads past that cache what is not needed again
// (8 x 64 planes of 1024^2, fp16 with a residual: 787 us for 807 in the
// opposite order, 756 with both).
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
//
// Bound by memory: 8 x 64 x 1024^2, fp16: sums 165 us (6.5 TB/s), results with a
// residual 542 (6.2); the backward of 16 x 128 x 256^2, bf16: 98 to 102 and
// 135 to 142 (5.3 to 5.5, 5.9 to 6.2).  Channels last 32 x 128^2 x 64, fp16: forward 13 + 28 us (5.2 and
// 4.9 TB/s), backward 35 + 36 (4.0 and 5.8), its sums as much by their arithmetic
// (28% of a wave's time in vector operations, four work-groups to a unit, the
// GELU body with two registers in scratch).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <numeric>

#include "../../include/fno_spectral_conv.h"
#include "fno_host.h"
#include "fno_norm.h"

namespace fno {
namespace {

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
// The element of the chunk where this thread's vector k starts.  Chunks hold
// less than 2^31 elements.
__device__ __forceinline__ uint32_t my_at(const NormArgs& a, int k, int vec) {
  return (uint32_t)(((int)threadIdx.x + k * a.A) * vec);
}

// f(j, channel, group) for the elements of this thread's vectors.
template <int V, bool UNI, typename F>
__device__ __forceinline__ void my_channels(const NormArgs& a, F f) {
  int c = V * ((int)threadIdx.x % a.L);
  if (!UNI) c %= a.C;
  int g = c / a.Cg, left = (g + 1) * a.Cg - c;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    f(j, c, g);
    ++c;
    if (!UNI && --left == 0) {
      left = a.Cg;
      if (++g == a.G) g = c = 0;
    }
  }
}

// UNI: a vector's channels are of one group (and C is a multiple of a vector).
// The second pass also tells whether vectors are aligned, as they then are.
enum { kAny = 0, kAligned = 1, kUni = 2 };
template <typename T, bool UNI>
__device__ __forceinline__ void flat_stats(const NormArgs& a, int64_t unit, Sums* lds) {  // [A][E]
  constexpr int V = kVec<T>, UN = 4, E = UNI ? 1 : V;
  const int64_t b = unit / a.n1, chunk = unit - b * a.n1;
  const Mine m = my_vectors(a, chunk, a.v1, V);
  const T* x = static_cast<const T*>(a.x) + b * a.R + m.base;
  Sums acc[E];
#pragma unroll
  for (int j = 0; j < E; ++j) acc[j] = Sums{0.0, 0.0};
  stream<UN>(m.count, [&](int k) { return load_vec<T, V>(x + my_at(a, k, V)); })
      .run([&](const Vec<T, V>& v, int) {
#pragma unroll
        for (int j = 0; j < V; ++j) add_value(&acc[UNI ? 0 : j], (float)v.e[j]);
      });
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

template <typename T, int ACT, int KIND>
__device__ __forceinline__ void flat_fwd(const NormArgs& a, int64_t unit, Stat* lds) {  // [G]
  constexpr bool UNI = KIND == kUni;
  constexpr int V = kVec<T>, UN = UNI ? 2 : 1;
  const int64_t b = unit / a.n1, chunk = unit - b * a.n1;
  const bool res = a.res != nullptr;
  const Mine m = my_vectors(a, chunk, a.v1, V);
  const T* x = static_cast<const T*>(a.x) + b * a.R + m.base;
  const T* r = res ? static_cast<const T*>(a.res) + b * a.R + m.base : nullptr;
  T* out = static_cast<T*>(a.out) + b * a.R + m.base;
  auto data = stream<UN>(m.count, [&](int k) {
    Pair<T, V> p;
    p.x = load_vec<T, V>(x + my_at(a, k, V));
    if (res) p.y = load_last<T, V>(r + my_at(a, k, V));  // (x: 37.9 us cached, 42.9 past it)
    return p;
  });
  load_groups(a, b, lds, [&](int g, const Sums& t) {
    const Stat st = stat_of(a, t);
    if (chunk == 0 && a.stats) write_stat(a, b * a.G + g, st);
    return st;
  });
  if (!m.count && !m.tail) return;
  Line l[V];
  my_channels<V, UNI>(a, [&](int j, int c, int g) {
    l[j] = line_of(a, lds[g], c);
    if (UNI && j) l[j].mu = l[0].mu;
  });
  data.run(
      [&](const Pair<T, V>& p, int k) {
        float y[V];
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = act_any<T>(on_line(l[j], p.x.e[j]), ACT);
        if (res)
#pragma unroll
          for (int j = 0; j < V; ++j) y[j] += (float)p.y.e[j];
        Vec<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.e[j] = (T)y[j];
        store_result<T, V>(out + my_at(a, k, V), o, KIND != kAny);
      });
  if (m.tail) {
    const int64_t at = ((int)threadIdx.x + m.count * a.A) * V;
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (m.base + at + j < a.R) {
        float y = act_any<T>(on_line(l[j], x[at + j]), ACT);
        if (res) y += (float)r[at + j];
        out[at + j] = (T)y;
      }
  }
}
template <typename T, int ACT, int KIND>
__global__ __launch_bounds__(NT, 4) void flat_fwd_kernel(NormArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  for (int64_t u = a.u0 + blockIdx.x; u < a.u1; u += gridDim.x) {
    flat_fwd<T, ACT, KIND>(a, a.u1 - 1 - u, reinterpret_cast<Stat*>(smem));
    __syncthreads();
  }
}

// lds [A][V]: by thread and element; ch [C]: gamma times the channel's sums.
template <typename T, int ACT, bool UNI>
__device__ __forceinline__ void flat_sums(const NormArgs& a, int64_t unit, float2* lds, Sums* ch) {
  constexpr int V = kVec<T>, UN = UNI ? 2 : 1;
  const int64_t b = unit / a.n1, chunk = unit - b * a.n1;
  const Mine m = my_vectors(a, chunk, a.v1, V);
  const T* x = static_cast<const T*>(a.x) + b * a.R + m.base;
  const T* g = static_cast<const T*>(a.gout) + b * a.R + m.base;
  auto data = stream<UN>(m.count, [&](int i) {
    return Pair<T, V>{load_vec<T, V>(x + my_at(a, i, V)), load_vec<T, V>(g + my_at(a, i, V))};
  });
  if ((int)threadIdx.x < a.A) {
    Coef k[V];
    float s[V], q[V];
    my_channels<V, UNI>(a, [&](int j, int c, int gr) {
      k[j] = bwd_coef<T>(a, b * a.G + gr, c);
      if (UNI && j) {
        k[j].mu = k[0].mu;
        k[j].s = k[0].s;
        k[j].rel = k[0].rel;
      }
      s[j] = q[j] = 0.0f;
    });
    data.run(
        [&](const Pair<T, V>& p, int) {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            float h, d;
            bwd_terms<ACT>(k[j], p.x.e[j], p.y.e[j], &h, &d);
            s[j] += h;
            q[j] = __builtin_fmaf(h, d, q[j]);
          }
        });
    if (m.tail) {
      const int64_t at = ((int)threadIdx.x + m.count * a.A) * V;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (m.base + at + j < a.R) {
          float h, d;
          bwd_terms<ACT>(k[j], x[at + j], g[at + j], &h, &d);
          s[j] += h;
          q[j] = __builtin_fmaf(h, d, q[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) lds[threadIdx.x * V + j] = bwd_sums(k[j], ACT, s[j], q[j]);
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
__global__ __launch_bounds__(NT, UNI ? 4 : 3) void flat_sums_kernel(NormArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  float2* lds = reinterpret_cast<float2*>(smem);
  for (int64_t u = a.u0 + blockIdx.x; u < a.u1; u += gridDim.x) {
    flat_sums<T, ACT, UNI>(a, u, lds, reinterpret_cast<Sums*>(lds + (size_t)NT * kVec<T>));
    __syncthreads();
  }
}

template <typename T, int ACT, int KIND>
__device__ __forceinline__ void flat_bwd(const NormArgs& a, int64_t unit, Means* lds) {  // [G]
  constexpr bool UNI = KIND == kUni;
  constexpr int V = kVec<T>, UN = UNI ? 2 : 1;
  const int64_t b = unit / a.n1, chunk = unit - b * a.n1;
  const Mine m = my_vectors(a, chunk, a.v1, V);
  const T* x = static_cast<const T*>(a.x) + b * a.R + m.base;
  const T* g = static_cast<const T*>(a.gout) + b * a.R + m.base;
  T* out = static_cast<T*>(a.out) + b * a.R + m.base;
  auto data = stream<UN>(m.count, [&](int i) {
    // (Groups that cross vectors: 44.3 us with cached loads for 16 x 241^2 x 20, 46.8 past the cache.)
    Pair<T, V> p;
    p.x = UNI ? load_last<T, V>(x + my_at(a, i, V)) : load_vec<T, V>(x + my_at(a, i, V));
    p.y = UNI ? load_last<T, V>(g + my_at(a, i, V)) : load_vec<T, V>(g + my_at(a, i, V));
    return p;
  });
  load_groups(a, b, lds, [&](int, const Sums& t) { return means_of(a, t); });
  if (!m.count && !m.tail) return;
  Coef k[V];
  Gx gk[V];
  my_channels<V, UNI>(a, [&](int j, int c, int gr) {
    k[j] = bwd_coef<T>(a, b * a.G + gr, c);
    gk[j] = gx_coef(k[j], lds[gr]);
    if (UNI && j) {
      k[j].mu = k[0].mu;
      k[j].s = k[0].s;
      gk[j].c0 = gk[0].c0;
      gk[j].c1 = gk[0].c1;
    }
  });
  data.run(
      [&](const Pair<T, V>& p, int i) {
        Vec<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float h, d;
          bwd_terms<ACT>(k[j], p.x.e[j], p.y.e[j], &h, &d);
          o.e[j] = (T)bwd_gx(gk[j], h, d);
        }
        store_result<T, V>(out + my_at(a, i, V), o, KIND != kAny);
      });
  if (m.tail) {
    const int64_t at = ((int)threadIdx.x + m.count * a.A) * V;
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (m.base + at + j < a.R) {
        float h, d;
        bwd_terms<ACT>(k[j], x[at + j], g[at + j], &h, &d);
        out[at + j] = (T)bwd_gx(gk[j], h, d);
      }
  }
}

template <typename T, int ACT, int KIND>
__global__ __launch_bounds__(NT, KIND == kUni ? 4 : 3) void flat_bwd_kernel(NormArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  if ((int)blockIdx.x >= a.main) return param_grads(a, (int)blockIdx.x - a.main);
  for (int64_t u = a.u0 + blockIdx.x; u < a.u1; u += a.main) {
    flat_bwd<T, ACT, KIND>(a, a.u1 - 1 - u, reinterpret_cast<Means*>(smem));
    __syncthreads();
  }
}

// Each group's entries joined by TEAM threads: a wave where a group has up to
// 256, else a work-group; four loads of a thread in flight (8192 entries of one group,
// 8 planes of 2^24: forward 136 us, 167 with a wave and one load).
template <int TEAM>
__global__ __launch_bounds__(NT) void join_kernel(NormArgs a) {
  const int lane = threadIdx.x & (TEAM - 1);
  for (int64_t g0 = (int64_t)blockIdx.x * (NT / TEAM); g0 < a.u1; g0 += (int64_t)gridDim.x * (NT / TEAM)) {
    const int64_t g = g0 + (int)threadIdx.x / TEAM;
    Sums v[4] = {};
    if (g < a.u1) {
      const Sums* p = a.part + g * a.n;
      for (int i = lane; i < a.n; i += 4 * TEAM) {
        Sums t[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = p[i + k * TEAM < a.n ? i + k * TEAM : i];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i + k * TEAM < a.n) v[k] = add(v[k], t[k]);
      }
    }
    const Sums t = team_sum<TEAM>(add(add(v[0], v[1]), add(v[2], v[3])));
    if (g < a.u1 && lane == 0) a.joined[g] = t;
  }
}

// --------------------------------------------------------------------------
// Channels last, wide: a thread takes W channels down the rows of a chunk
// --------------------------------------------------------------------------
// Three to five times the bytes' time: one channel to a load where C is no
// multiple of a vector (16 x 128^2 x 257, fp16: forward 190 us for 41, backward
// 272 for 61), else registers for two work-groups a unit in the backward's sums
// (8 x 64^2 x 4096: 231 for 81 and 420 for 122).
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

// f(row, vector of x, vector of the second tensor) for the thread's rows.
template <typename T, int W, typename F>
__device__ __forceinline__ void over_rows(const NormArgs& a, const Wide& w, const T* x, const T* y, F f) {
  stream<4>((int)w.rows, [&](int i) {
    Pair<T, W> p;
    p.x = load_vec<T, W>(x + w.at + (int64_t)i * a.C);
    if (y) p.y = load_vec<T, W>(y + w.at + (int64_t)i * a.C);
    return p;
  }).run([&](const Pair<T, W>& p, int i) { f((int64_t)i, p.x, p.y); });
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
                        float y = act_any<T>(on_line(l[j], v.e[j]), a.act);
                        if (a.res) y += (float)r.e[j];
                        o.e[j] = (T)y;
                      }
                      store_result<T, W>(out + i * a.C, o, a.nt);
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
    Sums t[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      k[j] = bwd_coef<T>(a, w.b * a.G + (w.c + j) / a.Cg, w.c + j);
      s[j] = q[j] = 0.0f;
      t[j] = Sums{0.0, 0.0};
    }
    auto flush = [&] {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        t[j] = add(t[j], Sums{s[j], q[j]});
        s[j] = q[j] = 0.0f;
      }
    };
    over_rows<T, W>(a, w, static_cast<const T*>(a.x), static_cast<const T*>(a.gout),
                    [&](int64_t i, const Vec<T, W>& x, const Vec<T, W>& g) {
#pragma unroll
                      for (int j = 0; j < W; ++j) {
                        const float d = distance(k[j], x.e[j]);
                        const float h = (float)g.e[j] *
                                        act_grad_any<T>(__builtin_fmaf(d, k[j].k, k[j].be), a.act);
                        s[j] += h;
                        q[j] = __builtin_fmaf(h, d, q[j]);
                      }
                      if (i % kChain == kChain - 1) flush();
                    });
    flush();
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const int64_t at = (w.b * a.C + w.c + j) * a.n1 + w.chunk;
      const Sums v = bwd_sums(k[j], a.act, t[j]);
      a.chan[at] = v;
      a.part[at] = Sums{(double)k[j].ga * v.s, (double)k[j].ga * v.q};
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
    Gx gk[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const int64_t bg = w.b * a.G + (w.c + j) / a.Cg;
      k[j] = bwd_coef<T>(a, bg, w.c + j);
      gk[j] = gx_coef(k[j], means_of(a, a.joined[bg]));
    }
    T* out = static_cast<T*>(a.out) + w.at;
    over_rows<T, W>(a, w, static_cast<const T*>(a.x), static_cast<const T*>(a.gout),
                    [&](int64_t i, const Vec<T, W>& x, const Vec<T, W>& g) {
                      Vec<T, W> o;
#pragma unroll
                      for (int j = 0; j < W; ++j) {
                        const float d = distance(k[j], x.e[j]);
                        const float h = (float)g.e[j] *
                                        act_grad_any<T>(__builtin_fmaf(d, k[j].k, k[j].be), a.act);
                        o.e[j] = (T)bwd_gx(gk[j], h, d);
                      }
                      store_result<T, W>(out + i * a.C, o, a.nt);
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

// This thread's full vectors of a segment, of x and (y not null) of y, UN ahead.
// (Backward of 16 x 128 planes of 256^2, bf16: 226 us with one ahead in the sums
// and three in the results; two in the sums 232, three 263 (registers); two in
// the results 232, one 228.  Forward: three 756, two 772, four 772.)
template <typename T, int TEAM, int UN, bool LAST>
__device__ __forceinline__ auto segment(const T* x, const T* y, int len) {
  constexpr int V = kVec<T>;
  const int lane = threadIdx.x & (TEAM - 1), full = len / V;
  return stream<UN>(lane < full ? (full - lane + TEAM - 1) / TEAM : 0, [=](int k) {
    const uint32_t e = (uint32_t)((lane + k * TEAM) * V);
    Pair<T, V> p;
    p.x = LAST ? load_last<T, V>(x + e) : load_vec<T, V>(x + e);
    if (y) p.y = LAST ? load_last<T, V>(y + e) : load_vec<T, V>(y + e);
    return p;
  });
}
// f(element, vector of x, vector of y) for them, then f1(element) for at most
// one element of the segment's last, partial vector.
template <typename T, int TEAM, typename S, typename F, typename F1>
__device__ __forceinline__ void over_segment(S& data, int len, F f, F1 f1) {
  constexpr int V = kVec<T>;
  const int lane = threadIdx.x & (TEAM - 1), full = len / V;
  data.run([&](const Pair<T, V>& p, int k) { f((lane + k * TEAM) * V, p.x, p.y); });
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
    auto data = segment<T, TEAM, 4, false>(x, (const T*)nullptr, s.len);
    over_segment<T, TEAM>(
        data, s.len,
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
    const Seg s = seg_of(a, a.u1 - 1 - u);
    const T* x = static_cast<const T*>(a.x) + s.at;
    const T* r = a.res ? static_cast<const T*>(a.res) + s.at : nullptr;
    auto data = segment<T, TEAM, 3, true>(x, r, s.len);
    const Stat st = stat_of(a, group_of<TEAM>(a, s.bg));
    if (a.stats && s.seg == 0 && s.c % a.Cg == 0 && (threadIdx.x & (TEAM - 1)) == 0) write_stat(a, s.bg, st);
    const Line l = line_of(a, st, s.c);
    T* out = static_cast<T*>(a.out) + s.at;
    over_segment<T, TEAM>(
        data, s.len,
        [&](int e, const Vec<T, V>& v, const Vec<T, V>& rv) {
          float y[V];
#pragma unroll
          for (int j = 0; j < V; ++j) y[j] = act_any<T>(on_line(l, v.e[j]), ACT);
          if (r)
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] += (float)rv.e[j];
          Vec<T, V> o;
#pragma unroll
          for (int j = 0; j < V; ++j) o.e[j] = (T)y[j];
          store_result<T, V>(out + e, o, a.nt);
        },
        [&](int e) {
          float y = act_any<T>(on_line(l, x[e]), ACT);
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
    const T* x = static_cast<const T*>(a.x) + s.at;
    const T* g = static_cast<const T*>(a.gout) + s.at;
    auto data = segment<T, TEAM, 1, false>(x, g, s.len);
    const Coef k = bwd_coef<T>(a, s.bg, s.c);
    float sh = 0.0f, sx = 0.0f;
    int n = 0;  // vectors (a wave's plane has at most 16 for a lane)
    Sums mine{0.0, 0.0};
    auto one = [&](T xv, T gv) {
      float h, d;
      bwd_terms<ACT>(k, xv, gv, &h, &d);
      sh += h;
      sx = __builtin_fmaf(h, d, sx);
    };
    auto flush = [&] {
      mine = add(mine, Sums{sh, sx});
      sh = sx = 0.0f;
    };
    over_segment<T, TEAM>(
        data, s.len,
        [&](int, const Vec<T, V>& xv, const Vec<T, V>& gv) {
#pragma unroll
          for (int j = 0; j < V; ++j) one(xv.e[j], gv.e[j]);
          if (TEAM == NT && ++n % (kChain / V) == 0) flush();
        },
        [&](int e) {
          flush();
          one(x[e], g[e]);
        });
    flush();
    const Sums t = team_sum<TEAM>(bwd_sums(k, ACT, mine));
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
    const Seg s = seg_of(a, a.u1 - 1 - u);
    const T* x = static_cast<const T*>(a.x) + s.at;
    const T* g = static_cast<const T*>(a.gout) + s.at;
    auto data = segment<T, TEAM, 3, true>(x, g, s.len);
    const Coef k = bwd_coef<T>(a, s.bg, s.c);
    const Gx gk = gx_coef(k, means_of(a, group_of<TEAM>(a, s.bg)));
    T* out = static_cast<T*>(a.out) + s.at;
    auto one = [&](T xv, T gv) {
      float h, d;
      bwd_terms<ACT>(k, xv, gv, &h, &d);
      return bwd_gx(gk, h, d);
    };
    over_segment<T, TEAM>(
        data, s.len,
        [&](int e, const Vec<T, V>& xv, const Vec<T, V>& gv) {
          Vec<T, V> o;
#pragma unroll
          for (int j = 0; j < V; ++j) o.e[j] = (T)one(xv.e[j], gv.e[j]);
          store_result<T, V>(out + e, o, a.nt);
        },
        [&](int e) { out[e] = (T)one(x[e], g[e]); });
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

enum Route { FLAT, WIDE, FIRST, RESIDENT };
constexpr int kFill = 1024;        // work-groups that fill the chip (four per compute unit)
constexpr int kFillFew = 768;      // three: the backward where groups cross vectors, by its
                                   // registers (16 x 241^2 x 20: 44.5 us, 50.7 with 1024)
constexpr int kMaxGrid = 1 << 20;  // work-groups of a launch; more work is looped over

struct NormPlan {
  NormArgs a;  // sizes only
  Route route;
  int vec;     // elements of a vector (wide: of a thread)
  bool uni;    // flat: a vector's channels are of one group
  int team;    // first
  int64_t units;  // work items of each pass
  bool first;     // channels first
};

NormPlan plan_of(const fno_norm_desc& d, bool bwd) {
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
  p.first = d.layout == FNO_LAYOUT_CHANNELS_FIRST;
  a.nt = (p.first ? a.P : a.R) % V == 0;
  if (norm_resident_fits(a, d.dtype, p.first, bwd)) {
    p.route = RESIDENT;
    a.nc = 1;
    return p;
  }
  if (p.first) {
    // A wave per plane up to 16 vectors a lane, else work-groups on segments
    // of eight vectors a thread: forward of 8 x 64 planes of 1024^2 in eight
    // groups, fp16 with a residual, 703 us; 747 with sixteen vectors, 774 with
    // six, 888 with four; backward of 16 x 128 planes of 256^2, bf16, 225, 232,
    // 232 and 248.  Longer ones where a group would have more than the 1024
    // entries that the second pass joins itself, unless work-groups are few
    // (the same planes in one group: 603 us with sixteen segments a plane, 635
    // with 64 and a launch that joins them).  Few or small planes leave compute
    // units idle: 2 x 16 x 90^2 runs in eight work-groups, 15 us forward and 21
    // backward, where a launch and its calls take 10.
    p.route = FIRST;
    p.team = a.P <= 64 * V * 16 ? 64 : NT;
    a.n1 = 1;
    if (p.team == NT)
      a.n1 = (int)std::max<int64_t>(
          {1, std::min(std::max<int64_t>(1024 / a.Cg, cdiv(8 * kFill, a.B * a.C)), a.P / (NT * V * 8)),
           cdiv(a.P, (int64_t)1 << 30)});
    a.rows = rup(cdiv(a.P, a.n1), (int64_t)NT * V);
    a.n1 = (int)cdiv(a.P, a.rows);
    a.n = a.Cg * a.n1;
    a.nc = a.n1;
    a.collapse = a.n > (p.team == NT ? 1024 : 256);
    p.units = a.B * a.C * a.n1;
    return p;
  }
  const int64_t L = a.C / std::gcd(a.C, V);
  if (L <= NT) {
    // Chunks of 16 vectors a thread (fp32, whose vectors take half the
    // operations: 8), between one and four times the work-groups that fill
    // the chip, but at least four vectors a thread.  A work-group's start and
    // end (its channels' coefficients, its sums joined) cost as much as five
    // vectors (33.5 M fp16 elements: forward 37.7 us with 1024 work-groups, 42.9
    // with 2048, 57 with 4096, backward 67.4, 72.7 and 91; as many fp32: 68.5,
    // 69 and 66).
    p.route = FLAT;
    a.L = (int)L;
    a.A = (int)(NT / L * L);
    p.uni = a.C % V == 0 && a.Cg % V == 0;
    const int64_t nv = cdiv(a.R, V), per = (int64_t)a.A * (V == 4 ? 8 : 16);
    const int fill = bwd && !p.uni ? kFillFew : kFill;
    const int64_t want = std::clamp<int64_t>(a.B * nv / per, fill, 4 * fill) / a.B;
    const int64_t room = std::max<int64_t>(1, nv / ((int64_t)a.A * 4));
    // (the backward's chunks also so that a thread adds at most kChain values of a channel)
    const int64_t n = std::max(std::clamp<int64_t>(want, 1, room),
                               cdiv(nv, bwd ? (int64_t)a.A * kChain : (int64_t)1 << 26));
    a.v1 = rup(cdiv(nv, n), a.A);
    a.n1 = (int)cdiv(nv, a.v1);
    a.n = a.nc = a.n1;
    a.collapse = (int64_t)a.n * a.G > 2048;
    p.units = a.B * a.n1;
    return p;
  }
  p.route = WIDE;
  p.vec = a.C % V == 0 ? V : 1;
  a.nt = p.vec == V;
  a.cols = (int)cdiv(a.C, (int64_t)NT * p.vec);
  const int64_t want = std::max<int64_t>(1, kFill / (a.B * a.cols));
  a.rows = cdiv(a.P, std::min(want, std::max<int64_t>(1, a.P / 8)));
  a.n1 = (int)cdiv(a.P, a.rows);
  a.n = a.Cg * a.n1;
  a.nc = a.n1;
  a.collapse = 1;
  p.units = a.B * a.n1 * a.cols;
  return p;
}

// Workspace: the groups' partial and joined sums, the channels' sums.
struct WsLayout {
  int64_t joined, chan, bytes;
};
WsLayout ws_of(const NormPlan& p, bool bwd) {
  const NormArgs& a = p.a;
  WsLayout w;
  w.joined = rup(std::max<int64_t>(1, a.B * a.G * a.n) * (int64_t)sizeof(Sums), 256);
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
  a.u1 = a.B * a.G;
  if (a.n <= 256) hipLaunchKernelGGL(join_kernel<64>, dim3(grid_of(cdiv(a.u1, 4))), dim3(NT), 0, L.s, a);
  else hipLaunchKernelGGL(join_kernel<NT>, dim3(grid_of(a.u1)), dim3(NT), 0, L.s, a);
}

template <typename T>
void launch_stats(NormLaunch& L) {
  NormArgs& a = L.p.a;
  const int64_t units = a.u1 - a.u0;
  if (L.p.route == FLAT) {
    const size_t lds = (size_t)a.A * (L.p.uni ? 1 : kVec<T>) * sizeof(Sums);
    auto k = L.p.uni ? flat_stats_kernel<T, true> : flat_stats_kernel<T, false>;
    hipLaunchKernelGGL(k, dim3(grid_of(units)), dim3(NT), lds, L.s, a);
  } else if (L.p.route == WIDE) {
    auto k = L.p.vec == 1 ? wide_stats_kernel<T, 1> : wide_stats_kernel<T, kVec<T>>;
    hipLaunchKernelGGL(k, dim3(grid_of(units)), dim3(NT), 0, L.s, a);
  } else {
    auto k = L.p.team == 64 ? first_stats_kernel<T, 64> : first_stats_kernel<T, NT>;
    hipLaunchKernelGGL(k, dim3(grid_of(cdiv(units, NT / L.p.team))), dim3(NT), 0, L.s, a);
  }
}

template <typename T, int ACT>
void launch_fwd2(NormLaunch& L) {
  NormArgs& a = L.p.a;
  const int64_t units = a.u1 - a.u0;
  if (L.p.route == FLAT) {
    auto k = L.p.uni ? flat_fwd_kernel<T, ACT, kUni> : a.nt ? flat_fwd_kernel<T, ACT, kAligned> : flat_fwd_kernel<T, ACT, kAny>;
    hipLaunchKernelGGL(k, dim3(grid_of(units)), dim3(NT), a.G * sizeof(Stat), L.s, a);
  } else if (L.p.route == WIDE) {
    auto k = L.p.vec == 1 ? wide_fwd_kernel<T, 1> : wide_fwd_kernel<T, kVec<T>>;
    hipLaunchKernelGGL(k, dim3(grid_of(units)), dim3(NT), 0, L.s, a);
  } else {
    auto k = L.p.team == 64 ? first_fwd_kernel<T, 64, ACT> : first_fwd_kernel<T, NT, ACT>;
    hipLaunchKernelGGL(k, dim3(grid_of(cdiv(units, NT / L.p.team))), dim3(NT), 0, L.s, a);
  }
}

template <typename T, int ACT>
void launch_sums(NormLaunch& L) {
  NormArgs& a = L.p.a;
  const int64_t units = a.u1 - a.u0;
  if (L.p.route == FLAT) {
    const size_t lds = (size_t)NT * kVec<T> * sizeof(float2) + a.C * sizeof(Sums);
    auto k = L.p.uni ? flat_sums_kernel<T, ACT, true> : flat_sums_kernel<T, ACT, false>;
    hipLaunchKernelGGL(k, dim3(grid_of(units)), dim3(NT), lds, L.s, a);
  } else if (L.p.route == WIDE) {
    auto k = L.p.vec == 1 ? wide_sums_kernel<T, 1> : wide_sums_kernel<T, kVec<T>>;
    hipLaunchKernelGGL(k, dim3(grid_of(units)), dim3(NT), 0, L.s, a);
  } else {
    auto k = L.p.team == 64 ? first_sums_kernel<T, 64, ACT> : first_sums_kernel<T, NT, ACT>;
    hipLaunchKernelGGL(k, dim3(grid_of(cdiv(units, NT / L.p.team))), dim3(NT), 0, L.s, a);
  }
}

// extra: work-groups beyond the slab's for the parameter gradients
template <typename T, int ACT>
void launch_bwd2(NormLaunch& L, int extra) {
  NormArgs& a = L.p.a;
  const int64_t units = a.u1 - a.u0;
  if (L.p.route == FLAT) {
    a.main = (int)grid_of(units);
    auto k = L.p.uni ? flat_bwd_kernel<T, ACT, kUni> : a.nt ? flat_bwd_kernel<T, ACT, kAligned> : flat_bwd_kernel<T, ACT, kAny>;
    hipLaunchKernelGGL(k, dim3(a.main + extra), dim3(NT), a.G * sizeof(Stat), L.s, a);
  } else if (L.p.route == WIDE) {
    a.main = (int)grid_of(units);
    auto k = L.p.vec == 1 ? wide_bwd_kernel<T, 1> : wide_bwd_kernel<T, kVec<T>>;
    hipLaunchKernelGGL(k, dim3(a.main + extra), dim3(NT), 0, L.s, a);
  } else {
    a.main = (int)grid_of(cdiv(units, NT / L.p.team));
    auto k = L.p.team == 64 ? first_bwd_kernel<T, 64, ACT> : first_bwd_kernel<T, NT, ACT>;
    hipLaunchKernelGGL(k, dim3(a.main + extra), dim3(NT), 0, L.s, a);
  }
}

template <typename T, int ACT>
void launch_both(NormLaunch& L, bool bwd) {
  NormArgs& a = L.p.a;
  a.u0 = 0;
  a.u1 = L.p.units;
  bwd ? launch_sums<T, ACT>(L) : launch_stats<T>(L);
  launch_join(L);
  a.u1 = L.p.units;
  if (bwd) launch_bwd2<T, ACT>(L, a.ggamma || a.gbeta ? a.C : 0);
  else launch_fwd2<T, ACT>(L);
}

template <typename T>
hipError_t by_act(NormLaunch& L, bool bwd) {
  switch (L.p.a.act) {
    case FNO_NORM_ACT_GELU: launch_both<T, FNO_NORM_ACT_GELU>(L, bwd); break;
    case FNO_NORM_ACT_SILU: launch_both<T, FNO_NORM_ACT_SILU>(L, bwd); break;
    default: launch_both<T, FNO_NORM_ACT_NONE>(L, bwd);
  }
  return hipGetLastError();
}

hipError_t by_type(NormLaunch& L, bool bwd) {
  if (L.p.route == RESIDENT) return norm_resident_launch(L.p.a, L.dt, L.p.first, bwd, L.s);
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
  *bytes = (size_t)ws_of(plan_of(*d, op == FNO_OP_BWD), op == FNO_OP_BWD).bytes;
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
  NormLaunch L{plan_of(*d, false), d->dtype, stream};
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
  NormLaunch L{plan_of(*d, true), d->dtype, stream};
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
