// What the kernels of the group norm share: vectors, activations, sums, the
// per-channel coefficients and the streams of loads (device code), and the
// launches of the kernels that keep a group on chip.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/fno_spectral_conv.h"
#include "fno_act.h"

namespace fno {

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
// The same where the call reads them for the last time: past the memory-side
// cache, which keeps what is still to be read.
template <typename T, int W>
__device__ __forceinline__ Vec<T, W> load_last(const T* p) {
  if constexpr (sizeof(Vec<T, W>) == 16) {
    typedef uint32_t U4 __attribute__((ext_vector_type(4), aligned(2)));
    return __builtin_bit_cast(Vec<T, W>, __builtin_nontemporal_load(reinterpret_cast<const U4*>(p)));
  }
  return load_vec<T, W>(p);
}
template <typename T, int W>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, W>& v) {
  __builtin_memcpy(__builtin_assume_aligned(p, sizeof(T)), &v, sizeof(v));
}
// A result that the call does not read again: past the memory-side cache where
// pieces are 16-byte aligned (`nt`), so that it does not push out what the
// second pass is about to read (33.5 M fp16 elements channels last: forward 44
// -> 38 us, as many fp32 76 -> 67).  Unaligned pieces are parts of memory's
// own pieces and better joined in the cache (241^2 with 20 channels, backward:
// 50 us, 55 past it).
template <typename T, int W>
__device__ __forceinline__ void store_result(T* p, const Vec<T, W>& v, int nt) {
  typedef uint32_t U4 __attribute__((ext_vector_type(4)));
  if constexpr (sizeof(v) == 16) {
    if (nt) {
      __builtin_nontemporal_store(__builtin_bit_cast(U4, v), reinterpret_cast<U4*>(p));
      return;
    }
  }
  store_vec<T, W>(p, v);
}

// --------------------------------------------------------------------------
// Activations
// --------------------------------------------------------------------------
// GELU of 16-bit tensors: z Phi(z) = max(z, 0) - |z| erfc(|z| / sqrt 2) / 2, with
// half of erfc by Abramowitz & Stegun 7.1.26 (absolute error at most 0.75e-7).
// inf for inf, NaN for -inf (-inf times 0), as the definition has it.
__device__ __forceinline__ float gelu_of(float z) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(z), 0.23164189f, 1.0f));
  float p = __builtin_fmaf(t, 0.5307027145f, -0.7265760135f);
  p = __builtin_fmaf(t, p, 0.7107068705f);
  p = __builtin_fmaf(t, p, -0.142248368f);
  p = __builtin_fmaf(t, p, 0.127414796f);
  const float e = __builtin_amdgcn_exp2f(z * (z * -0.72134752044448f));
  return __builtin_fmaf(-__builtin_fabsf(__builtin_fminf(z, 3.402823466e+38f)), p * t * e, __builtin_fmaxf(z, 0.0f));
}
// Its derivative Phi(z) + z phi(z) as 1/2 + z P(z^2) / Q(z^2) for |z| <= 5.6,
// constant beyond: a rational fit of degrees (5, 5) to the definition (least
// squares, reweighted to near the minimax of 1.1e-7), within 3.3e-7 of it
// everywhere in float.  One reciprocal and no exponential: 18 operations' time
// against 22 through erfc and exp(-z^2 / 2), where the passes are bound by it.
__device__ __forceinline__ float gelu_grad_of(float z) {
  const float c = __builtin_amdgcn_fmed3f(z, -5.6f, 5.6f), t = c * c;
  float p = __builtin_fmaf(t, 1.921672664e-07f, 3.589928644e-05f);
  p = __builtin_fmaf(t, p, 1.975132363e-05f);
  p = __builtin_fmaf(t, p, 1.422606847e-02f);
  p = __builtin_fmaf(t, p, -3.097535923e-02f);
  p = __builtin_fmaf(t, p, 7.978853454e-01f);
  float q = __builtin_fmaf(t, 8.928170334e-06f, 1.920517995e-04f);
  q = __builtin_fmaf(t, q, 3.522637464e-03f);
  q = __builtin_fmaf(t, q, 4.098374084e-02f);
  q = __builtin_fmaf(t, q, 2.945195774e-01f);
  q = __builtin_fmaf(t, q, 1.0f);
  return __builtin_fmaf(c * p, __builtin_amdgcn_rcpf(q), 0.5f);
}

// GELU of fp32 tensors, as exact as the type: below 1.5 in size Phi(z) - 1/2 = z
// A(z^2), beyond it the tail E = erfc(|z| / sqrt 2) / 2 = t P(t) exp(-z^2 / 2) with
// t = 1 / (1 + 0.3375 |z|).  A of degree 6 (relative error 2.7e-9) and P of degree
// 5 (1.9e-7, up to |z| = 14) fit the definition (least squares, reweighted to
// near the minimax).  On normally distributed z both results are within 4.2e-8
// of the definition in the 2-norm, the forms above within 8.3e-8 and 1.24e-7; fp32
// calls take 1% (planes of 1024^2) to 4% (backward of 16 x 241^2 x 20) longer.
struct Gelu32 {
  float half, tail, e;  // A(z^2), E, exp(-z^2 / 2)
  bool near;
};
__device__ __forceinline__ Gelu32 gelu32_terms(float z) {
  const float u = z * z, a = __builtin_fabsf(z);
  float h = __builtin_fmaf(u, 4.1155591e-07f, -8.71830338e-06f);
  h = __builtin_fmaf(u, h, 1.14356388e-04f);
  h = __builtin_fmaf(u, h, -1.18648849e-03f);
  h = __builtin_fmaf(u, h, 9.97324131e-03f);
  h = __builtin_fmaf(u, h, -6.6490335e-02f);
  h = __builtin_fmaf(u, h, 3.98942279e-01f);
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(a, 0.3375f, 1.0f));
  float p = __builtin_fmaf(t, -7.27348701e-02f, 1.19748334e-01f);
  p = __builtin_fmaf(t, p, 5.71845018e-02f);
  p = __builtin_fmaf(t, p, 1.26757348e-01f);
  p = __builtin_fmaf(t, p, 1.33728535e-01f);
  p = __builtin_fmaf(t, p, 1.3468849e-01f);
  const float e = __builtin_amdgcn_exp2f(z * (z * -0.72134752044448f));
  return Gelu32{h, p * t * e, e, a < 1.5f};
}
__device__ __forceinline__ float gelu32_of(float z) {
  const Gelu32 g = gelu32_terms(z);
  const float far = __builtin_fmaf(-__builtin_fabsf(__builtin_fminf(z, 3.402823466e+38f)), g.tail, __builtin_fmaxf(z, 0.0f));
  return g.near ? __builtin_fmaf(z * z, g.half, 0.5f * z) : far;
}
// Phi(z) + z phi(z)
__device__ __forceinline__ float gelu32_grad_of(float z) {
  const Gelu32 g = gelu32_terms(z);
  const float far = z >= 0.0f ? 1.0f - g.tail : g.tail;
  return __builtin_fmaf(z * 0.39894228040143268f, g.e, g.near ? __builtin_fmaf(z, g.half, 0.5f) : far);
}

// Of z formed from values of type T.
template <typename T>
__device__ __forceinline__ float act_any(float z, int act) {
  if (act == FNO_NORM_ACT_GELU) return sizeof(T) == 4 ? gelu32_of(z) : gelu_of(z);
  return act == FNO_NORM_ACT_SILU ? silu_f(z) : z;
}
template <typename T>
__device__ __forceinline__ float act_grad_any(float z, int act) {
  if (act == FNO_NORM_ACT_GELU) return sizeof(T) == 4 ? gelu32_grad_of(z) : gelu_grad_of(z);
  return act == FNO_NORM_ACT_SILU ? silu_grad_f(z) : 1.0f;
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
  int nt;                // every vector of the tensors is 16-byte aligned
  int act;
  float eps;
  // flat: L, A as above; vectors of a chunk (a multiple of A), chunks of a sample
  int L, A, n1;
  int64_t v1;
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
// to put(g, sum) by one thread; all threads of the work-group take part.  Two
// wait states behind a put, which may end in a 16-byte store and a branch: its
// data registers are not written sooner, wherever the branch leads.
template <int THREADS = NT, typename Entry, typename Put>
__device__ __forceinline__ void group_sums(int groups, int n, Entry entry, Put put) {
  __shared__ Sums red[THREADS / 64];
  if (groups > 4) {
    // a power of two of threads (at most a wave) per group
    int sub = 1;
    while (sub < 64 && sub * 2 * groups <= THREADS) sub *= 2;
    const int s = threadIdx.x & (sub - 1);
    for (int g0 = 0; g0 < groups; g0 += THREADS / sub) {
      const int g = g0 + (int)threadIdx.x / sub;
      Sums v{0.0, 0.0};
      if (g < groups)
        for (int i = s; i < n; i += sub) v = add(v, entry(g, i));
      for (int d = sub / 2; d > 0; d >>= 1) v = add(v, Sums{__shfl_xor(v.s, d), __shfl_xor(v.q, d)});
      if (g < groups && s == 0) {
        put(g, v);
        asm volatile("s_nop 1" ::: "memory");
      }
    }
    return;
  }
  for (int g = 0; g < groups; ++g) {
    Sums v{0.0, 0.0};
    for (int i = threadIdx.x; i < n; i += THREADS) v = add(v, entry(g, i));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = add(v, Sums{__shfl_xor(v.s, d), __shfl_xor(v.q, d)});
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
      for (int w = 1; w < THREADS / 64; ++w) red[0] = add(red[0], red[w]);
      put(g, red[0]);
    }
  }
}

// x and x^2 added in double: the variance loses (mean / sigma)^2 2^-53 of itself,
// however far a group's mean or a few of its values lie from the rest, and the
// unit's double additions run at the rate of float ones.
__device__ __forceinline__ void add_value(Sums* t, float x) {
  const double d = (double)x;
  t->s += d;
  t->q = __builtin_fma(d, d, t->q);
}

// A thread's items 0 .. count - 1, loaded ahead of their use: the first UN when
// the stream is made (before what the use needs is worked out), then the next
// UN while UN are used.  The loads stand outside every condition but that there
// are items; inside one the compiler moves them next to their use.  An item is
// loaded before any item from it on is used, so results may overwrite what was
// loaded.
template <int UN, typename Load>
struct Stream {
  int count;
  Load load;
  decltype(load(0)) cur[UN];
  __device__ __forceinline__ Stream(int n, Load l) : count(n), load(l) {
    if (count > 0)
#pragma unroll
      for (int u = 0; u < UN; ++u) cur[u] = load(u < count ? u : count - 1);
  }
  // use(item k, k) for each
  template <typename Use>
  __device__ __forceinline__ void run(Use use) {
    if (count <= 0) return;
    decltype(load(0)) next[UN];
    int k = 0;
#pragma unroll 2
    for (; k + UN <= count; k += UN) {
#pragma unroll
      for (int u = 0; u < UN; ++u) next[u] = load(k + UN + u < count ? k + UN + u : count - 1);
#pragma unroll
      for (int u = 0; u < UN; ++u) use(cur[u], k + u);
#pragma unroll
      for (int u = 0; u < UN; ++u) cur[u] = next[u];
    }
#pragma unroll
    for (int u = 0; u < UN - 1; ++u)
      if (k + u < count) use(cur[u], k + u);
  }
};
template <int UN, typename Load>
__device__ __forceinline__ Stream<UN, Load> stream(int count, Load load) {
  return Stream<UN, Load>(count, load);
}

// Vectors of x and of a second tensor.
template <typename T, int W>
struct Pair {
  Vec<T, W> x, y;
};

// x - mu.  The factor is one; it is hidden from the compiler so that the fp16
// conversion folds into the multiply-add.
__device__ __forceinline__ float less(float x, float mu) { return x - mu; }
__device__ __forceinline__ float less(_Float16 x, float mu) {
  float one = 1.0f;
  asm("" : "+s"(one));
  return __builtin_fmaf((float)x, one, -mu);
}
__device__ __forceinline__ float less(__bf16 x, float mu) { return (float)x - mu; }

// z = (x - mu) k + beta, k = r gamma.  (Not x k + (beta - mu k): where a
// group's spread is nothing beside its mean, that has mu k 2^-24 of error.)
struct Line {
  float mu, k, be;
};
__device__ __forceinline__ Line line_of(const NormArgs& a, const Stat& st, int c) {
  return Line{st.mean, a.gamma ? st.rstd * a.gamma[c] : st.rstd, a.beta ? a.beta[c] : 0.0f};
}
template <typename T>
__device__ __forceinline__ float on_line(const Line& l, T x) {
  return __builtin_fmaf(less(x, l.mu), l.k, l.be);
}

__device__ __forceinline__ void write_stat(const NormArgs& a, int64_t bg, const Stat& st) {
  a.stats[2 * bg] = st.mean;
  a.stats[2 * bg + 1] = st.rstd;
}

// What the backward needs of a channel: d = (x - mu) s, z = d k + beta with
// k = (r / s) gamma; h = g_out act'(z); the sums of h and of h d, r / s put to
// it at the end; gx = r (gamma h - a - xh m), m the group's mean of gamma h xh.
// s is the power of two below r, so that d, k and the sums are of the size of
// xh and gamma at any spread (with x - mu itself r^2 would come in, which leaves
// fp32 at spreads of 1e19 and, with eps 0, of 1e-19), and x s - mu s is one
// operation, rounded like x - mu.  An fp16 group's spread lies between 1e-13 and
// 1e5, which squared stay inside: s = 1.
template <typename T>
constexpr bool kNarrow = false;
template <>
inline constexpr bool kNarrow<_Float16> = true;

struct Coef {
  float mu, s;    // mu times s
  float rs, rel;  // r, r / s
  float k, ga, be;
};
template <typename T>
__device__ __forceinline__ Coef bwd_coef(const NormArgs& a, int64_t bg, int c) {
  const float mu = a.stats_in[2 * bg], rs = a.stats_in[2 * bg + 1];
  // (of an r below the normal numbers: the smallest of these; and mu s below 2^126,
  // where values that hardly differ are as large as the type has them)
  const uint32_t mask = 0x7f800000u, top = (379u << 23) - (__float_as_uint(mu) & mask);
  const float s = kNarrow<T> ? 1.0f : __uint_as_float(min(max(__float_as_uint(rs) & mask, 0x00800000u), top));
  const float rel = kNarrow<T> ? rs : rs / s;
  const float ga = a.gamma ? a.gamma[c] : 1.0f;
  return Coef{mu * s, s, rs, rel, rel * ga, ga, a.beta ? a.beta[c] : 0.0f};
}
template <typename T>
__device__ __forceinline__ float distance(const Coef& k, T x) {
  return kNarrow<T> ? less(x, k.mu) : __builtin_fmaf((float)x, k.s, -k.mu);
}
// (Both passes form h alike: in a group whose values hardly differ gx is the
// small difference of large terms, and would show any difference of the two.)
template <int ACT, typename T>
__device__ __forceinline__ void bwd_terms(const Coef& k, T x, T g, float* h, float* d) {
  *d = distance(k, x);
  *h = (float)g * act_grad_any<T>(__builtin_fmaf(*d, k.k, k.be), ACT);
}
// The sums of h and h xh.  Where the statistics are not finite, or behind an
// activation gamma or beta, they are not numbers: h itself may be finite there
// (the derivative of GELU is, for any z), and so would gx be.
__device__ __forceinline__ float bad_of(const Coef& k, int act) {
  const float bad = 0.0f * k.rel;
  return act == FNO_NORM_ACT_NONE ? bad : __builtin_fmaf(0.0f, k.k, __builtin_fmaf(0.0f, k.be, bad));
}
__device__ __forceinline__ float2 bwd_sums(const Coef& k, int act, float s, float q) {
  const float bad = bad_of(k, act);
  return make_float2(s + bad, __builtin_fmaf(q, k.rel, bad));
}
__device__ __forceinline__ Sums bwd_sums(const Coef& k, int act, const Sums& t) {
  const float bad = bad_of(k, act);
  return Sums{t.s + bad, __builtin_fma(t.q, (double)k.rel, (double)bad)};
}
// A thread adds h and h d in fp32, at most this many of a channel before it goes
// on in double: terms of one sign lose 2e-6 of their sum in 128 additions, 1.5e-5
// in 1024, 2.3e-4 in 16384.  (Held groups have 32; work items of the flat layout
// are cut to it.)
constexpr int kChain = 128;
// gx = r gamma h + c1 d + c0.
struct Means {
  float a, d;
};
struct Gx {
  float c0, c1, k;
};
__device__ __forceinline__ Gx gx_coef(const Coef& k, const Means& m) {
  return Gx{-k.rs * m.a, -(k.rs * m.d) * k.rel, k.rs * k.ga};
}
__device__ __forceinline__ float bwd_gx(const Gx& m, float h, float d) {
  return __builtin_fmaf(m.k, h, __builtin_fmaf(d, m.c1, m.c0));
}
__device__ __forceinline__ Means means_of(const NormArgs& a, const Sums& t) {
  const double m = (double)a.P * a.Cg;
  return Means{(float)(t.s / m), (float)(t.q / m)};
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

// Group norm with each group held by one work-group (fno_norm_res.hip).  fits:
// whether the kernels take this shape in this direction; launch: the whole call
// (forward with bwd false), `dtype` the tensors' fno_dtype.
bool norm_resident_fits(const NormArgs& a, int dtype, bool first, bool bwd);
hipError_t norm_resident_launch(const NormArgs& a, int dtype, bool first, bool bwd, hipStream_t s);

}  // namespace fno
