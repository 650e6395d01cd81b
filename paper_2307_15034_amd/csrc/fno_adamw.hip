// The optimizer step over many tensors at once (AdamW, states in 32 or 8
// bits) and the global gradient norm that steers it on the device.
//
// A launch takes a batch of tensors by value in its kernel arguments (no
// table to upload, nothing kept between calls): each work-group finds its
// tensor by a search over the batch's first-chunk numbers and works on one
// chunk of it.  The kernels stream every operand once; they are bound by HBM
// (67 M fp16 weights with masters: step 300 us, 6.7 TB/s, norm 46, 5.8; with
// 8-bit states 228 to 251, 4.9 to 5.4; read-out 59, 6.9; 268 M fp32 weights with
// 8-bit states 762 to 789, 5.5 to 5.7, read-out 265 to 287, 5.7 to 6.2), small lists by the latency of a chain of loads
// (5 us a step, 6 to 7 the norm).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/fno_spectral_conv.h"
#include "fno_host.h"

namespace fno {
namespace {

constexpr int kBatch = FNO_ADAMW_LAUNCH_TENSORS;
constexpr int kNormBatch = 128;              // tensors of a launch of the norm
constexpr int kBlk = FNO_ADAMW_BLOCK;
constexpr int64_t kPiece = 1024;             // elements that a work-group of the step loads at once:
                                             // a block of the 8-bit states per wave
constexpr int64_t kNormChunk = 8192;         // elements of a work-group of the norm
constexpr int64_t kMomentChunk = 4096;       // elements of a work-group that reads moments out
constexpr int64_t kMaxN = (int64_t)1 << 34;  // elements of a tensor
constexpr int64_t kMaxGrid = (int64_t)1 << 23;  // work-groups of a launch

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct AdamTensor {
  void* p;
  float* master;
  const void* g;
  void *m, *v;
  float *ms, *vs;
  int64_t n;
  int32_t pdt, gdt, bits;
  float wd;
};

struct AdamArgs {
  AdamTensor t[kBatch];
  int32_t first[kBatch + 1];  // first chunk of tensor i; first[count]: all chunks
  int32_t count;
};

struct AdamHyper {
  double lr, b1, b2, bias1, bias2;  // bias1 = 1 / (1 - b1^t), bias2 = 1 / sqrt(1 - b2^t)
  float eps;
};

// x^t by repeated squaring, the same on the host and on the device.
__host__ __device__ inline double int_pow(double x, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1) {
    if (t & 1) r *= x;
    x *= x;
  }
  return r;
}

typedef float f4 __attribute__((ext_vector_type(4)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef int8_t c4 __attribute__((ext_vector_type(4)));
typedef uint8_t u4 __attribute__((ext_vector_type(4)));
template <typename T>
struct Vec4;
template <>
struct Vec4<float> {
  typedef f4 type;
};
template <>
struct Vec4<_Float16> {
  typedef h4 type;
};
template <>
struct Vec4<__bf16> {
  typedef b4 type;
};

// Elements e .. e + 4 of an array of n (e a multiple of four): in one access
// where all four are there, one by one at the tensor's end (others read as 0).
template <typename V, typename T>
__device__ __forceinline__ V load4(const T* p, int64_t e, int64_t n) {
  if (e + 4 <= n) return *reinterpret_cast<const V*>(p + e);
  V v = {};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (e + j < n) v[j] = p[e + j];
  return v;
}

// An fp32 result rounded to the storage type: two roundings, as stated.  (The
// compiler otherwise folds a last product or sum and its conversion to fp16
// into one instruction with one rounding.)
template <typename T>
__device__ __forceinline__ T rounded(float x) {
  asm("" : "+v"(x));
  return (T)x;
}

// The tensor of chunk c: the last i with first[i] <= c.  Every lane looks at an
// entry (of N <= 128: at two), all in one or two loads.
template <int N>
__device__ __forceinline__ int find_tensor(const int32_t (&first)[N], int count, int c) {
  static_assert(N <= 129, "two entries per lane");
  const int lane = threadIdx.x & 63, last = count - 1;
  int i = __builtin_popcountll(__ballot(lane <= last && first[lane <= last ? lane : last] <= c));
  if (N > 65) {
    const int l2 = lane + 64;
    i += __builtin_popcountll(__ballot(l2 <= last && first[l2 <= last ? l2 : last] <= c));
  }
  return i - 1;
}

struct Consts {  // an element's step in floats
  float b1, c1, b2, c2, size, root, eps, gs, keep;
};

// One element's step; every operation rounded by itself (no contraction), so
// that the codes of 8-bit states do not depend on the compiler's choices.
__device__ inline float adam_element(const Consts& k, float p, float g, float* m, float* v, float* w) {
#pragma clang fp contract(off)
  g = g * k.gs;
  *m = *m * k.b1 + g * k.c1;
  *v = *v * k.b2 + (g * g) * k.c2;
  *w = __builtin_sqrtf(*v);
  return p * k.keep - (*m * k.size) / (*w * k.root + k.eps);
}

__device__ __forceinline__ Consts consts_of(const AdamHyper& h, const fno_adamw_control* ctl, float wd) {
  const double lr = ctl ? h.lr * (double)ctl->lr_factor : h.lr;
  Consts k;
  k.b1 = (float)h.b1;
  k.c1 = (float)(1.0 - h.b1);
  k.b2 = (float)h.b2;
  k.c2 = (float)(1.0 - h.b2);
  k.size = (float)(lr * (ctl ? ctl->bias1 : h.bias1));
  k.root = (float)(ctl ? ctl->bias2 : h.bias2);
  k.eps = h.eps;
  k.gs = ctl ? ctl->grad_scale : 1.0f;
  k.keep = (float)(1.0 - lr * (double)wd);
  return k;
}

// |x| as its bits: ordered like the values, with inf and then NaN on top.
__device__ inline uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

__device__ inline uint32_t wave_max(uint32_t x) {
  for (int d = 1; d < 64; d <<= 1) x = max(x, (uint32_t)__shfl_xor((int)x, d));
  return x;
}

__device__ inline float decode_m(float a, int q) {
#pragma clang fp contract(off)
  return (a * (1.0f / 16129.0f)) * (float)(q * (q < 0 ? -q : q));
}
__device__ inline float decode_v(float b, int q) {
#pragma clang fp contract(off)
  const float s = (b * (1.0f / 65025.0f)) * (float)(q * q);
  return s * s;
}
// Elements of an array of any type as floats, all loads before the first use.
template <int N>
__device__ __forceinline__ void load_any(const void* p, int dt, const uint32_t (&at)[N], float (&x)[N]) {
  uint32_t raw[N];
  if (dt == FNO_DTYPE_F32) {
#pragma unroll
    for (int j = 0; j < N; ++j) raw[j] = static_cast<const uint32_t*>(p)[at[j]];
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) raw[j] = static_cast<const uint16_t*>(p)[at[j]];
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    x[j] = dt == FNO_DTYPE_F32   ? __uint_as_float(raw[j])
           : dt == FNO_DTYPE_F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)raw[j])
                                 : __uint_as_float(raw[j] << 16);
}

// A code with its moment's sign; a second moment's, at least 1 where w > 0.
// (Blocks that hold a value that is not finite: some code within the range.)
__device__ __forceinline__ int8_t signed_code(float q, float m) {
  const int c = (int)__builtin_fminf(q, 127.0f);
  return (int8_t)(m < 0.0f ? -c : c);
}
__device__ __forceinline__ uint8_t unsigned_code(float q, float w) {
  return (uint8_t)(int)__builtin_fminf(__builtin_fmaxf(q, w > 0.0f ? 1.0f : 0.0f), 255.0f);
}

// rint(levels sqrt(x / top)), quotient, root and product rounded to fp32:
// the code of the fraction x / top; a top that is 0 or not a number gives
// some code (0 for 0; the scale then tells).
__device__ __forceinline__ float code_exact(float x, float top, float levels) {
#pragma clang fp contract(off)
  return rintf(__builtin_sqrtf(x / (top > 0.0f ? top : 1.0f)) * levels);
}

// The codes of four fractions.  A reciprocal of the block's top and the
// hardware's root are within 3.5 x 2^-23 of the rounded quotient's root, so
// the product with at most 255 levels is within 2^-13 of the exact one, and
// the nearest integer is the same unless a half lies that near.  Where one of
// the wave's values is (about one wave in nine), all take the divisions and
// rounded roots.  (These cost 60 operations an element for both moments: the
// step of 268 M fp32 parameters, then 827 us, took 987 with them everywhere.)
__device__ __forceinline__ void codes4(const f4& x, float top, float levels, f4* q) {
  const float r = __builtin_amdgcn_rcpf(top > 0.0f ? top : 1.0f);
  bool near = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float z = __builtin_amdgcn_sqrtf(x[j] * r) * levels;
    (*q)[j] = __builtin_rintf(z);
    near |= !(__builtin_fabsf(z - (*q)[j]) < 0.5f - 0x1p-13f);
  }
  if (__any(near)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) (*q)[j] = code_exact(x[j], top, levels);
  }
}

// Large lists (U 2) go past the memory-side cache both ways: each operand is
// read and written once, and through the cache the written lines would be
// pushed out by later reads (67 M fp16 weights with masters, clipped: 436 us
// through it, 430 with the results stored past it, 348 with the loads as well;
// 268 M fp32 weights with 8-bit states, step and read-out: 1093, 1107 and,
// with the parameters stored past it too, 1075).  Small lists stay in it from
// one step to the next.
template <int U, typename V>
__device__ __forceinline__ void put_result(V* p, const V& v) {
  if (U == 1) *p = v;
  else __builtin_nontemporal_store(v, p);
}
template <int U, typename V>
__device__ __forceinline__ V get_once(const V* p) {
  if (U == 1) return *p;
  return __builtin_nontemporal_load(p);
}

// A chunk that lies inside its tensor: each thread takes four consecutive
// elements at a time, so that a wave covers 256, a block of the 8-bit states;
// all loads of the chunk are in flight before the first element's step.
template <typename P, typename G, bool MASTER, int BITS, int U>
__device__ __forceinline__ void full_chunk(const AdamTensor& t, int64_t base, const Consts& k) {
  using PV = typename Vec4<P>::type;
  using GV = typename Vec4<G>::type;
  const int64_t e0 = base + 4 * threadIdx.x;
  P* pp = static_cast<P*>(t.p) + e0;
  const G* gp = static_cast<const G*>(t.g) + e0;
  float* master = t.master + e0;
  float *m32 = static_cast<float*>(t.m) + e0, *v32 = static_cast<float*>(t.v) + e0;
  int8_t* m8 = static_cast<int8_t*>(t.m) + e0;
  uint8_t* v8 = static_cast<uint8_t*>(t.v) + e0;
  const int64_t b0 = __builtin_amdgcn_readfirstlane((int)(e0 / kBlk));
  f4 pm[U], m[U], v[U];
  PV pl[U];
  GV g[U];
  c4 qm[U];
  u4 qv[U];
  float as[U], bs[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (MASTER) pm[u] = get_once<U>(reinterpret_cast<const f4*>(master + 1024 * u));
    else pl[u] = get_once<U>(reinterpret_cast<const PV*>(pp + 1024 * u));
    g[u] = get_once<U>(reinterpret_cast<const GV*>(gp + 1024 * u));
    if (BITS == 32) {
      m[u] = get_once<U>(reinterpret_cast<const f4*>(m32 + 1024 * u));
      v[u] = get_once<U>(reinterpret_cast<const f4*>(v32 + 1024 * u));
    } else {
      qm[u] = get_once<U>(reinterpret_cast<const c4*>(m8 + 1024 * u));
      qv[u] = get_once<U>(reinterpret_cast<const u4*>(v8 + 1024 * u));
      as[u] = t.ms[b0 + 4 * u];
      bs[u] = t.vs[b0 + 4 * u];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    f4 p, w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (BITS == 8) {
        m[u][j] = decode_m(as[u], qm[u][j]);
        v[u][j] = decode_v(bs[u], qv[u][j]);
      }
      float mj = m[u][j], vj = v[u][j], wj;
      p[j] = adam_element(k, MASTER ? pm[u][j] : (float)pl[u][j], (float)g[u][j], &mj, &vj, &wj);
      m[u][j] = mj;
      v[u][j] = vj;
      w[j] = wj;
    }
    if (MASTER) put_result<U>(reinterpret_cast<f4*>(master + 1024 * u), p);
    PV pr;
#pragma unroll
    for (int j = 0; j < 4; ++j) pr[j] = rounded<P>(p[j]);
    put_result<U>(reinterpret_cast<PV*>(pp + 1024 * u), pr);
    if (BITS == 32) {
      put_result<U>(reinterpret_cast<f4*>(m32 + 1024 * u), m[u]);
      put_result<U>(reinterpret_cast<f4*>(v32 + 1024 * u), v[u]);
    } else {
      f4 am, cm, cv;
      uint32_t ma = 0, mb = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        am[j] = __builtin_fabsf(m[u][j]);
        ma = max(ma, abs_bits(m[u][j]));
        mb = max(mb, abs_bits(w[j]));
      }
      const float A = __uint_as_float(wave_max(ma)), Bt = __uint_as_float(wave_max(mb));
      codes4(am, A, 127.0f, &cm);
      codes4(w, Bt, 255.0f, &cv);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        qm[u][j] = signed_code(cm[j], m[u][j]);
        qv[u][j] = unsigned_code(cv[j], w[j]);
      }
      put_result<U>(reinterpret_cast<c4*>(m8 + 1024 * u), qm[u]);
      put_result<U>(reinterpret_cast<u4*>(v8 + 1024 * u), qv[u]);
      if ((threadIdx.x & 63) == 0) {
        t.ms[b0 + 4 * u] = A;
        t.vs[b0 + 4 * u] = Bt;
      }
    }
  }
}

// The last piece of a tensor, of any types: elements lie across the lanes, 64 of
// a block at a time; loads past the end read the last element and are dropped,
// so that here too all of them are in flight at once.
template <int BITS>
__device__ __forceinline__ void last_piece(const AdamTensor& t, int64_t base, const Consts& k) {
  constexpr int N = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int left = (int)(t.n - base < kPiece ? t.n - base : kPiece);  // elements of the piece
  const int first = wave * kBlk + lane;
  float p[N], g[N], m[N], v[N];
  uint32_t at[N];  // from `base` on
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = first + 64 * i;
    at[i] = (uint32_t)(e < left ? e : left - 1);
  }
  const int ps = t.master || t.pdt == FNO_DTYPE_F32 ? 4 : 2, gs = t.gdt == FNO_DTYPE_F32 ? 4 : 2;
  load_any(static_cast<const char*>(t.master ? t.master : t.p) + base * ps, t.master ? FNO_DTYPE_F32 : t.pdt, at, p);
  load_any(static_cast<const char*>(t.g) + base * gs, t.gdt, at, g);
  float *m32 = static_cast<float*>(t.m) + base, *v32 = static_cast<float*>(t.v) + base;
  int8_t* m8 = static_cast<int8_t*>(t.m) + base;
  uint8_t* v8 = static_cast<uint8_t*>(t.v) + base;
  float *ms = t.ms + base / kBlk, *vs = t.vs + base / kBlk;
  if (BITS == 32) {
    load_any(m32, FNO_DTYPE_F32, at, m);
    load_any(v32, FNO_DTYPE_F32, at, v);
  } else {
    int qm[N], qv[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      qm[i] = m8[at[i]];
      qv[i] = v8[at[i]];
    }
    const float as = ms[at[0] / kBlk], bs = vs[at[0] / kBlk];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      m[i] = decode_m(as, qm[i]);
      v[i] = decode_v(bs, qv[i]);
    }
  }
  if (wave * kBlk >= left) return;  // the same for the wave's lanes
  uint32_t ma = 0, mb = 0;
  f4 am, wm;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float w;
    p[i] = adam_element(k, p[i], g[i], &m[i], &v[i], &w);
    am[i] = __builtin_fabsf(m[i]);
    wm[i] = w;
    if (first + 64 * i >= left) continue;
    ma = max(ma, abs_bits(m[i]));
    mb = max(mb, abs_bits(w));
    if (t.master) (t.master + base)[at[i]] = p[i];
    if (t.pdt == FNO_DTYPE_F32) (static_cast<float*>(t.p) + base)[at[i]] = p[i];
    else if (t.pdt == FNO_DTYPE_F16) (static_cast<_Float16*>(t.p) + base)[at[i]] = rounded<_Float16>(p[i]);
    else (static_cast<__bf16*>(t.p) + base)[at[i]] = rounded<__bf16>(p[i]);
    if (BITS == 32) {
      m32[at[i]] = m[i];
      v32[at[i]] = v[i];
    }
  }
  if (BITS == 32) return;
  const float A = __uint_as_float(wave_max(ma)), Bt = __uint_as_float(wave_max(mb));
  f4 cm, cv;
  codes4(am, A, 127.0f, &cm);
  codes4(wm, Bt, 255.0f, &cv);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (first + 64 * i >= left) continue;
    m8[at[i]] = signed_code(cm[i], m[i]);
    v8[at[i]] = unsigned_code(cv[i], wm[i]);
  }
  if (lane == 0) {
    ms[wave] = A;
    vs[wave] = Bt;
  }
}

template <typename P, typename G, bool MASTER, int U>
__device__ __forceinline__ void full_of(const AdamTensor& t, int64_t base, const Consts& k) {
  if (t.bits == 32) full_chunk<P, G, MASTER, 32, U>(t, base, k);
  else full_chunk<P, G, MASTER, 8, U>(t, base, k);
}

template <typename P, int U>
__device__ __forceinline__ void full_half(const AdamTensor& t, int64_t base, const Consts& k) {
  if (t.gdt == FNO_DTYPE_F32) {
    if (t.master) full_of<P, float, true, U>(t, base, k);
    else full_of<P, float, false, U>(t, base, k);
  } else {
    if (t.master) full_of<P, P, true, U>(t, base, k);
    else full_of<P, P, false, U>(t, base, k);
  }
}

// A work-group takes a chunk of U pieces.  Two per work-group stream a large
// list faster (67 M fp16 weights with masters, clipped: 3%), one keeps small
// lists' chains of loads short (24 tensors of 262 K elements in all: 10.9 us,
// 12.3 with two).
template <int U>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a, AdamHyper h,
                                                    const fno_adamw_control* ctl) {
  if (ctl && ctl->skip) return;
  // From the last chunk on: the gradient norm has just read the last gradients.
  const int blk = (int)gridDim.x - 1 - (int)blockIdx.x;
  const int i = find_tensor(a.first, a.count, blk);
  const AdamTensor& t = a.t[i];
  const int64_t base = (int64_t)(blk - a.first[i]) * (U * kPiece);
  const Consts k = consts_of(h, ctl, t.wd);
  if (base + U * kPiece > t.n) {
#pragma unroll 1
    for (int64_t b = base; b < base + U * kPiece && b < t.n; b += kPiece)
      if (t.bits == 32) last_piece<32>(t, b, k);
      else last_piece<8>(t, b, k);
  } else if (t.pdt == FNO_DTYPE_F32) {
    full_of<float, float, false, U>(t, base, k);
  } else if (t.pdt == FNO_DTYPE_F16) {
    full_half<_Float16, U>(t, base, k);
  } else {
    full_half<__bf16, U>(t, base, k);
  }
}

// 8-bit moments read out.
struct MomentArgs {
  AdamArgs a;
  void* mo[kBatch];
  void* vo[kBatch];
  int32_t dt;
};

// Eight elements of a thread at a time, so that a 16-bit result is stored in
// whole 16-byte pieces; all of a chunk's loads in flight at once.
template <typename T>
__device__ __forceinline__ void moments_chunk(const AdamTensor& t, int64_t base, T* mo, T* vo) {
  constexpr int U = (int)kMomentChunk / 2048;
  typedef T V __attribute__((ext_vector_type(8)));
  typedef int8_t C __attribute__((ext_vector_type(8)));
  typedef uint8_t D __attribute__((ext_vector_type(8)));
  const int8_t* pm = static_cast<const int8_t*>(t.m);
  const uint8_t* pv = static_cast<const uint8_t*>(t.v);
  if (base + kMomentChunk > t.n) {
    for (int64_t e = base + threadIdx.x; e < t.n; e += 256) {
      mo[e] = rounded<T>(decode_m(t.ms[e / kBlk], pm[e]));
      vo[e] = rounded<T>(decode_v(t.vs[e / kBlk], pv[e]));
    }
    return;
  }
  const int64_t e0 = base + 8 * threadIdx.x;
  C qm[U];
  D qv[U];
  float a[U], b[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    qm[u] = *reinterpret_cast<const C*>(pm + e0 + 2048 * u);
    qv[u] = *reinterpret_cast<const D*>(pv + e0 + 2048 * u);
    a[u] = t.ms[(e0 + 2048 * u) / kBlk];
    b[u] = t.vs[(e0 + 2048 * u) / kBlk];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    V m, v;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      m[j] = rounded<T>(decode_m(a[u], qm[u][j]));
      v[j] = rounded<T>(decode_v(b[u], qv[u][j]));
    }
    // past the memory-side cache: 268 M weights 1059 us with the step, 1073 through it
    __builtin_nontemporal_store(m, reinterpret_cast<V*>(mo + e0 + 2048 * u));
    __builtin_nontemporal_store(v, reinterpret_cast<V*>(vo + e0 + 2048 * u));
  }
}

__global__ __launch_bounds__(256) void moments_kernel(MomentArgs a) {
  const int i = find_tensor(a.a.first, a.a.count, (int)blockIdx.x);
  const AdamTensor& t = a.a.t[i];
  const int64_t base = (int64_t)((int)blockIdx.x - a.a.first[i]) * kMomentChunk;
  if (a.dt == FNO_DTYPE_F32)
    moments_chunk(t, base, static_cast<float*>(a.mo[i]), static_cast<float*>(a.vo[i]));
  else if (a.dt == FNO_DTYPE_F16)
    moments_chunk(t, base, static_cast<_Float16*>(a.mo[i]), static_cast<_Float16*>(a.vo[i]));
  else
    moments_chunk(t, base, static_cast<__bf16*>(a.mo[i]), static_cast<__bf16*>(a.vo[i]));
}

// v summed over the work-group's THREADS threads in a fixed order.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double red[THREADS / 64];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_down(v, d);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) s += red[i];
  return s;
}

// Sum of squares of each chunk of the gradients, in double: no fp32 gradient
// overflows it, so the sum is finite exactly where every value is.
template <typename G>
__device__ __forceinline__ double square_sum(const G* g, int64_t base, int64_t n) {
  using V = typename Vec4<G>::type;
  constexpr int U = 8;
  double s = 0.0;
  int64_t b = base;
  const int64_t end = base + kNormChunk < n ? base + kNormChunk : n;
  for (; b + 1024 * U <= end; b += 1024 * U) {
    V v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const V*>(g + b + 1024 * u + 4 * threadIdx.x);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = __builtin_fma((double)(float)v[u][j], (double)(float)v[u][j], s);
  }
  for (; b < end; b += 1024) {  // past the end: zeros
    const V v = load4<V>(g, b + 4 * threadIdx.x, n);
#pragma unroll
    for (int j = 0; j < 4; ++j) s = __builtin_fma((double)(float)v[j], (double)(float)v[j], s);
  }
  return s;
}

// A batch's gradients alone.
struct NormTensor {
  const void* g;
  int64_t n;
};
struct NormArgs {
  NormTensor t[kNormBatch];
  int32_t first[kNormBatch + 1];
  int8_t dt[kNormBatch];
  int32_t count;
};

struct NormOut {
  double* part;  // the whole list's sums, by chunk
  int64_t chunks;
  double b1, b2, max_norm, inv_scale;
  fno_adamw_control* ctl;
};

// The control block from the chunks' sums, by the THREADS threads of a
// work-group; `load` reads a sum.
template <int THREADS, typename Load>
__device__ __forceinline__ void finish_norm(const NormOut& o, Load load) {
  double s = 0.0;
#pragma unroll 8
  for (int64_t e = threadIdx.x; e < o.chunks; e += THREADS) s += load(o.part + e);
  const double sum = block_sum<THREADS>(s);
  if (threadIdx.x != 0) return;
  fno_adamw_control* ctl = o.ctl;
  const double norm = sqrt(sum) * o.inv_scale;
  const bool ok = sum <= 1.7976931348623157e308;  // false for inf and NaN
  ctl->grad_norm = (float)norm;
  ctl->grad_scale = (float)(norm > o.max_norm ? o.inv_scale * (o.max_norm / norm) : o.inv_scale);
  ctl->skip = ok ? 0 : 1;
  if (!ok) {
    ctl->skipped += 1;
    return;
  }
  const int64_t t = ctl->step + 1;
  ctl->step = t;
  ctl->bias1 = 1.0 / (1.0 - int_pow(o.b1, t));
  ctl->bias2 = 1.0 / sqrt(1.0 - int_pow(o.b2, t));
}

// JOIN: the work-group that ends last forms the norm.  Its sum was made
// visible to the device before it counted itself (release), and it reads the
// others' after it saw that all had (acquire); it leaves the count at zero.
template <bool JOIN>
__global__ __launch_bounds__(256) void grad_sq_kernel(NormArgs a, NormOut o, int64_t at) {
  const int i = find_tensor(a.first, a.count, (int)blockIdx.x);
  const NormTensor t = a.t[i];
  const int dt = a.dt[i];
  const int64_t base = (int64_t)((int)blockIdx.x - a.first[i]) * kNormChunk;
  double s;
  if (dt == FNO_DTYPE_F32) s = square_sum(static_cast<const float*>(t.g), base, t.n);
  else if (dt == FNO_DTYPE_F16) s = square_sum(static_cast<const _Float16*>(t.g), base, t.n);
  else s = square_sum(static_cast<const __bf16*>(t.g), base, t.n);
  s = block_sum<256>(s);
  if (!JOIN) {
    if (threadIdx.x == 0) o.part[at + blockIdx.x] = s;
    return;
  }
  __shared__ bool last;
  if (threadIdx.x == 0) {
    __hip_atomic_store(o.part + at + blockIdx.x, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int32_t before = __hip_atomic_fetch_add(&o.ctl->arrived, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    last = before == (int32_t)o.chunks - 1;
  }
  __syncthreads();
  if (!last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  finish_norm<256>(o, [](const double* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  });
  if (threadIdx.x == 0) o.ctl->arrived = 0;
}

__global__ __launch_bounds__(1024) void grad_norm_kernel(NormOut o) {
  finish_norm<1024>(o, [](const double* p) { return *p; });
}

// --------------------------------------------------------------------------
// Host side
// --------------------------------------------------------------------------
inline bool ok16(const void* p) { return p && ((uintptr_t)p & 15u) == 0; }
inline bool ok_dtype(int dt) { return dt >= FNO_DTYPE_F32 && dt <= FNO_DTYPE_BF16; }

bool check_list(const fno_adamw_tensor* t, int64_t count) {
  return count >= 0 && count <= ((int64_t)1 << 31) && (count == 0 || t);
}

bool check_grad(const fno_adamw_tensor& t) {
  if (t.n < 0 || t.n > kMaxN || !ok_dtype(t.param_dtype)) return false;
  if (t.grad_dtype != FNO_DTYPE_F32 && t.grad_dtype != t.param_dtype) return false;
  return t.n == 0 || ok16(t.grad);
}

bool check_states(const fno_adamw_tensor& t) {
  if (t.n < 0 || t.n > kMaxN || (t.state_bits != 32 && t.state_bits != 8)) return false;
  if (t.n == 0) return true;
  if (!ok16(t.exp_avg) || !ok16(t.exp_avg_sq) || t.exp_avg == t.exp_avg_sq) return false;
  return t.state_bits == 32 ? !t.exp_avg_scale && !t.exp_avg_sq_scale
                            : ok16(t.exp_avg_scale) && ok16(t.exp_avg_sq_scale);
}

bool check_hyper(const fno_adamw_desc* d) {
  return d && d->lr >= 0.0 && d->lr <= 1.7e308 && d->beta1 >= 0.0 && d->beta1 < 1.0 &&
         d->beta2 >= 0.0 && d->beta2 < 1.0 && d->eps >= 0.0 && d->eps <= 3.4e38;
}

bool check_tensor(const fno_adamw_tensor& t) {
  if (!check_grad(t) || !check_states(t)) return false;
  if (!(t.weight_decay >= 0.0f && t.weight_decay <= 3.4e38f)) return false;
  if (t.param_dtype == FNO_DTYPE_F32 && t.master) return false;
  return t.n == 0 || (ok16(t.param) && (!t.master || ok16(t.master)));
}

void put(AdamArgs* a, const fno_adamw_tensor& x) {
  a->t[a->count] = AdamTensor{x.param, x.master, x.grad, x.exp_avg, x.exp_avg_sq,
                              x.exp_avg_scale, x.exp_avg_sq_scale, x.n, x.param_dtype,
                              x.grad_dtype, x.state_bits, x.weight_decay};
}
void put(NormArgs* a, const fno_adamw_tensor& x) {
  a->t[a->count] = NormTensor{x.grad, x.n};
  a->dt[a->count] = (int8_t)x.grad_dtype;
}

// The next launch's tensors from list position *i on; returns its chunks.
template <typename Args>
int64_t next_batch(const fno_adamw_tensor* t, int64_t count, int64_t chunk, int64_t* i, Args* a) {
  constexpr int most = (int)(sizeof(a->t) / sizeof(a->t[0]));
  int64_t chunks = 0;
  a->count = 0;
  for (; *i < count && a->count < most; ++*i) {
    const fno_adamw_tensor& x = t[*i];
    if (x.n == 0) continue;
    const int64_t c = cdiv(x.n, chunk);
    if (a->count && chunks + c > kMaxGrid) break;
    put(a, x);
    a->first[a->count++] = (int32_t)chunks;
    chunks += c;
  }
  a->first[a->count] = (int32_t)chunks;
  return chunks;
}

int64_t norm_chunks(const fno_adamw_tensor* t, int64_t count) {
  int64_t c = 0;
  for (int64_t i = 0; i < count; ++i) c += cdiv(t[i].n, kNormChunk);
  return c;
}

// Runs `launch(args, chunks, list index of the first tensor)` over the batches of a list.
template <typename Args, typename F>
hipError_t over_batches(const fno_adamw_tensor* t, int64_t count, int64_t chunk, F launch) {
  Args a;
  for (int64_t i = 0; i < count;) {
    const int64_t from = i;
    const int64_t chunks = next_batch(t, count, chunk, &i, &a);
    if (chunks == 0) continue;
    launch(a, chunks, from);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

struct StepLaunch {
  const fno_adamw_tensor* t;
  int64_t count;
  AdamHyper h;
  const fno_adamw_control* ctl;
  hipStream_t s;
};

template <int U>
hipError_t launch_step_of(const StepLaunch& L) {
  return over_batches<AdamArgs>(L.t, L.count, U * kPiece, [&](const AdamArgs& a, int64_t chunks, int64_t) {
    hipLaunchKernelGGL(adamw_kernel<U>, dim3((unsigned)chunks), dim3(256), 0, L.s, a, L.h, L.ctl);
  });
}

hipError_t launch_step(void* ctx) {
  const StepLaunch& L = *static_cast<StepLaunch*>(ctx);
  int64_t n = 0;
  for (int64_t i = 0; i < L.count; ++i) n += L.t[i].n;
  return n < ((int64_t)1 << 22) ? launch_step_of<1>(L) : launch_step_of<2>(L);
}

struct NormLaunch {
  const fno_adamw_tensor* t;
  int64_t count;
  NormOut o;
  hipStream_t s;
};

// Up to kJoin chunks the last work-group of the sums forms the norm too (the
// launch that it saves is a third of a small model's step); beyond, counting
// every work-group would cost more than a launch of its own.
constexpr int64_t kJoin = 512;

hipError_t launch_norm(void* ctx) {
  const NormLaunch& L = *static_cast<NormLaunch*>(ctx);
  const bool join = L.o.chunks > 0 && L.o.chunks <= kJoin;
  int64_t at = 0;
  const hipError_t e =
      over_batches<NormArgs>(L.t, L.count, kNormChunk, [&](const NormArgs& a, int64_t chunks, int64_t) {
        hipLaunchKernelGGL(join ? grad_sq_kernel<true> : grad_sq_kernel<false>, dim3((unsigned)chunks),
                           dim3(256), 0, L.s, a, L.o, at);
        at += chunks;
      });
  if (e != hipSuccess || join) return e;
  hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(1024), 0, L.s, L.o);
  return hipGetLastError();
}

struct MomentLaunch {
  const fno_adamw_tensor* t;
  int64_t count;
  int dt;
  void* const* mo;
  void* const* vo;
  hipStream_t s;
};

hipError_t launch_moments(void* ctx) {
  const MomentLaunch& L = *static_cast<MomentLaunch*>(ctx);
  MomentArgs ma;
  ma.dt = L.dt;
  return over_batches<AdamArgs>(L.t, L.count, kMomentChunk, [&](const AdamArgs& a, int64_t chunks, int64_t from) {
    ma.a = a;
    for (int64_t i = from, j = 0; j < a.count; ++i) {
      if (L.t[i].n == 0) continue;
      ma.mo[j] = L.mo[i];
      ma.vo[j++] = L.vo[i];
    }
    hipLaunchKernelGGL(moments_kernel, dim3((unsigned)chunks), dim3(256), 0, L.s, ma);
  });
}

fno_status timed_status(const char* name, hipStream_t s, hipError_t (*launch)(void*), void* ctx) {
  const hipError_t e = timed_launch(name, s, launch, ctx);
  return e == hipSuccess ? FNO_OK : report_hip_error(e, name);
}

}  // namespace
}  // namespace fno

using namespace fno;

extern "C" fno_status fno_grad_norm_workspace_size(const fno_adamw_tensor* t, int64_t count,
                                                   size_t* bytes) {
  if (!check_list(t, count) || !bytes) return FNO_ERR_INVALID_ARGUMENT;
  for (int64_t i = 0; i < count; ++i)
    if (t[i].n < 0 || t[i].n > kMaxN) return FNO_ERR_INVALID_ARGUMENT;
  *bytes = (size_t)(cdiv(norm_chunks(t, count) * 8, 256) * 256 + 256);
  return FNO_OK;
}

extern "C" fno_status fno_grad_norm(const fno_adamw_desc* d, const fno_adamw_tensor* t,
                                    int64_t count, double max_norm, double inv_loss_scale,
                                    fno_adamw_control* control, void* ws, size_t ws_len,
                                    hipStream_t stream) {
  if (!check_hyper(d) || !check_list(t, count) || !ok16(control)) return FNO_ERR_INVALID_ARGUMENT;
  if (!(max_norm > 0.0) || !(inv_loss_scale > 0.0 && inv_loss_scale <= 3.4e38))
    return FNO_ERR_INVALID_ARGUMENT;
  for (int64_t i = 0; i < count; ++i)
    if (!check_grad(t[i])) return FNO_ERR_INVALID_ARGUMENT;
  size_t need = 0;
  const fno_status st = fno_grad_norm_workspace_size(t, count, &need);
  if (st != FNO_OK) return st;
  if (ws_len < need) return FNO_ERR_WORKSPACE_TOO_SMALL;
  if (!ok16(ws)) return FNO_ERR_INVALID_ARGUMENT;
  NormLaunch L{t, count,
               NormOut{static_cast<double*>(ws), norm_chunks(t, count), d->beta1, d->beta2, max_norm,
                       inv_loss_scale, control},
               stream};
  return timed_status("grad_norm", stream, launch_norm, &L);
}

extern "C" fno_status fno_adamw_step(const fno_adamw_desc* d, const fno_adamw_tensor* t,
                                     int64_t count, int64_t step, const fno_adamw_control* control,
                                     hipStream_t stream) {
  if (!check_hyper(d) || !check_list(t, count)) return FNO_ERR_INVALID_ARGUMENT;
  if (control ? !ok16(control) : step < 1) return FNO_ERR_INVALID_ARGUMENT;
  for (int64_t i = 0; i < count; ++i)
    if (!check_tensor(t[i])) return FNO_ERR_INVALID_ARGUMENT;
  if (count == 0) return FNO_OK;
  StepLaunch L{t, count, AdamHyper{d->lr, d->beta1, d->beta2, 0.0, 0.0, (float)d->eps}, control,
               stream};
  if (!control) {
    L.h.bias1 = 1.0 / (1.0 - int_pow(d->beta1, step));
    L.h.bias2 = 1.0 / std::sqrt(1.0 - int_pow(d->beta2, step));
  }
  return timed_status("adamw_step", stream, launch_step, &L);
}

extern "C" fno_status fno_adamw_moments(const fno_adamw_tensor* t, int64_t count, fno_dtype dtype,
                                        void* const* exp_avg_out, void* const* exp_avg_sq_out,
                                        hipStream_t stream) {
  if (!check_list(t, count) || !ok_dtype(dtype)) return FNO_ERR_INVALID_ARGUMENT;
  if (count && (!exp_avg_out || !exp_avg_sq_out)) return FNO_ERR_INVALID_ARGUMENT;
  for (int64_t i = 0; i < count; ++i) {
    if (!check_states(t[i]) || t[i].state_bits != 8) return FNO_ERR_INVALID_ARGUMENT;
    if (t[i].n && (!ok16(exp_avg_out[i]) || !ok16(exp_avg_sq_out[i]))) return FNO_ERR_INVALID_ARGUMENT;
  }
  if (count == 0) return FNO_OK;
  MomentLaunch L{t, count, (int)dtype, exp_avg_out, exp_avg_sq_out, stream};
  return timed_status("adamw_moments", stream, launch_moments, &L);
}
