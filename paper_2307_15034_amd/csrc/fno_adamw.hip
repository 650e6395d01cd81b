// The optimizer step over many tensors at once (AdamW, states in 32 or 8
// bits) and the global gradient norm that steers it on the device.
//
// A launch takes a batch of tensors by value in its kernel arguments (no
// table to upload, nothing kept between calls): each work-group finds its
// tensor by a search over the batch's first-chunk numbers and works on one
// chunk of it.  The kernels stream every operand once; they are bound by HBM.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/fno_spectral_conv.h"
#include "fno_host.h"

namespace fno {
namespace {

constexpr int kBatch = FNO_ADAMW_LAUNCH_TENSORS;
constexpr int kBlk = FNO_ADAMW_BLOCK;
constexpr int64_t kChunk = 2048;             // elements of a work-group
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
  double lr, b1, b2, size, root;  // size = lr / (1 - b1^t), root = 1 / sqrt(1 - b2^t)
  float eps, gs;
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

__host__ __device__ inline void bias_correct(AdamHyper* h, int64_t t) {
  h->size = h->lr / (1.0 - int_pow(h->b1, t));
  h->root = 1.0 / sqrt(1.0 - int_pow(h->b2, t));
}

__device__ inline float load_as_float(const void* p, int64_t i, int dt) {
  if (dt == FNO_DTYPE_F32) return static_cast<const float*>(p)[i];
  if (dt == FNO_DTYPE_F16) return (float)static_cast<const _Float16*>(p)[i];
  return (float)static_cast<const __bf16*>(p)[i];
}
__device__ inline void store_rounded(void* p, int64_t i, int dt, float v) {
  if (dt == FNO_DTYPE_F32) static_cast<float*>(p)[i] = v;
  else if (dt == FNO_DTYPE_F16) static_cast<_Float16*>(p)[i] = (_Float16)v;
  else static_cast<__bf16*>(p)[i] = (__bf16)v;
}

// The tensor of chunk c: the last i with first[i] <= c.
__device__ inline int find_tensor(const int32_t* first, int count, int c) {
  int lo = 0, hi = count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= c) lo = mid;
    else hi = mid - 1;
  }
  return lo;
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

__device__ inline Consts consts_of(const AdamHyper& h0, const fno_adamw_control* ctl, float wd) {
  AdamHyper h = h0;
  if (ctl) {
    h.lr *= (double)ctl->lr_factor;
    bias_correct(&h, ctl->step);
    h.gs = ctl->grad_scale;
  }
  Consts k;
  k.b1 = (float)h.b1;
  k.c1 = (float)(1.0 - h.b1);
  k.b2 = (float)h.b2;
  k.c2 = (float)(1.0 - h.b2);
  k.size = (float)h.size;
  k.root = (float)h.root;
  k.eps = h.eps;
  k.gs = h.gs;
  k.keep = (float)(1.0 - h.lr * (double)wd);
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
// Codes of the fractions |m| / A and sqrt(v) / B; top = 0 or a value that is
// not a number gives 0 (the scale then tells).
__device__ inline int code_of(float x, float top, float levels) {
#pragma clang fp contract(off)
  if (!(top > 0.0f)) return 0;
  const float q = rintf(__builtin_sqrtf(x / top) * levels);
  return q == q ? (int)q : 0;
}

__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a, AdamHyper h,
                                                    const fno_adamw_control* ctl) {
  if (ctl && ctl->skip) return;
  const int i = find_tensor(a.first, a.count, (int)blockIdx.x);
  const AdamTensor& t = a.t[i];
  const Consts k = consts_of(h, ctl, t.wd);
  const int64_t base = (int64_t)((int)blockIdx.x - a.first[i]) * kChunk;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (t.bits == 32) {
    for (int64_t e = base + threadIdx.x; e < base + kChunk && e < t.n; e += 256) {
      float m = static_cast<float*>(t.m)[e], v = static_cast<float*>(t.v)[e], w;
      float p = t.master ? t.master[e] : load_as_float(t.p, e, t.pdt);
      p = adam_element(k, p, load_as_float(t.g, e, t.gdt), &m, &v, &w);
      static_cast<float*>(t.m)[e] = m;
      static_cast<float*>(t.v)[e] = v;
      if (t.master) t.master[e] = p;
      store_rounded(t.p, e, t.pdt, p);
    }
    return;
  }
  for (int64_t b = base / kBlk + wave; b < (base + kChunk) / kBlk && b * kBlk < t.n; b += 4) {
    float m[4], w[4];
    const float as = t.ms[b], bs = t.vs[b];
    uint32_t am = 0, bm = 0;
    for (int j = 0; j < 4; ++j) {
      const int64_t e = b * kBlk + 64 * j + lane;
      m[j] = w[j] = 0.0f;
      if (e >= t.n) continue;
      m[j] = decode_m(as, static_cast<int8_t*>(t.m)[e]);
      float v = decode_v(bs, static_cast<uint8_t*>(t.v)[e]);
      float p = t.master ? t.master[e] : load_as_float(t.p, e, t.pdt);
      p = adam_element(k, p, load_as_float(t.g, e, t.gdt), &m[j], &v, &w[j]);
      if (t.master) t.master[e] = p;
      store_rounded(t.p, e, t.pdt, p);
      am = max(am, abs_bits(m[j]));
      bm = max(bm, abs_bits(w[j]));
    }
    const float A = __uint_as_float(wave_max(am)), Bt = __uint_as_float(wave_max(bm));
    for (int j = 0; j < 4; ++j) {
      const int64_t e = b * kBlk + 64 * j + lane;
      if (e >= t.n) continue;
      const int qm = code_of(__builtin_fabsf(m[j]), A, 127.0f);
      const int qv = code_of(w[j], Bt, 255.0f);
      static_cast<int8_t*>(t.m)[e] = (int8_t)(m[j] < 0.0f ? -qm : qm);
      static_cast<uint8_t*>(t.v)[e] = (uint8_t)(w[j] > 0.0f && qv < 1 ? 1 : qv);
    }
    if (lane == 0) {
      t.ms[b] = A;
      t.vs[b] = Bt;
    }
  }
}

// 8-bit moments read out.
struct MomentArgs {
  AdamArgs a;
  void* mo[kBatch];
  void* vo[kBatch];
  int32_t dt;
};

__global__ __launch_bounds__(256) void moments_kernel(MomentArgs a) {
  const int i = find_tensor(a.a.first, a.a.count, (int)blockIdx.x);
  const AdamTensor& t = a.a.t[i];
  const int64_t base = (int64_t)((int)blockIdx.x - a.a.first[i]) * kChunk;
  for (int64_t e = base + threadIdx.x; e < base + kChunk && e < t.n; e += 256) {
    store_rounded(a.mo[i], e, a.dt, decode_m(t.ms[e / kBlk], static_cast<int8_t*>(t.m)[e]));
    store_rounded(a.vo[i], e, a.dt, decode_v(t.vs[e / kBlk], static_cast<uint8_t*>(t.v)[e]));
  }
}

// Sum of squares of each chunk of the gradients, in double: no fp32 gradient
// overflows it, so the sum is finite exactly where every value is.
__global__ __launch_bounds__(256) void grad_sq_kernel(AdamArgs a, double* part) {
  __shared__ double red[256];
  const int i = find_tensor(a.first, a.count, (int)blockIdx.x);
  const AdamTensor& t = a.t[i];
  const int64_t base = (int64_t)((int)blockIdx.x - a.first[i]) * kChunk;
  double s = 0.0;
  for (int64_t e = base + threadIdx.x; e < base + kChunk && e < t.n; e += 256) {
    const double g = (double)load_as_float(t.g, e, t.gdt);
    s += g * g;
  }
  red[threadIdx.x] = s;
  __syncthreads();
  for (int d = 128; d > 0; d >>= 1) {
    if ((int)threadIdx.x < d) red[threadIdx.x] += red[threadIdx.x + d];
    __syncthreads();
  }
  if (threadIdx.x == 0) part[blockIdx.x] = red[0];
}

__global__ __launch_bounds__(256) void grad_norm_kernel(const double* part, int64_t n, double max_norm,
                                                        double inv_scale, fno_adamw_control* ctl) {
  __shared__ double red[256];
  double s = 0.0;
  for (int64_t e = threadIdx.x; e < n; e += 256) s += part[e];
  red[threadIdx.x] = s;
  __syncthreads();
  for (int d = 128; d > 0; d >>= 1) {
    if ((int)threadIdx.x < d) red[threadIdx.x] += red[threadIdx.x + d];
    __syncthreads();
  }
  if (threadIdx.x != 0) return;
  const double sum = red[0], norm = sqrt(sum) * inv_scale;
  const bool ok = sum <= 1.7976931348623157e308;  // false for inf and NaN
  ctl->grad_norm = (float)norm;
  ctl->grad_scale = (float)(norm > max_norm ? inv_scale * (max_norm / norm) : inv_scale);
  ctl->skip = ok ? 0 : 1;
  ctl->step += ok ? 1 : 0;
  ctl->skipped += ok ? 0 : 1;
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

bool check_tensor(const fno_adamw_tensor& t) {
  if (!check_grad(t) || !check_states(t)) return false;
  if (!(t.weight_decay >= 0.0f && t.weight_decay <= 3.4e38f)) return false;
  if (t.param_dtype == FNO_DTYPE_F32 && t.master) return false;
  return t.n == 0 || (ok16(t.param) && (!t.master || ok16(t.master)));
}

// The next launch's tensors from list position *i on; returns its chunks.
int64_t next_batch(const fno_adamw_tensor* t, int64_t count, int64_t* i, AdamArgs* a) {
  int64_t chunks = 0;
  a->count = 0;
  for (; *i < count && a->count < kBatch; ++*i) {
    const fno_adamw_tensor& x = t[*i];
    if (x.n == 0) continue;
    const int64_t c = cdiv(x.n, kChunk);
    if (a->count && chunks + c > kMaxGrid) break;
    a->t[a->count] = AdamTensor{x.param, x.master, x.grad, x.exp_avg, x.exp_avg_sq,
                                x.exp_avg_scale, x.exp_avg_sq_scale, x.n, x.param_dtype,
                                x.grad_dtype, x.state_bits, x.weight_decay};
    a->first[a->count++] = (int32_t)chunks;
    chunks += c;
  }
  a->first[a->count] = (int32_t)chunks;
  return chunks;
}

int64_t all_chunks(const fno_adamw_tensor* t, int64_t count) {
  int64_t c = 0;
  for (int64_t i = 0; i < count; ++i) c += cdiv(t[i].n, kChunk);
  return c;
}

// Runs `launch(args, chunks, list index of the first tensor)` over the batches of a list.
template <typename F>
hipError_t over_batches(const fno_adamw_tensor* t, int64_t count, F launch) {
  AdamArgs a;
  for (int64_t i = 0; i < count;) {
    const int64_t from = i;
    const int64_t chunks = next_batch(t, count, &i, &a);
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

hipError_t launch_step(void* ctx) {
  const StepLaunch& L = *static_cast<StepLaunch*>(ctx);
  return over_batches(L.t, L.count, [&](const AdamArgs& a, int64_t chunks, int64_t) {
    hipLaunchKernelGGL(adamw_kernel, dim3((unsigned)chunks), dim3(256), 0, L.s, a, L.h, L.ctl);
  });
}

struct NormLaunch {
  const fno_adamw_tensor* t;
  int64_t count;
  double max_norm, inv_scale;
  fno_adamw_control* ctl;
  double* part;
  hipStream_t s;
};

hipError_t launch_norm(void* ctx) {
  const NormLaunch& L = *static_cast<NormLaunch*>(ctx);
  int64_t at = 0;
  const hipError_t e =
      over_batches(L.t, L.count, [&](const AdamArgs& a, int64_t chunks, int64_t) {
        hipLaunchKernelGGL(grad_sq_kernel, dim3((unsigned)chunks), dim3(256), 0, L.s, a, L.part + at);
        at += chunks;
      });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(256), 0, L.s, L.part, at, L.max_norm,
                     L.inv_scale, L.ctl);
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
  return over_batches(L.t, L.count, [&](const AdamArgs& a, int64_t chunks, int64_t from) {
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
  *bytes = (size_t)(cdiv(all_chunks(t, count) * 8, 256) * 256 + 256);
  return FNO_OK;
}

extern "C" fno_status fno_grad_norm(const fno_adamw_tensor* t, int64_t count, double max_norm,
                                    double inv_loss_scale, fno_adamw_control* control, void* ws,
                                    size_t ws_len, hipStream_t stream) {
  if (!check_list(t, count) || !ok16(control)) return FNO_ERR_INVALID_ARGUMENT;
  if (!(max_norm > 0.0) || !(inv_loss_scale > 0.0 && inv_loss_scale <= 1.7e308))
    return FNO_ERR_INVALID_ARGUMENT;
  for (int64_t i = 0; i < count; ++i)
    if (!check_grad(t[i])) return FNO_ERR_INVALID_ARGUMENT;
  size_t need = 0;
  const fno_status st = fno_grad_norm_workspace_size(t, count, &need);
  if (st != FNO_OK) return st;
  if (ws_len < need) return FNO_ERR_WORKSPACE_TOO_SMALL;
  if (!ok16(ws)) return FNO_ERR_INVALID_ARGUMENT;
  NormLaunch L{t, count, max_norm, inv_loss_scale, control, static_cast<double*>(ws), stream};
  return timed_status("grad_norm", stream, launch_norm, &L);
}

extern "C" fno_status fno_adamw_step(const fno_adamw_desc* d, const fno_adamw_tensor* t,
                                     int64_t count, int64_t step, const fno_adamw_control* control,
                                     hipStream_t stream) {
  if (!d || !check_list(t, count)) return FNO_ERR_INVALID_ARGUMENT;
  if (!(d->lr >= 0.0 && d->lr <= 1.7e308) || !(d->beta1 >= 0.0 && d->beta1 < 1.0) ||
      !(d->beta2 >= 0.0 && d->beta2 < 1.0) || !(d->eps >= 0.0 && d->eps <= 3.4e38))
    return FNO_ERR_INVALID_ARGUMENT;
  if (control ? !ok16(control) : step < 1) return FNO_ERR_INVALID_ARGUMENT;
  for (int64_t i = 0; i < count; ++i)
    if (!check_tensor(t[i])) return FNO_ERR_INVALID_ARGUMENT;
  if (count == 0) return FNO_OK;
  StepLaunch L{t, count, AdamHyper{d->lr, d->beta1, d->beta2, 0.0, 0.0, (float)d->eps, 1.0f},
               control, stream};
  if (!control) bias_correct(&L.h, step);
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
