// Group norm with an activation (and the block's residual), forward and
// backward, in either layout.
//
//   xh = (x - mu) r,  r = 1 / sqrt(var + eps),  z = gamma xh + beta,
//   out = act(z) (+ residual)
//   h = g_out act'(z),  g_beta = sum h,  g_gamma = sum h xh,
//   gx = r (gamma h - a - xh d),  a, d = the group's means of gamma h, gamma h xh
//
// All kernels are bound by memory: an element costs 4 to 12 bytes and a few
// dozen vector operations.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/fno_spectral_conv.h"
#include "fno_act.h"
#include "fno_host.h"

namespace fno {
namespace {

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t rup(int64_t a, int64_t b) { return cdiv(a, b) * b; }

struct NormArgs {
  const void *x, *res, *gout;
  const float *gamma, *beta;
  void* out;        // out or gx
  float* stats;     // [B][G][2]
  float* chan;      // [B][C][2]: sums of h and h xh
  float* group;     // [B][G][2]: a and d
  float *ggamma, *gbeta;
  int64_t B, P;
  int C, G, last;
  float eps;
};

__device__ inline int64_t at(const NormArgs& a, int64_t b, int64_t c, int64_t p) {
  return a.last ? (b * a.P + p) * a.C + c : (b * a.C + c) * a.P + p;
}

// v over the work-group's 256 threads.
__device__ inline double block_sum(double v, double* red) {
  red[threadIdx.x] = v;
  __syncthreads();
  for (int d = 128; d > 0; d >>= 1) {
    if ((int)threadIdx.x < d) red[threadIdx.x] += red[threadIdx.x + d];
    __syncthreads();
  }
  const double s = red[0];
  __syncthreads();
  return s;
}

template <int ACT>
__device__ __forceinline__ float act_f(float z) {
  return ACT == FNO_NORM_ACT_GELU ? gelu_f(z) : ACT == FNO_NORM_ACT_SILU ? silu_f(z) : z;
}
template <int ACT>
__device__ __forceinline__ float act_grad_f(float z) {
  return ACT == FNO_NORM_ACT_GELU ? gelu_grad_f(z) : ACT == FNO_NORM_ACT_SILU ? silu_grad_f(z) : 1.0f;
}

template <typename T>
__global__ __launch_bounds__(256) void norm_stats_kernel(NormArgs a) {
  __shared__ double red[256];
  const int64_t b = blockIdx.x / a.G;
  const int g = blockIdx.x % a.G, cg = a.C / a.G;
  const T* x = static_cast<const T*>(a.x);
  const int64_t M = a.P * cg;
  double s = 0.0, q = 0.0;
  for (int64_t i = threadIdx.x; i < M; i += 256) {
    const int64_t p = a.last ? i / cg : i % a.P;
    const int64_t c = g * cg + (a.last ? i % cg : i / a.P);
    const double v = (double)(float)x[at(a, b, c, p)];
    s += v;
    q += v * v;
  }
  const double mean = block_sum(s, red) / (double)M;
  const double var = fmax(block_sum(q, red) / (double)M - mean * mean, 0.0);
  if (threadIdx.x == 0) {
    const bool ok = __builtin_fabs(mean) <= 1.7976931348623157e308;  // false for inf and NaN
    a.stats[2 * blockIdx.x] = ok ? (float)mean : __builtin_nanf("");
    a.stats[2 * blockIdx.x + 1] = ok ? (float)(1.0 / sqrt(var + (double)a.eps)) : __builtin_nanf("");
  }
}

template <typename T, int ACT>
__global__ __launch_bounds__(256) void norm_fwd_kernel(NormArgs a) {
  const int64_t n = a.B * a.P * a.C;
  const int cg = a.C / a.G;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t b = i / (a.P * a.C), r = i - b * a.P * a.C;
    const int c = (int)(a.last ? r % a.C : r / a.P);
    const float* st = a.stats + 2 * (b * a.G + c / cg);
    const float xh = ((float)static_cast<const T*>(a.x)[i] - st[0]) * st[1];
    const float z = xh * (a.gamma ? a.gamma[c] : 1.0f) + (a.beta ? a.beta[c] : 0.0f);
    float o = act_f<ACT>(z);
    if (a.res) o += (float)static_cast<const T*>(a.res)[i];
    static_cast<T*>(a.out)[i] = (T)o;
  }
}

// Sums of h and h xh of one (sample, channel).
template <typename T, int ACT>
__global__ __launch_bounds__(256) void norm_sums_kernel(NormArgs a) {
  __shared__ double red[256];
  const int64_t b = blockIdx.x / a.C;
  const int c = blockIdx.x % a.C;
  const float* st = a.stats + 2 * (b * a.G + c / (a.C / a.G));
  const float ga = a.gamma ? a.gamma[c] : 1.0f, be = a.beta ? a.beta[c] : 0.0f;
  double s = 0.0, q = 0.0;
  for (int64_t p = threadIdx.x; p < a.P; p += 256) {
    const int64_t i = at(a, b, c, p);
    const float xh = ((float)static_cast<const T*>(a.x)[i] - st[0]) * st[1];
    const float h = (float)static_cast<const T*>(a.gout)[i] * act_grad_f<ACT>(xh * ga + be);
    s += h;
    q += h * xh;
  }
  s = block_sum(s, red);
  q = block_sum(q, red);
  if (threadIdx.x == 0) {
    a.chan[2 * blockIdx.x] = (float)s;
    a.chan[2 * blockIdx.x + 1] = (float)q;
  }
}

// a and d of every group, and the parameter gradients.
__global__ __launch_bounds__(256) void norm_join_kernel(NormArgs a) {
  const int cg = a.C / a.G;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < a.B * a.G) {
    const int64_t b = i / a.G;
    double s = 0.0, q = 0.0;
    for (int j = 0; j < cg; ++j) {
      const int c = (int)(i - b * a.G) * cg + j;
      const double ga = a.gamma ? a.gamma[c] : 1.0;
      s += ga * a.chan[2 * (b * a.C + c)];
      q += ga * a.chan[2 * (b * a.C + c) + 1];
    }
    const double m = (double)a.P * cg;
    a.group[2 * i] = (float)(s / m);
    a.group[2 * i + 1] = (float)(q / m);
  }
  if (i < a.C) {
    double s = 0.0, q = 0.0;
    for (int64_t b = 0; b < a.B; ++b) {
      s += a.chan[2 * (b * a.C + i)];
      q += a.chan[2 * (b * a.C + i) + 1];
    }
    if (a.gbeta) a.gbeta[i] = (float)s;
    if (a.ggamma) a.ggamma[i] = (float)q;
  }
}

template <typename T, int ACT>
__global__ __launch_bounds__(256) void norm_bwd_kernel(NormArgs a) {
  const int64_t n = a.B * a.P * a.C;
  const int cg = a.C / a.G;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t b = i / (a.P * a.C), r = i - b * a.P * a.C;
    const int c = (int)(a.last ? r % a.C : r / a.P);
    const int64_t g = b * a.G + c / cg;
    const float rs = a.stats[2 * g + 1];
    const float xh = ((float)static_cast<const T*>(a.x)[i] - a.stats[2 * g]) * rs;
    const float ga = a.gamma ? a.gamma[c] : 1.0f;
    const float h = (float)static_cast<const T*>(a.gout)[i] *
                    act_grad_f<ACT>(xh * ga + (a.beta ? a.beta[c] : 0.0f));
    static_cast<T*>(a.out)[i] = (T)(rs * (ga * h - a.group[2 * g] - xh * a.group[2 * g + 1]));
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
  if (d->batch * d->channels > ((int64_t)1 << 23)) return FNO_ERR_UNSUPPORTED;
  return FNO_OK;
}

// Workspace: statistics, channel sums and group means.
size_t ws_bytes(const fno_norm_desc& d, bool bwd) {
  const int64_t groups = d.batch * d.groups, chans = d.batch * d.channels;
  return (size_t)(rup(8 * groups, 256) + (bwd ? rup(8 * chans, 256) : 0));
}

struct NormLaunch {
  NormArgs a;
  int dt, act;
  hipStream_t s;
};

unsigned grid_for(int64_t n) { return (unsigned)std::min<int64_t>(cdiv(n, 256), 16384); }

template <typename T, int ACT>
hipError_t fwd_t(const NormLaunch& L) {
  const NormArgs& a = L.a;
  hipLaunchKernelGGL(norm_stats_kernel<T>, dim3((unsigned)(a.B * a.G)), dim3(256), 0, L.s, a);
  hipLaunchKernelGGL((norm_fwd_kernel<T, ACT>), dim3(grid_for(a.B * a.P * a.C)), dim3(256), 0, L.s, a);
  return hipGetLastError();
}

template <typename T, int ACT>
hipError_t bwd_t(const NormLaunch& L) {
  const NormArgs& a = L.a;
  hipLaunchKernelGGL((norm_sums_kernel<T, ACT>), dim3((unsigned)(a.B * a.C)), dim3(256), 0, L.s, a);
  hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)cdiv(std::max<int64_t>(a.B * a.G, a.C), 256)),
                     dim3(256), 0, L.s, a);
  hipLaunchKernelGGL((norm_bwd_kernel<T, ACT>), dim3(grid_for(a.B * a.P * a.C)), dim3(256), 0, L.s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t by_act(const NormLaunch& L, bool bwd) {
  switch (L.act) {
    case FNO_NORM_ACT_GELU:
      return bwd ? bwd_t<T, FNO_NORM_ACT_GELU>(L) : fwd_t<T, FNO_NORM_ACT_GELU>(L);
    case FNO_NORM_ACT_SILU:
      return bwd ? bwd_t<T, FNO_NORM_ACT_SILU>(L) : fwd_t<T, FNO_NORM_ACT_SILU>(L);
    default:
      return bwd ? bwd_t<T, FNO_NORM_ACT_NONE>(L) : fwd_t<T, FNO_NORM_ACT_NONE>(L);
  }
}

hipError_t by_type(const NormLaunch& L, bool bwd) {
  return L.dt == FNO_DTYPE_F32   ? by_act<float>(L, bwd)
         : L.dt == FNO_DTYPE_F16 ? by_act<_Float16>(L, bwd)
                                 : by_act<__bf16>(L, bwd);
}
hipError_t launch_fwd(void* ctx) { return by_type(*static_cast<NormLaunch*>(ctx), false); }
hipError_t launch_bwd(void* ctx) { return by_type(*static_cast<NormLaunch*>(ctx), true); }

NormLaunch launch_of(const fno_norm_desc& d, hipStream_t s) {
  NormLaunch L{};
  L.a.B = d.batch;
  L.a.P = d.points;
  L.a.C = (int)d.channels;
  L.a.G = (int)d.groups;
  L.a.last = d.layout == FNO_LAYOUT_CHANNELS_LAST;
  L.a.eps = d.eps;
  L.dt = d.dtype;
  L.act = d.activation;
  L.s = s;
  return L;
}

}  // namespace
}  // namespace fno

using namespace fno;

extern "C" fno_status fno_group_norm_act_workspace_size(const fno_norm_desc* d, fno_op op,
                                                        size_t* bytes) {
  const fno_status st = check_desc(d);
  if (st != FNO_OK) return st;
  if (!bytes || (op != FNO_OP_FWD && op != FNO_OP_BWD)) return FNO_ERR_INVALID_ARGUMENT;
  *bytes = ws_bytes(*d, op == FNO_OP_BWD);
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
  if (ws_len < ws_bytes(*d, false)) return FNO_ERR_WORKSPACE_TOO_SMALL;
  if (!ok16(ws)) return FNO_ERR_INVALID_ARGUMENT;
  NormLaunch L = launch_of(*d, stream);
  L.a.x = x;
  L.a.gamma = gamma;
  L.a.beta = beta;
  L.a.res = residual;
  L.a.out = out;
  L.a.stats = stats ? stats : static_cast<float*>(ws);
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
  if (ws_len < ws_bytes(*d, true)) return FNO_ERR_WORKSPACE_TOO_SMALL;
  if (!ok16(ws)) return FNO_ERR_INVALID_ARGUMENT;
  NormLaunch L = launch_of(*d, stream);
  L.a.x = x;
  L.a.gamma = gamma;
  L.a.beta = beta;
  L.a.stats = const_cast<float*>(stats);
  L.a.gout = g_out;
  L.a.out = gx;
  L.a.ggamma = g_gamma;
  L.a.gbeta = g_beta;
  L.a.group = static_cast<float*>(ws);
  L.a.chan = reinterpret_cast<float*>(static_cast<char*>(ws) + rup(8 * d->batch * d->groups, 256));
  const hipError_t e = timed_launch("group_norm_act_bwd", stream, launch_bwd, &L);
  return e == hipSuccess ? FNO_OK : report_hip_error(e, "group_norm_act_bwd");
}
