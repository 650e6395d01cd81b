// Rounding to 8-bit codes with a scale for each block of 128, along the rows,
// along the columns (into the transpose), or for tiles, in one pass over x.
#include <algorithm>

#include "fno_fp8.h"
#include "fno_host.h"
#include "fno_norm.h"

namespace fno {
namespace {

constexpr int QT = 256;  // threads of a work-group

template <int CTRL>
__device__ __forceinline__ float lane_of(float v) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float join(float a, float b, bool add) {
  return add ? a + b : __builtin_fmaxf(a, b);
}
// Maximum over CG consecutive lanes, in all of them.
template <int CG>
__device__ __forceinline__ float near_max(float v) {
  v = __builtin_fmaxf(v, lane_of<0xB1>(v));
  if constexpr (CG >= 4) v = __builtin_fmaxf(v, lane_of<0x4E>(v));
  if constexpr (CG >= 8) v = __builtin_fmaxf(v, lane_of<0x141>(v));
  if constexpr (CG >= 16) v = __builtin_fmaxf(v, lane_of<0x140>(v));
  return v;
}
// Maximum (or sum) over the lanes of a wave CG apart that belong to one block of
// 128 rows (16 row groups), in all of them: rotations within 16 lanes, then rows
// and halves of the wave exchanged.
template <int CG>
__device__ __forceinline__ float far_join(float v, bool add) {
  if constexpr (CG == 2) v = join(v, lane_of<0x122>(v), add);
  if constexpr (CG <= 4) v = join(v, lane_of<0x124>(v), add);
  if constexpr (CG <= 8) v = join(v, lane_of<0x128>(v), add);
  {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v),
                                                    __builtin_bit_cast(unsigned, v), false, false);
    v = join(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]), add);
  }
  if constexpr (CG >= 4) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v),
                                                    __builtin_bit_cast(unsigned, v), false, false);
    v = join(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]), add);
  }
  return v;
}

__device__ __forceinline__ float finite_size(float v) {
  const float a = __builtin_fabsf(v);
  return a <= 3.402823466e+38f ? a : 0.0f;
}

__device__ __forceinline__ void put_scale(void* out, int64_t at, const BlockScale& s, bool pow2) {
  if (pow2)
    static_cast<uint8_t*>(out)[at] = (uint8_t)s.byte;
  else
    static_cast<float*>(out)[at] = s.scale;
}

// A work-group takes CG x 8 columns of 2048 / CG rows, a thread 8 x 8 of them:
// lanes next to each other hold neighbouring columns of the same rows.  A row's
// blocks are joined within a wave; a column's blocks of 128 rows are 16 threads,
// within a wave up to CG = 4, over two or four waves beyond.
template <typename T, int FMT, int CG>
__global__ __launch_bounds__(QT) void quantize_kernel(QuantArgs a) {
  constexpr int RG = QT / CG;                    // row groups of 8
  constexpr int BLOCKS = RG / 16;                // blocks of 128 rows
  constexpr int WAVES = CG <= 4 ? 1 : CG / 4;    // waves of a column's block
  __shared__ float red[2][4][CG * 8];
  const int cg = threadIdx.x % CG, rg = threadIdx.x / CG, wave = threadIdx.x >> 6;
  const int64_t tiles_c = (a.cols + CG * 8 - 1) / (CG * 8);
  const int64_t tr = blockIdx.x / tiles_c;
  const int c0 = (int)(blockIdx.x - tr * tiles_c) * (CG * 8) + cg * 8;
  const int64_t r0 = tr * (RG * 8) + rg * 8;
  const bool pow2 = a.pow2;
  float v[8][8];
  const T* x = static_cast<const T*>(a.x);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool on = r0 + i < a.rows;
    const T* row = x + (r0 + i) * a.cols;
    if (on && c0 + 8 <= a.cols) {
      T t[8];
      __builtin_memcpy(t, __builtin_assume_aligned(row + c0, sizeof(T)), sizeof(t));
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = (float)t[j];
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = on && c0 + j < a.cols ? (float)row[c0 + j] : 0.0f;
    }
  }
  if (a.act != FNO_NORM_ACT_NONE) {  // both are 0 at 0
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = act_any<T>(v[i][j], a.act);
  }
  const int64_t block_r = (r0 >> 7), block_c = c0 >> 7;
  // Largest sizes and sums of the columns' blocks.
  float top[8];
  if (a.codes_t || a.tile || a.part) {
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float m = 0.0f, s = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        m = __builtin_fmaxf(m, finite_size(v[i][j]));
        s += v[i][j];
      }
      top[j] = far_join<CG>(m, false);
      sum[j] = a.part ? far_join<CG>(s, true) : 0.0f;
    }
    if constexpr (WAVES > 1) {
      if ((threadIdx.x & 63) < CG) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          red[0][wave][cg * 8 + j] = top[j];
          red[1][wave][cg * 8 + j] = sum[j];
        }
      }
      __syncthreads();
      const int first = wave / WAVES * WAVES;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        top[j] = red[0][first][cg * 8 + j];
        sum[j] = red[1][first][cg * 8 + j];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) {
          top[j] = __builtin_fmaxf(top[j], red[0][first + w][cg * 8 + j]);
          sum[j] += red[1][first + w][cg * 8 + j];
        }
      }
    }
    if (a.part && rg % 16 == 0 && r0 < a.rows) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c0 + j < a.cols) a.part[block_r * a.cols + c0 + j] = sum[j];
    }
  }
  BlockScale one{};
  if (a.tile) {  // CG = 16: all threads' columns are one block
    float m = top[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) m = __builtin_fmaxf(m, top[j]);
    one = block_scale<FMT>(near_max<CG>(m), pow2);
    if (threadIdx.x == 0) {
      if (a.codes) put_scale(a.scale, block_c * a.blocks_r + block_r, one, pow2);
      if (a.codes_t) put_scale(a.scale_t, block_r * a.blocks_c + block_c, one, pow2);
    }
  }
  if (a.codes) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      BlockScale s = one;
      if (!a.tile) {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = __builtin_fmaxf(m, finite_size(v[i][j]));
        s = block_scale<FMT>(near_max<CG>(m), pow2);
      }
      if (r0 + i < a.rows) {
        if (!a.tile && cg == 0) put_scale(a.scale, block_c * a.rows + r0 + i, s, pow2);
        if (c0 < a.pitch) {
          uint2 q;
          q.x = pack4<FMT>(v[i][0] * s.inv, v[i][1] * s.inv, v[i][2] * s.inv, v[i][3] * s.inv);
          q.y = pack4<FMT>(v[i][4] * s.inv, v[i][5] * s.inv, v[i][6] * s.inv, v[i][7] * s.inv);
          *reinterpret_cast<uint2*>(a.codes + (r0 + i) * a.pitch + c0) = q;
        }
      }
    }
  }
  if (a.codes_t && r0 < a.pitch_t) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const BlockScale s = a.tile ? one : block_scale<FMT>(top[j], pow2);
      if (c0 + j < a.cols) {
        if (!a.tile && rg % 16 == 0 && r0 < a.rows)
          put_scale(a.scale_t, block_r * a.cols + c0 + j, s, pow2);
        uint2 q;
        q.x = pack4<FMT>(v[0][j] * s.inv, v[1][j] * s.inv, v[2][j] * s.inv, v[3][j] * s.inv);
        q.y = pack4<FMT>(v[4][j] * s.inv, v[5][j] * s.inv, v[6][j] * s.inv, v[7][j] * s.inv);
        *reinterpret_cast<uint2*>(a.codes_t + (int64_t)(c0 + j) * a.pitch_t + r0) = q;
      }
    }
  }
}

// Sums of the units' column sums, in double.
constexpr int kSumCols = 16, kSumRows = 64;
__global__ __launch_bounds__(kSumCols* kSumRows) void col_sum_kernel(const float* part, float* out,
                                                                     int64_t units, int cols) {
  __shared__ double red[kSumRows][kSumCols + 1];
  const int col = threadIdx.x % kSumCols, lane = threadIdx.x / kSumCols;
  const int64_t c = (int64_t)blockIdx.x * kSumCols + col;
  double s = 0.0;
  if (c < cols) {
#pragma unroll 4
    for (int64_t i = lane; i < units; i += kSumRows) s += (double)part[i * cols + c];
  }
  red[lane][col] = s;
  __syncthreads();
#pragma unroll
  for (int d = kSumRows / 2; d > 0; d >>= 1) {
    if (lane < d) red[lane][col] += red[lane + d][col];
    __syncthreads();
  }
  if (lane == 0 && c < cols) out[c] = (float)red[0][col];
}

// --------------------------------------------------------------------------
// Host side
// --------------------------------------------------------------------------
fno_status check_desc(const fno_fp8_quantize_desc* d) {
  if (!d) return FNO_ERR_INVALID_ARGUMENT;
  if (d->dtype < FNO_DTYPE_F32 || d->dtype > FNO_DTYPE_BF16) return FNO_ERR_INVALID_ARGUMENT;
  if (d->format != FNO_FP8_E4M3 && d->format != FNO_FP8_E5M2) return FNO_ERR_INVALID_ARGUMENT;
  if (d->scale_type != FNO_SCALE_POW2 && d->scale_type != FNO_SCALE_F32)
    return FNO_ERR_INVALID_ARGUMENT;
  if (d->blocks != FNO_BLOCKS_ROW && d->blocks != FNO_BLOCKS_TILE) return FNO_ERR_INVALID_ARGUMENT;
  if (d->activation < FNO_NORM_ACT_NONE || d->activation > FNO_NORM_ACT_SILU)
    return FNO_ERR_INVALID_ARGUMENT;
  if (d->rows < 1 || d->cols < 1 || d->rows > INT32_MAX || d->cols > INT32_MAX ||
      d->rows > ((int64_t)1 << 40) / d->cols)
    return FNO_ERR_INVALID_ARGUMENT;
  return FNO_OK;
}

struct QuantLaunch {
  QuantArgs a;
  int dtype, format;
  float* col_sums;
  hipStream_t stream;
};

template <typename T, int FMT, int CG>
hipError_t launch_tiles(const QuantLaunch& L) {
  const int64_t grid = fp8_cdiv(L.a.rows, QT / CG * 8) * fp8_cdiv(L.a.cols, CG * 8);
  quantize_kernel<T, FMT, CG><<<dim3((unsigned)grid), dim3(QT), 0, L.stream>>>(L.a);
  return hipGetLastError();
}
template <typename T, int FMT>
hipError_t launch_width(const QuantLaunch& L) {
  if (L.a.tile || L.a.cols > 64) return launch_tiles<T, FMT, 16>(L);
  if (L.a.cols > 32) return launch_tiles<T, FMT, 8>(L);
  if (L.a.cols > 16) return launch_tiles<T, FMT, 4>(L);
  return launch_tiles<T, FMT, 2>(L);
}
template <typename T>
hipError_t launch_format(const QuantLaunch& L) {
  return L.format == FNO_FP8_E4M3 ? launch_width<T, FNO_FP8_E4M3>(L) : launch_width<T, FNO_FP8_E5M2>(L);
}

hipError_t launch_quantize(void* ctx) {
  const QuantLaunch& L = *static_cast<QuantLaunch*>(ctx);
  const hipError_t e = L.dtype == FNO_DTYPE_F32   ? launch_format<float>(L)
                       : L.dtype == FNO_DTYPE_F16 ? launch_format<_Float16>(L)
                                                  : launch_format<__bf16>(L);
  if (e != hipSuccess || !L.col_sums) return e;
  col_sum_kernel<<<dim3((unsigned)fp8_cdiv(L.a.cols, kSumCols)), dim3(kSumCols * kSumRows), 0, L.stream>>>(
      L.a.part, L.col_sums, L.a.blocks_r, L.a.cols);
  return hipGetLastError();
}

size_t ws_bytes(const fno_fp8_quantize_desc& d) {
  return (size_t)std::max<int64_t>(256, fp8_cdiv(fp8_cdiv(d.rows, kBlock) * d.cols * 4, 256) * 256);
}

}  // namespace
}  // namespace fno

using namespace fno;

extern "C" int64_t fno_fp8_pitch(int64_t cols) { return cols < 0 ? 0 : fp8_pitch(cols); }

extern "C" fno_status fno_fp8_quantize_workspace_size(const fno_fp8_quantize_desc* d,
                                                      size_t* bytes) {
  const fno_status st = check_desc(d);
  if (st != FNO_OK) return st;
  if (!bytes) return FNO_ERR_INVALID_ARGUMENT;
  *bytes = ws_bytes(*d);
  return FNO_OK;
}

extern "C" fno_status fno_fp8_quantize(const fno_fp8_quantize_desc* d, const void* x, void* codes,
                                       void* scale, void* codes_t, void* scale_t, float* col_sums,
                                       void* ws, size_t ws_len, hipStream_t stream) {
  const fno_status st = check_desc(d);
  if (st != FNO_OK) return st;
  if (!fp8_ok16(x) || !fp8_null_or16(codes) || !fp8_null_or16(scale) || !fp8_null_or16(codes_t) ||
      !fp8_null_or16(scale_t) || !fp8_null_or16(col_sums))
    return FNO_ERR_INVALID_ARGUMENT;
  if (!codes != !scale || !codes_t != !scale_t || (!codes && !codes_t)) return FNO_ERR_INVALID_ARGUMENT;
  if (codes && codes == codes_t) return FNO_ERR_INVALID_ARGUMENT;
  if (col_sums) {
    if (ws_len < ws_bytes(*d)) return FNO_ERR_WORKSPACE_TOO_SMALL;
    if (!fp8_ok16(ws)) return FNO_ERR_INVALID_ARGUMENT;
  }
  QuantLaunch L{{}, d->dtype, d->format, col_sums, stream};
  QuantArgs& a = L.a;
  a.x = x;
  a.codes = static_cast<uint8_t*>(codes);
  a.codes_t = static_cast<uint8_t*>(codes_t);
  a.scale = scale;
  a.scale_t = scale_t;
  a.part = col_sums ? static_cast<float*>(ws) : nullptr;
  a.rows = d->rows;
  a.cols = (int)d->cols;
  a.pitch = fp8_pitch(d->cols);
  a.pitch_t = fp8_pitch(d->rows);
  a.act = d->activation;
  a.pow2 = d->scale_type == FNO_SCALE_POW2;
  a.tile = d->blocks == FNO_BLOCKS_TILE;
  a.blocks_r = fp8_cdiv(d->rows, kBlock);
  a.blocks_c = fp8_cdiv(d->cols, kBlock);
  const hipError_t e = timed_launch("fp8_quantize", stream, launch_quantize, &L);
  return e == hipSuccess ? FNO_OK : report_hip_error(e, "fp8_quantize");
}
