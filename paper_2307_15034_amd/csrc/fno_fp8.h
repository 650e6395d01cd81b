// What the kernels of the 8-bit products share: formats, block scales, and the
// arguments of the launches.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/fno_spectral_conv.h"

namespace fno {

constexpr int kBlock = FNO_FP8_BLOCK;

inline int64_t fp8_cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
__host__ __device__ inline int64_t fp8_pitch(int64_t cols) { return (cols + 15) & ~(int64_t)15; }
inline bool fp8_ok16(const void* p) { return p && ((uintptr_t)p & 15u) == 0; }
inline bool fp8_null_or16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// A block's scale from the largest of its finite sizes: the factor that values
// are multiplied with, and what is stored.
struct BlockScale {
  float inv, scale;
  unsigned byte;  // POW2
};
// POW2: a = m 2^E with 1 <= m < 2 and F = 1.75 2^T (T = 8 e4m3, 15 e5m2), so the
// least e with a <= F 2^e is E - T, one more where m > 1.75: a carry out of the
// fraction's bits past those of 1.75.
template <int FMT>
__device__ __forceinline__ BlockScale block_scale(float a, bool pow2) {
  constexpr int T = FMT == FNO_FP8_E4M3 ? 8 : 15;
  constexpr float F = FMT == FNO_FP8_E4M3 ? 448.0f : 57344.0f;
  BlockScale s{1.0f, 1.0f, 127u};
  if (a > 0.0f) {
    if (pow2) {
      int e = (int)((__builtin_bit_cast(unsigned, a) + 0x1fffffu) >> 23) - 127 - T;
      e = e < -126 ? -126 : e;
      s.byte = (unsigned)(e + 127);
      s.inv = __builtin_bit_cast(float, (unsigned)(127 - e) << 23);
    } else {
      const float q = a * (1.0f / F);  // (the fp32 reciprocal)
      s.scale = q < 0x1p-126f ? 0x1p-126f : q;
      s.inv = 1.0f / s.scale;
    }
  }
  return s;
}

template <int FMT>
__device__ __forceinline__ unsigned pack4(float a, float b, float c, float d) {
  int r = 0;
  if constexpr (FMT == FNO_FP8_E4M3) {
    r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  } else {
    r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
  }
  return (unsigned)r;
}

struct QuantArgs {
  const void* x;
  uint8_t *codes, *codes_t;
  void *scale, *scale_t;
  float* part;     // [units][cols]: column sums of each unit's rows, or null
  int64_t rows;
  int64_t pitch, pitch_t;
  int cols;
  int act, pow2, tile;
  int64_t blocks_r, blocks_c;  // blocks of 128 along the rows and the columns
  int64_t groups;              // work-groups of the launch
};

struct MatmulArgs {
  const uint8_t *a, *b;
  const void *scale_a, *scale_b;
  const void* z;
  const float* bias;
  void* out;
  float* part;          // [splits][M][N], where splits > 1
  int64_t pitch;        // of a's and b's rows
  int64_t M, N;
  int64_t scales_a, scales_b;  // scales of one block column
  int kb;               // blocks of 128 along the inner axis
  int splits, kb_per_split;
  int shift_a, shift_b; // a row's scale: row >> shift (0 rows, 7 tiles)
  int act, dtype;
  int64_t tiles_m, tiles_n;
};

}  // namespace fno
