// Rounding to 8-bit codes with a scale for each block of 128, along the rows,
// along the columns (into the transpose), or for tiles, in one pass over x.
#include <algorithm>
#include <type_traits>

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

// SiLU as exact as fp32: the exponential of the argument's product with log2 e and
// that product's own remainder, the reciprocal with one step of Newton's.
__device__ __forceinline__ float silu32_of(float z) {
  const float hi = z * -1.44269502f;
  const float lo = __builtin_fmaf(z, -1.92596299e-08f, __builtin_fmaf(z, -1.44269502f, -hi));
  float e = __builtin_amdgcn_exp2f(hi);
  e = __builtin_fmaf(e, lo * 0.693147182f, e);
  const float d = 1.0f + e;
  float r = __builtin_amdgcn_rcpf(d);
  r = __builtin_fmaf(r, __builtin_fmaf(-d, r, 1.0f), r);
  return __builtin_fabsf(z) < 87.0f ? z * r : silu_f(z);
}
// What is rounded to eight bits is formed in fp32 as exactly as fp32 tensors are,
// whatever the type of x: an error beside a border between two codes becomes a
// whole step of the code.
__device__ __forceinline__ float act32_of(float z, int act) {
  return act == FNO_NORM_ACT_GELU ? gelu32_of(z) : act == FNO_NORM_ACT_SILU ? silu32_of(z) : z;
}

// The 8 x 8 values of a thread.  16-bit values without an activation stay in
// pairs: sizes are compared as whole numbers, two at a time, and with powers of
// two the conversion takes pairs and divides them itself (exactly).  Three
// operations a value for both directions, where single floats take thirteen
// (33.5 M values both ways 27 us, with fp32 scales, so as single floats, 30; 67 M
// 48 and 55; from the memory-side cache.  67 M weights from memory 50, 5.4 TB/s).
template <typename T, int FMT, bool ACT, bool POW2>
struct Values {
  static constexpr bool PAIRS = sizeof(T) == 2 && !ACT && POW2;
  typedef T T2 __attribute__((ext_vector_type(2)));
  typedef short S2 __attribute__((ext_vector_type(2)));
  typedef unsigned short U2 __attribute__((ext_vector_type(2)));
  unsigned p[PAIRS ? 8 : 1][4];  // two values each
  float f[PAIRS ? 1 : 8][8];

  __device__ __forceinline__ void set(int i, const T (&t)[8], int act) {
    if constexpr (PAIRS) {
      __builtin_memcpy(p[i], t, sizeof(t));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] = ACT ? act32_of((float)t[j], act) : quiet(t[j]);
    }
  }
  // In fp32, a signaling NaN made quiet: fmax leaves out a quiet one, but of a
  // signaling one makes NaN, behind which the largest size so far is lost.  (fp16's
  // conversion quiets, so does arithmetic; bfloat16's is a shift.)
  static __device__ __forceinline__ float quiet(T v) {
    if constexpr (std::is_same_v<T, float>) {
      return __builtin_canonicalizef(v);
    } else if constexpr (std::is_same_v<T, _Float16>) {
      return (float)v;
    } else {
      return __builtin_canonicalizef(
          __builtin_bit_cast(float, (unsigned)__builtin_bit_cast(unsigned short, v) << 16));
    }
  }
  __device__ __forceinline__ float at(int i, int j) const {
    if constexpr (PAIRS)
      return number((unsigned short)(j & 1 ? p[i][j / 2] >> 16 : p[i][j / 2] & 0xffffu));
    else
      return f[i][j];
  }
  // The same values, of which the compiler does not know that: what is formed from
  // them on a rare path is not formed before it, and not kept behind it.
  __device__ __forceinline__ Values apart() const {
    Values v = *this;
    if constexpr (PAIRS) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(v.p[i][j]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(v.f[i][j]));
    }
    return v;
  }
  // Largest finite sizes.
  static constexpr unsigned short INF16 = std::is_same_v<T, _Float16> ? 0x7c00 : 0x7f80;
  static __device__ __forceinline__ U2 size2(unsigned v) { return __builtin_bit_cast(U2, v & 0x7fff7fffu); }
  static __device__ __forceinline__ float number(unsigned short bits) {
    T v;
    __builtin_memcpy(&v, &bits, 2);
    return (float)v;
  }
  __device__ __forceinline__ float row_top(int i) const {
    float m = 0.0f;
    bool odd;
    if constexpr (PAIRS) {
      const U2 a = __builtin_elementwise_max(__builtin_elementwise_max(size2(p[i][0]), size2(p[i][1])),
                                             __builtin_elementwise_max(size2(p[i][2]), size2(p[i][3])));
      const unsigned short b = a[0] > a[1] ? a[0] : a[1];
      odd = b >= INF16;
      m = number(b);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) m = __builtin_fmaxf(m, __builtin_fabsf(f[i][j]));
      odd = !(m <= 3.402823466e+38f);
    }
    if (odd) {
      const Values v = apart();
      m = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = __builtin_fmaxf(m, finite_size(v.at(i, j)));
    }
    return m;
  }
  __device__ __forceinline__ void col_tops(float (&m)[8]) const {
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      if constexpr (PAIRS) {
        U2 a = size2(p[0][j / 2]);
#pragma unroll
        for (int i = 1; i < 8; ++i) a = __builtin_elementwise_max(a, size2(p[i][j / 2]));
        odd |= a[0] >= INF16 || a[1] >= INF16;
        m[j] = number(a[0]);
        m[j + 1] = number(a[1]);
      } else {
        m[j] = m[j + 1] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          m[j] = __builtin_fmaxf(m[j], __builtin_fabsf(f[i][j]));
          m[j + 1] = __builtin_fmaxf(m[j + 1], __builtin_fabsf(f[i][j + 1]));
        }
        odd |= !(m[j] <= 3.402823466e+38f) || !(m[j + 1] <= 3.402823466e+38f);
      }
    }
    if (odd) {
      const Values v = apart();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m[j] = __builtin_fmaxf(m[j], finite_size(v.at(i, j)));
      }
    }
  }
  // Two pairs to four codes, divided by 2^e.
  static __device__ __forceinline__ unsigned four(unsigned pa, unsigned pb, float by) {
    T2 a, b;
    __builtin_memcpy(&a, &pa, 4);
    __builtin_memcpy(&b, &pb, 4);
    S2 r = {0, 0};
    if constexpr (std::is_same_v<T, _Float16>) {
      if constexpr (FMT == FNO_FP8_E4M3) {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, a, by, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, b, by, true);
      } else {
        r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f16(r, a, by, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f16(r, b, by, true);
      }
    } else if constexpr (sizeof(T) == 2) {
      if constexpr (FMT == FNO_FP8_E4M3) {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, a, by, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, b, by, true);
      } else {
        r = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(r, a, by, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(r, b, by, true);
      }
    }
    return __builtin_bit_cast(unsigned, r);
  }
  __device__ __forceinline__ uint2 row_codes(int i, const BlockScale& s) const {
    if constexpr (PAIRS) {
      const float by = __builtin_bit_cast(float, s.byte << 23);
      return uint2{four(p[i][0], p[i][1], by), four(p[i][2], p[i][3], by)};
    }
    return uint2{pack4<FMT>(at(i, 0) * s.inv, at(i, 1) * s.inv, at(i, 2) * s.inv, at(i, 3) * s.inv),
                 pack4<FMT>(at(i, 4) * s.inv, at(i, 5) * s.inv, at(i, 6) * s.inv, at(i, 7) * s.inv)};
  }
  __device__ __forceinline__ unsigned column2(int i, int j) const {  // rows i and i + 1
    return __builtin_amdgcn_perm(p[i + 1][j / 2], p[i][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
  }
  __device__ __forceinline__ uint2 col_codes(int j, const BlockScale& s) const {
    if constexpr (PAIRS) {
      const float by = __builtin_bit_cast(float, s.byte << 23);
      return uint2{four(column2(0, j), column2(2, j), by), four(column2(4, j), column2(6, j), by)};
    }
    return uint2{pack4<FMT>(at(0, j) * s.inv, at(1, j) * s.inv, at(2, j) * s.inv, at(3, j) * s.inv),
                 pack4<FMT>(at(4, j) * s.inv, at(5, j) * s.inv, at(6, j) * s.inv, at(7, j) * s.inv)};
  }
};

// Elements `by` to 7 to the front, zeros behind them (by 0 to 8).
template <typename T>
__device__ __forceinline__ void move_down(T (&t)[8], int by) {
#pragma unroll
  for (int d = 8; d > 0; d /= 2)
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = by & d ? (j + d < 8 ? t[j + d] : (T)0.0f) : t[j];
}

// A work-group takes CG x 8 columns of 2048 / CG rows, a thread 8 x 8 of them:
// lanes next to each other hold neighbouring columns of the same rows.  A row's
// blocks are joined within a wave; a column's blocks of 128 rows are 16 threads,
// within a wave up to CG = 4, over two or four waves beyond.  CG = 64, whose waves
// read 1 KB of a row at a time, is for codes of rows alone.
template <typename T, int FMT, int CG, bool ACT, bool POW2>
__global__ __launch_bounds__(QT) void quantize_kernel(QuantArgs a) {
  constexpr int RG = QT / CG;                    // row groups of 8
  constexpr bool COLUMNS = CG <= 16;
  constexpr int BLOCKS = COLUMNS ? RG / 16 : 1;  // blocks of 128 rows
  constexpr int WAVES = CG <= 4 ? 1 : CG / 4;    // waves of a column's block
  constexpr int BL = CG < 16 ? CG : 16;          // lanes of a row's block
  __shared__ float red[2][4][COLUMNS ? CG * 8 : 1];
  __shared__ __attribute__((aligned(16))) uint8_t turned[COLUMNS ? BLOCKS * CG * 8 * kBlock : 16];
  const int cg = threadIdx.x % CG, rg = threadIdx.x / CG, wave = threadIdx.x >> 6;
  const int64_t tiles_c = ((int64_t)a.cols + CG * 8 - 1) / (CG * 8);
  // A die's work-groups (every eighth) take consecutive tiles: what they write of a
  // line of memory meets in one cache.
  int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (id >= a.groups) return;
  const int64_t each = a.groups >> 3;
  if (id < each * 8) id = (id & 7) * each + (id >> 3);
  const int64_t tr = id / tiles_c;
  // (the last tile's columns may pass 2^31)
  const unsigned c0 = (unsigned)(id - tr * tiles_c) * (CG * 8) + cg * 8;
  const int64_t r0 = tr * (RG * 8) + rg * 8;
  constexpr bool pow2 = POW2;
  Values<T, FMT, ACT, POW2> v;
  const T* x = static_cast<const T*>(a.x);
  // All eight rows' loads before any is used, so none has a branch of its own: rows
  // behind the last repeat it and are zeroed, and where a row ends inside the eight
  // columns its last eight are read and moved down.
  T t[8][8];
  const int cols = a.cols, left = (int)((unsigned)cols - c0);  // columns from c0 on
  const bool whole = (cols & 7) == 0;
  if (cols >= 8) {
    const int at = left >= 8 ? (int)c0 : cols - 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = r0 + i < a.rows ? r0 + i : a.rows - 1;
      __builtin_memcpy(t[i], __builtin_assume_aligned(x + row * cols + at, sizeof(T)), sizeof(t[i]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = r0 + i < a.rows ? r0 + i : a.rows - 1;
#pragma unroll
      for (int j = 0; j < 8; ++j) t[i][j] = j < left ? x[row * cols + c0 + j] : (T)0.0f;
    }
  }
  const int off = !whole && cols >= 8 && left < 8 ? (left > 0 ? 8 - left : 8) : 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (!whole) move_down(t[i], off);
    const bool on = r0 + i < a.rows && left > 0;
    uint32_t w[sizeof(t[i]) / 4];
    __builtin_memcpy(w, t[i], sizeof(w));
#pragma unroll
    for (uint32_t& e : w) e = on ? e : 0u;  // 0 as behind an activation
    __builtin_memcpy(t[i], w, sizeof(w));
    v.set(i, t[i], a.act);
  }
  const int64_t block_r = (r0 >> 7), block_c = c0 >> 7;
  // Largest sizes and sums of the columns' blocks.
  float top[8];
  if (COLUMNS && (a.codes_t || a.tile || a.part)) {
    float sum[8];
    v.col_tops(top);
#pragma unroll
    for (int j = 0; j < 8; ++j) top[j] = far_join<CG>(top[j], false);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
    if (a.part) {
      const auto w = v.apart();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[j] += w.at(i, j);
        sum[j] = far_join<CG>(sum[j], true);
      }
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
        if ((int64_t)c0 + j < cols) a.part[block_r * cols + c0 + j] = sum[j];
    }
  }
  BlockScale one{};
  if (a.tile) {  // CG = 16: all threads' columns are one block
    float m = top[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) m = __builtin_fmaxf(m, top[j]);
    one = block_scale<FMT>(near_max<BL>(m), pow2);
    if (threadIdx.x == 0) {
      if (a.codes) put_scale(a.scale, block_c * a.blocks_r + block_r, one, pow2);
      if (a.codes_t) put_scale(a.scale_t, block_r * a.blocks_c + block_c, one, pow2);
    }
  }
  if (a.codes) {
    // each lane stores 8 / CG (at least one) of its rows' scales
    constexpr int EACH = CG >= 8 ? 1 : 8 / CG;
    BlockScale mine[EACH];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      BlockScale s = one;
      if (!a.tile) {
        s = block_scale<FMT>(near_max<BL>(v.row_top(i)), pow2);
        if (EACH == 1 ? cg % BL == i : cg == i / EACH) mine[i % EACH] = s;
      }
      if (r0 + i < a.rows && c0 < a.pitch) {
        *reinterpret_cast<uint2*>(a.codes + (r0 + i) * a.pitch + c0) = v.row_codes(i, s);
      }
    }
    if (!a.tile && cg % BL < 8) {
#pragma unroll
      for (int k = 0; k < EACH; ++k) {
        const int64_t row = r0 + cg % BL * EACH + k;
        if (row < a.rows && block_c < a.blocks_c) put_scale(a.scale, block_c * a.rows + row, mine[k], pow2);
      }
    }
  }
  if (COLUMNS && a.codes_t) {
    // Through LDS, so that 128 codes of a column leave as one run.  A column's
    // pieces of 8 are exchanged by the bits of its group of columns (banks).
    const int block = rg / 16, piece = rg % 16;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const BlockScale s = a.tile ? one : block_scale<FMT>(top[j], pow2);
      if (!a.tile && piece == 0 && r0 < a.rows && j < left)
        put_scale(a.scale_t, block_r * a.cols + c0 + j, s, pow2);
      *reinterpret_cast<uint2*>(turned + ((block * CG + cg) * 8 + j) * kBlock + (piece ^ cg) * 8) =
          v.col_codes(j, s);
    }
    __syncthreads();
    const int64_t first = tr * (RG * 8);
    const int64_t cfirst = c0 - cg * 8;
#pragma unroll
    for (int i = 0; i < BLOCKS * CG * 8 * 8 / QT; ++i) {
      const int t = threadIdx.x + i * QT, at = t & 7, line = t >> 3;  // line: block, column
      const int col = line % (CG * 8), of = col >> 3;
      const int64_t row = first + (line / (CG * 8)) * kBlock + at * 16;
      if (cfirst + col < a.cols && row < a.pitch_t) {
        uint4 q = *reinterpret_cast<const uint4*>(turned + line * kBlock + ((2 * at ^ of) & 14) * 8);
        if (of & 1) q = uint4{q.z, q.w, q.x, q.y};
        *reinterpret_cast<uint4*>(a.codes_t + (cfirst + col) * a.pitch_t + row) = q;
      }
    }
  }
}

// Sums of the units' column sums, in double.
// COLS columns for a work-group, four for a thread: few where units are many.
template <int COLS>
__global__ __launch_bounds__(1024) void col_sum_kernel(const float* part, float* out, int64_t units,
                                                       int cols) {
  constexpr int QUADS = COLS / 4, LANES = 1024 / QUADS;
  __shared__ double red[16][COLS];
  const int quad = threadIdx.x % QUADS, lane = threadIdx.x / QUADS;
  const int64_t group = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  const int64_t c = group * COLS + quad * 4;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  if (c + 4 <= cols) {
#pragma unroll 4
    for (int64_t i = lane; i < units; i += LANES) {
      float t[4];
      __builtin_memcpy(t, __builtin_assume_aligned(part + i * cols + c, 4), sizeof(t));
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] += (double)t[j];
    }
  } else {
    for (int64_t i = lane; i < units; i += LANES)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < cols) s[j] += (double)part[i * cols + c + j];
  }
#pragma unroll
  for (int d = QUADS; d < 64; d *= 2)
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] += __shfl_xor(s[j], d);
  if ((threadIdx.x & 63) < QUADS) {
#pragma unroll
    for (int j = 0; j < 4; ++j) red[threadIdx.x >> 6][quad * 4 + j] = s[j];
  }
  __syncthreads();
  const int64_t mine = group * COLS + threadIdx.x;
  if (threadIdx.x < COLS && mine < cols) {
    double t = red[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < 16; ++w) t += red[w][threadIdx.x];
    out[mine] = (float)t;
  }
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

// A launch's threads stay below 2^32 along an axis: more work-groups than a row of
// the grid holds go on in the next one (the last row's surplus leaves at once).
dim3 grid_of(int64_t groups) {
  constexpr int64_t kRow = 1 << 20;
  return groups <= kRow ? dim3((unsigned)groups) : dim3((unsigned)kRow, (unsigned)fp8_cdiv(groups, kRow));
}

template <typename T, int FMT, int CG>
hipError_t launch_tiles(const QuantLaunch& L) {
  QuantArgs a = L.a;
  a.groups = fp8_cdiv(a.rows, QT / CG * 8) * fp8_cdiv(a.cols, CG * 8);
  const dim3 g = grid_of(a.groups), t(QT);
  if (a.act == FNO_NORM_ACT_NONE)
    a.pow2 ? quantize_kernel<T, FMT, CG, false, true><<<g, t, 0, L.stream>>>(a)
           : quantize_kernel<T, FMT, CG, false, false><<<g, t, 0, L.stream>>>(a);
  else
    a.pow2 ? quantize_kernel<T, FMT, CG, true, true><<<g, t, 0, L.stream>>>(a)
           : quantize_kernel<T, FMT, CG, true, false><<<g, t, 0, L.stream>>>(a);
  return hipGetLastError();
}
template <typename T, int FMT>
hipError_t launch_width(const QuantLaunch& L) {
  if (!L.a.tile && !L.a.codes_t && !L.a.part && L.a.cols >= 512) return launch_tiles<T, FMT, 64>(L);
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
  if (L.a.blocks_r > 512)
    col_sum_kernel<4><<<grid_of(fp8_cdiv(L.a.cols, 4)), dim3(1024), 0, L.stream>>>(
        L.a.part, L.col_sums, L.a.blocks_r, L.a.cols);
  else
    col_sum_kernel<32><<<grid_of(fp8_cdiv(L.a.cols, 32)), dim3(1024), 0, L.stream>>>(
        L.a.part, L.col_sums, L.a.blocks_r, L.a.cols);
  return hipGetLastError();
}

bool too_many(const fno_fp8_quantize_desc& d) { return d.rows > (((int64_t)1 << 38) - 1) / d.cols; }

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
  if (too_many(*d)) return FNO_ERR_UNSUPPORTED;
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
  if (too_many(*d)) return FNO_ERR_UNSUPPORTED;
  if (col_sums) {
    if (ws_len < ws_bytes(*d)) return FNO_ERR_WORKSPACE_TOO_SMALL;
    if (!fp8_ok16(ws)) return FNO_ERR_INVALID_ARGUMENT;
  }
  if (any_twice({codes, scale, codes_t, scale_t, col_sums})) return FNO_ERR_INVALID_ARGUMENT;
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
