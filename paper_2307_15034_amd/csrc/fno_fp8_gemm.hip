// Products of 8-bit codes with block scales, out = (A B^T) act'(z) + bias, on the
// matrix cores.
//
// 16-bit results: 16 x 16 x 128 products of codes, whose inner length is one scale
// block.  That instruction joins eight neighbouring products at a time in fewer
// bits than fp32: each is cut towards zero to a multiple of 2^-13 of the power of
// two below the largest of the eight (measured, as for the 8-bit products of inner
// length 32); the eights are joined in fp32.  In the 2-norm the sums of normally
// distributed codes are 1.5e-5 off, a fourteenth of fp16's rounding of the result
// (with one value in a thousand twenty times as large 3.8e-5 to 4.6e-5; with values of
// one sign, which the cut all makes smaller, 2.5e-6).
// fp32 results, whose rounding is below that: the codes are widened to bfloat16,
// which holds them exactly, and multiplied at half the rate by products that keep
// fp32 throughout (8e-9 off).
//
// Powers of two as scales are the 8-bit instruction's own (one byte for each row
// of its operands), or the widening's, so the sums over all blocks stay in the
// accumulators.  fp32 scales multiply each block's product on the vector unit as
// it joins the sum.
//
// Rows of a tile are dealt to the matrix operands so that four operands' rows
// lie next to each other in memory: element i of operand 4 h + m is row 64 h + 4 i
// + m.  Four bytes next to each other then are the scales of four operands, and
// a lane ends with four consecutive columns of a row.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "fno_fp8.h"
#include "fno_host.h"
#include "fno_norm.h"

namespace fno {
namespace {

typedef int V8I __attribute__((ext_vector_type(8)));
typedef int V4I __attribute__((ext_vector_type(4)));
typedef float V4F __attribute__((ext_vector_type(4)));
typedef __bf16 V2B __attribute__((ext_vector_type(2)));
typedef __bf16 V8B __attribute__((ext_vector_type(8)));

// What chunks behind a row's last code read.
__device__ const uint4 kZeros = {0, 0, 0, 0};

// 16 bytes a lane from global memory into LDS, a wave's lanes one behind the other
// from `to` on (the same for the whole wave).  Written out, because behind the
// builtin the compiler waits for the copy before any read of LDS that may be its
// target, the other buffer's among them; here all_arrived() is the wait.
__device__ __forceinline__ void copy16_to_lds(uint64_t from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(from), "s"(to)
               : "memory", "m0");
}
// The same from a base of the whole wave's and an offset of the lane's.
__device__ __forceinline__ void copy16_to_lds(uint64_t base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(off), "s"(base), "s"(to)
               : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)__builtin_amdgcn_readfirstlane(
      (int)(uintptr_t)(const __attribute__((address_space(3))) void*)p);
}

// Waits for this wave's copies into LDS (which no other wait covers) and for the
// other waves.
__device__ __forceinline__ void all_arrived() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// Brings ROWS x 128 codes of a block column into LDS: row r's piece c of 16 at
// place c ^ (r / 4 mod 8) of the row, so that the lanes of an operand's load (rows
// 4 apart) spread over the banks.  Rows behind the last repeat it, pieces behind a
// row's last code are zeros.
template <int ROWS, int THREADS>
struct TileLoad {
  static constexpr int N = ROWS * 8 / THREADS;
  uint32_t off[N];  // of the thread's pieces, from the tile's first row on
  const uint8_t* codes;
  int64_t pitch;
  int most;         // last row
  bool near;        // offsets fit
  __device__ __forceinline__ TileLoad(const uint8_t* base, int64_t r0, int64_t rows, int64_t pitch_)
      : codes(base + r0 * pitch_), pitch(pitch_) {
    const int r = threadIdx.x >> 3, c = ((threadIdx.x & 7) ^ ((threadIdx.x >> 5) & 7)) << 4;
    most = rows - r0 < ROWS ? (int)(rows - r0) - 1 : ROWS - 1;
    near = pitch <= ((int64_t)1 << 31) / ROWS;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = r + i * (THREADS / 8) < most ? r + i * (THREADS / 8) : most;
      off[i] = (uint32_t)row * (uint32_t)pitch + c;
      asm volatile("" : "+v"(off[i]));  // one register each, not the product's two
    }
  }
  __device__ __forceinline__ void fetch(int kb, uint8_t* lds) const {
    const uint32_t to = lds_address(lds + (threadIdx.x & ~63) * 16);
    const int64_t at = (int64_t)kb * kBlock;
    if (near && at + kBlock <= pitch) {
      const uint64_t base = (uint64_t)codes + at;
#pragma unroll
      for (int i = 0; i < N; ++i) copy16_to_lds(base, off[i], to + i * THREADS * 16);
    } else {
      int t = threadIdx.x;
      asm volatile("" : "+v"(t));  // formed here, not kept over the caller's loop
      const int r = t >> 3, c = ((t & 7) ^ ((t >> 5) & 7)) << 4;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = r + i * (THREADS / 8) < most ? r + i * (THREADS / 8) : most;
        const uint64_t from = (uint64_t)codes + (uint64_t)row * (uint64_t)pitch + (uint64_t)(at + c);
        copy16_to_lds(at + c < pitch ? from : (uint64_t)&kZeros, to + i * THREADS * 16);
      }
    }
  }
};

template <typename T>
__device__ __forceinline__ void finish4(const MatmulArgs& g, int64_t row, int64_t col, V4F v,
                                        bool whole) {
  const int64_t at = row * g.N + col;
  T r[4];
  if (g.z) {
    const T* z = static_cast<const T*>(g.z) + at;
    if (whole) {
      __builtin_memcpy(r, __builtin_assume_aligned(z, sizeof(T)), sizeof(r));
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] *= act_grad_any<T>((float)r[j], g.act);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (col + j < g.N) v[j] *= act_grad_any<T>((float)z[j], g.act);
    }
  }
  if (g.bias) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (col + j < g.N) v[j] += g.bias[col + j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = (T)v[j];
  T* out = static_cast<T*>(g.out) + at;
  if (whole) {
    __builtin_memcpy(__builtin_assume_aligned(out, sizeof(T)), r, sizeof(r));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (col + j < g.N) out[j] = r[j];
  }
}
template <typename T>
__device__ __forceinline__ void finish1(const MatmulArgs& g, int64_t row, int64_t col, float v) {
  const int64_t at = row * g.N + col;
  if (g.z) v *= act_grad_any<T>((float)static_cast<const T*>(g.z)[at], g.act);
  if (g.bias) v += g.bias[col];
  static_cast<T*>(g.out)[at] = (T)v;
}
// A wave's part of the tile: four columns at a time of the rows that a lane holds,
// rows and columns behind the last left out.
template <typename T, int RM, int RN>
__device__ __forceinline__ void finish_tile(const MatmulArgs& g, const V4F (&acc)[RM][RN], int64_t row0,
                                            int64_t col0) {
#pragma unroll
  for (int q = 0; q < RN / 4; ++q) {
    const int64_t col = col0 + q * 64;
    const bool whole = col + 4 <= g.N && row0 < g.M;
    if (whole) {
      V4F bias = {0.0f, 0.0f, 0.0f, 0.0f};
      if (g.bias) __builtin_memcpy(&bias, __builtin_assume_aligned(g.bias + col, 4), 16);
      T* out = static_cast<T*>(g.out) + row0 * g.N + col;
      const T* z = static_cast<const T*>(g.z) + row0 * g.N + col;
      const int64_t left = g.M - row0;  // rows from row0 on
      struct T4 {
        T e[4];
      };
#pragma unroll
      for (int i = 0; i < RM; i += 2) {
        // eight rows of z at a time, all asked for before the first is used
        T4 t[2][4];
        if (g.z) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int64_t row = ((i + h) >> 2) * 64 + r * 4 + ((i + h) & 3);
              __builtin_memcpy(&t[h][r], __builtin_assume_aligned(z + (row < left ? row : 0) * g.N, sizeof(T)),
                               sizeof(T4));
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int64_t row = ((i + h) >> 2) * 64 + r * 4 + ((i + h) & 3);
            V4F v = {acc[i + h][q * 4][r], acc[i + h][q * 4 + 1][r], acc[i + h][q * 4 + 2][r],
                     acc[i + h][q * 4 + 3][r]};
            if (g.z) {
#pragma unroll
              for (int j = 0; j < 4; ++j) v[j] *= act_grad_any<T>((float)t[h][r].e[j], g.act);
            }
            T4 o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o.e[j] = (T)(v[j] + bias[j]);
            if (row < left) __builtin_memcpy(__builtin_assume_aligned(out + row * g.N, sizeof(T)), &o, sizeof(o));
          }
      }
    } else if (col < g.N && row0 < g.M) {
#pragma unroll
      for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int64_t row = row0 + (i >> 2) * 64 + r * 4 + (i & 3);
          if (row < g.M)
            finish4<T>(g, row, col, V4F{acc[i][q * 4][r], acc[i][q * 4 + 1][r], acc[i][q * 4 + 2][r], acc[i][q * 4 + 3][r]}, false);
        }
    }
  }
}
__device__ __forceinline__ void finish4_any(const MatmulArgs& g, int64_t row, int64_t col, V4F v) {
  const bool whole = col + 4 <= g.N;
  if (g.dtype == FNO_DTYPE_F32)
    finish4<float>(g, row, col, v, whole);
  else if (g.dtype == FNO_DTYPE_F16)
    finish4<_Float16>(g, row, col, v, whole);
  else
    finish4<__bf16>(g, row, col, v, whole);
}

// Work-groups go round the eight dies in turn: the tiles of a die are made
// consecutive ones, and those go through bands of eight tile rows, column by
// column, so that what a die reads at a time is read again from its cache.
__device__ __forceinline__ void tile_of(const MatmulArgs& g, int64_t id, int64_t* tm, int64_t* tn) {
  const int64_t total = g.tiles_m * g.tiles_n, each = total >> 3;
  if (id < each * 8) id = (id & 7) * each + (id >> 3);
  const int64_t band = id / (8 * g.tiles_n), m0 = band * 8;
  const int64_t rows = g.tiles_m - m0 < 8 ? g.tiles_m - m0 : 8;
  id -= band * 8 * g.tiles_n;
  *tn = id / rows;
  *tm = m0 + (id - *tn * rows);
}

// The 32 codes of a lane's operand in bfloat16, times a power of two.
template <int FMT>
__device__ __forceinline__ void widen(V8I codes, float scale, V8B (&out)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = codes[2 * i + (j >> 1)];
      V2B v;
      if constexpr (FMT == FNO_FP8_E4M3)
        v = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, true)
                  : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, false);
      else
        v = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(c, scale, true)
                  : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(c, scale, false);
      out[i][2 * j] = v[0];
      out[i][2 * j + 1] = v[1];
    }
}
template <int N, typename F, int... I>
__device__ __forceinline__ void unrolled_over(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
  unrolled_over<N>(f, std::make_integer_sequence<int, N>{});
}
// Byte m of four scales as a number (255: NaN).
__device__ __forceinline__ float scale_of(int four, int m) {
  const unsigned b = ((unsigned)four >> (8 * m)) & 255u;
  return __builtin_bit_cast(float, b == 255u ? 0x7fc00000u : b ? b << 23 : 0x00400000u);
}

// The tile's product.  Two stages of LDS: a block's tiles arrive while the one
// before is multiplied; the matrix cores bound it (256 x 256, eight waves of 128 x
// 64: their operands take 75% of LDS's rate; 128 x 128 tiles would take all of it).
// 16384 x 4096 x 4096: 237 to 265 us with powers of two (2.1 to 2.3 PFLOP/s), 389 to
// 395 with fp32 scales, which the vector unit bounds (eight operations for a 16 x 16
// product of 32 cycles).  Wide, 4096 x 4096 x 8192: 200 to 207 us (1.3 to 1.4 PFLOP/s).
template <int FA, int FB, bool F32S, bool WIDE, int BM, int BN, int WGM, int WGN, int STAGES = 2>
__global__ __launch_bounds__(64 * WGM * WGN, STAGES == 1 ? 3 : 1) void gemm_kernel(MatmulArgs g) {
  constexpr int THREADS = 64 * WGM * WGN;
  constexpr int TM = BM / WGM, TN = BN / WGN;  // a wave's part
  constexpr int HM = TM / 64, HN = TN / 64;
  __shared__ __attribute__((aligned(16))) uint8_t tile_a[STAGES][BM * kBlock], tile_b[STAGES][BN * kBlock];
  using S = std::conditional_t<F32S, float, uint8_t>;
  constexpr int SN = (BM + BN + THREADS - 1) / THREADS;  // scales a thread brings
  __shared__ __attribute__((aligned(16))) S scales[STAGES][BM + BN];
  const int lane = threadIdx.x & 63, i16 = lane & 15, kg = lane >> 4;
  const int wave = threadIdx.x >> 6, wm = wave / WGN, wn = wave % WGN;
  int64_t tm, tn;
  tile_of(g, blockIdx.x, &tm, &tn);
  const int64_t m0 = tm * BM, n0 = tn * BN;
  const int first = blockIdx.y * g.kb_per_split;
  const int last = first + g.kb_per_split < g.kb ? first + g.kb_per_split : g.kb;

  V4F acc[HM * 4][HN * 4];
#pragma unroll
  for (int i = 0; i < HM * 4; ++i)
#pragma unroll
    for (int j = 0; j < HN * 4; ++j) acc[i][j] = V4F{0.0f, 0.0f, 0.0f, 0.0f};

  // Thread t brings the scales of rows t, t + THREADS, ... of A's tile and then B's.
  uint64_t sat[SN];
  int64_t sstep[SN];
  S next_s[SN];
#pragma unroll
  for (int i = 0; i < SN; ++i) {
    const int t = threadIdx.x + i * THREADS;
    const bool of_a = t < BM;
    int64_t row = of_a ? m0 + t : n0 + t - BM;
    const int64_t most = (of_a ? g.M : g.N) - 1;
    row = (row < most ? row : most) >> (of_a ? g.shift_a : g.shift_b);
    sstep[i] = of_a ? g.scales_a : g.scales_b;
    sat[i] = (of_a ? (uint64_t)g.scale_a : (uint64_t)g.scale_b) +
             (uint64_t)(row + first * sstep[i]) * sizeof(S);
  }
  const TileLoad<BM, THREADS> from_a(g.a, m0, g.M, g.pitch);
  const TileLoad<BN, THREADS> from_b(g.b, n0, g.N, g.pitch);
  auto fetch = [&](int kb, uint8_t* a, uint8_t* b) {
#pragma unroll
    for (int i = 0; i < SN; ++i) {
      next_s[i] = *reinterpret_cast<const __attribute__((address_space(1))) S*>(sat[i]);
      sat[i] += (uint64_t)sstep[i] * sizeof(S);
    }
    from_a.fetch(kb, a);
    from_b.fetch(kb, b);
  };
  auto operand = [&](const uint8_t* lds, int row) {  // rows row + 4 i
    const uint8_t* p = lds + (row + i16 * 4) * kBlock;
    const V4I lo = *reinterpret_cast<const V4I*>(p + ((kg ^ (i16 & 7)) << 4));
    const V4I hi = *reinterpret_cast<const V4I*>(p + (((kg + 4) ^ (i16 & 7)) << 4));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // A block's products, operand by operand of A (LAST + 1 of them); each of A's
  // operands is read while the one before is multiplied.  B's operands of the next
  // block take the place of this one's as its last products go.
  constexpr int LAST = HM * 4 - 1;
  V8I fa, fb[WIDE ? 1 : HN * 4];
  V8B wb[WIDE ? HN * 4 : 1][4];
  int sa[HM], sb[HN];  // scales of four operands, a byte each
  V4F ra[F32S ? HM * 4 : 1], cb[F32S ? HN : 1];
  auto read_a = [&](int buf, int idx) {
    return operand(tile_a[buf], wm * TM + (idx >> 2) * 64 + (idx & 3));
  };
  auto read_b = [&](int buf, int j) {
    return operand(tile_b[buf], wn * TN + (j >> 2) * 64 + (j & 3));
  };
  auto read_scales = [&](int buf) {
    const S* s = scales[buf];
#pragma unroll
    for (int h = 0; h < HM; ++h) {
      if constexpr (F32S) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          ra[h * 4 + r] = *reinterpret_cast<const V4F*>(s + wm * TM + h * 64 + kg * 16 + r * 4);
      } else {
        sa[h] = *reinterpret_cast<const int*>(s + wm * TM + h * 64 + i16 * 4);
      }
    }
#pragma unroll
    for (int q = 0; q < HN; ++q) {
      if constexpr (F32S)
        cb[q] = *reinterpret_cast<const V4F*>(s + BM + wn * TN + q * 64 + i16 * 4);
      else
        sb[q] = *reinterpret_cast<const int*>(s + BM + wn * TN + q * 64 + i16 * 4);
    }
  };
  auto widen_b = [&](int buf) {
#pragma unroll
    for (int j = 0; j < HN * 4; ++j)
      widen<FB>(read_b(buf, j), F32S ? 1.0f : scale_of(sb[j >> 2], j & 3), wb[j]);
  };
  auto multiply = [&](auto index, auto reload, int buf) {
    constexpr int IDX = decltype(index)::value, H = IDX >> 2, M = IDX & 3;
    V8B wa[4];
    if constexpr (WIDE) widen<FA>(fa, F32S ? 1.0f : scale_of(sa[H], M), wa);
#pragma unroll
    for (int q = 0; q < HN; ++q)
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        V4F* c = &acc[IDX][q * 4 + n];
        if constexpr (WIDE || F32S) {
          V4F p = F32S ? V4F{0.0f, 0.0f, 0.0f, 0.0f} : *c;
          if constexpr (WIDE) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[i], wb[q * 4 + n][i], p, 0, 0, 0);
          } else {
            p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb[q * 4 + n], p, FA, FB, 0, 0, 0, 0);
          }
          if constexpr (F32S) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
              (*c)[r] = __builtin_fmaf(p[r], ra[H * 4 + r][M] * cb[q][n], (*c)[r]);
          } else {
            *c = p;
          }
        } else {
          // (the byte of the scales is part of the instruction)
          if (n == 0)
            *c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb[q * 4], *c, FA, FB, M, sa[H], 0, sb[q]);
          if (n == 1)
            *c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb[q * 4 + 1], *c, FA, FB, M, sa[H], 1, sb[q]);
          if (n == 2)
            *c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb[q * 4 + 2], *c, FA, FB, M, sa[H], 2, sb[q]);
          if (n == 3)
            *c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb[q * 4 + 3], *c, FA, FB, M, sa[H], 3, sb[q]);
        }
        if constexpr (decltype(reload)::value && !WIDE) {
          __builtin_amdgcn_sched_barrier(0);
          fb[q * 4 + n] = read_b(buf, q * 4 + n);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
  };
  using No = std::false_type;
  using Last = std::integral_constant<int, LAST>;
  // Operands 0 to LAST - 1; leaves the last one read.
  auto multiply_most = [&](int buf) {
    unrolled<LAST>([&](auto index) {
      const V8I next = read_a(buf, decltype(index)::value + 1);
      __builtin_amdgcn_sched_barrier(0);  // one operand ahead, not more: registers
      multiply(index, No{}, 0);
      __builtin_amdgcn_sched_barrier(0);
      fa = next;
    });
  };

  auto keep_scales = [&](int buf) {
#pragma unroll
    for (int i = 0; i < SN; ++i)
      if ((BM + BN) % THREADS == 0 || threadIdx.x + i * THREADS < BM + BN)
        scales[buf][threadIdx.x + i * THREADS] = next_s[i];
  };
  fetch(first, tile_a[0], tile_b[0]);
  keep_scales(0);
  all_arrived();
  if (STAGES > 1 && first + 1 < last) fetch(first + 1, tile_a[STAGES - 1], tile_b[STAGES - 1]);
  read_scales(0);
  if constexpr (WIDE) {
    widen_b(0);
  } else {
#pragma unroll
    for (int j = 0; j < HN * 4; ++j) fb[j] = read_b(0, j);
  }
  fa = read_a(0, 0);
  multiply_most(0);
  for (int kb = first + 1; STAGES > 1 && kb < last; ++kb) {  // (one stage: one block)
    const int cur = (kb - first) & (STAGES - 1);
    keep_scales(cur);
    all_arrived();  // this block's tiles are there, the last one's all read
    if (kb + 1 < last) fetch(kb + 1, tile_a[cur ^ (STAGES - 1)], tile_b[cur ^ (STAGES - 1)]);
    __builtin_amdgcn_sched_barrier(0);
    const V8I next = read_a(cur, 0);
    multiply(Last{}, std::true_type{}, cur);
    fa = next;
    read_scales(cur);
    if constexpr (WIDE) widen_b(cur);
    multiply_most(cur);
  }
  multiply(Last{}, No{}, 0);

  const int64_t row0 = m0 + wm * TM + kg * 16, col0 = n0 + wn * TN + i16 * 4;
  if (g.splits > 1) {
    MatmulArgs sum = g;  // plain fp32 sums
    sum.out = g.part + (int64_t)blockIdx.y * g.M * g.N;
    sum.z = nullptr;
    sum.bias = nullptr;
    finish_tile<float>(sum, acc, row0, col0);
  } else if (WIDE) {
    finish_tile<float>(g, acc, row0, col0);
  } else if (g.dtype == FNO_DTYPE_F16) {
    finish_tile<_Float16>(g, acc, row0, col0);
  } else {
    finish_tile<__bf16>(g, acc, row0, col0);
  }
}

// Few rows: the work is in reading B.  A work-group takes 16 of its rows, a wave
// every eighth block of them, straight from memory into the operands (row i of A
// and B: lanes i, i + 16, ..); the waves' sums meet in LDS, in their order.  One
// row of 4096 by 4096 x 4096: 5.5 us (3.1 TB/s of codes); split tiles and their join
// took 5.1 + 2.8.
constexpr int kRowWaves = 8;
template <int FA, int FB, bool F32S, bool WIDE, int MT>
__global__ __launch_bounds__(64 * kRowWaves) void few_rows_kernel(MatmulArgs g) {
  __shared__ V4F sums[kRowWaves][MT][64];
  const int lane = threadIdx.x & 63, i16 = lane & 15, kg = lane >> 4, wave = threadIdx.x >> 6;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int64_t bn = n0 + i16 < g.N ? n0 + i16 : g.N - 1;
  const uint8_t* b = g.b + bn * g.pitch;
  using S = std::conditional_t<F32S, float, uint8_t>;
  const S* sa = static_cast<const S*>(g.scale_a);
  const S* sb = static_cast<const S*>(g.scale_b) + (bn >> g.shift_b);
  const uint8_t* a[MT];
  int64_t am[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    am[t] = t * 16 + i16 < g.M ? t * 16 + i16 : g.M - 1;
    a[t] = g.a + am[t] * g.pitch;
  }
  auto operand = [&](const uint8_t* row, int kb) {
    const int64_t at = (int64_t)kb * kBlock + kg * 16;
    V4I lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
    if (at < g.pitch) lo = *reinterpret_cast<const V4I*>(row + at);
    if (at + 64 < g.pitch) hi = *reinterpret_cast<const V4I*>(row + at + 64);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  V4F acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = V4F{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll(MT == 1 ? 4 : 2)
  for (int kb = wave; kb < g.kb; kb += kRowWaves) {
    const V8I fb = operand(b, kb);
    const S ub = sb[kb * g.scales_b];
    V8B wb[4];
    if constexpr (WIDE) widen<FB>(fb, F32S ? 1.0f : scale_of((int)ub, 0), wb);
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const V8I fa = operand(a[t], kb);
      V4F p = F32S ? V4F{0.0f, 0.0f, 0.0f, 0.0f} : acc[t];
      S ua = 0;
      if constexpr (!F32S) ua = sa[kb * g.scales_a + (am[t] >> g.shift_a)];
      if constexpr (WIDE) {
        V8B wa[4];
        widen<FA>(fa, F32S ? 1.0f : scale_of((int)ua, 0), wa);
#pragma unroll
        for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[i], wb[i], p, 0, 0, 0);
      } else if constexpr (F32S) {
        p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb, p, FA, FB, 0, 0, 0, 0);
      } else {
        p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb, p, FA, FB, 0, (int)ua, 0, (int)ub);
      }
      if constexpr (F32S) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int64_t m = t * 16 + kg * 4 + r < g.M ? t * 16 + kg * 4 + r : g.M - 1;
          acc[t][r] = __builtin_fmaf(p[r], sa[kb * g.scales_a + (m >> g.shift_a)] * ub, acc[t][r]);
        }
      } else {
        acc[t] = p;
      }
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) sums[wave][t][lane] = acc[t];
  __syncthreads();
  // a thread for a result: row 4 q + r of its 16, column i
  for (int o = threadIdx.x; o < MT * 256; o += 64 * kRowWaves) {
    const int t = o >> 8, row16 = (o >> 4) & 15, col16 = o & 15;
    const int64_t row = t * 16 + row16, col = n0 + col16;
    if (row >= g.M || col >= g.N) continue;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) v += sums[w][t][(row16 >> 2) * 16 + col16][row16 & 3];
    if (g.dtype == FNO_DTYPE_F32)
      finish1<float>(g, row, col, v);
    else if (g.dtype == FNO_DTYPE_F16)
      finish1<_Float16>(g, row, col, v);
    else
      finish1<__bf16>(g, row, col, v);
  }
}

// Joins the splits' sums: four columns for `lanes` threads (a power of two up to
// 64), each of which adds every lanes-th split; a fixed order.
__global__ __launch_bounds__(256) void join_splits_kernel(MatmulArgs g, int lanes) {
  const int64_t per_row = (g.N + 3) / 4, total = g.M * per_row;
  const int lane = threadIdx.x & (lanes - 1);
  const int64_t step = (int64_t)gridDim.x * (256 / lanes);
  for (int64_t i = (int64_t)blockIdx.x * (256 / lanes) + threadIdx.x / lanes; i < total; i += step) {
    const int64_t row = i / per_row, col = (i - row * per_row) * 4;
    const bool whole = col + 4 <= g.N;
    V4F v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int s = lane; s < g.splits; s += lanes) {
      const float* p = g.part + ((int64_t)s * g.M + row) * g.N + col;
      if (whole) {
        float t[4];
        __builtin_memcpy(t, __builtin_assume_aligned(p, 4), 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += t[j];
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (col + j < g.N) v[j] += p[j];
      }
    }
    for (int d = 1; d < lanes; d *= 2)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += __shfl_xor(v[j], d);
    if (lane == 0) finish4_any(g, row, col, v);
  }
}

// --------------------------------------------------------------------------
// Host side
// --------------------------------------------------------------------------
fno_status check_desc(const fno_fp8_matmul_desc* d) {
  if (!d) return FNO_ERR_INVALID_ARGUMENT;
  for (int f : {d->format_a, d->format_b})
    if (f != FNO_FP8_E4M3 && f != FNO_FP8_E5M2) return FNO_ERR_INVALID_ARGUMENT;
  for (int b : {d->blocks_a, d->blocks_b})
    if (b != FNO_BLOCKS_ROW && b != FNO_BLOCKS_TILE) return FNO_ERR_INVALID_ARGUMENT;
  if (d->scale_type != FNO_SCALE_POW2 && d->scale_type != FNO_SCALE_F32)
    return FNO_ERR_INVALID_ARGUMENT;
  if (d->out_dtype < FNO_DTYPE_F32 || d->out_dtype > FNO_DTYPE_BF16) return FNO_ERR_INVALID_ARGUMENT;
  if (d->activation < FNO_NORM_ACT_NONE || d->activation > FNO_NORM_ACT_SILU)
    return FNO_ERR_INVALID_ARGUMENT;
  for (int64_t n : {d->rows, d->cols, d->inner})
    if (n < 1 || n > INT32_MAX) return FNO_ERR_INVALID_ARGUMENT;
  if (d->rows > ((int64_t)1 << 42) / d->cols) return FNO_ERR_INVALID_ARGUMENT;
  return FNO_OK;
}

enum Tile { TILE_128, TILE_256, TILE_NARROW, FEW_ROWS };
struct MatmulPlan {
  MatmulArgs g;
  Tile tile;
};

MatmulPlan plan_of(const fno_fp8_matmul_desc& d) {
  MatmulPlan p{};
  MatmulArgs& g = p.g;
  g.M = d.rows;
  g.N = d.cols;
  g.kb = (int)fp8_cdiv(d.inner, kBlock);
  g.pitch = fp8_pitch(d.inner);
  g.shift_a = d.blocks_a == FNO_BLOCKS_TILE ? 7 : 0;
  g.shift_b = d.blocks_b == FNO_BLOCKS_TILE ? 7 : 0;
  g.scales_a = g.shift_a ? fp8_cdiv(g.M, kBlock) : g.M;
  g.scales_b = g.shift_b ? fp8_cdiv(g.N, kBlock) : g.N;
  g.act = d.activation;
  g.dtype = d.out_dtype;
  // 256 x 256 where such tiles fill the chip's 256 compute units; 256 x 64 of one
  // stage where a row of codes is one block and columns are few (the work is in
  // the rows' bytes: more work-groups at a time); else 128 x 128.
  const bool pow2 = d.scale_type == FNO_SCALE_POW2;
  const int64_t of256 = fp8_cdiv(g.M, 256) * fp8_cdiv(g.N, 256);
  // Few rows: up to 64, while a wave's share of the inner axis stays short.  That is
  // for inner axes of channels; over many points (the gradient of 64 x 64 weights) the
  // border lies too far out: 2048 points 8 us, 8192 20, 32768 73, where split tiles
  // take 14 for 32897 (64 x 4096: 76 and 44).
  p.tile = g.M <= 64 && g.kb <= 256 && g.N < ((int64_t)1 << 26) ? FEW_ROWS
           : g.kb == 1 && g.N <= 64 && g.M > 128 ? TILE_NARROW
           : pow2 && of256 >= 192 && g.N > 128 ? TILE_256
                                               : TILE_128;
  const int bm = p.tile == FEW_ROWS ? 64 : p.tile == TILE_128 ? 128 : 256;
  const int bn = p.tile == FEW_ROWS ? 16 : p.tile == TILE_256 ? 256 : p.tile == TILE_NARROW ? 64 : 128;
  g.tiles_m = fp8_cdiv(g.M, bm);
  g.tiles_n = fp8_cdiv(g.N, bn);
  // Few tiles of a long inner axis: split along it, down to four blocks each.
  const int64_t tiles = g.tiles_m * g.tiles_n;
  g.splits = 1;
  const int64_t fill = p.tile == TILE_256 ? 256 : 512;  // work-groups that the chip holds at a time
  if (p.tile != FEW_ROWS && tiles <= fill / 2 && g.kb >= 8)
    g.splits = (int)std::max<int64_t>(1, std::min<int64_t>(fill / tiles, g.kb / 4));
  g.kb_per_split = (int)fp8_cdiv(g.kb, g.splits);
  g.splits = (int)fp8_cdiv(g.kb, g.kb_per_split);
  return p;
}

// Whether a launch's threads (512 or 256 for a tile) would pass 2^32.
bool too_many(const MatmulPlan& p) {
  const int64_t most = p.tile == TILE_256 || p.tile == FEW_ROWS ? (int64_t)1 << 23 : (int64_t)1 << 24;
  return p.g.tiles_m * p.g.tiles_n >= most;
}

struct MatmulLaunch {
  MatmulPlan p;
  int fa, fb;
  bool f32s;
  hipStream_t stream;
};

template <int FA, int FB, bool F32S, bool WIDE>
void launch_tile(const MatmulLaunch& L, dim3 grid) {
  const MatmulArgs& g = L.p.g;
  if (L.p.tile == FEW_ROWS) {
    g.M <= 16 ? few_rows_kernel<FA, FB, F32S, WIDE, 1><<<grid, dim3(64 * kRowWaves), 0, L.stream>>>(g)
              : few_rows_kernel<FA, FB, F32S, WIDE, 4><<<grid, dim3(64 * kRowWaves), 0, L.stream>>>(g);
  } else if (L.p.tile == TILE_NARROW) {
    gemm_kernel<FA, FB, F32S, WIDE, 256, 64, 4, 1, 1><<<grid, dim3(256), 0, L.stream>>>(g);
  } else if (L.p.tile == TILE_256) {
    if constexpr (!F32S) gemm_kernel<FA, FB, F32S, WIDE, 256, 256, 2, 4><<<grid, dim3(512), 0, L.stream>>>(g);
  } else {
    gemm_kernel<FA, FB, F32S, WIDE, 128, 128, 2, 2><<<grid, dim3(256), 0, L.stream>>>(g);
  }
}
template <int FA, int FB>
void launch_formats(const MatmulLaunch& L) {
  const MatmulArgs& g = L.p.g;
  const dim3 grid((unsigned)(g.tiles_m * g.tiles_n), (unsigned)g.splits);
  if (g.dtype == FNO_DTYPE_F32)
    L.f32s ? launch_tile<FA, FB, true, true>(L, grid) : launch_tile<FA, FB, false, true>(L, grid);
  else
    L.f32s ? launch_tile<FA, FB, true, false>(L, grid) : launch_tile<FA, FB, false, false>(L, grid);
}

hipError_t launch_matmul(void* ctx) {
  const MatmulLaunch& L = *static_cast<MatmulLaunch*>(ctx);
  // the instruction's format numbers are this ABI's: 0 e4m3, 1 e5m2
  if (L.fa == FNO_FP8_E4M3)
    L.fb == FNO_FP8_E4M3 ? launch_formats<0, 0>(L) : launch_formats<0, 1>(L);
  else
    L.fb == FNO_FP8_E4M3 ? launch_formats<1, 0>(L) : launch_formats<1, 1>(L);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || L.p.g.splits == 1) return e;
  // a thread for four columns where that fills the chip, else up to one for each
  // four splits
  const int64_t quads = L.p.g.M * fp8_cdiv(L.p.g.N, 4);
  int lanes = 1;
  while (lanes < 64 && lanes * 8 <= L.p.g.splits && quads * lanes < 128 * 1024) lanes *= 2;
  const int64_t groups = fp8_cdiv(quads * lanes, 256);
  join_splits_kernel<<<dim3((unsigned)std::min<int64_t>(groups, 1 << 20)), dim3(256), 0, L.stream>>>(L.p.g, lanes);
  return hipGetLastError();
}

size_t ws_bytes(const MatmulPlan& p) {
  if (p.g.splits == 1) return 256;
  return (size_t)(fp8_cdiv(p.g.splits * p.g.M * p.g.N * 4, 256) * 256);
}

}  // namespace
}  // namespace fno

using namespace fno;

extern "C" fno_status fno_fp8_matmul_workspace_size(const fno_fp8_matmul_desc* d, size_t* bytes) {
  const fno_status st = check_desc(d);
  if (st != FNO_OK) return st;
  if (!bytes) return FNO_ERR_INVALID_ARGUMENT;
  const MatmulPlan p = plan_of(*d);
  if (too_many(p)) return FNO_ERR_UNSUPPORTED;
  *bytes = ws_bytes(p);
  return FNO_OK;
}

extern "C" fno_status fno_fp8_matmul(const fno_fp8_matmul_desc* d, const void* a,
                                     const void* scale_a, const void* b, const void* scale_b,
                                     const void* z, const float* bias, void* out, void* ws,
                                     size_t ws_len, hipStream_t stream) {
  const fno_status st = check_desc(d);
  if (st != FNO_OK) return st;
  if (!fp8_ok16(a) || !fp8_ok16(scale_a) || !fp8_ok16(b) || !fp8_ok16(scale_b) || !fp8_ok16(out) ||
      !fp8_null_or16(z) || !fp8_null_or16(bias))
    return FNO_ERR_INVALID_ARGUMENT;
  if ((z != nullptr) != (d->activation != FNO_NORM_ACT_NONE)) return FNO_ERR_INVALID_ARGUMENT;
  MatmulLaunch L{plan_of(*d), d->format_a, d->format_b, d->scale_type == FNO_SCALE_F32, stream};
  if (L.p.g.splits > 1) {
    if (ws_len < ws_bytes(L.p)) return FNO_ERR_WORKSPACE_TOO_SMALL;
    if (!fp8_ok16(ws)) return FNO_ERR_INVALID_ARGUMENT;
  }
  if (too_many(L.p)) return FNO_ERR_UNSUPPORTED;
  MatmulArgs& g = L.p.g;
  g.a = static_cast<const uint8_t*>(a);
  g.b = static_cast<const uint8_t*>(b);
  g.scale_a = scale_a;
  g.scale_b = scale_b;
  g.z = z;
  g.bias = bias;
  g.out = out;
  g.part = static_cast<float*>(ws);
  const hipError_t e = timed_launch("fp8_matmul", stream, launch_matmul, &L);
  return e == hipSuccess ? FNO_OK : report_hip_error(e, "fp8_matmul");
}
