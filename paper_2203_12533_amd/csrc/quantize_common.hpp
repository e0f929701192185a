// What the quantisations to 8 and 4 bits share: a thread's 8 x 8 elements of a 128 x 128 tile, read once and kept as they are stored.
#pragma once
#include "common.hpp"

namespace pw {

constexpr int kTile = 128;             // rows and columns of a tile
constexpr int kPer = 8;                // rows of a thread, and columns

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

// Eight consecutive elements as they are, wherever they start; their magnitudes' bits in kWords words, in which the order of
// unsigned integers is that of the values, infinities and NaN above all numbers.
template <class T> struct Eight;
template <> struct Eight<float> {
  typedef uint32_t vec __attribute__((ext_vector_type(8), aligned(4)));
  typedef uint32_t word;
  static constexpr int kWords = 8;
  static __device__ __forceinline__ word magnitude(uint32_t v) { return v & 0x7fffffffu; }
  static __device__ __forceinline__ word finite(word m) { return m < 0x7f800000u ? m : 0u; }
  static __device__ __forceinline__ bool is_finite(word m) { return m < 0x7f800000u; }
  static __device__ __forceinline__ word larger(word a, word b) { return a > b ? a : b; }
};
template <> struct Eight<bf16> {
  typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
  typedef u16x2 word;
  static constexpr int kWords = 4;
  static __device__ __forceinline__ word magnitude(uint32_t v) { return __builtin_bit_cast(u16x2, v & 0x7fff7fffu); }
  static __device__ __forceinline__ word finite(word m) {
    return u16x2{(unsigned short)(m[0] < 0x7f80 ? m[0] : 0), (unsigned short)(m[1] < 0x7f80 ? m[1] : 0)};
  }
  static __device__ __forceinline__ bool is_finite(word m) { return m[0] < 0x7f80 && m[1] < 0x7f80; }
  static __device__ __forceinline__ word larger(word a, word b) { return __builtin_elementwise_max(a, b); }
};
template <class W> __device__ __forceinline__ W from_lane(W w, int lanes) {
  return __builtin_bit_cast(W, __shfl_xor(__builtin_bit_cast(int, w), lanes, kWave));
}

// 8-bit blocks of 128:
// e + 127 from the largest finite magnitude of a block, given as the bits of a float.
template <bool E5M2> __device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
  const int k = (int)(bits >> 23);                    // m 2^(k - 127), 1 <= m < 2 (k = 0: below 2^-126, clamped anyway)
  const int e = k - (E5M2 ? 15 : 8) + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < 0 ? 0u : (uint32_t)e;                    // at most 254 - 8 + 1
}

// Four bytes of v / 2^e from the bits of four values.
template <bool E5M2> __device__ __forceinline__ uint32_t pack_f32(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float scale) {
  s16x2 r = {0, 0};
  if constexpr (E5M2) {
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, __uint_as_float(a), __uint_as_float(b), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, __uint_as_float(c), __uint_as_float(d), scale, true);
  } else {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(a), __uint_as_float(b), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(c), __uint_as_float(d), scale, true);
  }
  return __builtin_bit_cast(uint32_t, r);
}

// Byte of (row, block) in a table of `rows` rows.
__device__ __forceinline__ int64_t scale_at(int64_t row, int64_t block, int64_t rows) {
  return block * ((rows + 63) & ~63LL) + (row & ~63LL) + (row & 15) * 4 + ((row & 63) >> 4);
}

// v[i]: columns c0 .. c0 + 7 of row r0 + i of x, in the tile at (row0, col0); zeros where there is no element.
template <class T>
__device__ __forceinline__ void load_8x8(typename Eight<T>::vec (&v)[kPer], const T* x, int64_t rows, int64_t cols, int64_t ldx, int64_t row0,
                                         int64_t col0, int64_t r0, int64_t c0) {
  using E = Eight<T>;
  constexpr bool BF16 = sizeof(T) == 2;
  constexpr int W = E::kWords;
  const T* const g = x + r0 * ldx + c0;
  if (row0 + kTile <= rows && col0 + kTile <= cols) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = *reinterpret_cast<const typename E::vec*>(g + i * ldx);
  } else if (cols >= kPer) {
    // Eight elements that exist, those of the last ones of a row that are not the lane's own shifted out: by 1, 2 and 4, as
    // the columns left over ask for (the same in all lanes), in the lane that has them.
    const int over = (int)(-cols & (kPer - 1));
    const bool tail = c0 < cols && c0 + kPer > cols;
    const int64_t from = c0 + kPer <= cols ? c0 : cols - kPer;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int64_t r = r0 + i < rows ? r0 + i : rows - 1;
      v[i] = *reinterpret_cast<const typename E::vec*>(x + r * ldx + from);
    }
#pragma unroll
    for (int s = 1; s < kPer; s *= 2) {
      if (over & s) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          typename E::vec m;
#pragma unroll
          for (int q = 0; q < W; ++q) {
            auto at = [&](int k) { return k < W ? v[i][k < W ? k : 0] : 0u; };
            if constexpr (BF16) m[q] = s == 1 ? at(q) >> 16 | at(q + 1) << 16 : at(q + s / 2);
            else m[q] = at(q + s);
          }
#pragma unroll
          for (int q = 0; q < W; ++q) v[i][q] = tail ? m[q] : v[i][q];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
#pragma unroll
      for (int q = 0; q < W; ++q) v[i][q] = r0 + i < rows && c0 < cols ? v[i][q] : 0u;
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      v[i] = 0;
      if (r0 + i < rows) {
#pragma unroll
        for (int j = 0; j < kPer; ++j)
          if (c0 + j < cols) {
            if constexpr (BF16) v[i][j / 2] |= (uint32_t)__builtin_bit_cast(unsigned short, g[i * ldx + j]) << (16 * (j % 2));
            else v[i][j] = __builtin_bit_cast(uint32_t, g[i * ldx + j]);
          }
      }
    }
  }
}

}  // namespace pw
