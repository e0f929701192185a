// Rows of activations, gradients or weights to 8-bit floating point with a scale for each block of 128 along the row, and - from
// the same read - the transposed array with blocks along what were the rows: the two operands that a layer's forward or
// data-gradient product and its weight-gradient product take (gemm_f8.hip).
//
// The scale of a block is 2^e with the smallest integer e in [-127, 127] for which max |x| <= M 2^e over the block's finite
// values; M = 448 (e4m3) or 57344 (e5m2), both 1.75 times a power of two, so that e follows from exponent and mantissa of the
// maximum without a division.  x 2^-e is exact and is rounded once, to nearest, ties to even.  A power of two costs up to one
// bit of range against an arbitrary scale and no precision; it is what the matrix cores apply for nothing (an E8M0 byte,
// e + 127).  NaN stays NaN; infinities become NaN in e4m3, which has none, and stay infinite in e5m2.
//
// Where scales are: byte (b * R + r / 64 * 64 + r % 16 * 4 + r % 64 / 16) for block b of row r, R = rows rounded up to 64: the four
// rows of a lane's four accumulator blocks side by side, so that the product fetches four scales with one load and picks one
// by an immediate.  Rows that do not exist have 0.
//
// Bound by memory: a block of 256 threads takes 128 x 128 elements, reads them once into registers, and writes 8 consecutive
// elements per lane; the transposed bytes turn in LDS.
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"

namespace pw {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 128;             // rows and columns of a block, and the length that shares a scale
constexpr int kPer = 8;                // rows of a thread, and columns
constexpr int kLdT = kTile + 8;        // bytes per row of the transposed tile in LDS

struct QuantParams {
  const void* x;
  int64_t rows, cols, ldx, ldq, ldqt;
  uint8_t *q, *qt, *q_scale, *qt_scale;
  int vec;                             // rows start on 16 bytes
};

template <class T> struct Eight;
template <> struct Eight<float> { typedef float type __attribute__((ext_vector_type(8), aligned(16))); };
template <> struct Eight<bf16> { typedef bf16x8 type; };

// Largest finite magnitude of a and b (b may be anything).
__device__ __forceinline__ float finite_max(float a, float b) {
  const float m = __builtin_fabsf(b);
  return m < __builtin_inff() ? fmaxf(a, m) : a;      // false for NaN
}
// e + 127 from the maximum of a block.
template <bool E5M2> __device__ __forceinline__ uint32_t scale_byte(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  const int k = (int)(bits >> 23);                    // amax = m 2^(k - 127), 1 <= m < 2 (k = 0: below 2^-126, clamped anyway)
  const int e = k - (E5M2 ? 15 : 8) + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < 0 ? 0u : (uint32_t)e;                    // at most 254 - 8 + 1
}
// 2^-e; e = -127 gives 2^127, e at most 120.
__device__ __forceinline__ float inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

template <bool E5M2> __device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  int r = 0;
  if constexpr (E5M2) {
    r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
  } else {
    r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  }
  return (uint32_t)r;
}

// Byte of (row, block) in a table of `rows` rows.
__device__ __forceinline__ int64_t scale_at(int64_t row, int64_t block, int64_t rows) {
  return block * ((rows + 63) & ~63LL) + (row & ~63LL) + (row & 15) * 4 + ((row & 63) >> 4);
}

// WEIGHT: one scale for the whole 128 x 128 block.  ROWS / COLS: which of the two outputs.
template <class T, bool E5M2, bool WEIGHT, bool ROWS, bool COLS>
__global__ __launch_bounds__(kThreads) void f8_quantize_kernel(QuantParams p) {
  __shared__ float col_max[4][kTile];
  __shared__ __attribute__((aligned(16))) uint8_t turned[COLS ? kTile * kLdT : 16];
  const int tid = threadIdx.x, wave = tid >> 6, c8 = tid & 15, r8 = tid >> 4;      // 16 x 16 threads of 8 x 8
  const int64_t row0 = (int64_t)blockIdx.y * kTile, col0 = (int64_t)blockIdx.x * kTile;
  const int64_t r0 = row0 + r8 * kPer, c0 = col0 + c8 * kPer;
  const T* const x = reinterpret_cast<const T*>(p.x);

  typename Eight<T>::type v[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    v[i] = {};
    const int64_t r = r0 + i;
    if (r < p.rows) {
      const T* const g = x + r * p.ldx + c0;
      if (p.vec && c0 + kPer <= p.cols) {
        v[i] = *reinterpret_cast<const typename Eight<T>::type*>(g);
      } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j)
          if (c0 + j < p.cols) v[i][j] = g[j];
      }
    }
  }

  uint32_t by_row[kPer], by_col[kPer];
  if constexpr (WEIGHT) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
#pragma unroll
      for (int j = 0; j < kPer; ++j) m = finite_max(m, (float)v[i][j]);
    m = wave_max(m);
    if ((tid & 63) == 0) col_max[0][wave] = m;
    __syncthreads();
    const uint32_t s = scale_byte<E5M2>(fmaxf(fmaxf(col_max[0][0], col_max[0][1]), fmaxf(col_max[0][2], col_max[0][3])));
#pragma unroll
    for (int i = 0; i < kPer; ++i) by_row[i] = by_col[i] = s;
  } else {
    if constexpr (ROWS) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        float m = 0.f;
#pragma unroll
        for (int j = 0; j < kPer; ++j) m = finite_max(m, (float)v[i][j]);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
        by_row[i] = scale_byte<E5M2>(m);
      }
    }
    if constexpr (COLS) {
      float m[kPer];
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        m[j] = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) m[j] = finite_max(m[j], (float)v[i][j]);
        m[j] = fmaxf(m[j], __shfl_xor(m[j], 16, 64));
        m[j] = fmaxf(m[j], __shfl_xor(m[j], 32, 64));
        if ((tid & 63) < 16) col_max[wave][c8 * kPer + j] = m[j];
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const int c = c8 * kPer + j;
        by_col[j] = scale_byte<E5M2>(fmaxf(fmaxf(col_max[0][c], col_max[1][c]), fmaxf(col_max[2][c], col_max[3][c])));
      }
    }
  }

  if constexpr (ROWS) {
    const int64_t width = (p.cols + 15) & ~15LL;          // zeros up to a multiple of 16
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int64_t r = r0 + i;
      const float k = inverse(by_row[i]);
      if (r < p.rows && c0 < width) {
        uint2 o;
        o.x = pack4<E5M2>((float)v[i][0] * k, (float)v[i][1] * k, (float)v[i][2] * k, (float)v[i][3] * k);
        o.y = pack4<E5M2>((float)v[i][4] * k, (float)v[i][5] * k, (float)v[i][6] * k, (float)v[i][7] * k);
        *reinterpret_cast<uint2*>(p.q + r * p.ldq + c0) = o;
      }
      if (c8 == 0 && r < ((p.rows + 63) & ~63LL)) p.q_scale[scale_at(r, blockIdx.x, p.rows)] = r < p.rows ? (uint8_t)by_row[i] : 0;
    }
  }
  if constexpr (COLS) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const float k = inverse(by_col[j]);
      uint2 o;
      o.x = pack4<E5M2>((float)v[0][j] * k, (float)v[1][j] * k, (float)v[2][j] * k, (float)v[3][j] * k);
      o.y = pack4<E5M2>((float)v[4][j] * k, (float)v[5][j] * k, (float)v[6][j] * k, (float)v[7][j] * k);
      *reinterpret_cast<uint2*>(turned + (c8 * kPer + j) * kLdT + r8 * kPer) = o;
      const int64_t c = c0 + j;
      if (r8 == 0 && c < ((p.cols + 63) & ~63LL)) p.qt_scale[scale_at(c, blockIdx.y, p.cols)] = c < p.cols ? (uint8_t)by_col[j] : 0;
    }
    __syncthreads();
    const int64_t width = (p.rows + 15) & ~15LL;
    for (int i = tid; i < kTile * (kTile / 8); i += kThreads) {
      const int c = i >> 4, piece = (i & 15) * 8;
      if (col0 + c < p.cols && row0 + piece < width)
        *reinterpret_cast<uint2*>(p.qt + (col0 + c) * p.ldqt + row0 + piece) = *reinterpret_cast<const uint2*>(turned + c * kLdT + piece);
    }
  }
}

}  // namespace

int64_t f8_scale_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0 || rows > (1LL << 30) || cols > (1LL << 30)) return -1;
  return (rows + 63) / 64 * 64 * ((cols + kTile - 1) / kTile);
}

hipError_t launch_f8_quantize(hipStream_t s, const F8QuantizeArgs& a) {
  const int64_t most = 1LL << 30;
  if ((a.dtype != kF32 && a.dtype != kBF16) || (a.format != kE4M3 && a.format != kE5M2) || (a.block_rows != 1 && a.block_rows != kTile))
    return hipErrorInvalidValue;
  if (!a.x || (!a.q && !a.qt) || a.rows < 0 || a.cols < 0 || a.rows > most || a.cols > most || a.ldx < a.cols) return hipErrorInvalidValue;
  if ((uintptr_t)a.x & (a.dtype == kBF16 ? 1 : 3)) return hipErrorInvalidValue;
  if (a.q && (!a.q_scale || ((uintptr_t)a.q & 15) || a.ldq % 16 || a.ldq < a.cols)) return hipErrorInvalidValue;
  if (a.qt && (!a.qt_scale || ((uintptr_t)a.qt & 15) || a.ldqt % 16 || a.ldqt < a.rows)) return hipErrorInvalidValue;
  if (a.rows == 0 || a.cols == 0) return hipSuccess;
  const int64_t gy = (a.rows + kTile - 1) / kTile;
  if (gy > 65535) return hipErrorInvalidValue;
  QuantParams p{a.x, a.rows, a.cols, a.ldx, a.ldq, a.ldqt, (uint8_t*)a.q, (uint8_t*)a.qt, a.q_scale, a.qt_scale, 0};
  p.vec = ((uintptr_t)a.x & 15) == 0 && a.ldx % (a.dtype == kBF16 ? 8 : 4) == 0;
  const dim3 grid((unsigned)((a.cols + kTile - 1) / kTile), (unsigned)gy);
  auto outputs = [&](auto t, auto e5m2, auto weight) {
    using T = decltype(t);
    constexpr bool E = decltype(e5m2)::value, W = decltype(weight)::value;
    if (a.q && a.qt) f8_quantize_kernel<T, E, W, true, true><<<grid, kThreads, 0, s>>>(p);
    else if (a.q) f8_quantize_kernel<T, E, W, true, false><<<grid, kThreads, 0, s>>>(p);
    else f8_quantize_kernel<T, E, W, false, true><<<grid, kThreads, 0, s>>>(p);
  };
  auto blocks = [&](auto t, auto e5m2) {
    if (a.block_rows == 1) outputs(t, e5m2, std::false_type{});
    else outputs(t, e5m2, std::true_type{});
  };
  auto formats = [&](auto t) {
    if (a.format == kE4M3) blocks(t, std::false_type{});
    else blocks(t, std::true_type{});
  };
  if (a.dtype == kF32) formats(float{});
  else formats(bf16{});
  return hipGetLastError();
}

}  // namespace pw
