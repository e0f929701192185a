// Rows of activations, gradients or weights to 4-bit floating point (e2m1) with a scale for each block of 32 along the row, and - from
// the same read - the transposed array with blocks along what were the rows: the two operands that a layer's forward or
// data-gradient product and its weight-gradient product take (gemm_f4.hip).
//
// The scale of a block is 2^e with the smallest integer e in [-127, 127] for which max |x| <= 6 2^e; 6 is 1.5 times a power of two, so
// that e follows from exponent and mantissa of the maximum without a division.  x 2^-e is exact and is rounded once, to nearest, ties to
// even (the only rounding here: one mantissa bit is what the format has).  It has no NaN and no infinity: a block that holds one gets the scale byte
// 255, which the matrix pipe takes for NaN, and codes of 0.
//
// Where scales are: byte (b / 4 * R + r / 64 * 64) * 4 + b % 4 * 64 + r % 16 * 4 + r % 64 / 16 for block b of row r, R = rows rounded up
// to 64.  A matrix instruction of 16 rows and 128 k wants in lane 16 q + l the scale of row l and block q: a word per lane holds
// those of the rows l, l + 16, l + 32, l + 48, and the 64 words of 64 rows and four blocks are neighbours.
//
// Bound by memory: a block of 256 threads takes 128 x 128 elements, 8 x 8 to a thread.  A wave has 32 rows of the tile, which is the
// block length, so that the maxima of both orientations are four exchanges between lanes and meet nowhere else.  8192 x 2048 bf16 into both 11.1 us
// (4.6 TB/s), 333 x 500 fp32 4.0, a launch.
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"
#include "quantize_common.hpp"

namespace pw {

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 32;             // length that shares a scale
struct F4QuantParams {
  const void* x;
  int64_t rows, cols, ldx, ldq, ldqt;  // ldq, ldqt in bytes
  uint8_t *q, *qt, *q_scale, *qt_scale;
};

// e + 127 from the largest magnitude of a block, given as the bits of a float; 255 for an infinity or NaN.
__device__ __forceinline__ uint32_t f4_scale_byte(uint32_t bits) {
  const int e = (int)(bits >> 23) - 2 + ((bits & 0x7fffffu) > 0x400000u ? 1 : 0);   // m 2^(k - 127): 1.5 2^2 2^(k - 2 - 127) holds m <= 1.5
  return bits >= 0x7f800000u ? 255u : e < 0 ? 0u : (uint32_t)e;
}

// Eight codes (a word) of eight values over 2^(byte - 127), 0 where the byte is 255.
template <class T> __device__ __forceinline__ uint32_t pack8(const uint32_t* w, uint32_t byte) {
  const float scale = __uint_as_float(byte << 23);
  uint32_t r = 0;
  if constexpr (sizeof(T) == 2) {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[0]), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[1]), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[2]), scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[3]), scale, 3);
  } else {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[0]), __uint_as_float(w[1]), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[2]), __uint_as_float(w[3]), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[4]), __uint_as_float(w[5]), scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[6]), __uint_as_float(w[7]), scale, 3);
  }
  return byte == 255 ? 0u : r;
}

// WEIGHT: one scale for 32 x 32 elements.  ROWS / COLS: which of the two outputs.
template <class T, bool WEIGHT, bool ROWS, bool COLS>
__global__ __launch_bounds__(kThreads) void f4_quantize_kernel(F4QuantParams p) {
  constexpr bool BF16 = sizeof(T) == 2;
  using E = Eight<T>;
  typedef typename E::word word;
  constexpr int W = E::kWords;
  __shared__ __attribute__((aligned(16))) uint8_t row_byte[4][kTile], col_byte[4][kTile];    // [block][row], [block][column]
  __shared__ __attribute__((aligned(16))) uint8_t turned[COLS ? kTile * kTile / 2 : 16];
  const int tid = threadIdx.x, wave = tid >> 6, c8 = tid & 15, r8 = tid >> 4;      // 16 x 16 threads of 8 x 8
  const int64_t row0 = (int64_t)blockIdx.y * kTile, col0 = (int64_t)blockIdx.x * kTile;
  const int64_t r0 = row0 + r8 * kPer, c0 = col0 + c8 * kPer;
  typename E::vec v[kPer];
  load_8x8<T>(v, reinterpret_cast<const T*>(p.x), p.rows, p.cols, p.ldx, row0, col0, r0, c0);

  // Largest magnitudes as the bits of floats: of the thread's rows among the 4 threads of 32 columns, and of its columns among the 4 of
  // 32 rows, which are in one wave.
  uint32_t by_row[kPer], by_col[kPer];
  {
    word rw[kPer], cw[W];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      rw[i] = E::magnitude(v[i][0]);
#pragma unroll
      for (int q = 1; q < W; ++q) rw[i] = E::larger(rw[i], E::magnitude(v[i][q]));
    }
    if constexpr (WEIGHT) {
      word m = rw[0];
#pragma unroll
      for (int i = 1; i < kPer; ++i) m = E::larger(m, rw[i]);
      m = E::larger(m, from_lane(m, 1));
      m = E::larger(m, from_lane(m, 2));
      m = E::larger(m, from_lane(m, 16));
      m = E::larger(m, from_lane(m, 32));
      uint32_t one;
      if constexpr (BF16) one = (uint32_t)(m[0] > m[1] ? m[0] : m[1]) << 16;
      else one = m;
#pragma unroll
      for (int i = 0; i < kPer; ++i) by_row[i] = by_col[i] = one;
    } else {
      if constexpr (ROWS) {
        if constexpr (BF16) {                                        // two rows to a word
#pragma unroll
          for (int i = 0; i < kPer; i += 2) {
            word m = E::larger(u16x2{rw[i][0], rw[i + 1][0]}, u16x2{rw[i][1], rw[i + 1][1]});
            m = E::larger(m, from_lane(m, 1));
            m = E::larger(m, from_lane(m, 2));
            by_row[i] = (uint32_t)m[0] << 16;
            by_row[i + 1] = (uint32_t)m[1] << 16;
          }
        } else {
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            word m = E::larger(rw[i], from_lane(rw[i], 1));
            by_row[i] = E::larger(m, from_lane(m, 2));
          }
        }
      }
      if constexpr (COLS) {
#pragma unroll
        for (int q = 0; q < W; ++q) {
          cw[q] = E::magnitude(v[0][q]);
#pragma unroll
          for (int i = 1; i < kPer; ++i) cw[q] = E::larger(cw[q], E::magnitude(v[i][q]));
          cw[q] = E::larger(cw[q], from_lane(cw[q], 16));
          cw[q] = E::larger(cw[q], from_lane(cw[q], 32));
          if constexpr (BF16) {
            by_col[2 * q] = (uint32_t)cw[q][0] << 16;
            by_col[2 * q + 1] = (uint32_t)cw[q][1] << 16;
          } else {
            by_col[q] = cw[q];
          }
        }
      }
    }
  }

  if constexpr (ROWS) {
    uint32_t bytes[kPer];
    uint2 packed = {0, 0};
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      bytes[i] = f4_scale_byte(by_row[i]);
      (i < 4 ? packed.x : packed.y) |= bytes[i] << (8 * (i & 3));
    }
    if ((c8 & 3) == 0) *reinterpret_cast<uint2*>(&row_byte[c8 >> 2][r8 * kPer]) = packed;
    const int64_t width = (p.cols + 31) & ~31LL;            // zeros up to a multiple of 32
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      uint32_t w[W];
#pragma unroll
      for (int q = 0; q < W; ++q) w[q] = v[i][q];
      const uint32_t o = pack8<T>(w, bytes[i]);
      if (r0 + i < p.rows && c0 < width) *reinterpret_cast<uint32_t*>(p.q + (r0 + i) * p.ldq + (c0 >> 1)) = o;
    }
  }
  if constexpr (COLS) {
    // Column c of the tile is 64 bytes, the 4 of rows 8 r8 .. at r8 ^ (c / 8): neighbouring columns' threads meet different banks.
    uint2 packed = {0, 0};
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t byte = f4_scale_byte(by_col[j]);
      (j < 4 ? packed.x : packed.y) |= byte << (8 * (j & 3));
      uint32_t w[W];
      if constexpr (BF16) {
#pragma unroll
        for (int q = 0; q < W; ++q) w[q] = __builtin_amdgcn_perm(v[2 * q + 1][j / 2], v[2 * q][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
      } else {
#pragma unroll
        for (int q = 0; q < W; ++q) w[q] = v[q][j];
      }
      *reinterpret_cast<uint32_t*>(turned + (c8 * kPer + j) * (kTile / 2) + ((r8 ^ c8) * 4)) = pack8<T>(w, byte);
    }
    if ((tid & 48) == 0) *reinterpret_cast<uint2*>(&col_byte[wave][c8 * kPer]) = packed;
  }
  __syncthreads();
  // Scales: a word to a thread, four rows 16 apart.  Rows and blocks that do not exist have 0.
  auto put_scales = [&](uint8_t* table, const uint8_t (*bytes)[kTile], int64_t first, int64_t n, int64_t block0, int64_t blocks, int t) {
    const int r = (t >> 6) * 64 + (t & 15), b = t >> 4 & 3;
    const int64_t R = (n + 63) & ~63LL;
    if (first + (r & 64) >= R) return;
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) w |= (uint32_t)(first + r + 16 * k < n && block0 + b < blocks ? bytes[b][r + 16 * k] : 0) << (8 * k);
    *reinterpret_cast<uint32_t*>(table + (block0 / 4 * R + ((first + r) & ~63LL)) * 4 + b * 64 + (r & 15) * 4) = w;
  };
  if (ROWS && tid < 128) put_scales(p.q_scale, row_byte, row0, p.rows, (int64_t)blockIdx.x * 4, (p.cols + 31) / 32, tid);
  if (COLS && tid >= 128) put_scales(p.qt_scale, col_byte, col0, p.cols, (int64_t)blockIdx.y * 4, (p.rows + 31) / 32, tid - 128);
  if constexpr (COLS) {
    const int64_t width = (p.rows + 31) & ~31LL;
#pragma unroll
    for (int n = 0; n < kTile * kTile / 32 / kThreads; ++n) {
      const int i = n * kThreads + tid, c = i >> 2, piece = (i & 3) * 4, turn = (c >> 3) & 15;
      const uint32_t* const from = reinterpret_cast<const uint32_t*>(turned + c * (kTile / 2));
      if (col0 + c < p.cols && row0 + piece * 8 < width)
        *reinterpret_cast<uint4*>(p.qt + (col0 + c) * p.ldqt + (row0 + piece * 8) / 2) =
            make_uint4(from[piece ^ turn], from[(piece + 1) ^ turn], from[(piece + 2) ^ turn], from[(piece + 3) ^ turn]);
    }
  }
}

}  // namespace

int64_t f4_scale_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0 || rows > (1LL << 30) || cols > (1LL << 30)) return -1;
  return (rows + 63) / 64 * 256 * ((cols + 127) / 128);
}

hipError_t launch_f4_quantize(hipStream_t s, const F4QuantizeArgs& a) {
  const int64_t most = 1LL << 30;
  if ((a.dtype != kF32 && a.dtype != kBF16) || (a.block_rows != 1 && a.block_rows != kBlock)) return hipErrorInvalidValue;
  if (!a.x || (!a.q && !a.qt) || a.rows < 0 || a.cols < 0 || a.rows > most || a.cols > most || a.ldx < a.cols) return hipErrorInvalidValue;
  if ((uintptr_t)a.x & (a.dtype == kBF16 ? 1 : 3)) return hipErrorInvalidValue;
  if (a.q && (!a.q_scale || (((uintptr_t)a.q_scale | (uintptr_t)a.q) & 15) || a.ldq % 32 || a.ldq < a.cols)) return hipErrorInvalidValue;
  if (a.qt && (!a.qt_scale || (((uintptr_t)a.qt_scale | (uintptr_t)a.qt) & 15) || a.ldqt % 32 || a.ldqt < a.rows)) return hipErrorInvalidValue;
  const int64_t gy = (a.rows + kTile - 1) / kTile;
  if (gy > 65535) return hipErrorInvalidValue;
  if (a.rows == 0 || a.cols == 0) return hipSuccess;
  const F4QuantParams p{a.x, a.rows, a.cols, a.ldx, a.ldq / 2, a.ldqt / 2, (uint8_t*)a.q, (uint8_t*)a.qt, a.q_scale, a.qt_scale};
  const dim3 grid((unsigned)((a.cols + kTile - 1) / kTile), (unsigned)gy);
  auto outputs = [&](auto t, auto weight) {
    using T = decltype(t);
    constexpr bool W = decltype(weight)::value;
    if (a.q && a.qt) f4_quantize_kernel<T, W, true, true><<<grid, kThreads, 0, s>>>(p);
    else if (a.q) f4_quantize_kernel<T, W, true, false><<<grid, kThreads, 0, s>>>(p);
    else f4_quantize_kernel<T, W, false, true><<<grid, kThreads, 0, s>>>(p);
  };
  auto blocks = [&](auto t) {
    if (a.block_rows == 1) outputs(t, std::false_type{});
    else outputs(t, std::true_type{});
  };
  if (a.dtype == kF32) blocks(float{});
  else blocks(bf16{});
  return hipGetLastError();
}

}  // namespace pw
