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
// Bound by memory: a block of 256 threads takes 128 x 128 elements, 8 x 8 to a thread, reads them once into registers and writes 8
// consecutive values per lane; the transposed bytes turn in LDS.  What it computes per element is kept to a few operations:
// maxima are taken of the magnitudes' bits, two bf16 at a time, and v_cvt_scalef32_pk_* divides by the scale and rounds two
// values at once.  8192 x 2048 bf16, both outputs, 12.1 to 12.5 us (67 MB, 5.5 TB/s; a copy of 1 GiB reaches 5.15); 2048 x 8192 fp32
// with 128 x 128 blocks 21.3 (101 MB).
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"
#include "quantize_common.hpp"

namespace pw {

namespace {

constexpr int kThreads = 256;
struct QuantParams {
  const void* x;
  int64_t rows, cols, ldx, ldq, ldqt;
  uint8_t *q, *qt, *q_scale, *qt_scale;
};

// Four bytes of v / 2^e from two words of two values.
template <bool E5M2> __device__ __forceinline__ uint32_t pack_bf16(uint32_t lo, uint32_t hi, float scale) {
  s16x2 r = {0, 0};
  const bf16x2 a = __builtin_bit_cast(bf16x2, lo), b = __builtin_bit_cast(bf16x2, hi);
  if constexpr (E5M2) {
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(r, a, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(r, b, scale, true);
  } else {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, a, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, b, scale, true);
  }
  return __builtin_bit_cast(uint32_t, r);
}

// WEIGHT: one scale for the whole 128 x 128 block.  ROWS / COLS: which of the two outputs.
template <class T, bool E5M2, bool WEIGHT, bool ROWS, bool COLS>
__global__ __launch_bounds__(kThreads) void f8_quantize_kernel(QuantParams p) {
  constexpr bool BF16 = sizeof(T) == 2;
  using E = Eight<T>;
  typedef typename E::word word;
  constexpr int W = E::kWords;
  __shared__ __attribute__((aligned(16))) uint32_t col_max[COLS && !WEIGHT ? 4 : 1][kTile];
  __shared__ __attribute__((aligned(16))) uint8_t row_byte[kTile], col_byte[kTile];
  __shared__ __attribute__((aligned(16))) uint8_t turned[COLS ? kTile * kTile : 16];
  const int tid = threadIdx.x, wave = tid >> 6, c8 = tid & 15, r8 = tid >> 4;      // 16 x 16 threads of 8 x 8
  const int64_t row0 = (int64_t)blockIdx.y * kTile, col0 = (int64_t)blockIdx.x * kTile;
  const int64_t r0 = row0 + r8 * kPer, c0 = col0 + c8 * kPer;

  typename E::vec v[kPer];
  load_8x8<T>(v, reinterpret_cast<const T*>(p.x), p.rows, p.cols, p.ldx, row0, col0, r0, c0);

  // Largest magnitudes of the thread's rows and columns; again, of finite values only, in a wave that has others.
  word by_row[kPer], by_col[W];
  auto maxima = [&](auto&& of) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      by_row[i] = of(v[i][0]);
#pragma unroll
      for (int q = 1; q < W; ++q) by_row[i] = E::larger(by_row[i], of(v[i][q]));
    }
    if constexpr (COLS && !WEIGHT) {
#pragma unroll
      for (int q = 0; q < W; ++q) {
        by_col[q] = of(v[0][q]);
#pragma unroll
        for (int i = 1; i < kPer; ++i) by_col[q] = E::larger(by_col[q], of(v[i][q]));
      }
    }
  };
  maxima([](uint32_t x) { return E::magnitude(x); });
  {
    word m = by_row[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) m = E::larger(m, by_row[i]);
    if (__any(!E::is_finite(m))) maxima([](uint32_t x) { return E::finite(E::magnitude(x)); });
  }
  auto bits_of = [](uint32_t m) { return BF16 ? m << 16 : m; };     // of a float
  if constexpr (WEIGHT) {
    word m = by_row[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) m = E::larger(m, by_row[i]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = E::larger(m, from_lane(m, o));
    uint32_t one;
    if constexpr (BF16) one = m[0] > m[1] ? m[0] : m[1];
    else one = m;
    if ((tid & 63) == 0) col_max[0][wave] = bits_of(one);
  } else {
    if constexpr (ROWS) {
      uint32_t row[kPer];
      if constexpr (BF16) {                                          // two rows to a word
#pragma unroll
        for (int i = 0; i < kPer; i += 2) {
          word m = E::larger(u16x2{by_row[i][0], by_row[i + 1][0]}, u16x2{by_row[i][1], by_row[i + 1][1]});
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) m = E::larger(m, from_lane(m, o));
          row[i] = m[0];
          row[i + 1] = m[1];
        }
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          word m = by_row[i];
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) m = E::larger(m, from_lane(m, o));
          row[i] = m;
        }
      }
      uint2 bytes = {0, 0};
#pragma unroll
      for (int i = 0; i < kPer; ++i) (i < 4 ? bytes.x : bytes.y) |= scale_byte<E5M2>(bits_of(row[i])) << (8 * (i & 3));
      if (c8 == 0) *reinterpret_cast<uint2*>(row_byte + r8 * kPer) = bytes;
    }
    if constexpr (COLS) {
#pragma unroll
      for (int q = 0; q < W; ++q) {
        word m = by_col[q];
        m = E::larger(m, from_lane(m, 16));
        m = E::larger(m, from_lane(m, 32));
        if ((tid & 63) < 16) {
          if constexpr (BF16) *reinterpret_cast<uint2*>(&col_max[wave][c8 * kPer + 2 * q]) = make_uint2(bits_of(m[0]), bits_of(m[1]));
          else col_max[wave][c8 * kPer + q] = m;
        }
      }
    }
  }
  __syncthreads();
  if (tid < kTile) {
    if constexpr (WEIGHT) {
      const uint32_t m = max(max(col_max[0][0], col_max[0][1]), max(col_max[0][2], col_max[0][3]));
      row_byte[tid] = col_byte[tid] = (uint8_t)scale_byte<E5M2>(m);
    } else if constexpr (COLS) {
      col_byte[tid] = (uint8_t)scale_byte<E5M2>(max(max(col_max[0][tid], col_max[1][tid]), max(col_max[2][tid], col_max[3][tid])));
    }
  }
  if constexpr (WEIGHT || COLS) __syncthreads();
  // Scales: a word to a thread, four rows 16 apart.  Rows that do not exist have 0.
  auto put_scales = [&](uint8_t* table, const uint8_t* bytes, int64_t first, int64_t n, int64_t block, int t) {
    const int r = (t >> 4) * 64 + (t & 15);
    if (first + (r & 64) >= ((n + 63) & ~63LL)) return;
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) w |= (uint32_t)(first + r + 16 * k < n ? bytes[r + 16 * k] : 0) << (8 * k);
    *reinterpret_cast<uint32_t*>(table + scale_at(first + r, block, n)) = w;
  };
  if (ROWS && tid < 32) put_scales(p.q_scale, row_byte, row0, p.rows, blockIdx.x, tid);
  if (COLS && tid >= 64 && tid < 96) put_scales(p.qt_scale, col_byte, col0, p.cols, blockIdx.y, tid - 64);

  auto scale_of = [](const uint2& b, int i) { return __uint_as_float((((i < 4 ? b.x : b.y) >> (8 * (i & 3))) & 255u) << 23); };
  if constexpr (ROWS) {
    const uint2 b = *reinterpret_cast<const uint2*>(row_byte + r8 * kPer);
    const int64_t width = (p.cols + 15) & ~15LL;          // zeros up to a multiple of 16
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float k = scale_of(b, i);
      uint2 o;
      if constexpr (BF16) o = make_uint2(pack_bf16<E5M2>(v[i][0], v[i][1], k), pack_bf16<E5M2>(v[i][2], v[i][3], k));
      else o = make_uint2(pack_f32<E5M2>(v[i][0], v[i][1], v[i][2], v[i][3], k), pack_f32<E5M2>(v[i][4], v[i][5], v[i][6], v[i][7], k));
      if (r0 + i < p.rows && c0 < width) *reinterpret_cast<uint2*>(p.q + (r0 + i) * p.ldq + c0) = o;
    }
  }
  if constexpr (COLS) {
    // Column c of the tile is 128 bytes, the 8 of rows 8 r8 .. at r8 ^ (c / 8): neighbouring columns' threads meet different banks.
    const uint2 b = *reinterpret_cast<const uint2*>(col_byte + c8 * kPer);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const float k = scale_of(b, j);
      uint2 o;
      if constexpr (BF16) {
        auto two = [&](int i) { return __builtin_amdgcn_perm(v[i + 1][j / 2], v[i][j / 2], j % 2 ? 0x07060302u : 0x05040100u); };
        o = make_uint2(pack_bf16<E5M2>(two(0), two(2), k), pack_bf16<E5M2>(two(4), two(6), k));
      } else {
        o = make_uint2(pack_f32<E5M2>(v[0][j], v[1][j], v[2][j], v[3][j], k), pack_f32<E5M2>(v[4][j], v[5][j], v[6][j], v[7][j], k));
      }
      *reinterpret_cast<uint2*>(turned + (c8 * kPer + j) * kTile + ((r8 ^ c8) * 8)) = o;
    }
    __syncthreads();
    const int64_t width = (p.rows + 15) & ~15LL;
#pragma unroll
    for (int n = 0; n < kTile * kTile / 16 / kThreads; ++n) {
      const int i = n * kThreads + tid, c = i >> 3, piece = (i & 7) * 2, turn = (c >> 3) & 15;
      const uint2 lo = *reinterpret_cast<const uint2*>(turned + c * kTile + ((piece ^ turn) * 8));
      const uint2 hi = *reinterpret_cast<const uint2*>(turned + c * kTile + (((piece + 1) ^ turn) * 8));
      if (col0 + c < p.cols && row0 + piece * 8 < width)
        *reinterpret_cast<uint4*>(p.qt + (col0 + c) * p.ldqt + row0 + piece * 8) = make_uint4(lo.x, lo.y, hi.x, hi.y);
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
  if (a.q && (!a.q_scale || ((uintptr_t)a.q_scale & 3) || ((uintptr_t)a.q & 15) || a.ldq % 16 || a.ldq < a.cols)) return hipErrorInvalidValue;
  if (a.qt && (!a.qt_scale || ((uintptr_t)a.qt_scale & 3) || ((uintptr_t)a.qt & 15) || a.ldqt % 16 || a.ldqt < a.rows)) return hipErrorInvalidValue;
  if (a.rows == 0 || a.cols == 0) return hipSuccess;
  const int64_t gy = (a.rows + kTile - 1) / kTile;
  if (gy > 65535) return hipErrorInvalidValue;
  const QuantParams p{a.x, a.rows, a.cols, a.ldx, a.ldq, a.ldqt, (uint8_t*)a.q, (uint8_t*)a.qt, a.q_scale, a.qt_scale};
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
