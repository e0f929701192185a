// Products of operands in 8-bit floating point with a power-of-two scale for each row and block of 128 along k
// (f8_quantize.hip), with the epilogues of the bf16 products:
//
//   C[m, n] = sum over blocks b of 2^(ea[m, b] + eb[n, b]) sum over k in b of A[m, k] B[n, k],   fp32 accumulation
//
// bf16 outputs come from v_mfma_scale_f32_16x16x128_f8f6f4, whose k depth is the block length: one instruction takes both
// operands' scales with it.  Lane l holds row l % 16 of its operand and 32 of the block's 128 k, and the E8M0 scale of that row;
// which 32 is the same for both operands, and all of a row's share one scale, so any order of k that both sides agree on is right.
//
// That pipe adds products in groups of eight consecutive k, aligned to the largest of the group and cut off 2^-13 below it
// (found with one large and one small product, and the same for every 8-bit matrix instruction, scaled or not): the sum is
// off by up to 7 * 2^-13 of sum |a b|, and by 1e-5 to 3e-5 of the result in the norm - far below the 2^-9 of a bf16 output and
// below what the operands' own rounding did (4e-2), but not fp32.  fp32 outputs are therefore formed on the bf16 pipe: a value
// q 2^e has at most four significant bits, so it is a bf16 number (exactly, within 2^-126 .. 2^127), its products are exact in
// fp32, and v_cvt_scalef32_pk_bf16_* makes two of them from two bytes with the scale applied.
#include <type_traits>

#include "common.hpp"
#include "gemm_common.hpp"
#include "kernels.hpp"

namespace pw {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct GemmF8Params {
  const uint8_t *A, *B, *sa, *sb;
  int64_t M, N, K, lda, ldb;
  int tiles_m, tiles_n;
  EpiParams epi;
};

// Bytes 4 d .. 4 d + 3 of a fragment as bf16 numbers, times 2^(byte - 127).
template <int FMT> __device__ __forceinline__ bf16x4 widen(int d, int scale_byte) {
  const float k = __uint_as_float((uint32_t)scale_byte << 23);
  bf16x2 lo, hi;
  if constexpr (FMT == 0) {
    lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d, k, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d, k, true);
  } else {
    lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(d, k, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(d, k, true);
  }
  return bf16x4{lo[0], lo[1], hi[0], hi[1]};
}
template <int FMT> __device__ __forceinline__ bf16x8 widen8(const i32x8& f, int s, int scale_byte) {
  const bf16x4 a = widen<FMT>(f[2 * s], scale_byte), b = widen<FMT>(f[2 * s + 1], scale_byte);
  return bf16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

template <int FA, int FB, bool EXACT>
__global__ __launch_bounds__(256) void gemm_f8_kernel(GemmF8Params p) {
  int tm, tn;
  tile_of_block(blockIdx.x, p.tiles_m * p.tiles_n, p.tiles_m, p.tiles_n, tm, tn);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, L = lane & 15, g = lane >> 4;
  const int64_t m0 = (int64_t)tm * 64 + (wave >> 1) * 32, n0 = (int64_t)tn * 64 + (wave & 1) * 32;
  const int64_t Ra = (p.M + 63) & ~63LL, Rb = (p.N + 63) & ~63LL;
  f32x4 acc[2][2] = {};
  for (int64_t k0 = 0, kb = 0; k0 < p.K; k0 += 128, ++kb) {
    i32x8 fa[2], fb[2];
    int sa[2], sb[2];
    auto load = [&](const uint8_t* base, int64_t ld, int64_t row, int64_t rows, i32x8& f) {
      if (row >= rows) row = rows - 1;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t k = k0 + 16 * (g + 4 * h);
        i32x4 v = {};
        if (k < p.K) v = *reinterpret_cast<const i32x4*>(base + row * ld + k);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[4 * h + e] = v[e];
      }
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t ra = m0 + 16 * i + L, rb = n0 + 16 * i + L;
      load(p.A, p.lda, ra, p.M, fa[i]);
      load(p.B, p.ldb, rb, p.N, fb[i]);
      sa[i] = p.sa[kb * Ra + (ra & ~63LL) + (ra & 15) * 4 + ((ra & 63) >> 4)];
      sb[i] = p.sb[kb * Rb + (rb & ~63LL) + (rb & 15) * 4 + ((rb & 63) >> 4)];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if constexpr (EXACT) {
#pragma unroll
          for (int s = 0; s < 4; ++s)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8<FB>(fb[j], s, sb[j]), widen8<FA>(fa[i], s, sa[i]), acc[i][j], 0, 0, 0);
        } else {
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[j], fa[i], acc[i][j], FB, FA, 0, sb[j], 0, sa[i]);
        }
      }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t m = m0 + 16 * i + L, n = n0 + 16 * j + 4 * g + r;
        if (m < p.M && n < p.N) epilogue1<true>(p.epi, m, n, acc[i][j][r]);
      }
}

}  // namespace

hipError_t launch_gemm_f8(hipStream_t s, const GemmF8Args& a) {
  const int64_t most = 1LL << 30;
  if (!a.A || !a.B || !a.a_scale || !a.b_scale || !a.C || a.M < 0 || a.N < 0 || a.K < 0 || a.M > most || a.N > most || a.K > most)
    return hipErrorInvalidValue;
  if ((a.a_format != kE4M3 && a.a_format != kE5M2) || (a.b_format != kE4M3 && a.b_format != kE5M2)) return hipErrorInvalidValue;
  if (a.epilogue < kEpiStore || a.epilogue > kEpiGeluBwd || (a.out_dtype != kF32 && a.out_dtype != kBF16)) return hipErrorInvalidValue;
  if (a.K % 16 || a.lda % 16 || a.ldb % 16 || a.ldc % 8 || a.lda < a.K || a.ldb < a.K || a.ldc < a.N) return hipErrorInvalidValue;
  if (((uintptr_t)a.A | (uintptr_t)a.B | (uintptr_t)a.C | (uintptr_t)a.C2 | (uintptr_t)a.aux | (uintptr_t)a.bias) & 15) return hipErrorInvalidValue;
  if (((uintptr_t)a.a_scale | (uintptr_t)a.b_scale) & 3) return hipErrorInvalidValue;
  if ((a.epilogue == kEpiBiasResidual || a.epilogue == kEpiGeluBwd) && !a.aux) return hipErrorInvalidValue;
  if (a.epilogue == kEpiBiasGelu && !a.C2) return hipErrorInvalidValue;
  if (a.accumulate && (a.out_dtype != kF32 || a.epilogue != kEpiStore)) return hipErrorInvalidValue;
  if (a.epilogue == kEpiBiasResidual && a.out_dtype != kF32) return hipErrorInvalidValue;
  if (a.M == 0 || a.N == 0) return hipSuccess;
  GemmF8Params p{};
  p.A = (const uint8_t*)a.A; p.B = (const uint8_t*)a.B; p.sa = a.a_scale; p.sb = a.b_scale;
  p.M = a.M; p.N = a.N; p.K = a.K; p.lda = a.lda; p.ldb = a.ldb;
  p.epi.mode = a.epilogue; p.epi.out_bf16 = a.out_dtype == kBF16; p.epi.accumulate = a.accumulate;
  p.epi.bias = a.bias; p.epi.aux = a.aux; p.epi.C = a.C; p.epi.C2 = a.C2; p.epi.ldc = a.ldc;
  const int64_t tm = (a.M + 63) / 64, tn = (a.N + 63) / 64;
  if (tm * tn > (1LL << 26)) return hipErrorInvalidValue;
  p.tiles_m = (int)tm;
  p.tiles_n = (int)tn;
  const int grid = (int)(tm * tn);
  auto go = [&](auto fa, auto fb) {
    constexpr int A = decltype(fa)::value, B = decltype(fb)::value;
    if (a.out_dtype == kF32) gemm_f8_kernel<A, B, true><<<grid, 256, 0, s>>>(p);
    else gemm_f8_kernel<A, B, false><<<grid, 256, 0, s>>>(p);
  };
  using e4m3 = std::integral_constant<int, 0>;
  using e5m2 = std::integral_constant<int, 1>;
  if (a.a_format == kE4M3) a.b_format == kE4M3 ? go(e4m3{}, e4m3{}) : go(e4m3{}, e5m2{});
  else a.b_format == kE4M3 ? go(e5m2{}, e4m3{}) : go(e5m2{}, e5m2{});
  return hipGetLastError();
}

}  // namespace pw
