// Products of operands in 4-bit floating point (e2m1) with a power-of-two scale for each row and block of 32 along k (f4_quantize.hip),
// with the epilogues of the bf16 products:
//
//   C[m, n] = sum over blocks b of 2^(ea[m, b] + eb[n, b]) sum over k in b of A[m, k] B[n, k],   fp32 accumulation
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 128 k of 4-bit operands in half the time of 8-bit ones: lane 16 q + l holds the 32
// values of row l in block q, 16 bytes, and that block's E8M0 scale.  A product of two e2m1 numbers is a multiple of 1/4 up to 36, eight
// bits, so nothing is lost among the products of a block, unlike in 8 bits (gemm_f8.hip): fp32 outputs come from the same instruction.
#include <type_traits>

#include "common.hpp"
#include "gemm_common.hpp"
#include "gemm_lds.hpp"
#include "kernels.hpp"

namespace pw {

namespace {

struct GemmF4Params {
  const uint8_t *A, *B, *sa, *sb;
  int64_t M, N, K, lda, ldb;              // lda, ldb in bytes
  int tiles_m, tiles_n;
  EpiParams epi;
};

constexpr int kF4BK = 2 * kRowBytes;      // k per tile: two matrix instructions deep
constexpr int kFmt = 4;                   // e2m1

// F32: fp32 outputs; bf16 ones take neither a residual nor an old value: the rest is not compiled.
template <bool F32> __device__ __forceinline__ void narrow(EpiParams& e) {
  e.out_bf16 = !F32;
  if (!F32) e.accumulate = 0;
}
// f(what the epilogue reads besides the bias), uniform over the launch.
template <bool F32, class F> __device__ __forceinline__ void with_extra(const EpiParams& e, F&& f) {
  if (e.mode == kEpiGeluBwd) return f(std::integral_constant<int, kExtraAuxBf16>{});
  if constexpr (F32) {
    if (e.mode == kEpiBiasResidual) return f(std::integral_constant<int, kExtraAuxF32>{});
    if (e.accumulate) return f(std::integral_constant<int, kExtraOldC>{});
  }
  f(std::integral_constant<int, kExtraNone>{});
}

// D[n][m] += B A^T of 128 k; byte IA of sa and IB of sb are the scales (the index has to be a constant).
__device__ __forceinline__ f32x4 mfma(const i32x4& b4, const i32x4& a4, f32x4 c, int ib, int sb, int ia, int sa) {
  const i32x8 b{b4[0], b4[1], b4[2], b4[3], 0, 0, 0, 0}, a{a4[0], a4[1], a4[2], a4[3], 0, 0, 0, 0};
#define PW_F4_CASE(IB, IA) if (ib == IB && ia == IA) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, kFmt, kFmt, IB, sb, IA, sa);
  PW_F4_CASE(0, 0) PW_F4_CASE(0, 1) PW_F4_CASE(0, 2) PW_F4_CASE(0, 3) PW_F4_CASE(1, 0) PW_F4_CASE(1, 1) PW_F4_CASE(1, 2) PW_F4_CASE(1, 3)
  PW_F4_CASE(2, 0) PW_F4_CASE(2, 1) PW_F4_CASE(2, 2) PW_F4_CASE(2, 3) PW_F4_CASE(3, 0) PW_F4_CASE(3, 1) PW_F4_CASE(3, 2)
#undef PW_F4_CASE
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, kFmt, kFmt, 3, sb, 3, sa);
}

// Few rows, and rows too far apart for 32-bit offsets.  What bounds a product of few rows is reading B once, so nothing is
// staged: a block owns 16 columns and 16 rows, its waves take every W-th 128 k, operands go from memory straight into
// fragments (four lanes read 64 consecutive bytes of a row), kAhead steps at a time, and the waves' sums meet in LDS in wave order.
// 1 x 8192 x 2048 4.9 us (3.8 to 4.3 where the operands of one call are those of the next), a launch.
constexpr int kAhead = 4;
template <int W, bool F32>
__global__ __launch_bounds__(64 * W) void gemm_f4_direct_kernel(GemmF4Params p) {
  __shared__ __attribute__((aligned(16))) float part[W][16][16 + 4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, L = lane & 15, g = lane >> 4;
  const int64_t m0 = (int64_t)(blockIdx.x / p.tiles_n) * 16, n0 = (int64_t)(blockIdx.x % p.tiles_n) * 16;
  const int64_t Ra = ((p.M + 63) & ~63LL) * 4, Rb = ((p.N + 63) & ~63LL) * 4;      // bytes of a table for 128 k
  auto in = [](int64_t r, int64_t rows) { return r < rows ? r : rows - 1; };
  auto scale_of = [&](const uint8_t* t, int64_t r) { return t + (r & ~63LL) * 4 + g * 64 + (r & 15) * 4 + ((r & 63) >> 4); };
  const int64_t ra = in(m0 + L, p.M), rb = in(n0 + L, p.N);
  const uint8_t* const pa = p.A + ra * p.lda + 16 * g;
  const uint8_t* const pb = p.B + rb * p.ldb + 16 * g;
  const uint8_t* const qa = scale_of(p.sa, ra);
  const uint8_t* const qb = scale_of(p.sb, rb);
  f32x4 acc = {};
  const int total = (int)((p.K + 127) / 128), blocks = (int)(p.K / 32);
  auto several = [&](int kb, auto count) {
    constexpr int U = decltype(count)::value;
    i32x4 fa[U], fb[U];
    int sa[U], sb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = kb + u * W;
      const bool there = k * 4 + g < blocks;       // a lane's block exists as a whole or not at all
      fa[u] = fb[u] = i32x4{};
      sa[u] = sb[u] = 0;
      if (there) {
        fb[u] = *reinterpret_cast<const i32x4*>(pb + (int64_t)k * 64);
        sb[u] = qb[k * Rb];
        fa[u] = *reinterpret_cast<const i32x4*>(pa + (int64_t)k * 64);
        sa[u] = qa[k * Ra];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) acc = mfma(fb[u], fa[u], acc, 0, sb[u], 0, sa[u]);
  };
  const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
  const bool mine = r < 16 && m0 + r < p.M && n0 + c < p.N;
  EpiParams epi = p.epi;
  narrow<F32>(epi);
  float bias = 0.f;                        // on its way with the operands
  if (mine && epi_has_bias(epi.mode) && epi.bias) bias = epi.bias[n0 + c];
  epi.bias = nullptr;
  int kb = wave;
  for (; kb + (kAhead - 1) * W < total; kb += kAhead * W) several(kb, std::integral_constant<int, kAhead>{});
  for (; kb < total; kb += W) several(kb, std::integral_constant<int, 1>{});
  *reinterpret_cast<f32x4*>(&part[wave][L][4 * g]) = acc;
  __syncthreads();
  if (mine) {
    float v = part[0][r][c];
#pragma unroll
    for (int w = 1; w < W; ++w) v += part[w][r][c];
    epilogue1<true>(epi, m0 + r, n0 + c, v + bias);
  }
}

// WM x WN waves to a tile of WM FM x WN FN blocks of 16 x 16; WK such groups split k between them (WK > 1: of one wave each).
template <int WM_, int WN_, int FM_, int FN_, int WK_, int NS_ = 2>
struct Tile {
  static constexpr int NS = NS_;                                                    // stages of LDS per group
  static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_, WK = WK_, G = WM * WN;
  static constexpr int BM = 16 * WM * FM, BN = 16 * WN * FN, kThreads = 64 * G * WK;
  static constexpr int kScalesA = BM < 64 ? 64 : BM;                                // whole groups of 64 rows
  static constexpr int kHalfScales = (kScalesA + BN) * 4, kPieces = 2 * kHalfScales / 16;   // bytes for 128 k; 16-byte pieces of a tile
  static constexpr int kSets = (kPieces + 63) / 64;                                 // loads by a wave
  static constexpr int kOperands = (BM + BN) * kRowBytes, kStage = kOperands + kSets * 1024;   // the scales lie behind the operands
  static constexpr int kLdP = BN + 4;
  static constexpr size_t kRing = (size_t)WK * NS * kStage;
  static constexpr int kRowsAtOnce = BM < 64 ? BM : 64;                             // of partial sums in LDS, where waves share a tile
  static constexpr size_t kParts = (size_t)(G > 1 ? kRowsAtOnce : WK * BM) * kLdP * 4;
  static constexpr size_t kSmem = (kRing > kParts ? kRing : kParts) + 1023 & ~(size_t)1023;
  static constexpr int kWavesPerSimd = WK == 1 ? 2 : 1;
  static_assert(WK == 1 || G == 1, "groups of one wave only");
  static_assert(kSets <= G && (kPieces % 64 == 0 || kSets == 2), "a wave fetches 64 pieces");
  static_assert(kSmem <= 160 * 1024, "LDS of a compute unit");
};
// What gemm_finish_tile sees of it.
template <class S> struct Finish {
  static constexpr int BM = S::G > 1 ? S::kRowsAtOnce : S::BM, BN = S::BN, WK = S::WK, kThreads = S::kThreads, kLdP = S::kLdP;
};

__device__ __forceinline__ i32x4 read_fragment(uint32_t at) {
  typedef __attribute__((address_space(3))) const i32x4* p;
  return *(p)(uintptr_t)at;
}
__device__ __forceinline__ int read_scales(uint32_t at) {
  typedef __attribute__((address_space(3))) const int* p;
  return *(p)(uintptr_t)at;
}

// ---- whole tiles of 256 x 256, one workgroup to a compute unit, one tile after the other ---------------------------------------------------
// What a launch of one tile per workgroup leaves idle is the time between tiles: the first loads of the next and the way of the
// results out, 10 of 22 us where k = 2048.  So a workgroup keeps its place and the k tiles of its output tiles form one stream: while the
// last k tiles of one are multiplied, the first of the next are on their way into LDS and into the first fragments, and the results
// leave from registers, in stores that nobody waits for.
// What lies behind k in the last k tile is never made zero: scales of 0 (2^-127) on both sides make a product of any two e2m1 numbers vanish
// (36 * 2^-254), so the lanes that would read behind the row read its beginning again, and one loop body serves every k tile.
// No single unit is full.  Where k is long (8192^3 bf16 229 us, 4.8 PFLOP/s) the matrix pipe is busy 61 % of the cycles, of which there are fewer (1.77 GHz,
// against 2.1 to 2.3 in the shorter launches: power), and LDS 29 %; waves stand at waits for 26 % of theirs and wait for their turn 39 %.  A k tile takes 1.6 us
// for 2048 cycles of matrix instructions on a SIMD.  8192 x 8192 x 2048, eight k tiles to an output tile, 74 us, 78 to 83 where no cache holds C: 38 % and 21 %;
// of the 17 us of an output tile about 4 go to converting and storing it.  2048 x 8192 x 8192 fp32 66 to 70 us: 39 % and 24 %.  With a second output (GELU) 98
// us at 8192 x 8192 x 2048, GELU backward 117, fp32 102 to 113, with a residual or an old value 162 to 166.  The fp32 form keeps 10 vector registers in memory.
template <int WM_, int WN_, int FM_, int FN_>
struct Stream {
  static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_, G = WM * WN, kThreads = 64 * G;
  static constexpr int BM = 16 * WM * FM, BN = 16 * WN * FN;
  static constexpr int kHalfScales = (BM + BN) * 4, kPieces = 2 * kHalfScales / 16, kSets = kPieces / 64;
  static constexpr int kOperands = (BM + BN) * kRowBytes, kStage = kOperands + kSets * 1024;
  static constexpr int kBiases = 2;                       // the next output tile's is on its way while one is used
  static constexpr size_t kSmem = 2 * kStage + kBiases * BN * 4;
  static_assert(kSets <= G && G % kSets == 0 && kPieces % 64 == 0 && kSmem <= 160 * 1024);
};

// Four consecutive columns of a row as bf16.
__device__ __forceinline__ uint2 pack4(const f32x4& v) {
  return make_uint2(__builtin_bit_cast(uint32_t, bf16x2{(bf16)v[0], (bf16)v[1]}), __builtin_bit_cast(uint32_t, bf16x2{(bf16)v[2], (bf16)v[3]}));
}
// Lane 16 q + l has columns 16 j + 4 q .. of row l, j = 0, 1; afterwards 8 q .. 8 q + 7 of the 32.
__device__ __forceinline__ uint4 join_columns(uint2 a, uint2 b) {
  auto turn = [](uint32_t& x, uint32_t& y) {
    const auto p = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    const auto r = __builtin_amdgcn_permlane16_swap(p[0], p[1], false, false);
    x = r[0];
    y = r[1];
  };
  turn(a.x, b.x);
  turn(a.y, b.y);
  return make_uint4(a.x, a.y, b.x, b.y);
}

// Results of a wave from registers: acc[i][j] is element (16 i + lane % 16, 16 j + 4 (lane / 16) + r) of its tile at (m0, n0).
// WHOLE: all of it exists; rows leave in pieces of 64 bytes.  Else vectors of four columns where four exist, and elements.
template <int FM, int FN, int KIND, bool F32, bool WHOLE>
__device__ __forceinline__ void store_tile(f32x4 (&acc)[FM][FN], const EpiParams& e, int64_t M, int64_t N, int64_t m0, int64_t n0, int lane) {
  static_assert(FN % 2 == 0);
  const int L = lane & 15, q = lane >> 4;
  const int64_t left = N - n0 - 4 * q;                    // columns from the lane's first on
  const int tail = (int)left & 3, last = left < 0 ? -1 : left >= 16 * FN ? FN : (int)left >> 4;   // the block of columns that the row ends in ...
  const bool odd = tail && last >= 0 && last < FN && left - 16 * last < 4;                   // ... among this lane's four
  const bool two = e.mode == kEpiBiasGelu;
  auto extra = [&](int64_t at) {                          // what the epilogue reads besides
    if constexpr (KIND == kExtraAuxBf16) {
      const uint2 u = *reinterpret_cast<const uint2*>(reinterpret_cast<const bf16*>(e.aux) + at);
      return make_uint4(u.x, u.y, 0, 0);
    } else {
      return *reinterpret_cast<const uint4*>(reinterpret_cast<const float*>(KIND == kExtraOldC ? e.C : e.aux) + at);
    }
  };
  auto with = [&](const f32x4& a, const uint4& x) {
    f32x4 v = a;
    if constexpr (KIND == kExtraAuxBf16) {
      const uint32_t w[2] = {x.x, x.y};
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] *= gelu_grad_f(__uint_as_float(r & 1 ? w[r / 2] & 0xffff0000u : w[r / 2] << 16));
    } else if constexpr (KIND != kExtraNone) {
      v += __builtin_bit_cast(f32x4, x);
    }
    return v;
  };
  auto gelu4 = [](const f32x4& v) { return f32x4{gelu_f(v[0]), gelu_f(v[1]), gelu_f(v[2]), gelu_f(v[3])}; };
  uint4 x[FN];
  auto fetch = [&](int i) {                               // a block of rows ahead
    if constexpr (KIND != kExtraNone) {
      const int64_t row = (m0 + 16 * i + L) * e.ldc + n0 + 4 * q;
#pragma unroll
      for (int j = 0; j < FN; ++j)
        if (WHOLE || (m0 + 16 * i + L < M && 16 * j + 4 <= left)) x[j] = extra(row + 16 * j);
    }
  };
  fetch(0);
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    const int64_t m = m0 + 16 * i + L, row = m * e.ldc + n0;
    f32x4 v[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) v[j] = with(acc[i][j], x[j]);
    if (i + 1 < FM) fetch(i + 1);
    if constexpr (WHOLE) {
      auto put = [&](void* to, auto&& value) {
        if constexpr (F32) {
#pragma unroll
          for (int j = 0; j < FN; ++j) *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(to) + row + 16 * j + 4 * q) = value(j);
        } else {
#pragma unroll
          for (int j = 0; j < FN; j += 2)
            *reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(to) + row + 16 * j + 8 * q) = join_columns(pack4(value(j)), pack4(value(j + 1)));
        }
      };
      put(e.C, [&](int j) { return v[j]; });
      if (two) put(e.C2, [&](int j) { return gelu4(v[j]); });
    } else {
      if (m < M) {
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          if (16 * j + 4 <= left) {
            const int64_t at = row + 16 * j + 4 * q;
            if constexpr (F32) {
              *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(e.C) + at) = v[j];
              if (two) *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(e.C2) + at) = gelu4(v[j]);
            } else {
              *reinterpret_cast<uint2*>(reinterpret_cast<bf16*>(e.C) + at) = pack4(v[j]);
              if (two) *reinterpret_cast<uint2*>(reinterpret_cast<bf16*>(e.C2) + at) = pack4(gelu4(v[j]));
            }
          }
        }
        if (odd) {
          f32x4 a = acc[i][0];
#pragma unroll
          for (int j = 1; j < FN; ++j) a = last == j ? acc[i][j] : a;
          EpiParams bare = e;
          bare.bias = nullptr;
#pragma unroll 1
          for (int r = 0; r < tail; ++r) epilogue1<true>(bare, m, n0 + 16 * last + 4 * q + r, r == 0 ? a[0] : r == 1 ? a[1] : a[2]);
        }
      }
    }
  }
  // What was loaded is there, and the compiler knows: it would wait for everything in every k tile otherwise, the direct loads among it.
  if (KIND != kExtraNone || !WHOLE) __builtin_amdgcn_s_waitcnt(0x0f70);
}

// The same number; what is computed from it is computed where it stands and not kept in registers across the loop.
__device__ __forceinline__ int fresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// The order of tiles, with the columns of each group of eight rows of tiles turned by an eighth of them (by four where that is less): what is written
// at one time is spread over whole rows of C.  Else the eight XCDs write the same few columns of rows that are a power of two apart, which share
// memory channels.  Into arrays that no cache holds, bf16, us, unturned and turned: 8192 x 8192 x 2048 92 and 83, 8192 x 8192 x 8192 251 and 237,
// 16384 x 16384 x 512 219 and 143, 8192 x 7168 x 2048 79.7 and 79.1.
__device__ __forceinline__ void stream_tile(int o, int tiles, int tiles_m, int tiles_n, int& tm, int& tn) {
  tile_of_block(o, tiles, tiles_m, tiles_n, tm, tn);
  tn += tm / 8 * (tiles_n > 32 ? tiles_n / 8 : 4) % tiles_n;
  if (tn >= tiles_n) tn -= tiles_n;
}
template <class S, bool F32>
__global__ __launch_bounds__(S::kThreads, S::G / 4) void gemm_f4_stream_kernel(GemmF4Params p) {
  constexpr int FM = S::FM, FN = S::FN, G = S::G, WN = S::WN;
  using OpA = Operand<S::BM, G, true>;
  using OpB = Operand<S::BN, G, false>;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  narrow<F32>(p.epi);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wm = wave / WN, wn = wave % WN, L = lane & 15, quarter = lane >> 4;
  const int tiles = p.tiles_m * p.tiles_n, n = (int)((p.K + kF4BK - 1) / kF4BK);
  const uint32_t ring = (uint32_t)(uintptr_t)(lds_ptr)smem, biases = ring + 2 * S::kStage;
  const float* const bias = epi_has_bias(p.epi.mode) ? p.epi.bias : nullptr;
  p.epi.bias = nullptr;                                     // in the sums already

  // Where loads are: k tile `kt` of output tile `to`, the `count`-th of this workgroup (at least two k tiles to one).  Scales of a k tile as in the kernel below.
  const int64_t Ra = ((p.M + 63) & ~63LL) * 4, Rb = ((p.N + 63) & ~63LL) * 4;
  const int piece = wave % S::kSets * 64 + lane, half = piece / (S::kPieces / 2), pos = piece % (S::kPieces / 2) * 16;
  const bool of_a = pos < S::BM * 4;
  const int scale_block = half * 4 + (pos >> 6 & 3);
  const int64_t step = of_a ? Ra : Rb;
  OpA oa;
  OpB ob;
  const uint8_t* sq;
  int kt = 0, to = blockIdx.x, count = 0;
  const bool partial = p.K % kF4BK != 0;
  auto begin = [&] {                                        // the loads of output tile `to`
    int tm, tn;
    stream_tile(to, tiles, p.tiles_m, p.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * S::BM, n0 = (int64_t)tn * S::BN;
    const int mine = fresh(lane);
    oa.init(p.A, p.lda, m0, p.M, 0, wave, mine);
    ob.init(p.B, p.ldb, n0, p.N, 0, wave, mine);
    const int64_t row_at = of_a ? m0 * 4 + pos : n0 * 4 + pos - S::BM * 4;
    sq = (of_a ? p.sa : p.sb) + (row_at < step ? row_at : step - 256 + (row_at & 255)) + half * step;
    if (bias) {                                             // 64 columns by a wave, the same ones by several
      const int64_t c = n0 + wave % (S::BN / 64) * 64 + mine;
      dma4(reinterpret_cast<const uint8_t*>(bias + (c < p.N ? c : p.N - 1)), biases + (count % S::kBiases) * (S::BN * 4) + wave % (S::BN / 64) * 256);
    }
  };
  constexpr int kPer = OpA::kPer + OpB::kPer, kLoads = kPer + 1;    // direct loads of a wave per k tile
  constexpr int kSecond = OpA::kPer / 2, kFirst = kPer - kSecond;   // the first: all but the second half of A
  // The last k tile of an output tile is a partial one: lanes whose place in it is behind the row go back to the tile's beginning.
  auto shorten = [&] {
    const int64_t left = (p.K - (int64_t)kt * kF4BK) / 2;
    const int mine = fresh(lane);
#pragma unroll
    for (int j = 0; j < OpB::kPer; ++j) ob.off[j] -= OpB::k_of(OpB::piece(wave, j), mine) < left ? 0 : OpB::k_of(OpB::piece(wave, j), mine);
#pragma unroll
    for (int j = 0; j < OpA::kPer; ++j) oa.off[j] -= OpA::k_of(OpA::piece(wave, j), mine) < left ? 0 : OpA::k_of(OpA::piece(wave, j), mine);
  };
  auto issue_one = [&](int m, uint32_t at) {                // load m of the k tile into the stage at `at`
    const uint32_t st = ring + at;
    if (m < OpB::kPer) ob.issue_one(m, st + S::BM * kRowBytes, wave);
    else oa.issue_one(m - OpB::kPer, st, wave);
    if (m == OpB::kPer - 1) {
      ob.base += kRowBytes;
      const bool there = (int64_t)kt * kF4BK + scale_block * 32 < p.K;
      dma16(there ? sq : reinterpret_cast<const uint8_t*>(kZeros), st + S::kOperands + wave % S::kSets * 1024);
      sq += 2 * step;
    }
    if (m == kPer - 1) {
      oa.base += kRowBytes;
      ++kt;
    }
  };

  const uint32_t row_a = ring + (wm * FM * 16 + L) * kRowBytes, row_b = ring + S::BM * kRowBytes + (wn * FN * 16 + L) * kRowBytes;
  const uint32_t c0 = (quarter ^ (L >> 1)) << 4, c1 = ((quarter + 4) ^ (L >> 1)) << 4;
  constexpr int GA = FM / 4, GB = FN / 4;                   // words of four scales for 128 k
  static_assert(FM % 4 == 0 && FN % 4 == 0);
  const uint32_t s_a = ring + S::kOperands + wm * FM * 64 + lane * 4, s_b = ring + S::kOperands + (S::BM + wn * FN * 16) * 4 + lane * 4;
  // All but the `later` direct loads asked for last are there, and this wave's LDS reads are done; then those of all waves.
  auto landed = [&](auto later) { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(later)::value) : "memory"); };
  auto meet = [&] {
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  f32x4 acc[FM][FN];
  i32x4 fa[2][2], fb[2][FN];                                // [k half][block]
  int sa[2][GA], sb[2][GB], nsa[2][GA], nsb[2][GB];
  struct At { uint32_t v[4]; };
  auto at_of = [&](uint32_t st) {                           // kept whole, so that what is constant in them goes into the instructions
    At r{{row_a + c0 + st, row_a + c1 + st, row_b + c0 + st, row_b + c1 + st}};
#pragma unroll
    for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(r.v[k]));
    return r;
  };
  auto read_a = [&](const At& at, int i) {
#pragma unroll
    for (int h = 0; h < 2; ++h) fa[h][i & 1] = read_fragment(at.v[h] + i * 16 * kRowBytes);
  };
  auto read_b = [&](const At& at, int j, int h) { fb[h][j] = read_fragment(at.v[2 + h] + j * 16 * kRowBytes); };
  auto read_scale = [&](uint32_t st, int g) {
    const int h = g / (GA + GB), w = g % (GA + GB);
    if (w < GA) nsa[h][w] = read_scales(s_a + st + h * S::kHalfScales + w * 256);
    else nsb[h][w - GA] = read_scales(s_b + st + h * S::kHalfScales + (w - GA) * 256);
  };
  auto take_scales = [&] {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int g = 0; g < GA; ++g) sa[h][g] = nsa[h][g];
#pragma unroll
      for (int g = 0; g < GB; ++g) sb[h][g] = nsb[h][g];
    }
  };
  // A k tile: a unit is one block of rows against all columns of the wave.  The next block's fragments are read while a unit runs, the next
  // k tile's columns take the place of this one's as those are used for the last time.  Columns and scales are in registers when the k tile
  // begins, so halfway (kHalf), where the waves meet, the place of the columns and of the first half of the rows is free for the k tile after
  // the next; that of the second half one unit before the end (kTurn), where the next k tile is there.  Loads go out between the MFMAs.
  // No branches inside: the compiler would move MFMAs past them.
  constexpr int kTurn = FM - 1, kHalf = FM / 2 - 1, kSlots = 2 * FN;
  static_assert(2 * (GA + GB) <= kSlots, "a slot for each word of scales");
  auto tile = [&](uint32_t st, uint32_t next) {
    const At here = at_of(st), there = at_of(next);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if (i == kHalf) {
        landed(std::integral_constant<int, kLoads>{});
        meet();
      }
      if (i == kTurn) {
        landed(std::integral_constant<int, kLoads>{});
        meet();
      }
#pragma unroll
      for (int hj = 0; hj < 2 * FN; ++hj) {
        const int h = hj / FN, jj = hj % FN;
        // back and forth: consecutive MFMAs share an operand; the last unit and the next tile's first in one order
        const int j = (i & 1) || i == 0 ? jj : FN - 1 - jj, slot = (i - kTurn) * 2 * FN + hj;
        __builtin_amdgcn_sched_barrier(0);
        if (i < FM - 1 && hj == (i == 0 ? 1 : 0)) read_a(here, i + 1);   // behind the first MFMA of a tile, so that its wait does not cover this
        if (slot >= 0) {
          if (slot < 2 * (GA + GB)) read_scale(next, slot);
          if (slot == 0) read_a(there, 0);
#pragma unroll
          for (int m = slot * kSecond / kSlots; m < (slot + 1) * kSecond / kSlots; ++m) issue_one(kFirst + m, st);
        }
        if (i >= kHalf && i < kTurn) {
          constexpr int slots = (kTurn - kHalf) * 2 * FN;
          const int at = (i - kHalf) * 2 * FN + hj;
#pragma unroll
          for (int m = at * kFirst / slots; m < (at + 1) * kFirst / slots; ++m) issue_one(m, st);
        }
        __builtin_amdgcn_sched_barrier(0);
        acc[i][j] = mfma(fb[h][j], fa[h][i & 1], acc[i][j], j % 4, sb[h][j / 4], i % 4, sa[h][i / 4]);
        if (i == FM - 1) {           // the fragment's last use
          __builtin_amdgcn_sched_barrier(0);
          read_b(there, j, h);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    take_scales();
  };
  begin();
#pragma unroll 1
  for (uint32_t at = 0; at <= S::kStage; at += S::kStage) {
    if (partial && kt == n - 1) shorten();
#pragma unroll
    for (int m = 0; m < kPer; ++m) issue_one(m, at);
  }
  landed(std::integral_constant<int, kLoads + kSecond>{});
  meet();
#pragma unroll
  for (int g = 0; g < 2 * (GA + GB); ++g) read_scale(0, g);
  take_scales();
  {
    const At here = at_of(0);
    read_a(here, 0);
#pragma unroll
    for (int j = 0; j < 2 * FN; ++j) read_b(here, j % FN, j / FN);
  }
  uint32_t st = 0;
  int done = 0;
  for (int o = blockIdx.x; o < tiles; o += gridDim.x, ++done) {
    // Sums begin with the bias, which is in LDS before the first operands are: 128 additions less.
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      typedef __attribute__((address_space(3))) const f32x4* at;
      f32x4 b = {0.f, 0.f, 0.f, 0.f};
      if (bias) b = *(at)(uintptr_t)(biases + (done % S::kBiases) * (S::BN * 4) + (wn * FN * 16 + 16 * j + 4 * (fresh(lane) >> 4)) * 4);
#pragma unroll
      for (int i = 0; i < FM; ++i) acc[i][j] = b;
    }
    for (int t = 0; t < n; ++t) {
      if (t + 2 == n) {                      // loads are two k tiles ahead; behind the last output tile they fetch it once more, for nobody
        if (to + (int)gridDim.x < tiles) to += gridDim.x;
        ++count;
        kt = 0;
        begin();
      }
      if (partial && kt == n - 1) shorten();
      tile(st, S::kStage - st);
      st = S::kStage - st;
    }
    int tm, tn;
    stream_tile(o, tiles, p.tiles_m, p.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * S::BM, n0 = (int64_t)tn * S::BN;
    const bool whole = m0 + S::BM <= p.M && n0 + S::BN <= p.N;
    with_extra<F32>(p.epi, [&](auto kind) {
      constexpr int K = decltype(kind)::value;
      if (whole) store_tile<FM, FN, K, F32, true>(acc, p.epi, p.M, p.N, m0 + wm * FM * 16, n0 + wn * FN * 16, fresh(lane));
      else store_tile<FM, FN, K, F32, false>(acc, p.epi, p.M, p.N, m0 + wm * FM * 16, n0 + wn * FN * 16, fresh(lane));
    });
  }
  landed(std::integral_constant<int, 0>{});  // nothing is on its way into LDS any more
}

// ---- one tile to a workgroup ----------------------------------------------------------------------------------------------------------------------
// Fragments are read one block of rows ahead of their use and MFMAs run across k tiles without a pause.  All of a k tile has been read from
// LDS one unit (a block of rows against all columns of the wave) before its end; there (kTurn) the waves of a group meet, the next k
// tile is there, and the stage of this one is free for k tile t + NS.  What bounds a launch of one round is a chain: loads, k tiles, the waves' sums where they
// share a tile, epilogue (1000 x 760 x 1056 with a residual, 192 tiles of 64 x 64, 6.0 us); 2048 x 2048 x 8192, 256 tiles of 128 x 128, 25.4 us,
// 2.7 PFLOP/s (fp32 29.0).
template <class S, bool F32>
__global__ __launch_bounds__(S::kThreads, S::kWavesPerSimd) void gemm_f4_tile_kernel(GemmF4Params p) {
  constexpr int FM = S::FM, FN = S::FN, G = S::G, WN = S::WN;
  using OpA = Operand<S::BM, G, false>;
  using OpB = Operand<S::BN, G, false>;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  narrow<F32>(p.epi);
  int tm, tn;
  tile_of_block(blockIdx.x, p.tiles_m * p.tiles_n, p.tiles_m, p.tiles_n, tm, tn);
  const int64_t m0 = (int64_t)tm * S::BM, n0 = (int64_t)tn * S::BN;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int grp = wave / G, gw = wave % G, wm = gw / WN, wn = gw % WN, L = lane & 15, quarter = lane >> 4;

  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int total = (int)((p.K + kF4BK - 1) / kF4BK), per = (total + S::WK - 1) / S::WK;
  const int first = grp * per, n = total - first < per ? (total - first < 0 ? 0 : total - first) : per;
  OpA oa;
  OpB ob;
  oa.init(p.A, p.lda, m0, p.M, first, gw, lane);
  ob.init(p.B, p.ldb, n0, p.N, first, gw, lane);
  const uint32_t ring = (uint32_t)(uintptr_t)(lds_ptr)smem + grp * (S::NS * S::kStage);
  // Scales of the tile, 16 bytes (a block's words of four rows) to a lane: for each 128 k first A's groups of 64 rows, then B's.  Every wave
  // fetches 64 pieces, the same ones as another where there are fewer (a branch here would let the compiler move MFMAs
  // past it); groups of 64 rows that do not exist come from the last one.
  const int64_t Ra = ((p.M + 63) & ~63LL) * 4, Rb = ((p.N + 63) & ~63LL) * 4;       // bytes of a table for 128 k
  const int piece = (gw % S::kSets * 64 + lane) % S::kPieces, half = piece / (S::kPieces / 2), pos = piece % (S::kPieces / 2) * 16;
  const bool of_a = pos < S::kScalesA * 4;
  const int64_t step = of_a ? Ra : Rb, row_at = of_a ? (m0 & ~63LL) * 4 + pos : n0 * 4 + pos - S::kScalesA * 4;
  const uint8_t* sq = (of_a ? p.sa : p.sb) + (row_at < step ? row_at : step - 256 + (row_at & 255)) + (2 * (int64_t)first + half) * step;
  const int scale_block = half * 4 + (pos >> 6 & 3);                                // of the tile's eight
  auto issue_scales = [&](int t, uint32_t st, bool whole) {
    const uint32_t to = st + S::kOperands + gw % S::kSets * 1024;
    const bool there = whole || (int64_t)(first + t) * kF4BK + scale_block * 32 < p.K;
    dma16(there ? sq : reinterpret_cast<const uint8_t*>(kZeros), to);
    sq += 2 * step;
  };
  // k tile t into the stage at `at`; zeros where it does not exist.
  auto issue = [&](int t, uint32_t at) {
    const int64_t left = (p.K - (int64_t)(first + t) * kF4BK) / 2;
    const uint32_t st = ring + at;
    ob.issue(left, st + S::BM * kRowBytes, gw, lane);
    ob.base += kRowBytes;
    issue_scales(t, st, false);
    oa.issue(left, st, gw, lane);
    oa.base += kRowBytes;
  };
  // Addresses of this lane's fragments: block j of an operand is 16 j rows of 128 bytes further on, which leaves the swizzle
  // of the row as it is.
  const uint32_t row_a = ring + (wm * FM * 16 + L) * kRowBytes, row_b = ring + S::BM * kRowBytes + (wn * FN * 16 + L) * kRowBytes;
  const uint32_t c0 = (quarter ^ (L >> 1)) << 4, c1 = ((quarter + 4) ^ (L >> 1)) << 4;
  constexpr int GA = (FM + 3) / 4, GB = (FN + 3) / 4;       // words of four scales for 128 k
  const int rows_at = (S::BM < 64 ? (int)(m0 & 63) : 0) + wm * FM * 16, cols_at = wn * FN * 16;   // of this wave, in the words' groups
  const uint32_t s_a = ring + S::kOperands + (rows_at & ~63) * 4 + lane * 4, s_b = ring + S::kOperands + (S::kScalesA + (cols_at & ~63)) * 4 + lane * 4;
  // A wave of fewer than 64 rows (columns) begins with a later byte of its word.
  auto word_a = [&](int v) { return FM % 4 ? v >> ((rows_at & 63) / 2) : v; };
  auto word_b = [&](int v) { return FN % 4 ? v >> ((cols_at & 63) / 2) : v; };
  constexpr int kPer = OpA::kPer + OpB::kPer, kLoads = kPer + 1;    // direct loads of a wave per k tile
  // All but the `later` direct loads asked for last are there, and this wave's LDS reads are done ...
  auto landed = [&](auto later) { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(later)::value) : "memory"); };
  auto meet = [&] {                            // ... and those of the group's other waves
    if (G > 1) __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  i32x4 fa[2][2], fb[2][FN];                   // [k half][block]
  int sa[2][GA], sb[2][GB], nsa[2][GA], nsb[2][GB];
  // Addresses of a tile's fragments: kept whole, so that what is constant in them goes into the instructions.
  struct At { uint32_t v[4]; };
  auto at_of = [&](uint32_t st) {
    At r{{row_a + c0 + st, row_a + c1 + st, row_b + c0 + st, row_b + c1 + st}};
#pragma unroll
    for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(r.v[k]));
    return r;
  };
  auto read_a = [&](const At& at, int i) {
#pragma unroll
    for (int h = 0; h < 2; ++h) fa[h][i & 1] = read_fragment(at.v[h] + i * 16 * kRowBytes);
  };
  auto read_b = [&](const At& at, int j, int h) { fb[h][j] = read_fragment(at.v[2 + h] + j * 16 * kRowBytes); };
  auto read_scale = [&](uint32_t st, int g) {
    const int h = g / (GA + GB), w = g % (GA + GB);
    if (w < GA) nsa[h][w] = read_scales(s_a + st + h * S::kHalfScales + w * 256);
    else nsb[h][w - GA] = read_scales(s_b + st + h * S::kHalfScales + (w - GA) * 256);
  };
  auto take_scales = [&] {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int g = 0; g < GA; ++g) sa[h][g] = word_a(nsa[h][g]);
#pragma unroll
      for (int g = 0; g < GB; ++g) sb[h][g] = word_b(nsb[h][g]);
    }
  };
  auto issue_one = [&](int t, int m, uint32_t at) {       // load m of the whole tile t
    const uint32_t st = ring + at;
    if (m < OpB::kPer) ob.issue_one(m, st + S::BM * kRowBytes, gw);
    else oa.issue_one(m - OpB::kPer, st, gw);
    if (m == OpB::kPer - 1) {
      ob.base += kRowBytes;
      issue_scales(t, st, true);
    }
    if (m == kPer - 1) oa.base += kRowBytes;
  };
  // STREAM: tile t + NS is a whole one; MORE: tile t + 1 exists (t + NS, where it does not, is made of zeros nobody reads).  No
  // branches inside: the compiler would move MFMAs past them.
  constexpr int kTurn = FM - 1, kSlots = (FM - kTurn) * 2 * FN;
  static_assert(FM % 2 == 0 && 2 * (GA + GB) <= 2 * FN, "two fragments of rows in turn; a slot for each word of scales");
  auto tile = [&](int t, uint32_t st, uint32_t next, auto streaming, auto follows) {
    constexpr bool STREAM = decltype(streaming)::value, more = decltype(follows)::value;
    const At here = at_of(st), there = at_of(next);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if (i == kTurn && more) {
        landed(std::integral_constant<int, (S::NS - 2) * kLoads>{});
        meet();
        if (!STREAM) issue(t + S::NS, st);
      }
#pragma unroll
      for (int hj = 0; hj < 2 * FN; ++hj) {
        const int h = hj / FN, jj = hj % FN;
        // back and forth: consecutive MFMAs share an operand; the last unit and the next tile's first in one order
        const int j = (i & 1) || i == 0 ? jj : FN - 1 - jj, slot = (i - kTurn) * 2 * FN + hj;
        __builtin_amdgcn_sched_barrier(0);
        if (i < FM - 1 && hj == (i == 0 ? 1 : 0)) read_a(here, i + 1);   // behind the first MFMA of a tile, so that its wait does not cover this
        if (slot >= 0 && more) {
          if (slot < 2 * (GA + GB)) read_scale(next, slot);
          if (slot == 0) read_a(there, 0);
          if (STREAM) {
#pragma unroll
            for (int m = slot * kPer / kSlots; m < (slot + 1) * kPer / kSlots; ++m) issue_one(t + S::NS, m, st);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        acc[i][j] = mfma(fb[h][j], fa[h][i & 1], acc[i][j], j % 4, sb[h][j / 4], i % 4, sa[h][i / 4]);
        if (i == FM - 1 && more) {           // the fragment's last use
          __builtin_amdgcn_sched_barrier(0);
          read_b(there, j, h);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) take_scales();
  };
  // A whole tile's bias is added before the staging: it comes during the last k tile, whose waits it only makes stricter.
  constexpr bool kBias = G > 1 && FN % 4 == 0;
  const bool whole = kBias && m0 + S::BM <= p.M && n0 + S::BN <= p.N, biased = whole && epi_has_bias(p.epi.mode) && p.epi.bias;
  f32x4 bias[FN];
  auto load_bias = [&] {
    if (!biased) return;
#pragma unroll
    for (int j = 0; j < FN; ++j) bias[j] = *reinterpret_cast<const f32x4*>(p.epi.bias + n0 + wn * FN * 16 + 4 * quarter + 16 * j);
  };
  if (n > 0) {
#pragma unroll
    for (int i = 0; i < S::NS; ++i) issue(i, i * S::kStage);
    landed(std::integral_constant<int, (S::NS - 1) * kLoads>{});
    meet();
#pragma unroll
    for (int g = 0; g < 2 * (GA + GB); ++g) read_scale(0, g);
    take_scales();
    const At here = at_of(0);
    read_a(here, 0);
#pragma unroll
    for (int j = 0; j < 2 * FN; ++j) read_b(here, j % FN, j / FN);
    constexpr std::true_type yes;
    constexpr std::false_type no;
    int t = 0;
    uint32_t st = 0;
    auto after = [](uint32_t at) { return at == (S::NS - 1) * S::kStage ? 0u : at + S::kStage; };
    for (; t + S::NS + 1 < n; ++t) {           // the last tile may be a partial one
      tile(t, st, after(st), yes, yes);
      st = after(st);
    }
    for (; t + 1 < n; ++t) {
      tile(t, st, after(st), no, yes);
      st = after(st);
    }
    if constexpr (kBias) load_bias();
    tile(t, st, 0, no, no);
    landed(std::integral_constant<int, 0>{});  // nothing is on its way into LDS any more
  } else if constexpr (kBias) {
    load_bias();
  }

  __syncthreads();
  float* const parts = reinterpret_cast<float*>(smem);
  auto finish = [&](int64_t m) {
    with_extra<F32>(p.epi, [&](auto kind) { gemm_finish_tile<Finish<S>, decltype(kind)::value>(parts, p, m, n0); });
  };
  if constexpr (kBias) {
    if (whole) {
      if (biased) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[i][j] += bias[j];
        p.epi.bias = nullptr;
      }
      with_extra<F32>(p.epi, [&](auto kind) {
        gemm_epilogue_staged_kind<FM / 2, FN / 2, decltype(kind)::value>(reinterpret_cast<bf16*>(smem), acc, p, m0 + wm * FM * 16,
                                                                         n0 + wn * FN * 16, wave, lane);
      });
      return;
    }
  }
  if constexpr (G == 1) {
    float* mine = parts + (grp * S::BM + L) * S::kLdP + 4 * quarter;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) *reinterpret_cast<f32x4*>(mine + 16 * i * S::kLdP + 16 * j) = acc[i][j];
    finish(m0);
  } else {
    constexpr int kAt = S::kRowsAtOnce / 16;     // blocks of rows that are in LDS at a time
#pragma unroll
    for (int c = 0; c < S::BM / S::kRowsAtOnce; ++c) {
#pragma unroll
      for (int i = 0; i < kAt; ++i) {
        constexpr int kPerWave = FM;
        const int blk = c * kAt + i;
        if (blk / kPerWave == wm) {
          float* mine = parts + (16 * i + L) * S::kLdP + wn * FN * 16 + 4 * quarter;
#pragma unroll
          for (int j = 0; j < FN; ++j) *reinterpret_cast<f32x4*>(mine + 16 * j) = acc[blk % kPerWave][j];
        }
      }
      if (m0 + c * S::kRowsAtOnce < p.M) finish(m0 + c * S::kRowsAtOnce);
      __syncthreads();
    }
  }
}

using Big = Stream<2, 4, 8, 4>;         // 256 x 256
using Mid = Tile<2, 2, 4, 4, 1>;        // 128 x 128, two workgroups to a compute unit
using Half = Tile<2, 2, 4, 2, 1, 3>;    // 128 x 64
using Split = Tile<1, 1, 4, 4, 4>;      // 64 x 64, k over four waves
using Few = Tile<1, 1, 2, 4, 4, 2>;     // 32 x 64, likewise

constexpr int kUnits = 256;             // compute units
hipError_t prepare_big() {
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(gemm_f4_stream_kernel<Big, false>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)Big::kSmem);
  return e != hipSuccess ? e : hipFuncSetAttribute(reinterpret_cast<const void*>(gemm_f4_stream_kernel<Big, true>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)Big::kSmem);
}
hipError_t launch_big(hipStream_t s, GemmF4Params p, bool f32) {
  const int64_t tm = (p.M + Big::BM - 1) / Big::BM, tn = (p.N + Big::BN - 1) / Big::BN;
  if (tm * tn > (1LL << 30)) return hipErrorInvalidValue;
  p.tiles_m = (int)tm;
  p.tiles_n = (int)tn;
  const int blocks = tm * tn < kUnits ? (int)(tm * tn) : kUnits;
  if (f32) gemm_f4_stream_kernel<Big, true><<<blocks, Big::kThreads, Big::kSmem, s>>>(p);
  else gemm_f4_stream_kernel<Big, false><<<blocks, Big::kThreads, Big::kSmem, s>>>(p);
  return hipGetLastError();
}
template <class S>
hipError_t prepare() {
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(gemm_f4_tile_kernel<S, false>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem);
  return e != hipSuccess ? e : hipFuncSetAttribute(reinterpret_cast<const void*>(gemm_f4_tile_kernel<S, true>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem);
}
constexpr int64_t kMostThreads = (1LL << 32) - 1;     // of a launch
template <class S>
hipError_t launch(hipStream_t s, GemmF4Params p, bool f32) {
  const int64_t tm = (p.M + S::BM - 1) / S::BM, tn = (p.N + S::BN - 1) / S::BN;
  if (tm * tn * S::kThreads > kMostThreads) return hipErrorInvalidValue;
  p.tiles_m = (int)tm;
  p.tiles_n = (int)tn;
  if (f32) gemm_f4_tile_kernel<S, true><<<(int)(tm * tn), S::kThreads, S::kSmem, s>>>(p);
  else gemm_f4_tile_kernel<S, false><<<(int)(tm * tn), S::kThreads, S::kSmem, s>>>(p);
  return hipGetLastError();
}
template <int W>
hipError_t launch_direct(hipStream_t s, GemmF4Params p, bool f32) {
  const int64_t tm = (p.M + 15) / 16, tn = (p.N + 15) / 16;
  if (tm * tn * 64 * W > kMostThreads) return hipErrorInvalidValue;
  p.tiles_m = (int)tm;
  p.tiles_n = (int)tn;
  if (f32) gemm_f4_direct_kernel<W, true><<<(int)(tm * tn), 64 * W, 0, s>>>(p);
  else gemm_f4_direct_kernel<W, false><<<(int)(tm * tn), 64 * W, 0, s>>>(p);
  return hipGetLastError();
}
enum Kernel { kDirect4, kDirect8, kFew, kSplit, kHalf, kMid, kBig };
// Which shape: the largest whose tiles give every compute unit one, as a launch of up to one round takes as long as one tile.  Measured in us on both
// sides of each step, on one set of data (k = 2048 unless it says so, bf16; other k from 288 on and fp32 outputs follow the same steps, whose
// places were not measured for them):
//   few rows and columns straight from memory, up to 512 blocks of 16 x 16 (1 x 8192 3.8, as tiles of 32 x 64 4.4, 16 x 8192 4.5 and 4.5; beyond, 1 x 16384
//     5.0 and 4.5, 3 x 32768 9.1 and 8.0), up to 256 if k is long (16 x 4096 x 4096 4.5 and 5.2, x 8192 7.2 and 6.8; beyond, 16 x 8192 x 4096 6.6 and 5.2,
//     128 x 1024 x 16384 19.8 and 10.0); eight waves share a long k (16 x 4096 x 8192 7.2, four 7.7), four a short one (3 x 32768 9.1, eight 11.6);
//   32 x 64 up to 256 tiles (256 x 2048 4.6, as 64 x 64 5.6; 1024 x 1024 7.6 and 5.8), 64 x 64 up to 256 (1024 x 1024 5.8, as 128 x 64 6.8; 1024 x 2048
//     10.0 and 7.2), 128 x 64 up to 256 (1024 x 2048 7.2, as 128 x 128 8.5; 2048 x 2048 10.5 and 9.3);
//   128 x 128 is there twice on a unit, so up to 128 tiles of 256 x 256 it needs one round (2816 x 2816, 121 of them, 14.7, as 256 x 256 19.3; 2816 x 3000,
//     132, 21.1 and 18.5); a second round of 256 x 256 that few units have part in costs more than the third of 128 x 128 (4096 x 5120, 320, 34.4 and 32.5;
//     4096 x 5376, 336, 35.4 and 36.3); from the third on it does not (8192 x 4608, 576, 56.0 and 56.1; 8192 x 8448, 1056, 92 and 100).
//   Operands of one row or column of tiles: half of a tile of 256 x 256 would be empty (128 x 131072 45.4, as 128 x 128 33.9; 131072 x 128 43.4 and 32.9;
//     131072 x 100, whose rows of C do not end with a tile, 39.6 and 46.9), and of 128 x 128 (131072 x 60 45.3, as 128 x 64 35.1).
Kernel choose(int64_t M, int64_t N, int64_t K, bool far_apart) {
  auto tiles = [&](int m, int n) { return ((M + m - 1) / m) * ((N + n - 1) / n); };
  const bool deep = K >= 4096;
  if (tiles(16, 16) <= (deep ? 256 : 512) || far_apart) return deep ? kDirect8 : kDirect4;
  if (tiles(Few::BM, Few::BN) <= 256) return kFew;
  if (tiles(Split::BM, Split::BN) <= 256) return kSplit;
  if (tiles(Half::BM, Half::BN) <= 256 || N <= Half::BN) return kHalf;
  const int64_t big = tiles(Big::BM, Big::BN);
  return K > kF4BK && M > Mid::BM && N != Mid::BN && big > 128 && (big <= 256 || big >= 336) ? kBig : kMid;
}
bool rows_far_apart(const GemmF4Args& a) { return a.lda / 2 > kMaxLd || a.ldb / 2 > kMaxLd; }

}  // namespace

hipError_t gemm_f4_init() {
  hipError_t e = prepare_big();
  if (e == hipSuccess) e = prepare<Mid>();
  if (e == hipSuccess) e = prepare<Half>();
  if (e == hipSuccess) e = prepare<Split>();
  if (e == hipSuccess) e = prepare<Few>();
  return e;
}

const char* gemm_f4_kernel(const GemmF4Args& a) {
  static const char* const names[] = {"direct, 4 waves", "direct, 8 waves", "32 x 64", "64 x 64", "128 x 64", "128 x 128", "256 x 256"};
  return names[choose(a.M, a.N, a.K, rows_far_apart(a))];
}

hipError_t launch_gemm_f4(hipStream_t s, const GemmF4Args& a) {
  const int64_t most = 1LL << 26;
  if (!a.A || !a.B || !a.a_scale || !a.b_scale || !a.C || a.M < 0 || a.N < 0 || a.K < 0 || a.M > most || a.N > most || a.K > (1LL << 30))
    return hipErrorInvalidValue;
  if (a.epilogue < kEpiStore || a.epilogue > kEpiGeluBwd || (a.out_dtype != kF32 && a.out_dtype != kBF16)) return hipErrorInvalidValue;
  if (a.K % 32 || a.lda % 32 || a.ldb % 32 || a.ldc % 8 || a.lda < a.K || a.ldb < a.K || a.ldc < a.N) return hipErrorInvalidValue;
  if (((uintptr_t)a.A | (uintptr_t)a.B | (uintptr_t)a.C | (uintptr_t)a.C2 | (uintptr_t)a.aux | (uintptr_t)a.bias | (uintptr_t)a.a_scale |
       (uintptr_t)a.b_scale) & 15) return hipErrorInvalidValue;
  if ((a.epilogue == kEpiBiasResidual || a.epilogue == kEpiGeluBwd) && !a.aux) return hipErrorInvalidValue;
  if (a.epilogue == kEpiBiasGelu && !a.C2) return hipErrorInvalidValue;
  if (a.accumulate && (a.out_dtype != kF32 || a.epilogue != kEpiStore)) return hipErrorInvalidValue;
  if (a.epilogue == kEpiBiasResidual && a.out_dtype != kF32) return hipErrorInvalidValue;
  if (a.M == 0 || a.N == 0) return hipSuccess;
  GemmF4Params p{};
  p.A = (const uint8_t*)a.A; p.B = (const uint8_t*)a.B; p.sa = a.a_scale; p.sb = a.b_scale;
  p.M = a.M; p.N = a.N; p.K = a.K; p.lda = a.lda / 2; p.ldb = a.ldb / 2;
  p.epi.mode = a.epilogue; p.epi.out_bf16 = a.out_dtype == kBF16; p.epi.accumulate = a.accumulate;
  p.epi.bias = a.bias; p.epi.aux = a.aux; p.epi.C = a.C; p.epi.C2 = a.C2; p.epi.ldc = a.ldc;
  const bool f32 = a.out_dtype == kF32;
  switch (choose(a.M, a.N, a.K, rows_far_apart(a))) {
    case kDirect4: return launch_direct<4>(s, p, f32);
    case kDirect8: return launch_direct<8>(s, p, f32);
    case kFew: return launch<Few>(s, p, f32);
    case kSplit: return launch<Split>(s, p, f32);
    case kHalf: return launch<Half>(s, p, f32);
    case kMid: return launch<Mid>(s, p, f32);
    case kBig: return launch_big(s, p, f32);
  }
  return hipErrorInvalidValue;
}

}  // namespace pw
