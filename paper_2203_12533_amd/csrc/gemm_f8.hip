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

// EXACT kernels have fp32 outputs and the others bf16 ones, which take neither a residual nor an old value: the rest is not compiled.
template <bool EXACT> __device__ __forceinline__ void narrow(EpiParams& e) {
  e.out_bf16 = !EXACT;
  if (!EXACT) e.accumulate = 0;
}
// f(what the epilogue reads besides the bias), uniform over the launch.
template <bool EXACT, class F> __device__ __forceinline__ void with_extra(const EpiParams& e, F&& f) {
  if (e.mode == kEpiGeluBwd) return f(std::integral_constant<int, kExtraAuxBf16>{});
  if constexpr (EXACT) {
    if (e.mode == kEpiBiasResidual) return f(std::integral_constant<int, kExtraAuxF32>{});
    if (e.accumulate) return f(std::integral_constant<int, kExtraOldC>{});
  }
  f(std::integral_constant<int, kExtraNone>{});
}

typedef __attribute__((address_space(3))) void* lds_ptr;
constexpr int kBK = 128;                  // k per tile: the length that shares a scale
constexpr int64_t kMaxLd = 1 << 23;       // rows of a tile are within 32 bits of byte offset

__device__ __attribute__((aligned(16))) const uint32_t kZeros[4] = {0, 0, 0, 0};

// Bytes from global memory straight into LDS at lds_off + 16 (4) * lane.
__device__ __forceinline__ void dma16(const uint8_t* g, uint32_t lds_off) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(g), "s"(lds_off) : "memory", "m0");
}
__device__ __forceinline__ void dma16_s(const uint8_t* base, uint32_t off, uint32_t lds_off) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(lds_off) : "memory", "m0");
}
__device__ __forceinline__ void dma4(const uint8_t* g, uint32_t lds_off) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(g), "s"(lds_off) : "memory", "m0");
}

// WM x WN waves to a tile of WM FM x WN FN blocks of 16 x 16; WK such groups split k between them (WK > 1: of one wave each).
template <int WM_, int WN_, int FM_, int FN_, int WK_, int NS_ = 2>
struct Tile {
  static constexpr int NS = NS_;                                                    // stages of LDS per group
  static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_, WK = WK_, G = WM * WN;
  static constexpr int BM = 16 * WM * FM, BN = 16 * WN * FN, kThreads = 64 * G * WK;
  static constexpr int kScalesA = BM < 64 ? 64 : BM, kScales = kScalesA + BN;       // bytes: whole groups of 64 rows
  static constexpr int kOperands = (BM + BN) * kBK, kStage = kOperands + (kScales + 255) / 256 * 256;   // the scales lie behind the operands
  static constexpr int kLdP = BN + 4;
  static constexpr size_t kRing = (size_t)WK * NS * kStage;
  static constexpr int kRowsAtOnce = BM < 64 ? BM : 64;                             // of partial sums in LDS, where waves share a tile
  static constexpr size_t kParts = (size_t)(G > 1 ? kRowsAtOnce : WK * BM) * kLdP * 4;
  static constexpr size_t kSmem = (kRing > kParts ? kRing : kParts) + 1023 & ~(size_t)1023;
  static constexpr int kWavesPerSimd = WK == 1 ? 2 : 1;
  static_assert(WK == 1 || G == 1, "groups of one wave only");
};
// What gemm_finish_tile sees of it.
template <class S> struct Finish {
  static constexpr int BM = S::G > 1 ? S::kRowsAtOnce : S::BM, BN = S::BN, WK = S::WK, kThreads = S::kThreads, kLdP = S::kLdP;
};

// One operand of a group's tile: R rows of 128 bytes, fetched by G waves in pieces of 1 KiB (8 rows); chunk c (16 bytes) of row
// r lies at position c ^ ((r >> 1) & 7) of the row, so that the 16 rows of a fragment read hit all banks.
// HALVES: the first half of a wave's pieces are the first 64 of each 128 rows.
template <int R, int G, bool HALVES>
struct Operand {
  static constexpr int kPer = R / 8 / G;
  static_assert(!HALVES || (G == 8 && kPer == 4), "two times 128 rows");
  __device__ __forceinline__ static int piece(int gw, int j) {
    return HALVES ? (gw >> 2) * 16 + (j >> 1) * 8 + (gw & 3) * 2 + (j & 1) : gw * kPer + j;
  }
  const uint8_t* base;
  uint32_t off[kPer];
  __device__ __forceinline__ static int k_of(int instr, int lane) { return ((lane & 7) ^ (((instr * 8 + (lane >> 3)) >> 1) & 7)) * 16; }
  __device__ __forceinline__ void init(const uint8_t* p, int64_t ld, int64_t row0, int64_t rows, int64_t first, int gw, int lane) {
    base = p + row0 * ld + first * kBK;
    const int last = (int)(rows - row0 < R ? rows - row0 : R) - 1;     // rows past the end are fetched from the last one
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int instr = piece(gw, j), r = instr * 8 + (lane >> 3);
      off[j] = (uint32_t)((r < last ? r : last) * (int)ld + k_of(instr, lane));
    }
  }
  __device__ __forceinline__ void issue_one(int j, uint32_t lds_off, int gw) const { dma16_s(base, off[j], lds_off + piece(gw, j) * 1024); }
  // The next k tile, of which `left` bytes exist (a multiple of 16; whole, partial or none): the rest comes from zeros.
  __device__ __forceinline__ void issue(int64_t left, uint32_t lds_off, int gw, int lane, int from = 0, int to = kPer) const {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (j < from || j >= to) continue;
      const uint8_t* const g = base + off[j];
      dma16(k_of(piece(gw, j), lane) < left ? g : reinterpret_cast<const uint8_t*>(kZeros), lds_off + piece(gw, j) * 1024);
    }
  }
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

// Few rows, and rows too far apart for 32-bit offsets.  What bounds a product of few rows is reading B once, so nothing is
// staged: a block owns 16 columns and 16 rows, its waves take every W-th k block, operands go from memory straight into
// fragments (four lanes read 64 consecutive bytes of a row), kAhead blocks at a time, and the waves' sums meet
// in LDS in wave order.  1 x 8192 x 2048: 5.4 to 5.6 us a pass, of which the launch is about 4.
constexpr int kAhead = 4;
template <int W, int FA, int FB, bool EXACT>
__global__ __launch_bounds__(64 * W) void gemm_f8_direct_kernel(GemmF8Params p) {
  __shared__ __attribute__((aligned(16))) float part[W][16][16 + 4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, L = lane & 15, g = lane >> 4;
  const int64_t m0 = (int64_t)(blockIdx.x / p.tiles_n) * 16, n0 = (int64_t)(blockIdx.x % p.tiles_n) * 16;
  const int64_t Ra = (p.M + 63) & ~63LL, Rb = (p.N + 63) & ~63LL;
  auto in = [](int64_t r, int64_t rows) { return r < rows ? r : rows - 1; };
  auto scale_of = [](const uint8_t* t, int64_t r) { return t + (r & ~63LL) + (r & 15) * 4 + ((r & 63) >> 4); };
  const int64_t ra = in(m0 + L, p.M), rb = in(n0 + L, p.N);
  const uint8_t* const pa = p.A + ra * p.lda + 16 * g;
  const uint8_t* const pb = p.B + rb * p.ldb + 16 * g;
  const uint8_t* const qa = scale_of(p.sa, ra);
  const uint8_t* const qb = scale_of(p.sb, rb);
  f32x4 acc = {};
  const int total = (int)((p.K + kBK - 1) / kBK);
  auto load = [&](const uint8_t* q, int kb) {
    i32x8 f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t k = (int64_t)kb * kBK;
      i32x4 v = {};
      if (k + 16 * g + 64 * h < p.K) v = *reinterpret_cast<const i32x4*>(q + k + 64 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[4 * h + e] = v[e];
    }
    return f;
  };
  auto several = [&](int kb, auto count) {
    constexpr int U = decltype(count)::value;
    i32x8 fa[U], fb[U];
    int sa[U], sb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = kb + u * W;
      fb[u] = load(pb, k);
      sb[u] = qb[k * Rb];
      fa[u] = load(pa, k);
      sa[u] = qa[k * Ra];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (EXACT) {
#pragma unroll
        for (int s = 0; s < 4; ++s)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8<FB>(fb[u], s, sb[u]), widen8<FA>(fa[u], s, sa[u]), acc, 0, 0, 0);
      } else {
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[u], fa[u], acc, FB, FA, 0, sb[u], 0, sa[u]);
      }
    }
  };
  const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
  const bool mine = r < 16 && m0 + r < p.M && n0 + c < p.N;
  EpiParams epi = p.epi;
  narrow<EXACT>(epi);
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

// 32 bytes of a lane's row: the chunks lane / 16 and 4 + lane / 16.
__device__ __forceinline__ i32x8 read_fragment(uint32_t at0, uint32_t at1, uint32_t off) {
  typedef __attribute__((address_space(3))) const i32x4* p;
  const i32x4 a = *(p)(uintptr_t)(at0 + off), b = *(p)(uintptr_t)(at1 + off);
  return i32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}
__device__ __forceinline__ int read_scales(uint32_t at) {
  typedef __attribute__((address_space(3))) const int* p;
  return *(p)(uintptr_t)at;
}
// D[n][m] += B A^T of one block of k; byte IA of sa and IB of sb are the scales (the index has to be a constant).
template <int FA, int FB> __device__ __forceinline__ f32x4 mfma(const i32x8& b, const i32x8& a, f32x4 c, int ib, int sb, int ia, int sa) {
#define PW_F8_CASE(IB, IA) if (ib == IB && ia == IA) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, FB, FA, IB, sb, IA, sa);
  PW_F8_CASE(0, 0) PW_F8_CASE(0, 1) PW_F8_CASE(0, 2) PW_F8_CASE(0, 3) PW_F8_CASE(1, 0) PW_F8_CASE(1, 1) PW_F8_CASE(1, 2) PW_F8_CASE(1, 3)
  PW_F8_CASE(2, 0) PW_F8_CASE(2, 1) PW_F8_CASE(2, 2) PW_F8_CASE(2, 3) PW_F8_CASE(3, 0) PW_F8_CASE(3, 1) PW_F8_CASE(3, 2)
#undef PW_F8_CASE
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, FB, FA, 3, sb, 3, sa);
}

template <class S, int FA, int FB, bool EXACT>
__global__ __launch_bounds__(S::kThreads, S::kWavesPerSimd) void gemm_f8_tile_kernel(GemmF8Params p) {
  constexpr int FM = S::FM, FN = S::FN, G = S::G, WN = S::WN;
  constexpr bool SPLIT = FM == 8;
  using OpA = Operand<S::BM, G, SPLIT>;
  using OpB = Operand<S::BN, G, false>;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  narrow<EXACT>(p.epi);
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

  const int total = (int)((p.K + kBK - 1) / kBK), per = (total + S::WK - 1) / S::WK;
  const int first = grp * per, n = total - first < per ? (total - first < 0 ? 0 : total - first) : per;
  OpA oa;
  OpB ob;
  oa.init(p.A, p.lda, m0, p.M, first, gw, lane);
  ob.init(p.B, p.ldb, n0, p.N, first, gw, lane);
  const uint32_t ring = (uint32_t)(uintptr_t)(lds_ptr)smem + grp * (S::NS * S::kStage);
  // Scales of the tile: kScalesA / 4 words of A's table, then BN / 4 of B's.  Every wave fetches 64 of them, the same ones as another
  // where there are fewer (a branch here would let the compiler move MFMAs past it); groups of 64 rows that do not exist come
  // from the last one.
  constexpr int kWords = S::kScales / 4, kSets = (kWords + 63) / 64;
  static_assert(kSets <= G && (kWords % 64 == 0 || kSets == 1), "a wave fetches 64 words");
  const int64_t Ra = (p.M + 63) & ~63LL, Rb = (p.N + 63) & ~63LL;
  const int word = (gw % kSets * 64 + lane) % kWords, w = word < S::kScalesA / 4 ? word : word - S::kScalesA / 4;
  const bool of_a = word < S::kScalesA / 4;
  const int64_t sp_step = of_a ? Ra : Rb, sp_row = (of_a ? m0 & ~63LL : n0) + (w >> 4) * 64;
  const uint8_t* const sp = (of_a ? p.sa : p.sb) + (sp_row < sp_step - 64 ? sp_row : sp_step - 64) + (w & 15) * 4;
  const uint8_t* sq = sp + first * sp_step;      // of the tile that is asked for next; the last one's again behind it
  auto issue_scales = [&](int t, uint32_t st, bool last) {
    dma4(sq, st + S::kOperands + gw % kSets * 256);
    if (!last || first + t + 1 < total) sq += sp_step;
  };
  // k tile t into the stage at `at`; zeros where it does not exist.  part: 1 all but the second half of A, 2 that, 0 both.
  auto issue = [&](int t, uint32_t at, int part) {
    const int64_t left = p.K - (int64_t)(first + t) * kBK;
    const uint32_t st = ring + at;
    if (part != 2) {
      ob.issue(left, st + S::BM * kBK, gw, lane);
      ob.base += kBK;
      issue_scales(t, st, true);
      oa.issue(left, st, gw, lane, 0, SPLIT ? OpA::kPer / 2 : OpA::kPer);
    }
    if (SPLIT && part != 1) oa.issue(left, st, gw, lane, OpA::kPer / 2);
    if (!SPLIT || part != 1) oa.base += kBK;
  };
  // Addresses of this lane's fragments: block j of an operand is 16 j rows of 128 bytes further on, which leaves the swizzle
  // of the row as it is.
  const uint32_t row_a = ring + (wm * FM * 16 + L) * kBK, row_b = ring + S::BM * kBK + (wn * FN * 16 + L) * kBK;
  const uint32_t c0 = (quarter ^ (L >> 1)) << 4, c1 = ((quarter + 4) ^ (L >> 1)) << 4;
  const uint32_t a0 = row_a + c0, a1 = row_a + c1, b0 = row_b + c0, b1 = row_b + c1;
  constexpr int GA = (FM + 3) / 4, GB = (FN + 3) / 4;       // words of four scales
  const int rows_at = (S::BM < 64 ? (int)(m0 & 63) : 0) + wm * FM * 16, cols_at = wn * FN * 16;   // of this wave, in the words' groups
  const uint32_t s_a = ring + S::kOperands + (rows_at & ~63) + L * 4, s_b = ring + S::kOperands + S::kScalesA + (cols_at & ~63) + L * 4;
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
  i32x8 fa[2], fb[FN];
  int sa[GA], sb[GB], nsa[GA], nsb[GB];
  // Addresses of a tile's fragments: kept whole, so that what is constant in them goes into the instructions.
  struct At { uint32_t v[4]; };
  auto at_of = [&](uint32_t st) {
    At r{{a0 + st, a1 + st, b0 + st, b1 + st}};
#pragma unroll
    for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(r.v[k]));
    return r;
  };
  auto read_a = [&](const At& at, int i) { fa[i & 1] = read_fragment(at.v[0], at.v[1], i * 16 * kBK); };
  auto read_b = [&](const At& at, int j) { fb[j] = read_fragment(at.v[2], at.v[3], j * 16 * kBK); };
  auto read_scale = [&](uint32_t st, int g) {
    if (g < GA) nsa[g] = read_scales(s_a + st + g * 64);
    else nsb[g - GA] = read_scales(s_b + st + (g - GA) * 64);
  };
  auto take_scales = [&] {
#pragma unroll
    for (int g = 0; g < GA; ++g) sa[g] = word_a(nsa[g]);
#pragma unroll
    for (int g = 0; g < GB; ++g) sb[g] = word_b(nsb[g]);
  };
  auto issue_one = [&](int t, int m, uint32_t at) {       // load m of the whole tile t
    const uint32_t st = ring + at;
    if (m < OpB::kPer) ob.issue_one(m, st + S::BM * kBK, gw);
    else oa.issue_one(m - OpB::kPer, st, gw);
    if (m == OpB::kPer - 1) {
      ob.base += kBK;
      issue_scales(t, st, false);
    }
    if (m == kPer - 1) oa.base += kBK;
  };
  bf16x8 wa[EXACT ? 2 : 1][4], wb[EXACT ? FN : 1][4];
  auto byte_of = [](const int* w, int i) { return (w[i / 4] >> (8 * (i % 4))) & 255; };
  // MFMAs run across k tiles without a pause.  A unit is one block of rows against all columns of the wave.
  //  8-bit pipe: the next block's fragments are read while a unit runs.  All of a tile has been read from LDS one unit before its
  //    end; the next tile's columns take the place of this one's as those are used for the last time.
  //  The same of 256 x 256, whose two stages fill LDS (SPLIT): the tile's columns and scales are in registers when it begins, so
  //    halfway, where the waves meet once more, their place and that of the first half of its rows is free for tile t + 2; that of
  //    the second half is at kTurn.  Loads are on their way for one and a half tiles then instead of one, and go out all the
  //    time: 8192 x 8192 x 8192 428 -> 402 us; with all waits for them taken out it takes 400, without the loads 332.
  //  bf16 pipe: the next block is widened while a unit runs and the one after it read; the columns are widened between the MFMAs
  //    of the first unit, and their bytes' registers are free from there on.  All of a tile has been read two units before its
  //    end.
  // There (kTurn) the waves meet, the next tile is there, and the stage of this one is free for tile t + NS, whose direct loads
  // go out between the MFMAs that are left.
  // What bounds the largest: power.  8192 x 8192 x 8192 runs at 1.8 GHz, 69 of 100 cycles with an MFMA, 2.8 PFLOP/s; of its 389
  // us the MFMAs alone take 292, reading fragments 40, bringing operands 70.  Addresses of fragments kept whole and a running
  // pointer to the scales, fewer instructions between the MFMAs, won 4 of 100.  Four waves of 128 x 128, which read a third
  // less from LDS, leave nothing to a SIMD while its wave waits: 395 us instead of 392 then, and 139 instead of 130 with k = 2048.
  // STREAM: tile t + NS is a whole one; MORE: tile t + 1 exists (t + NS, where it does not, is made of zeros nobody reads).  No
  // branches inside: the compiler would move MFMAs past them.
  constexpr int kTurn = EXACT ? FM - 2 : FM - 1, kSlots = (FM - kTurn) * FN;
  constexpr int kHalf = FM / 2 - 1, kSecond = SPLIT ? OpA::kPer / 2 : kPer, kFirst = kPer - kSecond;
  static_assert(FM % 2 == 0 && GA + GB <= FN && (!EXACT || 4 % FN == 0), "two fragments of rows in turn; a slot for each word of scales");
  auto tile = [&](int t, uint32_t st, uint32_t next, auto streaming, auto follows) {
    constexpr bool STREAM = decltype(streaming)::value, more = decltype(follows)::value;
    const At here = at_of(st), there = at_of(next);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if (SPLIT && i == kHalf) {
        landed(std::integral_constant<int, kLoads>{});
        meet();
        if (more && !STREAM) issue(t + S::NS, st, 1);
      }
      if (i == kTurn && more) {
        landed(std::integral_constant<int, SPLIT ? kLoads : (S::NS - 2) * kLoads>{});
        meet();
        if (!STREAM) issue(t + S::NS, st, SPLIT ? 2 : 0);
      }
#pragma unroll
      for (int jj = 0; jj < FN; ++jj) {
        // back and forth: consecutive MFMAs share an operand; the last unit and the next tile's first in one order
        const int j = (i & 1) || i == 0 ? jj : FN - 1 - jj, slot = (i - kTurn) * FN + jj;
        __builtin_amdgcn_sched_barrier(0);
        if (EXACT) {
          if (i < FM - 2 && jj == 0) read_a(here, i + 2);
        } else {                               // behind the first MFMA of a tile, so that its wait does not cover this
          if (i < FM - 1 && jj == (i == 0 ? 1 : 0)) read_a(here, i + 1);
        }
        if (slot >= 0 && more) {
          if (slot < GA + GB) read_scale(next, slot);
          if (slot == 0) read_a(there, 0);
          if (EXACT && slot == FN) read_a(there, 1);
          if (EXACT && (slot & 1)) read_b(there, slot >> 1);
          if (STREAM) {
#pragma unroll
            for (int m = slot * kSecond / kSlots; m < (slot + 1) * kSecond / kSlots; ++m) issue_one(t + S::NS, kFirst + m, st);
          }
        }
        if (SPLIT && STREAM && i >= kHalf && i < kTurn) {
          const int at = (i - kHalf) * FN + jj, slots = (kTurn - kHalf) * FN;
#pragma unroll
          for (int m = at * kFirst / slots; m < (at + 1) * kFirst / slots; ++m) issue_one(t + S::NS, m, st);
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (EXACT) {
          if (i == 0) {
#pragma unroll
            for (int s = 0; s < 4; ++s) wb[j][s] = widen8<FB>(fb[j], s, byte_of(sb, j));
          }
          if (i + 1 < FM || more) {
            const int k = i + 1 < FM ? byte_of(sa, i + 1) : word_a(nsa[0]) & 255;
#pragma unroll
            for (int s = jj * 4 / FN; s < (jj + 1) * 4 / FN; ++s) wa[(i + 1) & 1][s] = widen8<FA>(fa[(i + 1) & 1], s, k);
          }
#pragma unroll
          for (int s = 0; s < 4; ++s) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j][s], wa[i & 1][s], acc[i][j], 0, 0, 0);
        } else {
          acc[i][j] = mfma<FA, FB>(fb[j], fa[i & 1], acc[i][j], j % 4, sb[j / 4], i % 4, sa[i / 4]);
          if (i == FM - 1 && more) {           // the column block's last use
            __builtin_amdgcn_sched_barrier(0);
            read_b(there, j);
          }
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) take_scales();
  };
  // A whole tile's bias is added before the staging and not row by row behind it (1024 x 4096 x 2048 15.3 -> 14.5 us, 8192 x 8192 x
  // 2048 131.4 -> 129.6; without a bias 122.6 -> 123.4): it comes during the last k tile, whose waits it only makes stricter.  The bf16 pipe's loop has no
  // registers for it (2048 x 8192 x 8192 215 -> 228).
  constexpr bool kBias = G > 1 && FN % 4 == 0 && !EXACT;
  const bool whole = G > 1 && FN % 4 == 0 && m0 + S::BM <= p.M && n0 + S::BN <= p.N, biased = kBias && whole && epi_has_bias(p.epi.mode) && p.epi.bias;
  f32x4 bias[FN];
  auto load_bias = [&] {
    if (!biased) return;
#pragma unroll
    for (int j = 0; j < FN; ++j) bias[j] = *reinterpret_cast<const f32x4*>(p.epi.bias + n0 + wn * FN * 16 + 4 * quarter + 16 * j);
  };
  if (n > 0) {
#pragma unroll
    for (int i = 0; i < S::NS; ++i) issue(i, i * S::kStage, 0);
    landed(std::integral_constant<int, (S::NS - 1) * kLoads + (SPLIT ? kSecond : 0)>{});
    meet();
#pragma unroll
    for (int g = 0; g < GA + GB; ++g) read_scale(0, g);
    take_scales();
    const At here = at_of(0);
    read_a(here, 0);
#pragma unroll
    for (int j = 0; j < FN; ++j) read_b(here, j);
    if constexpr (EXACT) {
      read_a(here, 1);
#pragma unroll
      for (int s = 0; s < 4; ++s) wa[0][s] = widen8<FA>(fa[0], s, byte_of(sa, 0));
    }
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
    with_extra<EXACT>(p.epi, [&](auto kind) { gemm_finish_tile<Finish<S>, decltype(kind)::value>(parts, p, m, n0); });
  };
  if constexpr (G > 1 && FN % 4 == 0) {
    if (whole) {
      if (kBias && biased) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[i][j] += bias[j];
        p.epi.bias = nullptr;
      }
      with_extra<EXACT>(p.epi, [&](auto kind) {
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

using Big = Tile<2, 4, 8, 4, 1>;        // 256 x 256
using Mid = Tile<2, 2, 4, 4, 1>;        // 128 x 128, two workgroups to a compute unit
using MidOne = Tile<2, 2, 4, 4, 1, 4>;  // the same with four stages, one workgroup to a unit
using Half = Tile<2, 2, 4, 2, 1, 3>;    // 128 x 64
using Split = Tile<1, 1, 4, 4, 4>;      // 64 x 64, k over four waves
using Few = Tile<1, 1, 2, 4, 4, 3>;     // 32 x 64, likewise

template <class S, int FA, int FB, bool EXACT>
hipError_t prepare() {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(gemm_f8_tile_kernel<S, FA, FB, EXACT>), hipFuncAttributeMaxDynamicSharedMemorySize,
                             (int)S::kSmem);
}
template <int FA, int FB, class S, class... Rest>
hipError_t prepare_both() {
  hipError_t e = prepare<S, FA, FB, false>();
  if (e == hipSuccess) e = prepare<S, FA, FB, true>();
  if constexpr (sizeof...(Rest) > 0) {
    if (e == hipSuccess) e = prepare_both<FA, FB, Rest...>();
  }
  return e;
}
template <int FA, int FB>
hipError_t prepare_formats() {
  hipError_t e = prepare<Big, FA, FB, false>();
  if (e == hipSuccess) e = prepare<MidOne, FA, FB, false>();
  return e == hipSuccess ? prepare_both<FA, FB, Mid, Half, Split, Few>() : e;
}
constexpr int64_t kMostThreads = (1LL << 32) - 1;     // of a launch
template <class S, int FA, int FB, bool EXACT>
hipError_t launch(hipStream_t s, GemmF8Params p) {
  const int64_t tm = (p.M + S::BM - 1) / S::BM, tn = (p.N + S::BN - 1) / S::BN;
  if (tm * tn * S::kThreads > kMostThreads) return hipErrorInvalidValue;
  p.tiles_m = (int)tm;
  p.tiles_n = (int)tn;
  gemm_f8_tile_kernel<S, FA, FB, EXACT><<<(int)(tm * tn), S::kThreads, S::kSmem, s>>>(p);
  return hipGetLastError();
}
template <int W, int FA, int FB>
hipError_t launch_direct(hipStream_t s, GemmF8Params p, bool exact) {
  const int64_t tm = (p.M + 15) / 16, tn = (p.N + 15) / 16;
  if (tm * tn * 64 * W > kMostThreads) return hipErrorInvalidValue;
  p.tiles_m = (int)tm;
  p.tiles_n = (int)tn;
  if (exact) gemm_f8_direct_kernel<W, FA, FB, true><<<(int)(tm * tn), 64 * W, 0, s>>>(p);
  else gemm_f8_direct_kernel<W, FA, FB, false><<<(int)(tm * tn), 64 * W, 0, s>>>(p);
  return hipGetLastError();
}
// Which shape: the largest whose tiles give every compute unit one, as a launch of up to one round takes as long as one tile.
// us (rows x columns x k, bf16 out unless it says fp32):
//   direct    1 x 8192 x 2048 5.4 (Few 5.8), 1 x 32768 x 2048 13.6 (15.3), 4 x 8192 x 2048 5.8 (5.8), 16 x 2048 x 2048
//             4.9 (5.7), 32 x 2048 x 2048 5.2 (5.7), 16 x 8192 x 2048 6.8 (6.3); eight waves from k = 4096 on: 1 x 2048 x 8192 7.8 (four: 8.8),
//             1 x 8192 x 4096 8.5 (9.8).  Few rows of a long k lose a little to one rule for all k: 1 x 8192 x 8192 13.7 (Few 13.2)
//   Few       256 x 2048 x 2048 6.0 (Split 6.9), fp32 7.5 (8.7), 64 x 2048 x 8192 11.3 (14.5), fp32 14.0 (18.8); 512 x 2048 x 2048, two rounds, 10.2 (7.1)
//   Split     512 x 2048 x 2048 7.1 (Half 8.9), 1024 x 1024 x 1024 5.9 (6.9), fp32 7.4 (9.6); 1024 x 2048 x 2048 13.1 (9.6)
//   Half      1024 x 2048 x 2048 9.6 (Mid 14.1, MidOne 12.9), fp32 16.3 (20.7)
//   MidOne    1024 x 4096 x 2048 14.1 (Mid 15.2, Half 14.9), 2048 x 2048 x 8192 36.8 (43.5, 40.6); fp32, Mid against Half: 67.2 (73.4)
//   Mid       1500 x 4096 x 2048 18.2 (MidOne 24.5, Half 21.1, Big 26.6), fp32 30.2 (Half 33.4); 128 tiles of 256 x 256, 2048 x 4096 x 2048,
//             19.8 (Big 27.2)
//   Big       a round from 144 tiles on, 2304 x 4096 x 2048 27.5 (Mid 29.4), 2816 x 3840 x 8192 80 (92); beyond one where few of the last
//             are idle: 272 tiles, 4352 x 4096 x 2048, 50.1 (44.5), 320 50.6 (45.1), 352 50.9 (49.2), 384 51.8 (50.9), 1024 119 (140)
template <int FA, int FB>
hipError_t choose(hipStream_t s, const GemmF8Params& p, bool exact) {
  auto tiles = [&](int m, int n) { return ((p.M + m - 1) / m) * ((p.N + n - 1) / n); };
  if (p.M < 4 || tiles(16, 16) <= 256 || p.lda > kMaxLd || p.ldb > kMaxLd)
    return p.K >= 4096 ? launch_direct<8, FA, FB>(s, p, exact) : launch_direct<4, FA, FB>(s, p, exact);
  if (tiles(Few::BM, Few::BN) <= 256) return exact ? launch<Few, FA, FB, true>(s, p) : launch<Few, FA, FB, false>(s, p);
  if (tiles(Split::BM, Split::BN) <= 256) return exact ? launch<Split, FA, FB, true>(s, p) : launch<Split, FA, FB, false>(s, p);
  if (tiles(Half::BM, Half::BN) <= 256) return exact ? launch<Half, FA, FB, true>(s, p) : launch<Half, FA, FB, false>(s, p);
  if (exact) return launch<Mid, FA, FB, true>(s, p);
  const int64_t big = tiles(Big::BM, Big::BN), slots = (big + 255) / 256 * 256;
  if (big <= 256 ? big >= 144 : 100 * big > 72 * slots) return launch<Big, FA, FB, false>(s, p);
  return tiles(Mid::BM, Mid::BN) <= 256 ? launch<MidOne, FA, FB, false>(s, p) : launch<Mid, FA, FB, false>(s, p);
}

}  // namespace

hipError_t gemm_f8_init() {
  hipError_t e = prepare_formats<0, 0>();
  if (e == hipSuccess) e = prepare_formats<0, 1>();
  if (e == hipSuccess) e = prepare_formats<1, 0>();
  if (e == hipSuccess) e = prepare_formats<1, 1>();
  return e;
}

hipError_t launch_gemm_f8(hipStream_t s, const GemmF8Args& a) {
  const int64_t most = 1LL << 26;
  if (!a.A || !a.B || !a.a_scale || !a.b_scale || !a.C || a.M < 0 || a.N < 0 || a.K < 0 || a.M > most || a.N > most || a.K > (1LL << 30))
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
  const bool exact = a.out_dtype == kF32;
  if (a.a_format == kE4M3) return a.b_format == kE4M3 ? choose<0, 0>(s, p, exact) : choose<0, 1>(s, p, exact);
  return a.b_format == kE4M3 ? choose<1, 0>(s, p, exact) : choose<1, 1>(s, p, exact);
}

}  // namespace pw
