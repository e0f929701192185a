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
template <int WM_, int WN_, int FM_, int FN_, int WK_, bool PIPELINED_ = false>
struct Tile {
  static constexpr bool kPipelined = PIPELINED_;
  static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_, WK = WK_, G = WM * WN;
  static constexpr int BM = 16 * WM * FM, BN = 16 * WN * FN, kThreads = 64 * G * WK;
  static constexpr int kOperands = (BM + BN) * kBK, kStage = kOperands + (BM + BN + 255) / 256 * 256;   // bytes; the scales lie behind the operands
  static constexpr int kLdP = BN + 4;
  static constexpr size_t kRing = (size_t)WK * 2 * kStage;
  static constexpr int kRowsAtOnce = BM < 64 ? BM : 64;                             // of partial sums in LDS, where waves share a tile
  static constexpr size_t kParts = (size_t)(G > 1 ? kRowsAtOnce : WK * BM) * kLdP * 4;
  static constexpr size_t kSmem = (kRing > kParts ? kRing : kParts) + 1023 & ~(size_t)1023;
  static_assert(WK == 1 || G == 1, "groups of one wave only");
};
// What gemm_finish_tile sees of it.
template <class S> struct Finish {
  static constexpr int BM = S::G > 1 ? S::kRowsAtOnce : S::BM, BN = S::BN, WK = S::WK, kThreads = S::kThreads, kLdP = S::kLdP;
};

// One operand of a group's tile: R rows of 128 bytes, fetched by G waves in pieces of 1 KiB (8 rows); chunk c (16 bytes) of row
// r lies at position c ^ ((r >> 1) & 7) of the row, so that the 16 rows of a fragment read hit all banks.
template <int R, int G>
struct Operand {
  static constexpr int kPer = R / 8 / G;
  const uint8_t* base;
  uint32_t off[kPer];
  __device__ __forceinline__ static int k_of(int instr, int lane) { return ((lane & 7) ^ (((instr * 8 + (lane >> 3)) >> 1) & 7)) * 16; }
  __device__ __forceinline__ void init(const uint8_t* p, int64_t ld, int64_t row0, int64_t rows, int64_t first, int gw, int lane) {
    base = p + row0 * ld + first * kBK;
    const int last = (int)(rows - row0 < R ? rows - row0 : R) - 1;     // rows past the end are fetched from the last one
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int instr = gw * kPer + j, r = instr * 8 + (lane >> 3);
      off[j] = (uint32_t)((r < last ? r : last) * (int)ld + k_of(instr, lane));
    }
  }
  __device__ __forceinline__ void issue_one(int j, uint32_t lds_off, int gw) const { dma16_s(base, off[j], lds_off + (gw * kPer + j) * 1024); }
  // The next k tile, of which `left` bytes exist (a multiple of 16; whole, partial or none): the rest comes from zeros.
  __device__ __forceinline__ void issue(int64_t left, uint32_t lds_off, int gw, int lane) const {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint8_t* const g = base + off[j];
      dma16(k_of(gw * kPer + j, lane) < left ? g : reinterpret_cast<const uint8_t*>(kZeros), lds_off + (gw * kPer + j) * 1024);
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
// staged: a block owns 16 columns and 16 FM rows, its waves take every fourth k block, operands go from memory straight into
// fragments (a lane has 32 consecutive bytes of its row, four lanes a line), kAhead blocks at a time, and the waves' sums meet
// in LDS in wave order.
constexpr int kAhead = 4, kDirectWaves = 4;
template <int FM, int FA, int FB, bool EXACT>
__global__ __launch_bounds__(64 * kDirectWaves) void gemm_f8_direct_kernel(GemmF8Params p) {
  __shared__ __attribute__((aligned(16))) float part[kDirectWaves][FM][16][16 + 4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, L = lane & 15, g = lane >> 4;
  const int64_t m0 = (int64_t)(blockIdx.x / p.tiles_n) * (16 * FM), n0 = (int64_t)(blockIdx.x % p.tiles_n) * 16;
  const int64_t Ra = (p.M + 63) & ~63LL, Rb = (p.N + 63) & ~63LL;
  auto in = [](int64_t r, int64_t rows) { return r < rows ? r : rows - 1; };
  auto scale_of = [](const uint8_t* t, int64_t r) { return t + (r & ~63LL) + (r & 15) * 4 + ((r & 63) >> 4); };
  const int64_t rb = in(n0 + L, p.N);
  const uint8_t* const pb = p.B + rb * p.ldb + 32 * g;
  const uint8_t* const qb = scale_of(p.sb, rb);
  const uint8_t *pa[FM], *qa[FM];
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int64_t ra = in(m0 + 16 * i + L, p.M);
    pa[i] = p.A + ra * p.lda + 32 * g;
    qa[i] = scale_of(p.sa, ra);
  }
  f32x4 acc[FM] = {};
  const int total = (int)((p.K + kBK - 1) / kBK);
  auto load = [&](const uint8_t* q, int kb) {
    i32x8 f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t k = (int64_t)kb * kBK;
      i32x4 v = {};
      if (k + 32 * g + 16 * h < p.K) v = *reinterpret_cast<const i32x4*>(q + k + 16 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[4 * h + e] = v[e];
    }
    return f;
  };
  auto several = [&](int kb, auto count) {
    constexpr int U = decltype(count)::value;
    i32x8 fb[U], fa[U][FM];
    int sb[U], sa[U][FM];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = kb + u * kDirectWaves;
      fb[u] = load(pb, k);
      sb[u] = qb[k * Rb];
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        fa[u][i] = load(pa[i], k);
        sa[u][i] = qa[i][k * Ra];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        if constexpr (EXACT) {
#pragma unroll
          for (int s = 0; s < 4; ++s)
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8<FB>(fb[u], s, sb[u]), widen8<FA>(fa[u][i], s, sa[u][i]), acc[i], 0, 0, 0);
        } else {
          acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[u], fa[u][i], acc[i], FB, FA, 0, sb[u], 0, sa[u][i]);
        }
      }
  };
  int kb = wave;
  for (; kb + (kAhead - 1) * kDirectWaves < total; kb += kAhead * kDirectWaves) several(kb, std::integral_constant<int, kAhead>{});
  for (; kb < total; kb += kDirectWaves) several(kb, std::integral_constant<int, 1>{});
#pragma unroll
  for (int i = 0; i < FM; ++i) *reinterpret_cast<f32x4*>(&part[wave][i][L][4 * g]) = acc[i];
  __syncthreads();
  const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    float v = part[0][i][r][c];
#pragma unroll
    for (int w = 1; w < kDirectWaves; ++w) v += part[w][i][r][c];
    const int64_t m = m0 + 16 * i + r, n = n0 + c;
    if (m < p.M && n < p.N) epilogue1<true>(p.epi, m, n, v);
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
__global__ __launch_bounds__(S::kThreads, S::WK == 1 ? 2 : 1) void gemm_f8_tile_kernel(GemmF8Params p) {
  constexpr int FM = S::FM, FN = S::FN, G = S::G, WN = S::WN;
  using OpA = Operand<S::BM, G>;
  using OpB = Operand<S::BN, G>;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
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
  const uint32_t ring = (uint32_t)(uintptr_t)(lds_ptr)smem + grp * (2 * S::kStage);
  // Scales of the tile: BM / 4 words of A's table, then BN / 4 of B's.  Every wave fetches 64 of them, the same ones as another
  // where there are fewer (a branch here would let the compiler move MFMAs past it); groups of 64 rows that do not exist come
  // from the last one.
  constexpr int kWords = (S::BM + S::BN) / 4, kSets = (kWords + 63) / 64;
  static_assert(kSets <= G && (kWords % 64 == 0 || kSets == 1), "a wave fetches 64 words");
  const int64_t Ra = (p.M + 63) & ~63LL, Rb = (p.N + 63) & ~63LL;
  const int word = (gw % kSets * 64 + lane) % kWords, w = word < S::BM / 4 ? word : word - S::BM / 4;
  const bool of_a = word < S::BM / 4;
  const int64_t sp_step = of_a ? Ra : Rb, sp_row = (of_a ? m0 : n0) + (w >> 4) * 64;
  const uint8_t* const sp = (of_a ? p.sa : p.sb) + (sp_row < sp_step - 64 ? sp_row : sp_step - 64) + (w & 15) * 4;
  auto issue_scales = [&](int t, uint32_t st) {
    const int kb = first + t < total ? first + t : total - 1;
    dma4(sp + kb * sp_step, st + S::kOperands + gw % kSets * 256);
  };
  auto issue = [&](int t) {
    const int64_t left = p.K - (int64_t)(first + t) * kBK;
    const uint32_t st = ring + (t & 1) * S::kStage;
    oa.issue(left, st, gw, lane);
    ob.issue(left, st + S::BM * kBK, gw, lane);
    oa.base += kBK;
    ob.base += kBK;
    issue_scales(t, st);
  };
  // Addresses of this lane's fragments: block j of an operand is 16 j rows of 128 bytes further on, which leaves the swizzle
  // of the row as it is.
  const uint32_t row_a = ring + (wm * FM * 16 + L) * kBK, row_b = ring + S::BM * kBK + (wn * FN * 16 + L) * kBK;
  const uint32_t c0 = (quarter ^ (L >> 1)) << 4, c1 = ((quarter + 4) ^ (L >> 1)) << 4;
  const uint32_t a0 = row_a + c0, a1 = row_a + c1, b0 = row_b + c0, b1 = row_b + c1;
  constexpr int GA = (FM + 3) / 4, GB = (FN + 3) / 4;       // words of four scales
  const uint32_t s_a = ring + S::kOperands + wm * FM * 16 + L * 4, s_b = ring + S::kOperands + S::BM + wn * FN * 16 + L * 4;
  auto landed_and_met = [&] {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    if (G > 1) __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  if constexpr (S::kPipelined && !EXACT) {
    // MFMAs run across k tiles without a pause.  A unit is one block of rows against all columns of the wave; the fragments of the
    // next block are read while it runs.  All of a tile has been asked for one unit before its end: there the waves meet, the
    // next tile is there, and the stage of this one is free for the one after next, whose direct loads go out between the
    // MFMAs of the last unit; the next tile's columns take the place of this one's as those are used for the last time.
    static_assert(FM % 2 == 0 && GA + GB <= FN, "two fragments of rows in turn; a slot for each word of scales");
    constexpr int kPer = OpA::kPer + OpB::kPer;
    i32x8 fa[2], fb[FN];
    int sa[GA], sb[GB], nsa[GA], nsb[GB];
    auto read_a = [&](uint32_t st, int i) { fa[i & 1] = read_fragment(a0 + st, a1 + st, i * 16 * kBK); };
    auto read_b = [&](uint32_t st, int j) { fb[j] = read_fragment(b0 + st, b1 + st, j * 16 * kBK); };
    auto read_scale = [&](uint32_t st, int g) {
      if (g < GA) nsa[g] = read_scales(s_a + st + g * 64);
      else nsb[g - GA] = read_scales(s_b + st + (g - GA) * 64);
    };
    auto take_scales = [&] {
#pragma unroll
      for (int g = 0; g < GA; ++g) sa[g] = nsa[g];
#pragma unroll
      for (int g = 0; g < GB; ++g) sb[g] = nsb[g];
    };
    auto issue_one = [&](int t, int m) {       // of the whole tile t
      const uint32_t st = ring + (t & 1) * S::kStage;
      if (m < OpA::kPer) oa.issue_one(m, st, gw);
      else ob.issue_one(m - OpA::kPer, st + S::BM * kBK, gw);
      if (m == kPer - 1) {
        oa.base += kBK;
        ob.base += kBK;
        issue_scales(t, st);
      }
    };
    // STREAM: tile t + 2 is a whole one; MORE: tile t + 1 exists (t + 2, where it does not, is made of zeros nobody reads).  No
    // branches inside: the compiler would move MFMAs past them.
    auto tile = [&](int t, auto streaming, auto follows) {
      constexpr bool STREAM = decltype(streaming)::value, more = decltype(follows)::value;
      const uint32_t st = (t & 1) * S::kStage, next = S::kStage - st;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        if (i == FM - 1 && more) {
          landed_and_met();
          if (!STREAM) issue(t + 2);
        }
#pragma unroll
        for (int jj = 0; jj < FN; ++jj) {
          // back and forth: consecutive MFMAs share an operand; the last unit and the next tile's first in one order
          const int j = (i & 1) || i == 0 ? jj : FN - 1 - jj;
          __builtin_amdgcn_sched_barrier(0);
          // behind the first MFMA of a tile, so that its wait does not cover what is asked for here
          if (i < FM - 1 && jj == (i == 0 ? 1 : 0)) read_a(st, i + 1);
          if (i == FM - 1 && more) {
            if (jj < GA + GB) read_scale(next, jj);
            if (jj == 0) read_a(next, 0);
            if (STREAM) {
#pragma unroll
              for (int m = jj * kPer / FN; m < (jj + 1) * kPer / FN; ++m) issue_one(t + 2, m);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
          acc[i][j] = mfma<FA, FB>(fb[j], fa[i & 1], acc[i][j], j % 4, sb[j / 4], i % 4, sa[i / 4]);
          if (i == FM - 1 && more) {           // the column block's last use
            __builtin_amdgcn_sched_barrier(0);
            read_b(next, j);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (more) take_scales();
    };
    if (n > 0) issue(0);
    landed_and_met();
    if (n > 1) issue(1);
    if (n > 0) {
#pragma unroll
      for (int g = 0; g < GA + GB; ++g) read_scale(0, g);
      take_scales();
      read_a(0, 0);
#pragma unroll
      for (int j = 0; j < FN; ++j) read_b(0, j);
    }
    constexpr std::true_type yes;
    constexpr std::false_type no;
    int t = 0;
    for (; t + 3 < n; ++t) tile(t, yes, yes);  // the last tile may be a partial one
    for (; t + 1 < n; ++t) tile(t, no, yes);
    if (t < n) tile(t, no, no);
    landed_and_met();
  } else {
    if (n > 0) issue(0);
    landed_and_met();
    for (int t = 0; t < n; ++t) {
      const uint32_t st = (t & 1) * S::kStage;
      if (t + 1 < n) issue(t + 1);
      int sa[GA], sb[GB];
      i32x8 fb[FN];
#pragma unroll
      for (int g = 0; g < GA; ++g) sa[g] = read_scales(s_a + st + g * 64);
#pragma unroll
      for (int g = 0; g < GB; ++g) sb[g] = read_scales(s_b + st + g * 64);
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[j] = read_fragment(b0, b1, st + j * 16 * kBK);
      if constexpr (EXACT) {
        bf16x8 wb[FN][4];
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int s = 0; s < 4; ++s) wb[j][s] = widen8<FB>(fb[j], s, (sb[j / 4] >> (8 * (j % 4))) & 255);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
          const i32x8 fa = read_fragment(a0, a1, st + i * 16 * kBK);
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const bf16x8 wa = widen8<FA>(fa, s, (sa[i / 4] >> (8 * (i % 4))) & 255);
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j][s], wa, acc[i][j], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < FM; ++i) {
          const i32x8 fa = read_fragment(a0, a1, st + i * 16 * kBK);
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[i][j] = mfma<FA, FB>(fb[j], fa, acc[i][j], j % 4, sb[j / 4], i % 4, sa[i / 4]);
        }
      }
      landed_and_met();
    }
  }

  __syncthreads();
  float* const parts = reinterpret_cast<float*>(smem);
  auto finish = [&](int64_t m) {
    switch (epi_extra_kind(p.epi)) {            // uniform over the launch
      case kExtraAuxBf16: gemm_finish_tile<Finish<S>, kExtraAuxBf16>(parts, p, m, n0); break;
      case kExtraAuxF32: gemm_finish_tile<Finish<S>, kExtraAuxF32>(parts, p, m, n0); break;
      case kExtraOldC: gemm_finish_tile<Finish<S>, kExtraOldC>(parts, p, m, n0); break;
      default: gemm_finish_tile<Finish<S>, kExtraNone>(parts, p, m, n0); break;
    }
  };
  if (S::kPipelined && m0 + S::BM <= p.M && n0 + S::BN <= p.N) {
    gemm_epilogue_staged<(FM + 1) / 2, (FN + 3) / 4 * 2>(reinterpret_cast<bf16*>(smem), acc, p, m0 + wm * FM * 16, n0 + wn * FN * 16, wave, lane);
    return;
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

using Big = Tile<2, 4, 8, 4, 1, true>;       // 256 x 256
using Mid = Tile<2, 2, 4, 4, 1>;       // 128 x 128, two workgroups per compute unit
using Split = Tile<1, 1, 4, 4, 4>;     // 64 x 64, k over four waves

template <class S, int FA, int FB, bool EXACT>
hipError_t prepare() {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(gemm_f8_tile_kernel<S, FA, FB, EXACT>), hipFuncAttributeMaxDynamicSharedMemorySize,
                             (int)S::kSmem);
}
template <int FA, int FB>
hipError_t prepare_formats() {
  hipError_t e = prepare<Big, FA, FB, false>();
  if (e == hipSuccess) e = prepare<Mid, FA, FB, false>();
  if (e == hipSuccess) e = prepare<Mid, FA, FB, true>();
  if (e == hipSuccess) e = prepare<Split, FA, FB, false>();
  if (e == hipSuccess) e = prepare<Split, FA, FB, true>();
  return e;
}
template <class S, int FA, int FB, bool EXACT>
hipError_t launch(hipStream_t s, GemmF8Params p) {
  const int64_t tm = (p.M + S::BM - 1) / S::BM, tn = (p.N + S::BN - 1) / S::BN;
  if (tm * tn > (1LL << 26)) return hipErrorInvalidValue;
  p.tiles_m = (int)tm;
  p.tiles_n = (int)tn;
  gemm_f8_tile_kernel<S, FA, FB, EXACT><<<(int)(tm * tn), S::kThreads, S::kSmem, s>>>(p);
  return hipGetLastError();
}
template <int FM, int FA, int FB>
hipError_t launch_direct(hipStream_t s, GemmF8Params p, bool exact) {
  const int64_t tm = (p.M + 16 * FM - 1) / (16 * FM), tn = (p.N + 15) / 16;
  if (tm * tn > (1LL << 30)) return hipErrorInvalidValue;
  p.tiles_m = (int)tm;
  p.tiles_n = (int)tn;
  if (exact) gemm_f8_direct_kernel<FM, FA, FB, true><<<(int)(tm * tn), 64 * kDirectWaves, 0, s>>>(p);
  else gemm_f8_direct_kernel<FM, FA, FB, false><<<(int)(tm * tn), 64 * kDirectWaves, 0, s>>>(p);
  return hipGetLastError();
}
template <int FA, int FB>
hipError_t choose(hipStream_t s, const GemmF8Params& p, bool exact) {
  auto tiles = [&](int m, int n) { return ((p.M + m - 1) / m) * ((p.N + n - 1) / n); };
  if (p.M <= 16) return launch_direct<1, FA, FB>(s, p, exact);
  if (p.M <= 32 || p.lda > kMaxLd || p.ldb > kMaxLd) return launch_direct<2, FA, FB>(s, p, exact);
  if (tiles(128, 128) <= 128) return exact ? launch<Split, FA, FB, true>(s, p) : launch<Split, FA, FB, false>(s, p);
  if (exact) return launch<Mid, FA, FB, true>(s, p);
  if (tiles(256, 256) >= 150) return launch<Big, FA, FB, false>(s, p);
  return launch<Mid, FA, FB, false>(s, p);
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
  const bool exact = a.out_dtype == kF32;
  if (a.a_format == kE4M3) return a.b_format == kE4M3 ? choose<0, 0>(s, p, exact) : choose<0, 1>(s, p, exact);
  return a.b_format == kE4M3 ? choose<1, 0>(s, p, exact) : choose<1, 1>(s, p, exact);
}

}  // namespace pw
