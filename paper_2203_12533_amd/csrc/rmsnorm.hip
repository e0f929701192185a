// Root-mean-square norm with the residual's addition in front and an 8-bit output behind, and its backward pass:
//
//   x' = x + y,  r = 1 / sqrt(mean x'^2 + eps),  h = x' r g,  q = h in 8 bits with a scale for each 128 columns (f8_quantize.hip)
//   dx = dres + r (dh g - xh mean(dh g xh)),  xh = x' r;   dg = sum over rows of dh xh
//
// Bound by memory: a row is read once into registers (a wave to a row of up to 2048 columns, a block beyond), four consecutive columns to a
// lane, so that every load and store of 4, 2 or 1 byte an element covers whole lines; 32 lanes hold a block of 128 columns, whose largest
// magnitude takes five moves between lanes.  8192 x 2048 bf16 with x' and 8 bits, nothing of it cached: forward 43.4 us (5.0 TB/s), backward 51 (5.3); rows
// read like everything else 51 and 53.  One row: 5.0 to 5.6 us, a launch.  Rows of 8193 columns on that do not fill 16384 hold some of theirs in memory (forward
// with an 8-bit output 16 to 21 registers, backward 78 to 83): 4096 x 12000 bf16 132 and 333 us (4.8 and 2.4 TB/s), 4096 x 16384 161 and 211 (5.4 and 5.1).
// What the separate passes would move besides: x' once more for the norm, h once more for the quantisation.  Sums, r and h are fp32; q rounds h once, and so
// does h in bf16.
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"
#include "lanes.hpp"
#include "quantize_common.hpp"

namespace pw {

namespace {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));        // wherever an element may be
typedef unsigned short u16x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(2)));

// Columns c .. c + 3 of a row of d: four elements as they are stored, asked for without a question, from the row's last four columns where those
// wanted are not all there, and put in their place, zeros behind the row, when they are used: a branch at each load makes it wait for the one before
// (8192 x 1000 backward 48 us, this 29; forward 21 and 25, of 2001 columns 24.7 and 21.6).  ONCE: nothing reads them again, and they leave the caches
// to what is written. Rows that are a team's vectors exactly need none of it; rows of fewer than four columns are one lane's.
enum Edge { kWhole, kAny, kTiny };
__device__ __forceinline__ int last4(int c, int d) { return c + 4 <= d ? c : d - 4; }
template <class T, Edge EDGE> struct Stored;
template <Edge EDGE> struct Stored<float, EDGE> {
  typedef f32x4u type;
  template <bool ONCE> static __device__ __forceinline__ type load(const float* p, int c, int d) {
    if constexpr (EDGE == kTiny) return type{p[0], d > 1 ? p[1] : 0.f, d > 2 ? p[2] : 0.f, 0.f};
    const type* const at = reinterpret_cast<const type*>(p + (EDGE == kWhole ? c : last4(c, d)));
    return ONCE ? __builtin_nontemporal_load(at) : *at;
  }
  static __device__ __forceinline__ f32x4 wide(const type& w, int c, int d) {
    f32x4 v = w;
    const int off = EDGE == kWhole ? 0 : EDGE == kTiny ? c : c - last4(c, d);
    if (off > 0) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = off == 1 && e < 3 ? w[(e + 1) & 3] : off == 2 && e < 2 ? w[(e + 2) & 3] : off == 3 && e < 1 ? w[3] : 0.f;
    }
    return v;
  }
};
template <Edge EDGE> struct Stored<bf16, EDGE> {
  typedef u32x2u type;
  template <bool ONCE> static __device__ __forceinline__ type load(const bf16* p, int c, int d) {
    if constexpr (EDGE == kTiny) {
      auto at = [&](int e) { return e < d ? (uint32_t)__builtin_bit_cast(unsigned short, p[e]) : 0u; };
      return type{at(0) | at(1) << 16, at(2)};
    }
    const type* const at = reinterpret_cast<const type*>(p + (EDGE == kWhole ? c : last4(c, d)));
    return ONCE ? __builtin_nontemporal_load(at) : *at;
  }
  static __device__ __forceinline__ f32x4 wide(const type& w, int c, int d) {
    type v = w;
    const int off = EDGE == kWhole ? 0 : EDGE == kTiny ? c : c - last4(c, d);
    if (off > 0) {
      const uint64_t x = off < 4 ? ((uint64_t)w[1] << 32 | w[0]) >> (16 * off) : 0;
      v = type{(uint32_t)x, (uint32_t)(x >> 32)};
    }
    return f32x4{__uint_as_float(v[0] << 16), __uint_as_float(v[0] & 0xffff0000u), __uint_as_float(v[1] << 16), __uint_as_float(v[1] & 0xffff0000u)};
  }
};
template <Edge EDGE> __device__ __forceinline__ void store4(float* p, int c, int d, const f32x4& v) {
  if (EDGE == kWhole || c + 4 <= d) {
    *reinterpret_cast<f32x4u*>(p + c) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (c + e < d) p[c + e] = v[e];
  }
}
template <Edge EDGE> __device__ __forceinline__ void store4(bf16* p, int c, int d, const f32x4& v) {
  const bf16x4 o = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
  if (EDGE == kWhole || c + 4 <= d) {
    *reinterpret_cast<u16x4u*>(p + c) = __builtin_bit_cast(u16x4u, o);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (c + e < d) p[c + e] = o[e];
  }
}

struct RmsFwdParams {
  const float* x;
  const void* y;
  const float* g;
  float* x_out;
  void* h;
  uint8_t *q, *scale;
  float* rstd;
  int64_t rows, ldx, ldh, ldq;
  int d;
  float eps;
};

// NT threads to a row, VEC times four columns to a thread; a block of 64 threads per row has four rows.  F8: 0 no 8-bit output, 1 e4m3, 2 e5m2.
template <int NT> constexpr int kBlock = NT < 256 ? 256 : NT;
template <class T, int NT, int VEC, int F8, Edge EDGE>
__global__ __launch_bounds__(kBlock<NT>) void rmsnorm_fwd_kernel(RmsFwdParams p) {
  typedef Stored<float, EDGE> Wide;
  typedef Stored<T, EDGE> Narrow;
  constexpr int kTeams = kBlock<NT> / NT, kWaves = NT / 64;
  __shared__ float red[3][NT > 64 ? kWaves : 1];
  const int team = NT < 256 ? threadIdx.x / NT : 0, t = threadIdx.x % NT, d = p.d;
  const int64_t step = (int64_t)gridDim.x * kTeams;
  const float inv_d = 1.f / (float)d;
  f32x4 v[VEC];
  typename Wide::type nx[VEC];
  typename Narrow::type ny[VEC];
  // The next row of this team travels while the current one is reduced and stored.
  auto fetch = [&](int64_t n) {
    const float* const xr = p.x + n * p.ldx;
#pragma unroll
    for (int i = 0; i < VEC; ++i) nx[i] = Wide::template load<true>(xr, 4 * (t + i * NT), d);
    if (p.y) {
      const T* const yr = reinterpret_cast<const T*>(p.y) + n * p.ldh;
#pragma unroll
      for (int i = 0; i < VEC; ++i) ny[i] = Narrow::template load<true>(yr, 4 * (t + i * NT), d);
    }
  };
  // Over the team; the sums of two calls in turn lie apart, so that one barrier is enough.
  auto across = [&](float s, int place) {
    s = lanes_sum(s);
    if constexpr (NT > 64) {
      if ((t & 63) == 0) red[place][t >> 6] = s;
      __syncthreads();
      s = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) s += red[place][w];
    }
    return s;
  };
  int64_t n = (int64_t)blockIdx.x * kTeams + team;
  if (NT == 64 && n >= p.rows) return;
  if (n < p.rows) fetch(n);
  int phase = 0;
  for (; n < p.rows; n += step, phase ^= 1) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      v[i] = Wide::wide(nx[i], 4 * (t + i * NT), d);
      if (p.y) v[i] += Narrow::wide(ny[i], 4 * (t + i * NT), d);
    }
    if (n + step < p.rows) fetch(n + step);
#pragma unroll
    for (int i = 0; i < VEC; ++i) s += (v[i][0] * v[i][0] + v[i][1] * v[i][1]) + (v[i][2] * v[i][2] + v[i][3] * v[i][3]);
    s = across(s, phase);
    float r = 1.f / sqrtf(s * inv_d + p.eps);
    // Squares that leave the range of 32 bits: once more, of values scaled by a power of two (uniform over the team).
    const float mean = s * inv_d + p.eps;
    if (!(mean > 0x1p-110f && s < INFINITY)) {
      const float k = s < INFINITY ? 0x1p100f : 0x1p-80f;
      s = 0.f;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const f32x4 w = v[i] * k;
        s += (w[0] * w[0] + w[1] * w[1]) + (w[2] * w[2] + w[3] * w[3]);
      }
      r = k / sqrtf(across(s, 2) * inv_d + p.eps * k * k);
    }
    if (p.rstd && t == 0) p.rstd[n] = r;
    if (p.x_out) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) store4<EDGE>(p.x_out + n * p.ldx, 4 * (t + i * NT), d, v[i]);
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const int c = 4 * (t + i * NT);
      f32x4 h = v[i] * r;
      h *= Wide::wide(Wide::template load<false>(p.g, c, d), c, d);
      if (p.h) store4<EDGE>(reinterpret_cast<T*>(p.h) + n * p.ldh, c, d, h);
      if constexpr (F8 != 0) {
        constexpr bool E5M2 = F8 == 2;
        uint32_t m = 0;
        if (EDGE != kWhole && c + 4 > d) {   // zeros behind the row, also where r is NaN
#pragma unroll
          for (int e = 0; e < 4; ++e) h[e] = c + e < d ? h[e] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t a = __float_as_uint(h[e]) & 0x7fffffffu;
          m = max(m, a < 0x7f800000u ? a : 0u);
        }
        const uint32_t byte = scale_byte<E5M2>(lanes_max_bits<32>(m));
        const uint32_t o = pack_f32<E5M2>(__float_as_uint(h[0]), __float_as_uint(h[1]), __float_as_uint(h[2]), __float_as_uint(h[3]),
                                          __uint_as_float(byte << 23));
        if (c < ((d + 15) & ~15)) *reinterpret_cast<uint32_t*>(p.q + n * p.ldq + c) = o;
        const int first = c & ~127;          // column of the block
        if ((t & 31) == 0 && c < d) p.scale[scale_at(n, first >> 7, p.rows)] = (uint8_t)byte;
        if (n == p.rows - 1 && first < d) {  // rows that do not exist
          const int64_t end = (p.rows + 63) & ~63LL;
          for (int64_t k = p.rows + (t & 31); k < end; k += 32) p.scale[scale_at(k, first >> 7, p.rows)] = 0;
        }
      }
    }
  }
}

// f(threads to a row, vectors to a thread).  A wave to a row where there are enough rows to fill the chip, else a block, whose threads have less
// of it to wait for.
template <class F> void by_size(int64_t rows, int64_t d, F&& f) {
  using std::integral_constant;
  const bool many = rows >= 1024;
  if (d <= 256) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (d <= 512 && many) f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  else if (d <= 1024 && many) f(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  else if (d <= 2048 && many) f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  else if (d <= 1024) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (d <= 2048) f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (d <= 4096) f(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  else if (d <= 8192 && many) f(integral_constant<int, 256>{}, integral_constant<int, 8>{});
  else if (d <= 8192) f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  else f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}
template <int NT, int VEC, class F> void by_edge(int64_t d, F&& f) {
  using std::integral_constant;
  if (d == 4 * NT * VEC) return f(integral_constant<Edge, kWhole>{});
  if constexpr (NT == 64 && VEC == 1)
    if (d < 4) return f(integral_constant<Edge, kTiny>{});
  f(integral_constant<Edge, kAny>{});
}
constexpr int64_t kMaxCols = 16384, kMaxRows = (1LL << 31) - 1;

// ---- backward ----------------------------------------------------------------------------------------------------
// ROWS rows at a time to a team of NT threads; dg's running sums stay in registers, a team's go to ws[team][:] and a second kernel adds the
// teams in order (the same bits on every run); one team writes dg itself.
struct RmsBwdParams {
  const void* dh;
  const float *x, *g, *rstd, *dres;
  float* dx;
  void* dy;
  float* part;                               // [teams][stride], or null: dg is not wanted
  int64_t rows, ldx, ldh, stride;
  int d, accumulate;                         // accumulate: one team adds into dg
};
template <class T, int NT, int VEC, int ROWS, Edge EDGE>
__global__ __launch_bounds__(NT) void rmsnorm_bwd_kernel(RmsBwdParams p) {
  typedef Stored<float, EDGE> Wide;
  typedef Stored<T, EDGE> Narrow;
  constexpr int kWaves = NT / 64;
  __shared__ float red[2][ROWS][kWaves];
  const int t = threadIdx.x, d = p.d;
  const int64_t step = (int64_t)gridDim.x * ROWS;
  const float inv_d = 1.f / (float)d;
  f32x4 gv[VEC], acc[VEC];
  typename Wide::type xv[ROWS][VEC], rv[ROWS][VEC];
  typename Narrow::type dv[ROWS][VEC];
  float rs[ROWS];
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    gv[i] = Wide::wide(Wide::template load<false>(p.g, 4 * (t + i * NT), d), 4 * (t + i * NT), d);
    acc[i] = f32x4{};
  }
  auto fetch = [&](int64_t n0) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int64_t n = n0 + r;
      if (n >= p.rows) break;                // uniform
      rs[r] = p.rstd[n];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int c = 4 * (t + i * NT);
        xv[r][i] = Wide::template load<true>(p.x + n * p.ldx, c, d);
        dv[r][i] = Narrow::template load<true>(reinterpret_cast<const T*>(p.dh) + n * p.ldh, c, d);
        if (p.dres) rv[r][i] = Wide::template load<true>(p.dres + n * p.ldx, c, d);
      }
    }
  };
  int64_t n0 = (int64_t)blockIdx.x * ROWS;
  constexpr bool kAhead = NT < 1024;         // 128 registers to a thread hold a row's arrays once
  if (kAhead && n0 < p.rows) fetch(n0);
  int phase = 0;
  for (; n0 < p.rows; n0 += step, phase ^= 1) {
    if (!kAhead) fetch(n0);
    f32x4 xh[ROWS][VEC], dg[ROWS][VEC], dr[ROWS][VEC];
    float sum[ROWS], rr[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      sum[r] = 0.f;
      rr[r] = rs[r];
      if (n0 + r >= p.rows) continue;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int c = 4 * (t + i * NT);
        const f32x4 dh = Narrow::wide(dv[r][i], c, d);
        xh[r][i] = Wide::wide(xv[r][i], c, d) * rr[r];
        if (p.dres) dr[r][i] = Wide::wide(rv[r][i], c, d);
        acc[i] += dh * xh[r][i];
        dg[r][i] = dh * gv[i];
        const f32x4 m = dg[r][i] * xh[r][i];
        sum[r] += (m[0] + m[1]) + (m[2] + m[3]);
      }
    }
    if (kAhead && n0 + step < p.rows) fetch(n0 + step);   // the next rows travel while these are reduced and stored
#pragma unroll
    for (int r = 0; r < ROWS; ++r) sum[r] = lanes_sum(sum[r]);
    if constexpr (kWaves > 1) {
      if ((t & 63) == 0) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) red[phase][r][t >> 6] = sum[r];
      }
      __syncthreads();
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        sum[r] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum[r] += red[phase][r][w];
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int64_t n = n0 + r;
      if (n >= p.rows) break;
      const float m = sum[r] * inv_d;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int c = 4 * (t + i * NT);
        f32x4 o = (dg[r][i] - xh[r][i] * m) * rr[r];
        if (p.dres) o += dr[r][i];
        store4<EDGE>(p.dx + n * p.ldx, c, d, o);
        if (p.dy) store4<EDGE>(reinterpret_cast<T*>(p.dy) + n * p.ldh, c, d, o);
      }
    }
  }
  if (!p.part) return;
  float* const out = p.part + (int64_t)blockIdx.x * p.stride;
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    const int c = 4 * (t + i * NT);
    if (p.accumulate) acc[i] += Wide::wide(Wide::template load<false>(out, c, d), c, d);
    store4<EDGE>(out, c, d, acc[i]);
  }
}
constexpr int kBwdTeams = 512;
// Rows that a team takes at a time: what its registers hold twice over, with two waves to a SIMD; fewer where rows do not fill the vectors, which takes registers
// too (us with 4 or 2 rows and with 2 or 1: 3000 x 2001 bf16 28.4 and 25.2, 8192 x 1500 53.4 and 44.8, 3000 x 2500 42.5 and 33.3; 8192 x 2048, whole, 50.3 with
// 4 and 51.5 with 2).
template <int NT, int VEC, Edge EDGE> constexpr int kBwdRows =
    NT != 256 ? (VEC <= 2 ? 4 : 1) : EDGE == kWhole || VEC == 1 ? (VEC <= 2 ? 4 : 2) : VEC == 2 ? 2 : 1;
// Threads to a row, vectors to a thread: registers are shared among more threads than in the forward pass, which holds less of a row.
template <class F> void by_width_bwd(int64_t d, F&& f) {
  using std::integral_constant;
  if (d <= 256) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (d <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  else if (d <= 1024) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (d <= 2048) f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (d <= 4096) f(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  else if (d <= 8192) f(integral_constant<int, 512>{}, integral_constant<int, 4>{});
  else f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}
int bwd_rows(int64_t d) {
  int rows = 0;
  by_width_bwd(d, [&](auto nt, auto vec) {
    constexpr int NT = decltype(nt)::value, VEC = decltype(vec)::value;
    by_edge<NT, VEC>(d, [&](auto edge) { rows = kBwdRows<NT, VEC, decltype(edge)::value>; });
  });
  return rows;
}
int64_t bwd_teams(int64_t rows, int64_t d) {
  const int per = bwd_rows(d);
  const int64_t teams = (rows + per - 1) / per, most = d <= 512 ? 4 * kBwdTeams : kBwdTeams;
  return teams < most ? teams : most;
}

hipError_t check(const RmsnormArgs& a) {
  if ((a.dtype != kF32 && a.dtype != kBF16) || !a.g || a.rows < 0 || a.rows > kMaxRows || a.cols < 1 || a.cols > kMaxCols || a.ldx < a.cols ||
      a.ldh < a.cols || !(a.eps >= 0.f) || ((uintptr_t)a.g & 3))
    return hipErrorInvalidValue;
  return hipSuccess;
}
bool misaligned(const void* p, int dtype) { return (uintptr_t)p & (dtype == kBF16 ? 1 : 3); }

}  // namespace

hipError_t launch_rmsnorm_fwd(hipStream_t s, const RmsnormArgs& a, const float* x, const void* y, float* x_out, void* h, const F8Out& q, float* rstd) {
  if (check(a) != hipSuccess || !x || (!h && !q.q)) return hipErrorInvalidValue;
  if (misaligned(x, kF32) || misaligned(y, a.dtype) || misaligned(x_out, kF32) || misaligned(h, a.dtype) || misaligned(rstd, kF32))
    return hipErrorInvalidValue;
  if (q.q && ((q.format != kE4M3 && q.format != kE5M2) || !q.scale || ((uintptr_t)q.scale & 3) || ((uintptr_t)q.q & 15) || q.ldq % 16 ||
              q.ldq < a.cols || a.rows > (1LL << 30)))
    return hipErrorInvalidValue;
  if (a.rows == 0) return hipSuccess;
  const RmsFwdParams p{x, y, a.g, x_out, h, (uint8_t*)q.q, q.scale, rstd, a.rows, a.ldx, a.ldh, q.ldq, (int)a.cols, a.eps};
  auto run = [&](auto t, auto f8) {
    by_size(a.rows, a.cols, [&](auto nt, auto vec) {
      constexpr int NT = decltype(nt)::value, VEC = decltype(vec)::value, kTeams = kBlock<NT> / NT;
      const int64_t blocks = (a.rows + kTeams - 1) / kTeams, most = NT == 1024 ? 512 : NT == 256 ? 2048 : 1024;
      const unsigned grid = (unsigned)(blocks < most ? blocks : most);
      by_edge<NT, VEC>(a.cols, [&](auto edge) {
        rmsnorm_fwd_kernel<decltype(t), NT, VEC, decltype(f8)::value, decltype(edge)::value><<<grid, kBlock<NT>, 0, s>>>(p);
      });
    });
  };
  auto format = [&](auto t) {
    if (!q.q) run(t, std::integral_constant<int, 0>{});
    else if (q.format == kE4M3) run(t, std::integral_constant<int, 1>{});
    else run(t, std::integral_constant<int, 2>{});
  };
  if (a.dtype == kF32) format(float{});
  else format(bf16{});
  return hipGetLastError();
}

int64_t rmsnorm_bwd_ws_floats(int64_t rows, int64_t cols) {
  if (rows < 0 || rows > kMaxRows || cols < 1 || cols > kMaxCols) return -1;
  const int64_t teams = bwd_teams(rows, cols);
  return teams > 1 ? teams * ((cols + 3) & ~3LL) : 0;
}

hipError_t launch_rmsnorm_bwd(hipStream_t s, const RmsnormArgs& a, const void* dh, const float* x, const float* rstd, const float* dres, float* dx,
                              void* dy, float* dg, float* ws, int accumulate) {
  if (check(a) != hipSuccess || !dh || !x || !rstd || !dx) return hipErrorInvalidValue;
  if (misaligned(dh, a.dtype) || misaligned(x, kF32) || misaligned(rstd, kF32) || misaligned(dres, kF32) || misaligned(dx, kF32) ||
      misaligned(dy, a.dtype) || misaligned(dg, kF32))
    return hipErrorInvalidValue;
  const int64_t teams = bwd_teams(a.rows, a.cols);
  if (dg && teams > 1 && (!ws || ((uintptr_t)ws & 15))) return hipErrorInvalidValue;
  if (a.rows == 0) return dg && !accumulate ? launch_reduce_parts(s, dg, dg, 0, 0, a.cols, 0) : hipSuccess;   // zeros
  const int64_t stride = (a.cols + 3) & ~3LL;
  const bool alone = teams == 1;
  const RmsBwdParams p{dh, x, a.g, rstd, dres, dx, dy, dg ? (alone ? dg : ws) : nullptr, a.rows, a.ldx, a.ldh, stride, (int)a.cols,
                       alone && accumulate};
  auto run = [&](auto t) {
    by_width_bwd(a.cols, [&](auto nt, auto vec) {
      constexpr int NT = decltype(nt)::value, VEC = decltype(vec)::value;
      by_edge<NT, VEC>(a.cols, [&](auto edge) {
        rmsnorm_bwd_kernel<decltype(t), NT, VEC, kBwdRows<NT, VEC, decltype(edge)::value>, decltype(edge)::value><<<(unsigned)teams, NT, 0, s>>>(p);
      });
    });
  };
  if (a.dtype == kF32) run(float{});
  else run(bf16{});
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || !dg || alone ? e : launch_reduce_parts(s, ws, dg, (int)teams, stride, a.cols, accumulate);
}

}  // namespace pw
