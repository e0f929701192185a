// Gated linear recurrence along a sequence, every channel on its own:
//
//   a_t = sigmoid(f_t),  h_t = a_t h_(t-1) + (1 - a_t) x_t,  y_t = h_t
//
// and backward, with r_t = a_t g_t what step t hands to the step before it:
//
//   g_t = dy_t + r_(t+1),  dx_t = g_t (1 - a_t),  df_t = g_t (h_(t-1) - x_t) a_t (1 - a_t),  dh_0 = r_1.
//
// A step is the map h -> a h + v, and maps compose: (P, S) after (p, s) is (P p, P s + S).  A thread takes 16 consecutive
// steps of its two channels into registers and composes them, the two halves of a wave exchange their maps, the waves of a
// block hand theirs over through LDS, and every thread then runs its steps again from the state in front of them: inputs are
// read once, nothing but outputs is written.  A block has 64 channels, so that a row of it is a whole cache line of bf16, and a
// tile of 32 steps for each of its up to 8 waves; it walks down its tiles with the state in registers.  The forward pass keeps
// the state in front of each tile (fp32, one value per channel and tile); the backward pass starts every tile from it and
// walks upwards.
//
// The least traffic is three arrays forward and five backward.  bf16 tiles come by direct loads into LDS while the one before
// is at work (registers hold one tile: 205 of 256 in the backward pass, which leaves it two waves to a SIMD; the forward pass is
// kept to 128, so that two blocks of a second round fit a unit: 12 x 1024 x 2048 50.2 us -> 46.9, now 46.3).  8 x 1024 x 2048 bf16:
// 27.4 us forward (3.7 TB/s; a copy reaches 5.15), 48.7 backward, 41 right behind the forward pass of the same arrays.  256 blocks of 8 waves are one to a unit, so the forward pass too has two waves to a SIMD there, of the four
// that its registers allow; of 28 us it took 23 without stores, 25 without exponentials, 19 without both: neither hides all of the
// other.  fp32 comes without loads ahead: 50.4 and 81.8 us (4.0 and 4.1 TB/s).  Blocks of 32 channels, two to a unit, read and write
// half lines: 33 and 52 us.  A second tile ahead wins nothing.  16 steps to a thread halve the exchanges that 8 steps take.
//
// Few channels leave compute units idle.  The sequence is then cut into segments of whole tiles (plan_of): a first launch
// composes each segment into one map, the second composes the maps in front of its segment (behind it, backward) and goes on as
// above.  1 x 16384 x 512 bf16: 24.0 us forward, 31.5 backward; fp32 37.6 and 57.6.
//
// Steps behind the end of a sequence (lens) are the identity map with outputs of zero, whatever their inputs hold: in their place a
// row of the tile is read (its first, where none is before the end) and dropped.
// Sums, states and gates are fp32; y, df and dx are rounded once.  All orders are fixed: the same bits on every run.
#include <type_traits>
#include <utility>

#include "common.hpp"
#include "kernels.hpp"

namespace pw {

namespace {

constexpr int kSteps = 16;         // consecutive steps of a thread
constexpr int kFew = 2;             // steps that a tile of hardly any is cut down to
constexpr int kVec = 2;            // channels of a thread
constexpr int kLanes = 32;         // lanes side by side along the channels; a wave's parts follow one another in time
constexpr int kParts = kWave / kLanes, kLevels = 1;
static_assert(1 << kLevels == kParts, "parts meet in pairs");
constexpr int kWaveSteps = kSteps * kParts;
constexpr int kMostWaves = 8;
constexpr int kChannels = kVec * kLanes;
constexpr int64_t kMostLd = 1 << 21;     // a tile's rows are within 32 bits of offset

int waves_of(int T) {
  const int w = (int)(((int64_t)T + kWaveSteps - 1) / kWaveSteps);
  return w < 1 ? 1 : (w > kMostWaves ? kMostWaves : w);
}
int tile_of(int T) { return waves_of(T) * kWaveSteps; }
int tiles_of(int T) { return (int)(((int64_t)T + tile_of(T) - 1) / tile_of(T)); }

struct Params {
  const void *f, *x, *dy;
  void *y, *df, *dx;
  int64_t ldf, ldx, ldy, lddf, lddx;     // ldy: of y (forward) or dy (backward)
  const float *h0, *dh_end;
  float *h_end, *dh0, *states;
  float2* maps;                          // [block of channels][segments][kChannels]
  const int32_t* lens;
  int T, D, tiles, segments, seg_tiles;
  uint32_t groups, base;                 // groups of channels of a sequence; the launch's first block of channels
  int dma;                               // pairs of bf16 channels start on four bytes everywhere
};

// The channels of a thread, wherever they start.
template <class T> struct Raw;
template <> struct Raw<bf16> { typedef __bf16 type __attribute__((ext_vector_type(kVec), aligned(2))); };
template <> struct Raw<float> { typedef float type __attribute__((ext_vector_type(kVec), aligned(4))); };
// Gates and their products are positive, as sigmoid and its products are: where one falls below what fp32 holds it stays there, so
// that an infinite state is one behind it too (0 times it would be NaN).  Of a finite one a shut gate leaves 2^-125.
constexpr float kLeast = 0x1p-149f;
__device__ __forceinline__ float positive(float p) { return __builtin_fmaxf(p, kLeast); }
// e^-f, at most 2^125, whose reciprocal is not yet cut to 0; NaN with f.  Off by 2 |f| 2^-24 of itself: the argument is rounded.
__device__ __forceinline__ float decay(float f) {
  return __builtin_amdgcn_exp2f(__builtin_elementwise_minimum(-1.4426950408889634f * f, 125.f));
}
// a = sigmoid(f) and z = 1 - a; neither comes from a difference that cancels.
__device__ __forceinline__ void gate(float f, float& a, float& z) {
  const float e = decay(f);
  a = __builtin_amdgcn_rcpf(1.f + e);
  z = __builtin_fmaf(e, a, kLeast);
}
// The same in one register: the smaller of the two, negative where that is a.  The other one is 1 minus it, to half a unit.
__device__ __forceinline__ float packed_gate(float f) {
  const float e = decay(f), a = __builtin_amdgcn_rcpf(1.f + e);
  return e > 1.f ? -a : __builtin_fmaf(e, a, kLeast);
}
__device__ __forceinline__ void unpack_gate(float g, float& a, float& z) {
  const float other = 1.f - __builtin_fabsf(g);
  const bool of_a = (int)__float_as_uint(g) < 0;
  a = of_a ? -g : other;
  z = of_a ? other : g;
}

struct Where {
  int64_t b;
  int c, n, shift, sub, wave, part, li, nw, len; // n: channels of the lane that exist; it reads them `shift` further left,
  bool whole;                                    // where a row ends.  whole: every lane of the block has all of its channels
};
__device__ __forceinline__ Where where(const Params& p) {
  Where w;
  const uint32_t id = p.base + blockIdx.x;
  const int g = (int)(id % p.groups);
  w.b = id / p.groups;
  w.wave = threadIdx.x >> 6;
  w.part = (threadIdx.x / kLanes) % kParts;
  w.li = threadIdx.x % kLanes;
  w.sub = kParts * w.wave + w.part;
  w.nw = blockDim.x >> 6;
  w.c = (g * kLanes + w.li) * kVec;
  w.n = p.D - w.c < 0 ? 0 : (p.D - w.c < kVec ? p.D - w.c : kVec);
  w.whole = (g + 1) * kChannels <= p.D;
  const int last = p.D - kVec > 0 ? p.D - kVec : 0;
  w.shift = w.c > last ? w.c - last : 0;
  w.len = p.T;
  if (p.lens) {
    const int l = p.lens[w.b];
    w.len = l < 0 ? 0 : (l > p.T ? p.T : l);
  }
  return w;
}

// One array seen by a thread: its steps of a tile are rows of `ld` elements behind a wave-uniform base, at an offset that stays
// the same from tile to tile (32 bits hold it: kMostLd).  What is read begins with the last channels of a row where the lane's
// own are not all there.
template <class T>
struct Column {
  const char* base;                              // row 0 of the sequence
  int64_t row;                                   // bytes
  uint32_t col, off;
  __device__ __forceinline__ Column(const void* p, int64_t ld, const Where& w, int T_, bool written = false)
      : base(reinterpret_cast<const char*>(p) + w.b * T_ * ld * (int64_t)sizeof(T)), row(ld * (int64_t)sizeof(T)),
        col((uint32_t)(written ? w.c : w.c - w.shift) * (uint32_t)sizeof(T)), off((uint32_t)(w.sub * kSteps) * (uint32_t)row + col) {}
  __device__ __forceinline__ const char* at(int tile0, int i) const { return base + (tile0 + i) * row + off; }
};
// Own channels first (in a lane without channels anything will do).  Branches are kept out of the loops over steps: they keep the
// loads of a tile from being asked for together.
template <class T> __device__ __forceinline__ void align(const Where& w, typename Raw<T>::type (&r)[kSteps]) {
  static_assert(kVec == 2, "a shift of one");
  if (!w.whole) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) r[i][0] = w.shift ? r[i][1] : r[i][0];
  }
}
// The steps of the tile that begins at step tile0.  WHOLE: all steps exist; else those that do not come out as zeros (fetched in
// their place is another row of the tile).
template <class T, bool WHOLE>
__device__ __forceinline__ void fetch(const Column<T>& q, const Where& w, const Params& p, int tile0, typename Raw<T>::type (&r)[kSteps]) {
  typedef typename Raw<T>::type raw;
  const int end = w.len - tile0, top = end > 0 ? end - 1 : 0;
  auto place = [&](int i) {
    const int t = w.sub * kSteps + i;
    return WHOLE ? q.at(tile0, i) : q.base + tile0 * q.row + ((uint32_t)(t < top ? t : top) * (uint32_t)q.row + q.col);
  };
  auto load = [&](auto count) {
    if (p.D >= kVec) {
#pragma unroll
      for (int i = 0; i < decltype(count)::value; ++i) r[i] = *reinterpret_cast<const raw*>(place(i));
    } else {
#pragma unroll
      for (int i = 0; i < decltype(count)::value; ++i) r[i][0] = *reinterpret_cast<const T*>(place(i));
    }
  };
  if constexpr (WHOLE) {
    load(std::integral_constant<int, kSteps>{});
    align<T>(w, r);
  } else {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) r[i] = raw{};
    if (end > kFew) load(std::integral_constant<int, kSteps>{});
    else load(std::integral_constant<int, kFew>{});
    align<T>(w, r);
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int j = 0; j < kVec; ++j) r[i][j] = w.sub * kSteps + i < end ? r[i][j] : (T)0.f;
  }
}
// FULL: every lane of the block has all of its channels.
template <class T, bool WHOLE, bool FULL>
__device__ __forceinline__ void put(const Column<T>& q, const Where& w, int tile0, int T_, int i, const float* v) {
  if (!WHOLE && tile0 + w.sub * kSteps + i >= T_) return;
  T* const g = reinterpret_cast<T*>(const_cast<char*>(q.at(tile0, i)));
  if (FULL || w.n == kVec) {
    typename Raw<T>::type r;
#pragma unroll
    for (int j = 0; j < kVec; ++j) r[j] = (T)v[j];
    *reinterpret_cast<typename Raw<T>::type*>(g) = r;
  } else if (w.n) {
    *g = (T)v[0];
  }
}

// Maps of a stretch of steps: of the state walking down (DIRS & 1) and of r walking up (DIRS & 2); both have the same product.
enum { kDown = 1, kUp = 2 };
template <int DIRS> struct Map { float p[kVec], s[DIRS == 3 ? 2 : 1][kVec]; };
template <int DIRS, int D> constexpr int sum_of() { return DIRS == 3 && D == kUp ? 1 : 0; }

template <int DIRS> __device__ __forceinline__ Map<DIRS> exchanged(const Map<DIRS>& m, int lanes) {
  Map<DIRS> o;
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    o.p[j] = __shfl_xor(m.p[j], lanes, kWave);
#pragma unroll
    for (int d = 0; d < (DIRS == 3 ? 2 : 1); ++d) o.s[d][j] = __shfl_xor(m.s[d][j], lanes, kWave);
  }
  return o;
}
template <int DIRS, int D> __device__ __forceinline__ void apply(const Map<DIRS>& m, float (&h)[kVec]) {
#pragma unroll
  for (int j = 0; j < kVec; ++j) h[j] = __builtin_fmaf(m.p[j], h[j], m.s[sum_of<DIRS, D>()][j]);
}
// The map of two neighbouring stretches, `mine` the earlier one or not.
template <int DIRS> __device__ __forceinline__ Map<DIRS> joined(const Map<DIRS>& mine, const Map<DIRS>& other, bool earlier) {
  Map<DIRS> r;
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    r.p[j] = positive(mine.p[j] * other.p[j]);
    auto after = [&](float first, float p, float s) { return __builtin_fmaf(p, first, s); };
    if (DIRS & kDown) {
      constexpr int d = sum_of<DIRS, kDown>();
      r.s[d][j] = earlier ? after(mine.s[d][j], other.p[j], other.s[d][j]) : after(other.s[d][j], mine.p[j], mine.s[d][j]);
    }
    if (DIRS & kUp) {
      constexpr int d = sum_of<DIRS, kUp>();
      r.s[d][j] = earlier ? after(other.s[d][j], mine.p[j], mine.s[d][j]) : after(mine.s[d][j], other.p[j], other.s[d][j]);
    }
  }
  return r;
}

// down: the state in front of the block's tile, up: the r handed in from behind it; each is replaced by the one on the other
// side.  in_down, in_up: what reaches this thread's steps, whose map is `mine`.  slot: LDS of this tile, [waves][lanes].
template <int DIRS>
__device__ __forceinline__ void compose(Map<DIRS>* slot, const Where& w, const Map<DIRS>& mine, float (&down)[kVec], float (&in_down)[kVec],
                                        float (&up)[kVec], float (&in_up)[kVec]) {
  Map<DIRS> others[kLevels], all = mine;
#pragma unroll
  for (int l = 0; l < kLevels; ++l) {
    others[l] = exchanged(all, kLanes << l);
    all = joined(all, others[l], ((w.part >> l) & 1) == 0);
  }
  if (w.part == 0) slot[w.wave * kLanes + w.li] = all;
  // What the waves exchange is in LDS: loads and stores of other data stay on their way.
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  const int wave = __builtin_amdgcn_readfirstlane(w.wave);
  const Map<DIRS>* const at = slot + w.li;
  if (DIRS & kDown) {
    for (int k = 0; k < wave; ++k) apply<DIRS, kDown>(at[k * kLanes], down);
#pragma unroll
    for (int j = 0; j < kVec; ++j) in_down[j] = down[j];
    for (int k = wave; k < w.nw; ++k) apply<DIRS, kDown>(at[k * kLanes], down);
#pragma unroll
    for (int l = kLevels - 1; l >= 0; --l)
      if ((w.part >> l) & 1) apply<DIRS, kDown>(others[l], in_down);
  }
  if (DIRS & kUp) {
    for (int k = w.nw - 1; k > wave; --k) apply<DIRS, kUp>(at[k * kLanes], up);
#pragma unroll
    for (int j = 0; j < kVec; ++j) in_up[j] = up[j];
    for (int k = wave; k >= 0; --k) apply<DIRS, kUp>(at[k * kLanes], up);
#pragma unroll
    for (int l = kLevels - 1; l >= 0; --l)
      if (!((w.part >> l) & 1)) apply<DIRS, kUp>(others[l], in_up);
  }
}

__device__ __forceinline__ float2* maps_of(const Params& p, const Where& w) {
  return p.maps + (int64_t)blockIdx.x * p.segments * kChannels + w.li * kVec;
}
// What reaches segment `seg`: the maps of the slots 1 .. seg (down) or segments - 2 .. seg (up), the first of which is a
// constant: what leaves the first (last) segment.  That one has a slot to itself, 0 (segments - 1), with what comes in.  Each part of
// a wave composes a stretch of them, then they meet as they do in a tile.
template <int D>
__device__ __forceinline__ void segment_carry(Map<D>* slot, const Where& w, const Params& p, int seg, float (&carry)[kVec]) {
  const int subs = kParts * w.nw, from = D == kDown && seg > 0 ? 1 : seg;
  const int n = D == kDown ? seg + 1 - from : (seg < p.segments - 1 ? p.segments - 1 - seg : 1), per = (n + subs - 1) / subs;
  Map<D> m;
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    m.p[j] = 1.f;
    m.s[0][j] = 0.f;
    carry[j] = 0.f;
  }
  for (int i = 0; i < per; ++i) {
    const int k = D == kDown ? w.sub * per + i : n - 1 - ((subs - 1 - w.sub) * per + i);
    if (D == kDown ? k < n : k >= 0) {
      const float2* q = maps_of(p, w) + (from + k) * kChannels;
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        if (j < w.n) {
          const float2 v = q[j];
          m.s[0][j] = __builtin_fmaf(v.x, m.s[0][j], v.y);
          m.p[j] = positive(m.p[j] * v.x);
        }
      }
    }
  }
  float in[kVec], none[kVec] = {}, none2[kVec];
  if constexpr (D == kDown) compose<D>(slot, w, m, carry, in, none, none2);
  else compose<D>(slot, w, m, none, none2, carry, in);
}

// The next tile of N bf16 arrays on its way into LDS, without registers: a wave fetches the steps its own threads will take,
// 256 bytes at a time, and a lane finds its two channels of step i of array n at [n][i][lane].
template <int N> struct Ahead {
  typedef __attribute__((address_space(3))) void* lds_ptr;
  static constexpr int kBytes = N * kSteps * kWave * 4;   // of a wave
  uint32_t (*mine)[kSteps][kWave];               // this wave's part
  uint32_t at;                                   // its offset in LDS
  __device__ __forceinline__ Ahead(uint8_t* lds, const Where& w) {
    mine = reinterpret_cast<uint32_t (*)[kSteps][kWave]>(lds + w.wave * kBytes);
    at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr)mine);
  }
  __device__ __forceinline__ void ask(int n, const Column<bf16>& q, int tile0) const {
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(q.off), "s"(q.base + (tile0 + i) * q.row),
                   "s"(at + (n * kSteps + i) * (kWave * 4)) : "memory", "m0");
  }
  __device__ __forceinline__ void take(int n, const Where& w, Raw<bf16>::type (&r)[kSteps]) const {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) r[i] = __builtin_bit_cast(bf16x2, mine[n][i][threadIdx.x & 63]);
    align<bf16>(w, r);
  }
  // Between take() of one tile and ask() for the next: what was read is in registers.
  __device__ __forceinline__ static void taken() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
  // In front of the tile's stores, behind which this would wait for those.
  __device__ __forceinline__ static void landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
};
// Gates of the steps of a tile; a = 1 where there is no step.  In a tile of few steps (kFew) no lane computes more.
template <bool WHOLE, class F> __device__ __forceinline__ void for_steps(const Where& w, int tile0, F&& f) {
  if (WHOLE || w.len - tile0 > kFew) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) f(i);
  } else {
#pragma unroll
    for (int i = 0; i < kFew; ++i) f(i);
  }
}
template <class T, bool WHOLE>
__device__ __forceinline__ void gates(const typename Raw<T>::type (&rf)[kSteps], const Where& w, int tile0, float (&a)[kSteps][kVec],
                                      float (&z)[kSteps][kVec]) {
  if (!WHOLE) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        a[i][j] = 1.f;
        z[i][j] = 0.f;
      }
  }
  for_steps<WHOLE>(w, tile0, [&](int i) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      float ai, zi;
      gate((float)rf[i][j], ai, zi);
      const bool there = WHOLE || tile0 + w.sub * kSteps + i < w.len;
      a[i][j] = there ? ai : 1.f;
      z[i][j] = there ? zi : 0.f;
    }
  });
}
template <class T, bool WHOLE>
__device__ __forceinline__ void packed_gates(const typename Raw<T>::type (&rf)[kSteps], const Where& w, int tile0, float (&g)[kSteps][kVec]) {
  if (!WHOLE) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int j = 0; j < kVec; ++j) g[i][j] = 0.f;
  }
  for_steps<WHOLE>(w, tile0, [&](int i) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const float gi = packed_gate((float)rf[i][j]);
      g[i][j] = WHOLE || tile0 + w.sub * kSteps + i < w.len ? gi : 0.f;
    }
  });
}
// One value per channel of a [B, .., D] array of floats.
__device__ __forceinline__ void get_row(const float* p, const Where& w, float (&v)[kVec]) {
#pragma unroll
  for (int j = 0; j < kVec; ++j) v[j] = j < w.n ? p[w.c + j] : 0.f;
}
__device__ __forceinline__ void put_row(float* p, const Where& w, const float (&v)[kVec]) {
#pragma unroll
  for (int j = 0; j < kVec; ++j)
    if (j < w.n) p[w.c + j] = v[j];
}

// SUMMARY: only the map of the block's segment, into slot seg + 1.
template <class T, bool SUMMARY>
__global__ __launch_bounds__(64 * kMostWaves, 4) void scan_fwd_kernel(Params p) {
  constexpr bool DMA = sizeof(T) == 2;
  __shared__ __attribute__((aligned(16))) Map<kDown> slots[2][kMostWaves * kLanes];
  extern __shared__ __attribute__((aligned(16))) uint8_t next[];
  typedef typename Raw<T>::type raw;
  const Where w = where(p);
  const int seg = blockIdx.z, tile = w.nw * kWaveSteps;
  const int first = seg * p.seg_tiles, last = first + p.seg_tiles < p.tiles ? first + p.seg_tiles : p.tiles;
  float h[kVec] = {}, prod[kVec], up[kVec] = {}, in_up[kVec];
#pragma unroll
  for (int j = 0; j < kVec; ++j) prod[j] = 1.f;
  float2* const maps = maps_of(p, w);
  const Column<T> qf(p.f, p.ldf, w, p.T), qx(p.x, p.ldx, w, p.T), qy(p.y, p.ldy, w, p.T, true);
  const Ahead<2> ahead(next, w);
  auto all_of = [&](int k) { return (k + 1) * tile <= w.len; };      // wave-uniform
  auto ask = [&](int k) {
    if constexpr (DMA) {
      if (p.dma && all_of(k)) {
        ahead.ask(0, qf, k * tile);
        ahead.ask(1, qx, k * tile);
      }
    }
  };
  if (first < last) ask(first);          // a sequence of no steps hands its state through
  if (SUMMARY || p.segments == 1) {
    if (p.h0 && seg == 0) get_row(p.h0 + w.b * p.D, w, h);
    if (SUMMARY && seg == 0 && w.sub == 0) {
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (j < w.n) maps[j] = make_float2(0.f, h[j]);
    }
  } else {
    segment_carry<kDown>(slots[1], w, p, seg, h);
  }
  if (DMA) ahead.landed();
  auto step = [&](int k, auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    Map<kDown>* const slot = slots[(k - first) & 1];
    raw rf[kSteps], rx[kSteps];
    if (DMA && WHOLE && p.dma) {
      if constexpr (DMA) {
        ahead.take(0, w, rf);
        ahead.take(1, w, rx);
        ahead.taken();
      }
    } else {
      fetch<T, WHOLE>(qf, w, p, k * tile, rf);
      fetch<T, WHOLE>(qx, w, p, k * tile, rx);
    }
    if (k + 1 < last) ask(k + 1);
    float a[kSteps][kVec], v[kSteps][kVec], in[kVec];
    gates<T, WHOLE>(rf, w, k * tile, a, v);
    Map<kDown> m;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      m.p[j] = 1.f;
      m.s[0][j] = 0.f;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        v[i][j] *= (float)rx[i][j];
        m.s[0][j] = __builtin_fmaf(a[i][j], m.s[0][j], v[i][j]);
        m.p[j] *= a[i][j];
      }
      m.p[j] = positive(m.p[j]);
    }
    float before[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) before[j] = h[j];
    compose<kDown>(slot, w, m, h, in, up, in_up);
    if (DMA) ahead.landed();
    if (!SUMMARY && p.states && w.sub == 0) put_row(p.states + (w.b * p.tiles + k) * p.D, w, before);
    if constexpr (SUMMARY) {
      for (int i = 0; i < w.nw; ++i)
#pragma unroll
        for (int j = 0; j < kVec; ++j) prod[j] = positive(prod[j] * slot[i * kLanes + w.li].p[j]);
    } else {
      auto emit = [&](auto full) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          float o[kVec];
#pragma unroll
          for (int j = 0; j < kVec; ++j) {
            in[j] = __builtin_fmaf(a[i][j], in[j], v[i][j]);
            o[j] = WHOLE || k * tile + w.sub * kSteps + i < w.len ? in[j] : 0.f;
          }
          put<T, WHOLE, decltype(full)::value>(qy, w, k * tile, p.T, i, o);
        }
      };
      if (w.whole) emit(std::true_type{});
      else emit(std::false_type{});
    }
  };
  for (int k = first; k < last; ++k) {
    if (all_of(k)) step(k, std::true_type{});
    else step(k, std::false_type{});
  }
  if (w.sub == 0) {
    if constexpr (SUMMARY) {
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (j < w.n) maps[(seg + 1) * kChannels + j] = make_float2(seg == 0 ? 0.f : prod[j], h[j]);
    } else if (p.h_end && seg == p.segments - 1) {
      put_row(p.h_end + w.b * p.D, w, h);
    }
  }
}

// SUMMARY: the map of r over the block's segment seg + 1, into slot seg (the last slot holds dh_end).
template <class T, bool SUMMARY>
__global__ __launch_bounds__(64 * kMostWaves, 2) void scan_bwd_kernel(Params p) {
  constexpr bool DMA = sizeof(T) == 2;
  constexpr int DIRS = SUMMARY ? kUp : kUp | kDown, N = SUMMARY ? 2 : 3;
  __shared__ __attribute__((aligned(16))) Map<DIRS> slots[2][kMostWaves * kLanes];
  extern __shared__ __attribute__((aligned(16))) uint8_t next[];
  typedef typename Raw<T>::type raw;
  const Where w = where(p);
  const int seg = SUMMARY ? blockIdx.z + 1 : blockIdx.z, tile = w.nw * kWaveSteps;
  const int first = seg * p.seg_tiles, last = first + p.seg_tiles < p.tiles ? first + p.seg_tiles : p.tiles;
  const bool behind = seg == p.segments - 1;
  float r[kVec] = {}, prod[kVec];
#pragma unroll
  for (int j = 0; j < kVec; ++j) prod[j] = 1.f;
  float2* const maps = maps_of(p, w);
  const Column<T> qf(p.f, p.ldf, w, p.T), qx(p.x, p.ldx, w, p.T), qd(p.dy, p.ldy, w, p.T), of(p.df, p.lddf, w, p.T, true),
      ox(p.dx, p.lddx, w, p.T, true);
  const Ahead<N> ahead(next, w);
  auto all_of = [&](int k) { return (k + 1) * tile <= w.len; };      // wave-uniform
  auto ask = [&](int k) {
    if constexpr (DMA) {
      if (p.dma && all_of(k)) {
        ahead.ask(0, qf, k * tile);
        ahead.ask(1, qd, k * tile);
        if constexpr (!SUMMARY) ahead.ask(2, qx, k * tile);
      }
    }
  };
  if (first < last) ask(last - 1);
  if (SUMMARY || p.segments == 1) {
    if (p.dh_end && behind) get_row(p.dh_end + w.b * p.D, w, r);
    if (SUMMARY && behind && w.sub == 0) {
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (j < w.n) maps[seg * kChannels + j] = make_float2(0.f, r[j]);
    }
  } else {
    segment_carry<kUp>(reinterpret_cast<Map<kUp>*>(slots[1]), w, p, seg, r);
  }
  if (DMA) ahead.landed();
  auto step = [&](int k, auto all) {
    constexpr bool WHOLE = decltype(all)::value;
    raw rf[kSteps], rx[kSteps], rd[kSteps];
    float h[kVec] = {}, g[kSteps][kVec], in[kVec], hin[kVec];
    if (!SUMMARY) get_row(p.states + (w.b * p.tiles + k) * p.D, w, h);
    if (DMA && WHOLE && p.dma) {
      if constexpr (DMA) {
        ahead.take(0, w, rf);
        ahead.take(1, w, rd);
        if constexpr (!SUMMARY) ahead.take(2, w, rx);
        ahead.taken();
      }
    } else {
      fetch<T, WHOLE>(qf, w, p, k * tile, rf);
      fetch<T, WHOLE>(qd, w, p, k * tile, rd);
      if (!SUMMARY) fetch<T, WHOLE>(qx, w, p, k * tile, rx);
    }
    if (k > first) ask(k - 1);
    packed_gates<T, WHOLE>(rf, w, k * tile, g);
    Map<DIRS> m;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      m.p[j] = 1.f;
      float up = 0.f, down = 0.f, a, z;
#pragma unroll
      for (int i = kSteps - 1; i >= 0; --i) {
        unpack_gate(g[i][j], a, z);
        up = a * ((float)rd[i][j] + up);
        m.p[j] *= a;
      }
      m.p[j] = positive(m.p[j]);
      m.s[sum_of<DIRS, kUp>()][j] = up;
      if constexpr (!SUMMARY) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          unpack_gate(g[i][j], a, z);
          down = __builtin_fmaf(a, down, z * (float)rx[i][j]);
        }
        m.s[sum_of<DIRS, kDown>()][j] = down;
      }
    }
    // Only what is packed stays in registers while the waves meet.
    __builtin_amdgcn_sched_barrier(0);
    Map<DIRS>* const slot = slots[(last - 1 - k) & 1];
    compose<DIRS>(slot, w, m, h, hin, r, in);
    if (DMA) ahead.landed();
    if constexpr (SUMMARY) {
      for (int i = 0; i < w.nw; ++i)
#pragma unroll
        for (int j = 0; j < kVec; ++j) prod[j] = positive(prod[j] * slot[i * kLanes + w.li].p[j]);
    } else {
      float before[kSteps][kVec], a, z;
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
          asm volatile("" : "+v"(g[i][j]));                 // unpacked again here, not kept from above
          unpack_gate(g[i][j], a, z);
          const float xi = (float)rx[i][j];
          before[i][j] = hin[j] - xi;                       // h_(t-1) - x_t
          hin[j] = __builtin_fmaf(a, hin[j], z * xi);
        }
      auto emit = [&](auto full) {
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
          float vf[kVec], vx[kVec];
          const bool there = WHOLE || k * tile + w.sub * kSteps + i < w.len;
#pragma unroll
          for (int j = 0; j < kVec; ++j) {
            unpack_gate(g[i][j], a, z);
            const float gr = (float)rd[i][j] + in[j];
            vx[j] = there ? gr * z : 0.f;
            vf[j] = there ? vx[j] * a * before[i][j] : 0.f;
            in[j] = a * gr;
          }
          put<T, WHOLE, decltype(full)::value>(of, w, k * tile, p.T, i, vf);
          put<T, WHOLE, decltype(full)::value>(ox, w, k * tile, p.T, i, vx);
        }
      };
      if (w.whole) emit(std::true_type{});
      else emit(std::false_type{});
    }
  };
  for (int k = last - 1; k >= first; --k) {
    if (all_of(k)) step(k, std::true_type{});
    else step(k, std::false_type{});
  }
  if (w.sub == 0) {
    if constexpr (SUMMARY) {
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (j < w.n) maps[(seg - 1) * kChannels + j] = make_float2(behind ? 0.f : prod[j], r[j]);
    } else if (p.dh0 && seg == 0) {
      put_row(p.dh0 + w.b * p.D, w, r);
    }
  }
}

// Blocks of channels run a round of one per compute unit at a time.  Those of the last round are cut into segments where they
// leave three quarters of the units idle or more, which costs reading the gates and one more array again: as many segments as
// still fit a round, no more than there are tiles.  Forward and backward in us, bf16, cut and not, of 2048 channels:
// 1 x 1024 steps 12.9 + 17.1 and 19.0 + 28.8, 9 x 1024 44.3 + 67.9 and 47.4 + 74.8, 10 x 4096 147 + 224 and 170 + 268; half a
// round or three tiles win nothing: 4 x 2048 45.3 + 65.0 and 42.4 + 70.3, 10 x 768 36.5 + 57.3 and 34.4 + 58.0.
constexpr int kUnits = 256, kCutFrom = 4;
struct Plan { int64_t whole, rest; int segments; };        // blocks of channels taken whole, the others, and into how many
Plan plan_of(int64_t B, int T, int D) {
  const int64_t blocks = B * ((D + kChannels - 1) / kChannels), left = blocks % kUnits, tiles = tiles_of(T);
  if (left == 0 || left > kUnits / 4 || tiles < kCutFrom) return {blocks, 0, 1};
  int64_t n = kUnits / left;
  if (n > tiles) n = tiles;
  const int64_t per = (tiles + n - 1) / n;
  return {blocks - left, left, (int)((tiles + per - 1) / per)};
}
bool dims_ok(int64_t B, int64_t T, int64_t D) {
  return B >= 0 && T >= 0 && D >= 0 && B <= 65535 && T <= (1 << 30) && D <= kMostLd;
}
bool args_ok(const ScanArgs& a) {
  if (a.dtype != kF32 && a.dtype != kBF16) return false;
  if (!dims_ok(a.B, a.T, a.D) || !a.f || !a.x || a.ldf < a.D || a.ldx < a.D || a.ldf > kMostLd || a.ldx > kMostLd) return false;
  const uintptr_t el = a.dtype == kBF16 ? 1 : 3;
  return !(((uintptr_t)a.f | (uintptr_t)a.x) & el) && !(((uintptr_t)a.h0 | (uintptr_t)a.lens) & 3);
}
Params params_of(const ScanArgs& a, float* ws) {
  Params p{};
  p.f = a.f; p.x = a.x; p.ldf = a.ldf; p.ldx = a.ldx;
  p.h0 = a.h0; p.lens = a.lens;
  p.T = a.T; p.D = a.D;
  p.groups = ((uint32_t)a.D + kChannels - 1) / kChannels;
  p.tiles = tiles_of(a.T);
  p.maps = reinterpret_cast<float2*>(ws);
  return p;
}
// The launches of a plan: launch(params, blocks, segments, summaries).
template <class F> void run(const Plan& plan, Params p, F&& launch) {
  constexpr int64_t most = 1 << 22;            // threads of a launch are counted in 32 bits
  p.segments = 1;
  p.seg_tiles = p.tiles;
  for (int64_t done = 0; done < plan.whole; done += most) {
    p.base = (uint32_t)done;
    launch(p, plan.whole - done < most ? plan.whole - done : most, 1, false);
  }
  if (!plan.rest) return;
  p.base = (uint32_t)plan.whole;
  p.segments = plan.segments;
  p.seg_tiles = (p.tiles + plan.segments - 1) / plan.segments;
  launch(p, plan.rest, plan.segments - 1, true);
  launch(p, plan.rest, plan.segments, false);
}

}  // namespace

hipError_t scan_init() {
  const std::pair<const void*, int> k[] = {{reinterpret_cast<const void*>(scan_fwd_kernel<bf16, true>), Ahead<2>::kBytes},
                                           {reinterpret_cast<const void*>(scan_fwd_kernel<bf16, false>), Ahead<2>::kBytes},
                                           {reinterpret_cast<const void*>(scan_bwd_kernel<bf16, true>), Ahead<2>::kBytes},
                                           {reinterpret_cast<const void*>(scan_bwd_kernel<bf16, false>), Ahead<3>::kBytes}};
  for (const auto& f : k) {
    const hipError_t e = hipFuncSetAttribute(f.first, hipFuncAttributeMaxDynamicSharedMemorySize, kMostWaves * f.second);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

int64_t scan_state_floats(int64_t B, int64_t T, int64_t D) {
  return dims_ok(B, T, D) ? (T == 0 ? 0 : B * tiles_of((int)T) * D) : -1;
}
int64_t scan_ws_floats(int64_t B, int64_t T, int64_t D) {
  if (!dims_ok(B, T, D)) return -1;
  if (B == 0 || T == 0 || D == 0) return 0;
  const Plan p = plan_of(B, (int)T, (int)D);
  return 2 * p.rest * p.segments * kChannels;
}

hipError_t launch_scan_fwd(hipStream_t s, const ScanArgs& a, void* y, int64_t ldy, float* h_end, float* states, float* ws) {
  if (!args_ok(a) || !y || ldy < a.D || ldy > kMostLd || ((uintptr_t)y & (a.dtype == kBF16 ? 1 : 3))) return hipErrorInvalidValue;
  if ((((uintptr_t)h_end | (uintptr_t)states) & 3) || ((uintptr_t)ws & 7)) return hipErrorInvalidValue;
  if (a.B == 0 || a.D == 0) return hipSuccess;
  Params p = params_of(a, ws);
  const Plan plan = plan_of(a.B, a.T, a.D);
  if (plan.rest && !ws) return hipErrorInvalidValue;
  p.y = y; p.ldy = ldy; p.h_end = h_end; p.states = states;
  p.dma = a.D % 2 == 0 && !(((uintptr_t)a.f | (uintptr_t)a.x) & 3) && !((a.ldf | a.ldx) & 1);
  const int waves = waves_of(a.T);
  auto go = [&](auto t) {
    using T = decltype(t);
    run(plan, p, [&](const Params& q, int64_t blocks, int segments, bool summaries) {
      const dim3 grid((unsigned)blocks, 1, (unsigned)segments);
      const auto lds = [&](int bytes) { return sizeof(T) == 2 ? (size_t)waves * bytes : 0; };
      if (summaries) scan_fwd_kernel<T, true><<<grid, 64 * waves, lds(Ahead<2>::kBytes), s>>>(q);
      else scan_fwd_kernel<T, false><<<grid, 64 * waves, lds(Ahead<2>::kBytes), s>>>(q);
    });
  };
  if (a.dtype == kBF16) go(bf16{});
  else go(float{});
  return hipGetLastError();
}

hipError_t launch_scan_bwd(hipStream_t s, const ScanArgs& a, const void* dy, int64_t lddy, const float* dh_end, const float* states,
                           void* df, int64_t lddf, void* dx, int64_t lddx, float* dh0, float* ws) {
  if (!args_ok(a) || !dy || !df || !dx || lddy < a.D || lddf < a.D || lddx < a.D || lddy > kMostLd || lddf > kMostLd ||
      lddx > kMostLd)
    return hipErrorInvalidValue;
  if (((uintptr_t)dy | (uintptr_t)df | (uintptr_t)dx) & (a.dtype == kBF16 ? 1 : 3)) return hipErrorInvalidValue;
  if ((((uintptr_t)dh_end | (uintptr_t)states | (uintptr_t)dh0) & 3) || ((uintptr_t)ws & 7)) return hipErrorInvalidValue;
  if (a.B == 0 || a.D == 0) return hipSuccess;
  Params p = params_of(a, ws);
  const Plan plan = plan_of(a.B, a.T, a.D);
  if ((!states && a.T > 0) || (plan.rest && !ws)) return hipErrorInvalidValue;
  p.dy = dy; p.ldy = lddy; p.dh_end = dh_end; p.states = const_cast<float*>(states);
  p.dma = a.D % 2 == 0 && !(((uintptr_t)a.f | (uintptr_t)a.x | (uintptr_t)dy) & 3) && !((a.ldf | a.ldx | lddy) & 1);
  p.df = df; p.lddf = lddf; p.dx = dx; p.lddx = lddx; p.dh0 = dh0;
  const int waves = waves_of(a.T);
  auto go = [&](auto t) {
    using T = decltype(t);
    run(plan, p, [&](const Params& q, int64_t blocks, int segments, bool summaries) {
      const dim3 grid((unsigned)blocks, 1, (unsigned)segments);
      const auto lds = [&](int bytes) { return sizeof(T) == 2 ? (size_t)waves * bytes : 0; };
      if (summaries) scan_bwd_kernel<T, true><<<grid, 64 * waves, lds(Ahead<2>::kBytes), s>>>(q);
      else scan_bwd_kernel<T, false><<<grid, 64 * waves, lds(Ahead<3>::kBytes), s>>>(q);
    });
  };
  if (a.dtype == kBF16) go(bf16{});
  else go(float{});
  return hipGetLastError();
}

}  // namespace pw
