// Gated linear recurrence along a sequence, every channel on its own:
//
//   a_t = sigmoid(f_t),  h_t = a_t h_(t-1) + (1 - a_t) x_t,  y_t = h_t
//
// and backward, with r_t = a_t g_t what step t hands to the step before it:
//
//   g_t = dy_t + r_(t+1),  dx_t = g_t (1 - a_t),  df_t = g_t (h_(t-1) - x_t) a_t (1 - a_t),  dh_0 = r_1.
//
// A step is the map h -> a h + v, and maps compose: (P, S) after (p, s) is (P p, P s + S).  A thread takes 8 consecutive
// steps of its channels into registers and composes them, the waves of a block hand their maps over through LDS, and every
// thread then runs its steps again from the state in front of them: inputs are read once, nothing but outputs is written.
// A block of up to 16 waves has 64 channels (two to a lane, so that a row is 128 or 256 bytes) and a tile of 16 steps per
// wave; it walks down its tiles with the state in registers.  The forward pass keeps the state in front of each tile
// (fp32, one value per channel and tile); the backward pass starts every tile from it and walks upwards.
//
// Few channels leave compute units idle.  The sequence is then cut into segments of whole tiles: a first launch composes
// each segment into one map, the second composes the maps in front of its segment (behind it, backward) and goes on as above.
//
// Steps behind the end of a sequence (lens) are the identity map with outputs of zero; their inputs are not read.
// Sums, states and gates are fp32; y, df and dx are rounded once.  All orders are fixed: the same bits on every run.
#include <initializer_list>
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"

namespace pw {

namespace {

constexpr int kSteps = 8;          // consecutive steps of a thread
constexpr int kMostWaves = 16;
constexpr int kLanes = 32;         // lanes side by side along the channels; the wave's other half has the next 8 steps

int waves_of(int T) {
  const int w = (T + 2 * kSteps - 1) / (2 * kSteps);
  return w < 1 ? 1 : (w > kMostWaves ? kMostWaves : w);
}
int tile_of(int T) { return waves_of(T) * 2 * kSteps; }
int tiles_of(int T) { return (T + tile_of(T) - 1) / tile_of(T); }

struct Params {
  const void *f, *x, *dy;
  void *y, *df, *dx;
  int64_t ldf, ldx, ldy, lddf, lddx;     // ldy: of y (forward) or dy (backward)
  const float *h0, *dh_end;
  float *h_end, *dh0, *states;
  float2* maps;                          // [B][segments][D]
  const int32_t* lens;
  int T, D, tiles, segments, seg_tiles;
};

// Two or one adjacent channels.
template <class T, int VEC> struct Raw;
template <> struct Raw<bf16, 2> { typedef bf16x2 type; };
template <> struct Raw<bf16, 1> { typedef bf16 type; };
template <> struct Raw<float, 2> { typedef float type __attribute__((ext_vector_type(2))); };
template <> struct Raw<float, 1> { typedef float type; };
template <class T, int VEC> __device__ __forceinline__ float lane_of(const typename Raw<T, VEC>::type& r, int j) {
  if constexpr (VEC == 2) return (float)r[j];
  else return (float)r;
}
template <class T, int VEC> __device__ __forceinline__ void put(T* p, const float* v) {
  typename Raw<T, VEC>::type r;
  if constexpr (VEC == 2) {
    r[0] = (T)v[0];
    r[1] = (T)v[1];
  } else {
    r = (T)v[0];
  }
  *reinterpret_cast<typename Raw<T, VEC>::type*>(p) = r;
}

// a = sigmoid(f) and z = 1 - a, each to full relative precision.
__device__ __forceinline__ void gate(float f, float& a, float& z) {
  const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * __builtin_fabsf(f));
  const float big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
  a = f >= 0.f ? big : small;
  z = f >= 0.f ? small : big;
  if (f != f) a = z = f;
}

struct Where {
  int64_t b;
  int c, sub, wave, half, li, nw, len;
  bool on;                               // the lane has channels
};
template <int VEC> __device__ __forceinline__ Where where(const Params& p) {
  Where w;
  w.b = blockIdx.y;
  w.wave = threadIdx.x >> 6;
  w.half = (threadIdx.x >> 5) & 1;
  w.li = threadIdx.x & (kLanes - 1);
  w.sub = 2 * w.wave + w.half;
  w.nw = blockDim.x >> 6;
  w.c = (blockIdx.x * kLanes + w.li) * VEC;
  w.on = w.c < p.D;
  w.len = p.T;
  if (p.lens) {
    const int l = p.lens[w.b];
    w.len = l < 0 ? 0 : (l > p.T ? p.T : l);
  }
  return w;
}

// The eight steps from t0 on of an array's channels.  Steps that do not exist come out as zeros: what is fetched in their
// place is the sequence's last row (or its first place in memory, where it has no step) and is not looked at.
template <class T, int VEC>
__device__ __forceinline__ void fetch(const void* base, int64_t ld, const Where& w, const Params& p, int t0,
                                      typename Raw<T, VEC>::type (&r)[kSteps]) {
  typedef typename Raw<T, VEC>::type raw;
  const T* const q = reinterpret_cast<const T*>(base) + w.b * p.T * ld + (w.on ? w.c : 0);
  const int end = t0 - w.sub * kSteps + w.nw * 2 * kSteps;      // of the block's tile
  if (end <= w.len) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) r[i] = *reinterpret_cast<const raw*>(q + (t0 + i) * ld);
  } else {
    const int top = w.len > 0 ? w.len - 1 : 0;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const raw v = *reinterpret_cast<const raw*>(q + (t0 + i < top ? t0 + i : top) * ld);
      r[i] = t0 + i < w.len ? v : raw{};
    }
  }
}

// Maps of the waves of a block, one array per composed quantity.
template <int VEC> struct Maps { float p[VEC], s[VEC]; };

template <int VEC>
__device__ __forceinline__ Maps<VEC> other_half(const Maps<VEC>& m) {
  Maps<VEC> o;
#pragma unroll
  for (int j = 0; j < VEC; ++j) {
    o.p[j] = __shfl_xor(m.p[j], 32, 64);
    o.s[j] = __shfl_xor(m.s[j], 32, 64);
  }
  return o;
}

// carry: the state in front of the block's tile (FORWARD) or handed in from behind it; replaced by the one on the other
// side.  in: what reaches this thread's eight steps.  mine: the map of those.  slot: LDS of this tile, [waves][lanes].
template <int VEC, bool FORWARD>
__device__ __forceinline__ void compose(Maps<VEC>* slot, const Where& w, const Maps<VEC>& mine, float (&carry)[VEC], float (&in)[VEC]) {
  const Maps<VEC> other = other_half(mine);
  const bool first = FORWARD ? w.half == 0 : w.half == 1;      // the half that the state reaches first
  Maps<VEC> both;
#pragma unroll
  for (int j = 0; j < VEC; ++j) {
    both.p[j] = mine.p[j] * other.p[j];
    both.s[j] = first ? __builtin_fmaf(other.p[j], mine.s[j], other.s[j]) : __builtin_fmaf(mine.p[j], other.s[j], mine.s[j]);
  }
  if (w.half == 0) slot[w.wave * kLanes + w.li] = both;
  __syncthreads();
  float h[VEC], at[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) at[j] = h[j] = carry[j];
  for (int i = 0; i < w.nw; ++i) {
    const int k = FORWARD ? i : w.nw - 1 - i;
    const Maps<VEC> m = slot[k * kLanes + w.li];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      if (k == w.wave) at[j] = h[j];
      h[j] = __builtin_fmaf(m.p[j], h[j], m.s[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < VEC; ++j) {
    carry[j] = h[j];
    in[j] = first ? at[j] : __builtin_fmaf(other.p[j], at[j], other.s[j]);
  }
}

// What reaches segment `seg`: the maps of the slots 0 .. seg (FORWARD) or segments - 1 .. seg, the first of which is a
// constant.  Each wave composes a stretch of them, then the waves meet as they do in a tile.
template <int VEC, bool FORWARD>
__device__ __forceinline__ void segment_carry(Maps<VEC>* slot, const Where& w, const Params& p, int seg, float (&carry)[VEC]) {
  const int n = FORWARD ? seg + 1 : p.segments - seg, per = (n + 2 * w.nw - 1) / (2 * w.nw);
  Maps<VEC> m;
#pragma unroll
  for (int j = 0; j < VEC; ++j) {
    m.p[j] = 1.f;
    m.s[j] = 0.f;
    carry[j] = 0.f;
  }
  for (int i = 0; i < per; ++i) {
    const int k = FORWARD ? w.sub * per + i : n - 1 - ((2 * w.nw - 1 - w.sub) * per + i);
    const bool there = FORWARD ? k < n : k >= 0;
    if (w.on && there) {
      const float2* q = p.maps + (w.b * p.segments + (FORWARD ? k : seg + k)) * p.D + w.c;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float2 v = q[j];
        m.s[j] = __builtin_fmaf(v.x, m.s[j], v.y);
        m.p[j] *= v.x;
      }
    }
  }
  float in[VEC];
  compose<VEC, FORWARD>(slot, w, m, carry, in);
}

template <class T, int VEC>
__device__ __forceinline__ void gates(const typename Raw<T, VEC>::type (&rf)[kSteps], const Where& w, int t0, float (&a)[kSteps][VEC],
                                      float (&z)[kSteps][VEC]) {
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      gate(lane_of<T, VEC>(rf[i], j), a[i][j], z[i][j]);
      if (t0 + i >= w.len) {
        a[i][j] = 1.f;
        z[i][j] = 0.f;
      }
    }
}

// SUMMARY: only the map of the block's segment, into slot seg + 1.
template <class T, int VEC, bool SUMMARY>
__global__ __launch_bounds__(64 * kMostWaves) void scan_fwd_kernel(Params p) {
  __shared__ __attribute__((aligned(16))) Maps<VEC> slots[2][kMostWaves * kLanes];
  const Where w = where<VEC>(p);
  const int seg = blockIdx.z, tile = w.nw * 2 * kSteps;
  const int first = seg * p.seg_tiles, last = first + p.seg_tiles < p.tiles ? first + p.seg_tiles : p.tiles;
  float h[VEC] = {}, in[VEC], prod[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) prod[j] = 1.f;
  if (SUMMARY || p.segments == 1) {
    if (p.h0 && seg == 0 && w.on) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) h[j] = p.h0[w.b * p.D + w.c + j];
    }
    if (SUMMARY && seg == 0 && w.on && w.sub == 0) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) p.maps[w.b * p.segments * p.D + w.c + j] = make_float2(0.f, h[j]);
    }
  } else {
    segment_carry<VEC, true>(slots[1], w, p, seg, h);
  }
  int t0 = first * tile + w.sub * kSteps, parity = 0;
  typename Raw<T, VEC>::type rf[kSteps], rx[kSteps];
  if (first < last) {                    // a sequence of no steps hands its state through
    fetch<T, VEC>(p.f, p.ldf, w, p, t0, rf);
    fetch<T, VEC>(p.x, p.ldx, w, p, t0, rx);
  }
  for (int k = first; k < last; ++k, t0 += tile, parity ^= 1) {
    float a[kSteps][VEC], v[kSteps][VEC];
    gates<T, VEC>(rf, w, t0, a, v);
    Maps<VEC> m;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      m.p[j] = 1.f;
      m.s[j] = 0.f;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        v[i][j] *= lane_of<T, VEC>(rx[i], j);
        m.s[j] = __builtin_fmaf(a[i][j], m.s[j], v[i][j]);
        m.p[j] *= a[i][j];
      }
    }
    if (k + 1 < last) {
      fetch<T, VEC>(p.f, p.ldf, w, p, t0 + tile, rf);
      fetch<T, VEC>(p.x, p.ldx, w, p, t0 + tile, rx);
    }
    if (!SUMMARY && p.states && w.on && w.sub == 0) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) p.states[(w.b * p.tiles + k) * p.D + w.c + j] = h[j];
    }
    compose<VEC, true>(slots[parity], w, m, h, in);
    if constexpr (SUMMARY) {
      // the product over the tile: composed once more with a state of one and sums of zero
      Maps<VEC>* slot = slots[parity];
      for (int i = 0; i < w.nw; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) prod[j] *= slot[i * kLanes + w.li].p[j];
    } else if (w.on) {
      T* const y = reinterpret_cast<T*>(p.y) + (w.b * p.T + t0) * p.ldy + w.c;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        float o[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          in[j] = __builtin_fmaf(a[i][j], in[j], v[i][j]);
          o[j] = t0 + i < w.len ? in[j] : 0.f;
        }
        if (t0 + i < p.T) put<T, VEC>(y + i * p.ldy, o);
      }
    }
  }
  if (w.on && w.sub == 0) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      if (SUMMARY) p.maps[(w.b * p.segments + seg + 1) * p.D + w.c + j] = make_float2(seg == 0 ? 0.f : prod[j], h[j]);
      else if (p.h_end && seg == p.segments - 1) p.h_end[w.b * p.D + w.c + j] = h[j];
    }
  }
}

// SUMMARY: the map of r over the block's segment seg + 1, into slot seg (the last slot holds dh_end).
template <class T, int VEC, bool SUMMARY>
__global__ __launch_bounds__(64 * kMostWaves) void scan_bwd_kernel(Params p) {
  __shared__ __attribute__((aligned(16))) Maps<VEC> slots[2][2][kMostWaves * kLanes];   // [parity][backward, forward]
  const Where w = where<VEC>(p);
  const int seg = SUMMARY ? blockIdx.z + 1 : blockIdx.z, tile = w.nw * 2 * kSteps;
  const int first = seg * p.seg_tiles, last = first + p.seg_tiles < p.tiles ? first + p.seg_tiles : p.tiles;
  const bool behind = seg == p.segments - 1;
  float r[VEC] = {}, in[VEC], prod[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) prod[j] = 1.f;
  if (SUMMARY || p.segments == 1) {
    if (p.dh_end && behind && w.on) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) r[j] = p.dh_end[w.b * p.D + w.c + j];
    }
    if (SUMMARY && behind && w.on && w.sub == 0) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) p.maps[(w.b * p.segments + seg) * p.D + w.c + j] = make_float2(0.f, r[j]);
    }
  } else {
    segment_carry<VEC, false>(slots[1][0], w, p, seg, r);
  }
  int t0 = (last - 1) * tile + w.sub * kSteps, parity = 0;
  typename Raw<T, VEC>::type rf[kSteps], rx[kSteps], rd[kSteps];
  for (int k = last - 1; k >= first; --k, t0 -= tile, parity ^= 1) {
    fetch<T, VEC>(p.f, p.ldf, w, p, t0, rf);
    fetch<T, VEC>(p.dy, p.ldy, w, p, t0, rd);
    float a[kSteps][VEC], z[kSteps][VEC];
    Maps<VEC> m;
    if constexpr (SUMMARY) {
      gates<T, VEC>(rf, w, t0, a, z);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        m.p[j] = 1.f;
        m.s[j] = 0.f;
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
          m.s[j] = a[i][j] * (lane_of<T, VEC>(rd[i], j) + m.s[j]);
          m.p[j] *= a[i][j];
        }
      }
      compose<VEC, false>(slots[parity][0], w, m, r, in);
      for (int i = 0; i < w.nw; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) prod[j] *= slots[parity][0][i * kLanes + w.li].p[j];
    } else {
      fetch<T, VEC>(p.x, p.ldx, w, p, t0, rx);
      float h[VEC] = {};
      if (w.on) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) h[j] = p.states[(w.b * p.tiles + k) * p.D + w.c + j];
      }
      gates<T, VEC>(rf, w, t0, a, z);
      Maps<VEC> mf;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        m.p[j] = 1.f;
        m.s[j] = mf.s[j] = 0.f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          mf.s[j] = __builtin_fmaf(a[i][j], mf.s[j], z[i][j] * lane_of<T, VEC>(rx[i], j));
        }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
          m.s[j] = a[i][j] * (lane_of<T, VEC>(rd[i], j) + m.s[j]);
          m.p[j] *= a[i][j];
        }
        mf.p[j] = m.p[j];
      }
      float hin[VEC];
      compose<VEC, false>(slots[parity][0], w, m, r, in);
      compose<VEC, true>(slots[parity][1], w, mf, h, hin);
      if (w.on) {
        float before[kSteps][VEC];
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const float xi = lane_of<T, VEC>(rx[i], j);
            before[i][j] = hin[j] - xi;                       // h_(t-1) - x_t
            hin[j] = __builtin_fmaf(a[i][j], hin[j], z[i][j] * xi);
          }
        T* const df = reinterpret_cast<T*>(p.df) + (w.b * p.T + t0) * p.lddf + w.c;
        T* const dx = reinterpret_cast<T*>(p.dx) + (w.b * p.T + t0) * p.lddx + w.c;
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
          float of[VEC], ox[VEC];
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const float g = lane_of<T, VEC>(rd[i], j) + in[j];
            const bool there = t0 + i < w.len;
            ox[j] = there ? g * z[i][j] : 0.f;
            of[j] = there ? ox[j] * a[i][j] * before[i][j] : 0.f;
            in[j] = a[i][j] * g;
          }
          if (t0 + i < p.T) {
            put<T, VEC>(df + i * p.lddf, of);
            put<T, VEC>(dx + i * p.lddx, ox);
          }
        }
      }
    }
  }
  if (w.on && w.sub == 0) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      if (SUMMARY) p.maps[(w.b * p.segments + seg - 1) * p.D + w.c + j] = make_float2(behind ? 0.f : prod[j], r[j]);
      else if (p.dh0 && seg == 0) p.dh0[w.b * p.D + w.c + j] = r[j];
    }
  }
}

// How many segments: as many as bring the launch to a block per compute unit, and no more than there are tiles.
int segments_of(int64_t B, int T, int D) {
  const int64_t blocks = B * ((D + 2 * kLanes - 1) / (2 * kLanes)), tiles = tiles_of(T);
  int64_t n = blocks >= 192 ? 1 : (256 + blocks - 1) / blocks;
  if (n > tiles) n = tiles;
  if (n <= 1) return 1;
  const int64_t per = (tiles + n - 1) / n;
  return (int)((tiles + per - 1) / per);
}
bool dims_ok(int64_t B, int64_t T, int64_t D) {
  return B >= 0 && T >= 0 && D >= 0 && B <= 65535 && T <= (1 << 30) && D <= (1 << 24);
}
bool args_ok(const ScanArgs& a) {
  if (a.dtype != kF32 && a.dtype != kBF16) return false;
  if (!dims_ok(a.B, a.T, a.D) || !a.f || !a.x || a.ldf < a.D || a.ldx < a.D) return false;
  const uintptr_t el = a.dtype == kBF16 ? 1 : 3;
  return !(((uintptr_t)a.f | (uintptr_t)a.x) & el) && !(((uintptr_t)a.h0 | (uintptr_t)a.lens) & 3);
}
Params params_of(const ScanArgs& a, float* ws) {
  Params p{};
  p.f = a.f; p.x = a.x; p.ldf = a.ldf; p.ldx = a.ldx;
  p.h0 = a.h0; p.lens = a.lens;
  p.T = a.T; p.D = a.D;
  p.tiles = tiles_of(a.T);
  p.segments = segments_of(a.B, a.T, a.D);
  p.seg_tiles = (p.tiles + p.segments - 1) / p.segments;
  p.maps = reinterpret_cast<float2*>(ws);
  return p;
}
// Two channels to a lane where every row starts on a pair.
template <class T> bool pairs(std::initializer_list<const void*> ptrs, std::initializer_list<int64_t> lds, int D) {
  uintptr_t bits = 0;
  for (const void* q : ptrs) bits |= (uintptr_t)q;
  int64_t odd = D;
  for (int64_t l : lds) odd |= l;
  return bits % (2 * sizeof(T)) == 0 && (odd & 1) == 0;
}

}  // namespace

int64_t scan_state_floats(int64_t B, int64_t T, int64_t D) {
  return dims_ok(B, T, D) ? (T == 0 ? 0 : B * tiles_of((int)T) * D) : -1;
}
int64_t scan_ws_floats(int64_t B, int64_t T, int64_t D) {
  if (!dims_ok(B, T, D)) return -1;
  if (B == 0 || T == 0 || D == 0) return 0;
  const int64_t n = segments_of(B, (int)T, (int)D);
  return n == 1 ? 0 : 2 * B * n * D;
}

hipError_t launch_scan_fwd(hipStream_t s, const ScanArgs& a, void* y, int64_t ldy, float* h_end, float* states, float* ws) {
  if (!args_ok(a) || !y || ldy < a.D || ((uintptr_t)y & (a.dtype == kBF16 ? 1 : 3))) return hipErrorInvalidValue;
  if ((((uintptr_t)h_end | (uintptr_t)states) & 3) || ((uintptr_t)ws & 7)) return hipErrorInvalidValue;
  if (a.B == 0 || a.D == 0) return hipSuccess;
  Params p = params_of(a, ws);
  if (p.segments > 1 && !ws) return hipErrorInvalidValue;
  p.y = y; p.ldy = ldy; p.h_end = h_end; p.states = states;
  const int threads = 64 * waves_of(a.T);
  auto go = [&](auto t, auto vec) {
    using T = decltype(t);
    constexpr int V = decltype(vec)::value;
    const unsigned groups = (unsigned)((a.D + V * kLanes - 1) / (V * kLanes));
    if (p.segments > 1) scan_fwd_kernel<T, V, true><<<dim3(groups, a.B, p.segments - 1), threads, 0, s>>>(p);
    scan_fwd_kernel<T, V, false><<<dim3(groups, a.B, p.segments), threads, 0, s>>>(p);
  };
  using one = std::integral_constant<int, 1>;
  using two = std::integral_constant<int, 2>;
  if (a.dtype == kBF16) pairs<bf16>({a.f, a.x, y}, {a.ldf, a.ldx, ldy}, a.D) ? go(bf16{}, two{}) : go(bf16{}, one{});
  else pairs<float>({a.f, a.x, y}, {a.ldf, a.ldx, ldy}, a.D) ? go(float{}, two{}) : go(float{}, one{});
  return hipGetLastError();
}

hipError_t launch_scan_bwd(hipStream_t s, const ScanArgs& a, const void* dy, int64_t lddy, const float* dh_end, const float* states,
                           void* df, int64_t lddf, void* dx, int64_t lddx, float* dh0, float* ws) {
  if (!args_ok(a) || !dy || !df || !dx || lddy < a.D || lddf < a.D || lddx < a.D) return hipErrorInvalidValue;
  if (((uintptr_t)dy | (uintptr_t)df | (uintptr_t)dx) & (a.dtype == kBF16 ? 1 : 3)) return hipErrorInvalidValue;
  if ((((uintptr_t)dh_end | (uintptr_t)states | (uintptr_t)dh0) & 3) || ((uintptr_t)ws & 7)) return hipErrorInvalidValue;
  if (a.B == 0 || a.D == 0) return hipSuccess;
  Params p = params_of(a, ws);
  if ((!states && a.T > 0) || (p.segments > 1 && !ws)) return hipErrorInvalidValue;
  p.dy = dy; p.ldy = lddy; p.dh_end = dh_end; p.states = const_cast<float*>(states);
  p.df = df; p.lddf = lddf; p.dx = dx; p.lddx = lddx; p.dh0 = dh0;
  const int threads = 64 * waves_of(a.T);
  auto go = [&](auto t, auto vec) {
    using T = decltype(t);
    constexpr int V = decltype(vec)::value;
    const unsigned groups = (unsigned)((a.D + V * kLanes - 1) / (V * kLanes));
    if (p.segments > 1) scan_bwd_kernel<T, V, true><<<dim3(groups, a.B, p.segments - 1), threads, 0, s>>>(p);
    scan_bwd_kernel<T, V, false><<<dim3(groups, a.B, p.segments), threads, 0, s>>>(p);
  };
  using one = std::integral_constant<int, 1>;
  using two = std::integral_constant<int, 2>;
  if (a.dtype == kBF16)
    pairs<bf16>({a.f, a.x, dy, df, dx}, {a.ldf, a.ldx, lddy, lddf, lddx}, a.D) ? go(bf16{}, two{}) : go(bf16{}, one{});
  else
    pairs<float>({a.f, a.x, dy, df, dx}, {a.ldf, a.ldx, lddy, lddf, lddx}, a.D) ? go(float{}, two{}) : go(float{}, one{});
  return hipGetLastError();
}

}  // namespace pw
