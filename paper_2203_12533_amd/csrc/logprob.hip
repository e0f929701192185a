// Log probabilities of given tokens, entropy and the likeliest alternatives of rows of logits, from one read, and the gradient of the logits:
//
//   d_v = s (z_v - max z),  S = sum e^d,  logp = d_t - log S,  H = log S - (sum e^d d) / S          (both terms of H are >= 0: nothing cancels)
//   dz_v = s [dlogp ([v = t] - p_v) - dentropy p_v (log p_v + H)],  p_v = e^(d_v - log S)
//
// In base 2: d = z k - max k with k = s log2 e, one fused multiply-add, whose product is exact; that max k is rounded shifts all of a row
// alike, by an amount that is known and taken off log S.  Every thread keeps a running maximum, S and sum of its own; they meet once per row.  Sums are fp32, of at most
// vocab / threads terms before they meet in a tree.
//
// Alternatives.  A chunk of the row is in registers; the block's threads form 64 groups, and the k-th largest of the groups' maxima (the upper 16
// bits of it) is a bound that k elements at least reach: usually few more do.  They go to a list in LDS with a key of value and index, 64 bits,
// no two alike, so that the order in which they arrive does not matter; later chunks add what reaches the bound.  A list that is full
// gets a tighter bound, and where that does not help - values that fall into few groups - the chunk's k best are taken out one by
// one.  Ranks in the list are counted at the end.
//
// Bound by memory: forward one read, backward one read and one write.
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"
#include "lanes.hpp"

// Products are rounded where they stand: a difference of two equal ones has to be 0 (as fma(a, k, -(a k)) it is not).
#pragma clang fp contract(off)

namespace pw {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4u2 __attribute__((ext_vector_type(4), aligned(2)));      // wherever an element may be
typedef uint32_t u32x4u4 __attribute__((ext_vector_type(4), aligned(4)));
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFloor = -1000.f;            // exp2 of it is 0, and 0 times it too, unlike of -infinity

// 16 bytes of a row: E elements.
template <class T> struct Vec;
template <> struct Vec<float> {
  static constexpr int E = 4;
  static constexpr uint32_t kFill = 0xff800000u;                                // -infinity
  static __device__ __forceinline__ u32x4 load(const float* p) { return *reinterpret_cast<const u32x4u4*>(p); }
  static __device__ __forceinline__ void store(float* p, const u32x4& v) { *reinterpret_cast<u32x4u4*>(p) = v; }
  static __device__ __forceinline__ float get(const u32x4& v, int e) { return __uint_as_float(v[e]); }
  static __device__ __forceinline__ void put(u32x4& v, int e, float x) { v[e] = __float_as_uint(x); }
  static __device__ __forceinline__ void fill(u32x4& v, int e, float x) { v[e] = __float_as_uint(x); }
};
template <> struct Vec<bf16> {
  static constexpr int E = 8;
  static constexpr uint32_t kFill = 0xff80ff80u;
  static __device__ __forceinline__ u32x4 load(const bf16* p) { return *reinterpret_cast<const u32x4u2*>(p); }
  static __device__ __forceinline__ void store(bf16* p, const u32x4& v) { *reinterpret_cast<u32x4u2*>(p) = v; }
  static __device__ __forceinline__ float get(const u32x4& v, int e) { return __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16); }
};
// Columns c .. of a row of n; -infinity behind its end.
template <class T> __device__ __forceinline__ u32x4 load_vec(const T* row, int64_t c, int64_t n) {
  constexpr int E = Vec<T>::E;
  if (c + E <= n) return Vec<T>::load(row + c);
  u32x4 v = {Vec<T>::kFill, Vec<T>::kFill, Vec<T>::kFill, Vec<T>::kFill};
#pragma unroll
  for (int e = 0; e < E - 1; ++e)
    if (c + e < n) {
      if constexpr (E == 8) {
        const uint32_t x = __builtin_bit_cast(unsigned short, row[c + e]);
        v[e / 2] = e & 1 ? (v[e / 2] & 0xffffu) | x << 16 : (v[e / 2] & 0xffff0000u) | x;
      } else {
        v[e] = __float_as_uint(row[c + e]);
      }
    }
  return v;
}

// The larger; NaN where there is one.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Where s z overflows, or comes near it, z - max is formed first; a maximum within these bounds leaves room for every product.
__device__ __forceinline__ float safe_bound(float k) { return 1e38f / fmaxf(k, 1.f); }

// Order of values and, among equals, of indices from the lowest on, as integers.
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) {
  const uint32_t b = __float_as_uint(v + 0.f);          // one zero
  return (uint64_t)(b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u)) << 32 | (0xffffffffu - index);
}
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o ^ ((int32_t)o < 0 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ uint32_t index_of(uint64_t key) { return 0xffffffffu - (uint32_t)key; }

constexpr int kMaxTop = 32, kCap = 1024;
struct LogprobFwdParams {
  const void* z;
  int64_t ldz, rows, vocab;
  const int32_t* targets;
  float scale, k;              // k = scale * log2 e
  float *logp, *entropy, *stats;
  int top;
  int32_t* top_id;
  float* top_logp;
};

// Three numbers of a set of logits: maximum, S and sum of e^d d (base 2) against it.
struct Soft { float m, s, t; };
__device__ __forceinline__ float shift_of(float m, float bound, float k) { return fmaxf(m, -bound) * k; }
// What the rounding of max k left over: the d of the sums are this much too large.
__device__ __forceinline__ float shift_error(float m, float bound, float k) { return __builtin_fmaf(fmaxf(m, -bound), k, -shift_of(m, bound, k)); }
__device__ __forceinline__ Soft rebase(const Soft& a, float m, float bound, float k) {
  const float d = larger(shift_of(a.m, bound, k) - shift_of(m, bound, k), kFloor), f = __builtin_amdgcn_exp2f(d);
  return {m, a.s * f, f * __builtin_fmaf(d, a.s, a.t)};
}

template <class T, int NT, int U>
__global__ __launch_bounds__(NT, 4) void logprob_fwd_kernel(LogprobFwdParams p) {
  constexpr int E = Vec<T>::E, kWaves = NT / 64;
  constexpr int64_t kChunk = (int64_t)NT * U * E;
  __shared__ float group_max[64];
  __shared__ Soft wave_soft[2][kWaves];
  __shared__ uint64_t list[kCap + kMaxTop], wave_key[2][kWaves];
  __shared__ int count;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, top = p.top;
  const int64_t row = blockIdx.x, V = p.vocab;
  const T* const z = reinterpret_cast<const T*>(p.z) + row * p.ldz;
  const float k = p.k, bound = safe_bound(k);
  const int target = p.targets ? p.targets[row] : -1;
  const bool given = target >= 0 && target < V;
  float zt = 0.f;
  if (given && t == 0 && p.logp) zt = to_f32(z[target]);
  if (t == 0) count = 0;

  u32x4 v[U], nx[U];
  auto fetch = [&](int64_t c0) {
#pragma unroll
    for (int u = 0; u < U; ++u) nx[u] = load_vec(z, c0 + ((int64_t)u * NT + t) * E, V);
  };
  Soft mine = {-INFINITY, 0.f, 0.f};
  float thr = -__FLT_MAX__;                              // finite: -infinity is no alternative
  float vec_max[U], chunk_max;

  // A bound that the k best of the chunk reach: upper bits of the k-th largest of 64 groups' maxima.  All waves find the same.  Two of the
  // block's barriers lie between two writes of group_max.
  auto bound_of_chunk = [&] {
    const float g = lanes_max<NT / 64>(chunk_max);
    if (t % (NT / 64) == 0) group_max[t / (NT / 64)] = g;
    __syncthreads();
    const uint32_t mine16 = (uint32_t)(key_of(group_max[lane], 0) >> 48);
    uint32_t best = 0;
#pragma unroll
    for (int b = 15; b >= 0; --b) {
      const uint32_t tryit = best | 1u << b;
      if (__popcll(__ballot(mine16 >= tryit)) >= top) best = tryit;
    }
    return value_of((uint64_t)best << 48);               // NaN's bits are never reached: maxima leave NaN out
  };
  auto push = [&](int64_t c0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!__any(vec_max[u] >= thr)) continue;
      if (vec_max[u] >= thr) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float x = Vec<T>::get(v[u], e);
          if (x >= thr) {
            const int at = atomicAdd(&count, 1);
            if (at < kCap) list[at] = key_of(x, (uint32_t)(c0 + ((int64_t)u * NT + t) * E + e));
          }
        }
      }
    }
  };
  // Ranks of what is in the list, of which n at most kCap + kMaxTop; f(rank, key).
  auto ranked = [&](int n, auto&& f) {
    for (int i = t; i < n; i += NT) {
      const uint64_t key = list[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += list[j] > key;
      f(rank, key);
    }
  };
  // The k best of the list alone stay in it.  Called by all, behind a barrier; ends with one.
  auto compact = [&](int n) {
    constexpr int kPer = (kCap + kMaxTop + NT - 1) / NT;
    int to[kPer], m = 0;
    uint64_t keys[kPer];
    ranked(n, [&](int rank, uint64_t key) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (i == m) to[i] = rank, keys[i] = key;
      ++m;
    });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (i < m && to[i] < top) list[to[i]] = keys[i];
    if (t == 0) count = n < top ? n : top;
    __syncthreads();
  };
  // The k best of the chunk to the end of a list of n, one by one, from memory: rows that come here are odd ones.
  auto extract = [&](int n, int64_t c0) {
    uint64_t last = ~0ull;
    int found = 0;
    for (; found < top; ++found) {
      uint64_t best = 0;
      for (int64_t c = c0 + t; c < V && c < c0 + kChunk; c += NT) {
        const float x = to_f32(z[c]);
        const uint64_t key = x >= -__FLT_MAX__ ? key_of(x, (uint32_t)c) : 0;
        if (key < last && key > best) best = key;
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const uint64_t other = __shfl_xor((unsigned long long)best, o, 64);
        best = other > best ? other : best;
      }
      if (lane == 0) wave_key[found & 1][wave] = best;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) best = wave_key[found & 1][w] > best ? wave_key[found & 1][w] : best;
      if (best == 0) break;
      last = best;
      if (t == 0) list[n + found] = best;
    }
    if (t == 0) count = n + found;
    __syncthreads();
    return n + found;
  };

  fetch(0);
  for (int64_t c0 = 0; c0 < V; c0 += kChunk) {
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = nx[u];
    if (c0 + kChunk < V) fetch(c0 + kChunk);             // travels while this one is reduced
    chunk_max = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      vec_max[u] = Vec<T>::get(v[u], 0);
#pragma unroll
      for (int e = 1; e < E; ++e) vec_max[u] = fmaxf(vec_max[u], Vec<T>::get(v[u], e));
      chunk_max = fmaxf(chunk_max, vec_max[u]);
      __builtin_amdgcn_sched_barrier(0);
    }
    mine = rebase(mine, fmaxf(mine.m, chunk_max), bound, k);
    const float mk = shift_of(mine.m, bound, k);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = larger(__builtin_fmaf(Vec<T>::get(v[u], e), k, -mk), kFloor), x = __builtin_amdgcn_exp2f(d);
        mine.s += x;
        mine.t = __builtin_fmaf(x, d, mine.t);
        if (e == E - 1) __builtin_amdgcn_sched_barrier(0);
      }
    if (top > 0) {
      if (c0 == 0) thr = fmaxf(thr, bound_of_chunk());   // (its barrier is behind the one write of count, too)
      const int before = c0 == 0 ? 0 : count;            // nobody writes it between the last barrier and the next
      if (c0 > 0) __syncthreads();
      push(c0);
      __syncthreads();
      int n = count;
      if (n > kCap) {                                    // uniform, as everything below
        thr = fmaxf(thr, bound_of_chunk());              // (a barrier: everybody has read count)
        if (t == 0) count = before;
        __syncthreads();
        push(c0);
        __syncthreads();
        n = count;
        if (n > kCap) {
          __syncthreads();
          n = extract(before, c0);
        }
      }
      if (n > kCap / 2) {
        __syncthreads();
        compact(n);
        if (count == top) thr = fmaxf(thr, value_of(list[top - 1]));
      }
    }
  }

  // All of the row: within a wave, then between waves.
  {
    const float m = lanes_max(mine.m);
    Soft a = rebase(mine, m, bound, k);
    a.s = lanes_sum(a.s);
    a.t = lanes_sum(a.t);
    if (lane == 0) wave_soft[0][wave] = a;
  }
  __syncthreads();
  Soft all = {-INFINITY, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) all.m = fmaxf(all.m, wave_soft[0][w].m);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const Soft a = rebase(wave_soft[0][w], all.m, bound, k);
    all.s += a.s;
    all.t += a.t;
  }
  const bool extreme = !(fabsf(all.m) <= bound);
  if (extreme && fabsf(all.m) < INFINITY) {              // once more, with z - max first
    float s = 0.f, st = 0.f;
    for (int64_t c = t; c < V; c += NT) {
      const float d = larger((to_f32(z[c]) - all.m) * k, kFloor), x = __builtin_amdgcn_exp2f(d);
      s += x;
      st = __builtin_fmaf(x, d, st);
    }
    s = lanes_sum(s);
    st = lanes_sum(st);
    if (lane == 0) wave_soft[1][wave] = Soft{0.f, s, st};
    __syncthreads();
    all.s = all.t = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      all.s += wave_soft[1][w].s;
      all.t += wave_soft[1][w].t;
    }
  }
  const bool none = all.m == -INFINITY && all.s == 0.f;  // (a NaN beside makes S one)
  const float nan = __builtin_nanf("");
  if (all.m == INFINITY || (all.m == -INFINITY && !none)) all.s = nan;
  const float log2s = __builtin_amdgcn_logf(all.s), lse = (log2s - (extreme ? 0.f : shift_error(all.m, bound, k))) * kLn2;
  auto log_p = [&](float x) { return none ? -INFINITY : (x - all.m) * p.scale - lse; };    // only what is out of range itself overflows
  if (t == 0) {
    if (p.logp) p.logp[row] = given ? log_p(zt) : 0.f;
    if (p.entropy) p.entropy[row] = none ? 0.f : (log2s - all.t / all.s) * kLn2;
    if (p.stats) *reinterpret_cast<float2*>(p.stats + 2 * row) = make_float2(all.m, none ? 0.f : lse);
  }
  if (top > 0) {
    const bool bad = !(all.s == all.s);
    const int n = bad ? 0 : count;                       // (barriers lie behind the last write)
    ranked(n, [&](int rank, uint64_t key) {
      if (rank < top) {
        p.top_id[row * top + rank] = (int32_t)index_of(key);
        p.top_logp[row * top + rank] = log_p(value_of(key));
      }
    });
    for (int i = n + t; i < top; i += NT) {
      p.top_id[row * top + i] = -1;
      p.top_logp[row * top + i] = bad ? nan : -INFINITY;
    }
  }
}

// ---- backward ----------------------------------------------------------------------------------------------------
struct LogprobBwdParams {
  const void* z;
  void* dz;
  int64_t ldz, lddz, rows, vocab, segments;
  const int32_t* targets;
  float scale, k;
  const float *stats, *entropy, *dlogp, *dentropy;
};
constexpr int kBwdThreads = 256, kBwdVecs = 4;
template <class T>
__global__ __launch_bounds__(kBwdThreads) void logprob_bwd_kernel(LogprobBwdParams p) {
  constexpr int E = Vec<T>::E, U = kBwdVecs;
  constexpr int64_t kSeg = (int64_t)kBwdThreads * U * E;
  const float k = p.k, bound = safe_bound(k);
  for (int64_t b = blockIdx.x; b < p.rows * p.segments; b += gridDim.x) {
    const int64_t row = b / p.segments, c0 = (b - row * p.segments) * kSeg + (int64_t)threadIdx.x * E, V = p.vocab;
    const T* const z = reinterpret_cast<const T*>(p.z) + row * p.ldz;
    T* const dz = reinterpret_cast<T*>(p.dz) + row * p.lddz;
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t c = c0 + (int64_t)u * kBwdThreads * E;
      if (c < V) v[u] = load_vec(z, c, V);
    }
    const float2 st = *reinterpret_cast<const float2*>(p.stats + 2 * row);
    const int target = p.targets ? p.targets[row] : -1;
    const bool given = target >= 0 && target < V && p.dlogp;
    const float dl = given ? p.dlogp[row] * p.scale : 0.f, de = p.dentropy ? p.dentropy[row] * p.scale : 0.f;
    const bool none = st.x == -INFINITY && st.y == 0.f, extreme = !(fabsf(st.x) <= bound);
    const float mk = shift_of(st.x, bound, k), log2s = st.y * kLog2e + (extreme ? 0.f : shift_error(st.x, bound, k));
    // dz = p (a0 + a1 log2 p) + [v = t] dl
    const float a0 = -(dl + (p.dentropy ? de * p.entropy[row] : 0.f)), a1 = -de * kLn2;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t c = c0 + (int64_t)u * kBwdThreads * E;
      if (c >= V) break;
      float o[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float x = Vec<T>::get(v[u], e);
        const float d = larger((extreme ? (x - st.x) * k : __builtin_fmaf(x, k, -mk)) - log2s, kFloor), q = __builtin_amdgcn_exp2f(d);
        o[e] = none ? 0.f : q * __builtin_fmaf(a1, d, a0);
      }
      if (given && !none && target >= c && target < c + E) {
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = target == c + e ? o[e] + dl : o[e];
      }
      u32x4 w;
      if constexpr (E == 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)o[2 * i], (bf16)o[2 * i + 1]});
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(o[i]);
      }
      if (c + E <= V) {
        Vec<T>::store(dz + c, w);
      } else {
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
          if (c + e < V) dz[c + e] = from_f32<T>(o[e]);
      }
    }
  }
}

hipError_t check(const LogprobArgs& a) {
  if ((a.dtype != kF32 && a.dtype != kBF16) || !a.z || a.rows < 0 || a.rows > (1LL << 31) - 1 || a.vocab < 1 || a.vocab > (1LL << 28) ||
      a.ldz < a.vocab || !(a.scale > 0.f && a.scale < INFINITY) || ((uintptr_t)a.z & (a.dtype == kBF16 ? 1 : 3)) || ((uintptr_t)a.targets & 3))
    return hipErrorInvalidValue;
  return hipSuccess;
}

}  // namespace

int64_t logprob_ws_floats(int64_t rows, int64_t vocab, int k) {
  if (rows < 0 || rows > (1LL << 31) - 1 || vocab < 1 || vocab > (1LL << 28) || k < 0 || k > kMaxTop) return -1;
  return 0;
}

hipError_t launch_logprob_fwd(hipStream_t s, const LogprobArgs& a, float* logp, float* entropy, float* stats, int k, int32_t* top_id, float* top_logp,
                              float* ws) {
  if (check(a) != hipSuccess || k < 0 || k > kMaxTop || (k > 0 && (!top_id || !top_logp)) || (k == 0 && (top_id || top_logp)) ||
      (logp && !a.targets) || (!logp && !entropy && !stats && k == 0))
    return hipErrorInvalidValue;
  if (((uintptr_t)logp | (uintptr_t)entropy | (uintptr_t)top_id | (uintptr_t)top_logp) & 3 || (uintptr_t)stats & 7) return hipErrorInvalidValue;
  (void)ws;
  if (a.rows == 0) return hipSuccess;
  const LogprobFwdParams p{a.z, a.ldz, a.rows, a.vocab, a.targets, a.scale, a.scale * kLog2e, logp, entropy, stats, k, top_id, top_logp};
  auto run = [&](auto t) {
    using T = decltype(t);
    if (a.rows <= 256 && a.vocab > 8192) logprob_fwd_kernel<T, 1024, 4><<<(unsigned)a.rows, 1024, 0, s>>>(p);
    else logprob_fwd_kernel<T, 256, 8><<<(unsigned)a.rows, 256, 0, s>>>(p);
  };
  if (a.dtype == kF32) run(float{});
  else run(bf16{});
  return hipGetLastError();
}

hipError_t launch_logprob_bwd(hipStream_t s, const LogprobArgs& a, const float* stats, const float* entropy, const float* dlogp, const float* dentropy,
                              void* dz, int64_t lddz) {
  if (check(a) != hipSuccess || !stats || !dz || lddz < a.vocab || (dlogp && !a.targets) || (dentropy && !entropy)) return hipErrorInvalidValue;
  if (((uintptr_t)dlogp | (uintptr_t)entropy | (uintptr_t)dentropy) & 3 || (uintptr_t)stats & 7 || (uintptr_t)dz & (a.dtype == kBF16 ? 1 : 3))
    return hipErrorInvalidValue;
  if (a.rows == 0) return hipSuccess;
  const int64_t seg = (int64_t)kBwdThreads * kBwdVecs * (a.dtype == kBF16 ? 8 : 4), segments = (a.vocab + seg - 1) / seg;
  const LogprobBwdParams p{a.z, dz, a.ldz, lddz, a.rows, a.vocab, segments, a.targets, a.scale, a.scale * kLog2e, stats, entropy, dlogp, dentropy};
  const int64_t blocks = a.rows * segments, most = 1 << 20;
  const unsigned grid = (unsigned)(blocks < most ? blocks : most);
  if (a.dtype == kF32) logprob_bwd_kernel<float><<<grid, kBwdThreads, 0, s>>>(p);
  else logprob_bwd_kernel<bf16><<<grid, kBwdThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace pw
