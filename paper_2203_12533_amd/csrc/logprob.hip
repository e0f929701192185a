// Log probabilities of given tokens, entropy and the likeliest alternatives of rows of logits, from one read, and the gradient of the logits:
//
//   d_v = s (z_v - max z),  S = sum e^d,  logp = d_t - log S,  H = log S - (sum e^d d) / S          (both terms of H are >= 0: nothing cancels)
//   dz_v = s [dlogp ([v = t] - p_v) - dentropy p_v (log p_v + H)],  p_v = e^(d_v - log S)
//
// In base 2: d = z k - max k with k = s log2 e, one fused multiply-add, whose product is exact; that max k is rounded shifts all of a row alike, by
// an amount of at most 1/4 that is known and taken off log S (in H it cancels).  What rounding then leaves of log S and H below 0 becomes 0, so that no
// probability is above 1.  Every thread keeps a running maximum, S and sum of its own; they meet once per row, in a tree.  A
// part of a row (32 terms of a thread) is summed in fp32 and joins the running pair in 64 bits: equal terms, as logits in few bits give, round the same way
// every time, and log S of a chain of 16384 fp32 additions was off by 8e-5.
//
// Alternatives.  Every wave keeps a list in LDS of what can be among the k best of its columns, without a word to the others: with a part of the row in
// registers, the k-th largest of its 64 lanes' maxima (the upper 16 bits of it) is a bound that k elements at least reach, and usually few more do.  Those go to
// the list as keys of value and index, 64 bits, no two alike, placed by a ballot; what comes later in the row adds what reaches the bound.  A list that is full
// gets a tighter bound, and where that does not help - values that fall into few lanes - the k best are taken out one by one, from memory: with 8 of them 2110
// us for 8192 rows of 32768 bf16 of one value, and 1750 where a mask of the type's lowest value leaves 200 neighbours of each row (a mask of -infinity 85, since
// that is no alternative; other rows 107).  At the end one wave takes the lists together, drops what is below such a bound of all, and ranks the rest by
// counting (every wave its own list first, in order: 174 us for 8192 rows of 32768 bf16 and k = 32, this then 147).
//
// Bound by memory: forward one read, backward one read and one write, the forward one nearly as much by its 40 or so cycles per element and lane
// (exp2 takes four slots of ten); vectors that lie behind the row as a whole are left out (8192 x 9000 bf16, 8 alternatives, 74 us with them, 55
// without).  The last 256 MB of logits, what the large cache holds, are read so that they stay there, and the backward call goes backwards and finds
// them; all else is read, and the gradient written, past the caches.  8192 rows of 32768 bf16: forward 92 us without alternatives (5.8 TB/s), 107
// with 8, 125 with 32; forward with 8 and backward 261 to 266, with every access an ordinary one, forwards, 338.  4096 rows of fp32: 94 and 252, so 321.
// Few rows are cut into segments, a block each, and joined by a second launch (4 rows of 32768 fp32, 20 alternatives: 10.6 us; as one block of 1024
// threads 12.2); a call of one launch is bound by latency (1 x 4000: 5.6 us).
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
  typedef u32x4u4 At;
  static __device__ __forceinline__ float get(const u32x4& v, int e) { return __uint_as_float(v[e]); }
  static __device__ __forceinline__ void put(u32x4& v, int e, float x) { v[e] = __float_as_uint(x); }
  static __device__ __forceinline__ void fill(u32x4& v, int e, float x) { v[e] = __float_as_uint(x); }
};
template <> struct Vec<bf16> {
  static constexpr int E = 8;
  static constexpr uint32_t kFill = 0xff80ff80u;
  typedef u32x4u2 At;
  static __device__ __forceinline__ float get(const u32x4& v, int e) { return __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16); }
};
// Columns c .. of a row of n (2^28 at most: offsets of bytes are 32 bits beside a uniform address); -infinity behind its end.
// KEEP: to stay in the caches.
template <bool KEEP, class T> __device__ __forceinline__ u32x4 load_vec(const T* row, uint32_t c, uint32_t n) {
  constexpr int E = Vec<T>::E;
  if (c + E <= n) {
    const auto p = reinterpret_cast<const typename Vec<T>::At*>(reinterpret_cast<const char*>(row) + c * (uint32_t)sizeof(T));
    return KEEP ? *p : __builtin_nontemporal_load(p);
  }
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

// Rows whose maximum is further from 0 are read again, with z - max formed first: up to 2^22 the rounding of max k shifts d by 1/4 at most, beyond it
// the sums would lose their bits and overflow.
float safe_bound(float k) { return fminf(4194304.f / k, 1e38f); }

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

// f(key, how many of the n in the list are larger) for the keys i, i + step, ...  M: at most so many of them are a thread's. 
template <int M, class F> __device__ __forceinline__ void ranks(const uint64_t* list, int n, int i, int step, F&& f) {
  uint64_t key[M];
  int rank[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    key[m] = i + m * step < n ? list[i + m * step] : ~0ull;
    rank[m] = 0;
  }
#pragma unroll 8
  for (int j = 0; j < n; ++j) {
    const uint64_t other = list[j];
#pragma unroll
    for (int m = 0; m < M; ++m) rank[m] += other > key[m];
  }
#pragma unroll
  for (int m = 0; m < M; ++m)
    if (i + m * step < n) f(key[m], rank[m]);
}

constexpr int kMaxTop = 32;
struct LogprobFwdParams {
  const void* z;
  int64_t ldz, rows, vocab;
  const int32_t* targets;
  float scale, k, bound;       // k = scale * log2 e, bound = safe_bound(k)
  float *logp, *entropy, *stats;
  int top;
  int32_t* top_id;
  float* top_logp;
  int segments;                // that a row is cut into, one to a block; > 1: what they find goes to `parts`, [row][segment] of 4 + 2 top floats
  int64_t segment;             // elements
  float* parts;
  int64_t kept;                // rows from this one on are left in the caches
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
// S and sum of a thread over as many parts as there are, against a maximum that moved by d.
struct Long { double s, t; };
__device__ __forceinline__ Long rebase(const Long& a, float d) {
  const double f = __builtin_amdgcn_exp2f(d);
  return {f * a.s, f * __builtin_fma((double)d, a.s, a.t)};
}

// The logit of a row's given token, for one thread: asked for before anything else, as one load waits for the other.
struct Given { bool is; float z; };
template <class T> __device__ __forceinline__ Given given_of(const LogprobFwdParams& p, int64_t row) {
  if (!p.targets || !p.logp) return {false, 0.f};
  const int target = p.targets[row];
  if (target < 0 || target >= p.vocab) return {false, 0.f};
  return {true, to_f32((reinterpret_cast<const T*>(p.z) + row * p.ldz)[target])};
}

// What becomes of a row when its parts are together: `all` of the fast sums, the list of n keys that hold the best (LDS, the first wave's).
// The whole block calls; `given` is its first thread's.
template <class T, int NT>
__device__ __forceinline__ void finish_row(const LogprobFwdParams& p, int64_t row, Soft all, const uint64_t* list, int n, Soft* wave_soft,
                                           const Given& given) {
  constexpr int kWaves = NT / 64;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, top = p.top;
  const T* const z = reinterpret_cast<const T*>(p.z) + row * p.ldz;
  const float k = p.k, bound = p.bound;
  const bool extreme = !(fabsf(all.m) <= bound);
  if (extreme && fabsf(all.m) < INFINITY) {              // once more, with z - max first
    double own = 0.0, own_t = 0.0;
    for (int64_t c = t; c < p.vocab; c += NT) {
      const float d = larger((to_f32(z[c]) - all.m) * k, kFloor), x = __builtin_amdgcn_exp2f(d);
      own += x;
      own_t = __builtin_fma((double)x, (double)d, own_t);
    }
    const float s = lanes_sum((float)own), st = lanes_sum((float)own_t);
    if (lane == 0) wave_soft[wave] = Soft{0.f, s, st};
    __syncthreads();
    all.s = all.t = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      all.s += wave_soft[w].s;
      all.t += wave_soft[w].t;
    }
  }
  const bool none = all.m == -INFINITY && all.s == 0.f;  // (a NaN beside makes S one)
  const float nan = __builtin_nanf("");
  if (all.m == INFINITY || (all.m == -INFINITY && !none)) all.s = nan;
  // S has a term of 1, so that log S >= 0 (and H); larger() keeps a NaN.
  const float log2s = __builtin_amdgcn_logf(all.s), lse = larger((log2s - (extreme ? 0.f : shift_error(all.m, bound, k))) * kLn2, 0.f);
  auto log_p = [&](float x) { return none ? -INFINITY : __builtin_fmaf(x - all.m, p.scale, -lse); };    // only what is out of range itself overflows
  if (t == 0) {
    if (p.logp) p.logp[row] = given.is ? log_p(given.z) : 0.f;
    if (p.entropy) p.entropy[row] = none ? 0.f : larger((log2s - all.t / all.s) * kLn2, 0.f);
    if (p.stats) *reinterpret_cast<float2*>(p.stats + 2 * row) = make_float2(all.m, none ? 0.f : lse);
  }
  if (top > 0 && wave == 0) {
    const bool bad = !(all.s == all.s);
    if (bad) n = 0;
    auto put = [&](uint64_t key, int rank) {
      if (rank < top) {
        p.top_id[row * top + rank] = (int32_t)index_of(key);
        p.top_logp[row * top + rank] = log_p(value_of(key));
      }
    };
    for (int i = lane; i < n; i += 64) ranks<1>(list, n, i, 64, put);
    for (int i = n + lane; i < top; i += 64) {
      p.top_id[row * top + i] = -1;
      p.top_logp[row * top + i] = bad ? nan : -INFINITY;
    }
  }
}

// LDS of one wave: what its lanes wrote is there for the others.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// To the front of a list in LDS: those of a wave's keys (0: none), M to a lane, whose upper 16 bits reach the k-th largest of the lanes' maxima.  The k
// best are among them; how many they are is returned.
template <int M> __device__ __forceinline__ int shortlist(const uint64_t (&key)[M], int top, uint64_t* list) {
  uint64_t most = 0;
#pragma unroll
  for (int m = 0; m < M; ++m) most = key[m] > most ? key[m] : most;
  const uint32_t mine16 = (uint32_t)(most >> 48);
  uint32_t least = 0;
#pragma unroll
  for (int b = 15; b >= 0; --b) {
    const uint32_t tryit = least | 1u << b;
    if (__popcll(__ballot(mine16 >= tryit)) >= top) least = tryit;
  }
  int n = 0;
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const bool take = key[m] != 0 && (uint32_t)(key[m] >> 48) >= least;
    const uint64_t who = __ballot(take);
    if (take) list[n + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] = key[m];
    n += __popcll(who);
  }
  wave_sync();
  return n;
}

// NT threads of a block, U vectors of 16 bytes to one in a chunk; a wave's list has kPlaces places, and kMaxTop more for a k best of a chunk.  Six blocks of 256
// to a unit, two registers spilled for it (8192 x 32768 bf16 107.1 us with 8 alternatives, 124.4 with 32; five 106.1 and 130.6).
constexpr int kPlaces = 256;
template <class T, int NT, int U, bool TOP>
__global__ __launch_bounds__(NT, NT == 256 ? 6 : 4) void logprob_fwd_kernel(LogprobFwdParams p) {
  constexpr int E = Vec<T>::E, kWaves = NT / 64;
  constexpr uint32_t kChunk = NT * U * E;
  __shared__ Soft wave_soft[2][kWaves];
  __shared__ uint64_t lists[TOP ? kWaves : 1][TOP ? kPlaces + kMaxTop : 1], best_keys[TOP ? kWaves * kMaxTop : 1];
  __shared__ int counts[kWaves];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), top = TOP ? p.top : 0;
  // A division's result is in vector registers, which are short here.
  const uint32_t in_row = __builtin_amdgcn_readfirstlane(p.segments > 1 ? blockIdx.x / (uint32_t)p.segments : blockIdx.x);
  const int64_t row = in_row;
  const uint32_t seg = blockIdx.x - in_row * (uint32_t)p.segments;
  const uint32_t from = seg * (uint32_t)p.segment, V = (uint32_t)(from + p.segment < p.vocab ? from + p.segment : p.vocab);   // of this block: from .. V - 1
  const T* const z = reinterpret_cast<const T*>(p.z) + row * p.ldz;
  const float k = p.k, bound = p.bound;
  const bool keep = row >= p.kept;
  uint64_t* const list = lists[TOP ? wave : 0];
  Given given = {};
  if (t == 0 && p.segments == 1) given = given_of<T>(p, row);
  int n = 0;                                             // keys in it

  u32x4 v[U], nx[U];
  auto fetch = [&](uint32_t c0) {
    const uint32_t c = c0 + (uint32_t)t * E;
#pragma unroll
    for (int u = 0; u < U; ++u) nx[u] = keep ? load_vec<true>(z, c + u * NT * E, V) : load_vec<false>(z, c + u * NT * E, V);
  };
  Long mine = {0.0, 0.0};
  float so_far = -INFINITY;                              // the maximum
  float thr = -__FLT_MAX__;                              // finite: -infinity is no alternative
  float vec_max[U], chunk_max;

  // A bound that the k best of the wave reach: upper bits of the k-th largest of its lanes' maxima, of the chunk or of all so far.
  auto bound_of = [&](float lane_max) {
    const uint32_t mine16 = (uint32_t)(key_of(lane_max, 0) >> 48);
    uint32_t best = 0;
#pragma unroll
    for (int b = 15; b >= 0; --b) {
      const uint32_t tryit = best | 1u << b;
      if (__popcll(__ballot(mine16 >= tryit)) >= top) best = tryit;
    }
    return value_of((uint64_t)best << 48);               // NaN's bits are never reached: maxima leave NaN out
  };
  auto push = [&](uint32_t c0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!__any(vec_max[u] >= thr)) continue;
      uint32_t col = c0 + (uint32_t)(u * NT + t) * E;
      asm volatile("" : "+v"(col));                      // not kept for every u across the loop
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float x = Vec<T>::get(v[u], e);
        const uint64_t who = __ballot(x >= thr);
        if (who == 0) continue;
        const int at = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
        if (x >= thr && at < kPlaces) list[at] = key_of(x, col + e);
        n += __popcll(who);
      }
    }
  };
  // The k best of the list alone stay in it, in order.
  auto compact = [&] {
    wave_sync();
    auto put = [&](uint64_t key, int rank) {
      if (rank < top) best_keys[wave * kMaxTop + rank] = key;
    };
#pragma unroll 1
    for (int i = 0; i < n; i += 128) ranks<2>(list, n, i + lane, 64, put);
    wave_sync();
    n = n < top ? n : top;
    if (lane < n) list[lane] = best_keys[wave * kMaxTop + lane];
    wave_sync();
  };
  // The k best of the wave's part of the chunk to the end of the list, one by one, from memory.
  auto extract = [&](uint32_t c0) {
    uint64_t last = ~0ull;
#pragma unroll 1
    for (int found = 0; found < top; ++found) {
      uint64_t best = 0;
#pragma unroll 1
      for (int i = 0; i < U * E; ++i) {
        const uint32_t c = c0 + (uint32_t)((i / E) * NT + t) * E + i % E;
        if (c >= V) continue;
        const float x = to_f32(z[c]);
        const uint64_t key = x >= -__FLT_MAX__ ? key_of(x, c) : 0;
        if (key < last && key > best) best = key;
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const uint64_t other = __shfl_xor((unsigned long long)best, o, 64);
        best = other > best ? other : best;
      }
      if (best == 0) break;
      last = best;
      if (lane == 0) list[n] = best;
      ++n;
    }
  };

  fetch(from);
#pragma unroll 1
  for (uint32_t c0 = from; c0 < V; c0 += kChunk) {
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
    const float most = fmaxf(so_far, chunk_max), mk = shift_of(most, bound, k), change = larger(shift_of(so_far, bound, k) - mk, kFloor);
    so_far = most;
    mine = rebase(mine, change);
    float s = 0.f, st = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u > 0 && c0 + u * NT * E >= V) break;          // uniform: the row's last chunk
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = larger(__builtin_fmaf(Vec<T>::get(v[u], e), k, -mk), kFloor), x = __builtin_amdgcn_exp2f(d);
        s += x;
        st = __builtin_fmaf(x, d, st);
        if (e == E - 1) __builtin_amdgcn_sched_barrier(0);
      }
    }
    mine = {mine.s + s, mine.t + st};
    if constexpr (TOP) {                                 // uniform over the wave
      thr = fmaxf(thr, bound_of(so_far));
      const int before = n;
      push(c0);
      if (n > kPlaces) {
        n = before;
        thr = fmaxf(thr, bound_of(chunk_max));
        push(c0);
        if (n > kPlaces) {
          n = before;
          extract(c0);
        }
      }
      if (n > kPlaces / 2) {
        compact();
        if (n == top) thr = fmaxf(thr, value_of(list[top - 1]));
      }
    }
  }

  // All of the segment: within a wave, then between waves.
  {
    const float m = lanes_max(so_far);
    Soft a = rebase(Soft{so_far, (float)mine.s, (float)mine.t}, m, bound, k);
    a.s = lanes_sum(a.s);
    a.t = lanes_sum(a.t);
    if (lane == 0) wave_soft[0][wave] = a;
  }
  if (TOP && lane == 0) counts[wave] = n;                // kPlaces / 2 at most
  __syncthreads();
  int keys = 0;                                          // the first wave's: what can be among the block's k best
  if constexpr (TOP) {
    if (wave == 0) {
      constexpr int kPer = kPlaces / 2 / 64;
      uint64_t key[kWaves * kPer];
#pragma unroll
      for (int i = 0; i < kWaves * kPer; ++i) key[i] = i % kPer * 64 + lane < counts[i / kPer] ? lists[i / kPer][i % kPer * 64 + lane] : 0;
      keys = shortlist(key, top, lists[0]);              // all of them are in registers: the lists' place is free
    }
  }
  Soft all = {-INFINITY, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) all.m = fmaxf(all.m, wave_soft[0][w].m);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const Soft a = rebase(wave_soft[0][w], all.m, bound, k);
    all.s += a.s;
    all.t += a.t;
  }
  if (p.segments == 1) {
    finish_row<T, NT>(p, row, all, lists[0], keys, wave_soft[1], given);
    return;
  }
  float* const out = p.parts + (int64_t)blockIdx.x * (4 + 2 * p.top);
  if (t == 0) *reinterpret_cast<float2*>(out) = make_float2(all.m, all.s), out[2] = all.t;
  if constexpr (TOP) {
    if (wave > 0) return;
    uint64_t* const to = reinterpret_cast<uint64_t*>(out + 4);
    for (int i = lane; i < keys; i += 64)
      ranks<1>(lists[0], keys, i, 64, [&](uint64_t key, int rank) {
        if (rank < top) to[rank] = key;
      });
    for (int i = keys + lane; i < top; i += 64) to[i] = 0;  // no key
  }
}

// The segments of a row together, at most kSegments of at most kMaxTop keys each, by one wave: of the keys those are ranked that reach the k-th largest of
// the lanes' maxima.
constexpr int kSegments = 32, kJoin = 64;
template <class T>
__global__ __launch_bounds__(kJoin) void logprob_join_kernel(LogprobFwdParams p) {
  constexpr int kPer = kSegments * kMaxTop / kJoin;
  __shared__ uint64_t list[kSegments * kMaxTop];
  __shared__ Soft wave_soft[1];
  const int lane = threadIdx.x, top = p.top;
  const int64_t row = blockIdx.x;
  const float* const in = p.parts + row * p.segments * (4 + 2 * top);
  const float k = p.k, bound = p.bound;
  Given given = {};
  if (lane == 0) given = given_of<T>(p, row);
  Soft all = {-INFINITY, 0.f, 0.f};
  if (lane < p.segments) {
    const float* const q = in + lane * (4 + 2 * top);
    all = Soft{q[0], q[1], q[2]};
  }
  uint64_t key[kPer];
#pragma unroll
  for (int m = 0; m < kPer; ++m) {
    const int i = m * kJoin + lane, s = top > 0 ? i / top : 0;
    key[m] = i < p.segments * top ? *reinterpret_cast<const uint64_t*>(in + s * (4 + 2 * top) + 4 + 2 * (i - s * top)) : 0;
  }
  all = rebase(all, lanes_max(all.m), bound, k);
  all.s = lanes_sum(all.s);
  all.t = lanes_sum(all.t);
  const int n = top > 0 ? shortlist(key, top, list) : 0;
  finish_row<T, kJoin>(p, row, all, list, n, wave_soft, given);
}

// ---- backward ----------------------------------------------------------------------------------------------------
struct LogprobBwdParams {
  const void* z;
  void* dz;
  int64_t ldz, lddz, rows, vocab, segments;
  const int32_t* targets;
  float scale, k, bound;
  const float *stats, *entropy, *dlogp, *dentropy;
  int64_t kept;                // rows from this one on may be in a cache
};
// A block takes one part of a row after the other, four of them where there are many: 8192 x 32768 bf16 157 us behind the forward pass, a block to each part
// 190, 4096 rows of fp32 159 and 181; eight waves to a SIMD by holding registers down (fp32 with five 190 in parts).
constexpr int kBwdThreads = 256, kBwdVecs = 4;
template <class T>
__global__ __launch_bounds__(kBwdThreads, 8) void logprob_bwd_kernel(LogprobBwdParams p) {
  constexpr int E = Vec<T>::E, U = kBwdVecs;
  constexpr int64_t kSeg = (int64_t)kBwdThreads * U * E;
  const float k = p.k, bound = p.bound;
  // Backwards: the last rows may be in a cache.
  for (int64_t b = p.rows * p.segments - 1 - blockIdx.x; b >= 0; b -= gridDim.x) {
    const int64_t row = b / p.segments, c0 = (b - row * p.segments) * kSeg + (int64_t)threadIdx.x * E, V = p.vocab;
    const T* const z = reinterpret_cast<const T*>(p.z) + row * p.ldz;
    T* const dz = reinterpret_cast<T*>(p.dz) + row * p.lddz;
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t c = c0 + (int64_t)u * kBwdThreads * E;
      if (c < V) v[u] = row >= p.kept ? load_vec<true>(z, c, V) : load_vec<false>(z, c, V);
    }
    const float2 st = *reinterpret_cast<const float2*>(p.stats + 2 * row);
    const int target = p.targets ? p.targets[row] : -1;
    const bool given = target >= 0 && target < V && p.dlogp;
    const float dl = given ? p.dlogp[row] * p.scale : 0.f, de = p.dentropy ? p.dentropy[row] * p.scale : 0.f;
    const bool none = st.x == -INFINITY && st.y == 0.f, extreme = !(fabsf(st.x) <= bound);
    const float mk = shift_of(st.x, bound, k), log2s = st.y * kLog2e + (extreme ? 0.f : shift_error(st.x, bound, k));
    // dz = p (a0 + a1 log2 p) + [v = t] dl.  A row like any other takes one multiply-add for log2 p, against c1 = max k + log2 S rounded to 32 bits: what
    // that leaves, c2, goes into a0 and a1.
    const float a0 = -(dl + (p.dentropy ? de * p.entropy[row] : 0.f)), a1 = -de * kLn2;
    const float c1 = mk + log2s, b1 = c1 - mk, c2 = (mk - (c1 - b1)) + (log2s - b1), f = __builtin_amdgcn_exp2f(-c2);
    const float f0 = f * (a0 - a1 * c2), f1 = f * a1;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t c = c0 + (int64_t)u * kBwdThreads * E;
      if (c >= V) break;
      float o[E];
      if (!(none || extreme)) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float d = larger(__builtin_fmaf(Vec<T>::get(v[u], e), k, -c1), kFloor);
          o[e] = __builtin_amdgcn_exp2f(d) * __builtin_fmaf(f1, d, f0);
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float d = larger((Vec<T>::get(v[u], e) - st.x) * k - log2s, kFloor);
          o[e] = none ? 0.f : __builtin_amdgcn_exp2f(d) * __builtin_fmaf(a1, d, a0);
        }
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
        __builtin_nontemporal_store((typename Vec<T>::At)w, reinterpret_cast<typename Vec<T>::At*>(dz + c));
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
      a.ldz < a.vocab || !(a.scale > 0.f && a.scale <= 0x1p127f) || ((uintptr_t)a.z & (a.dtype == kBF16 ? 1 : 3)) || ((uintptr_t)a.targets & 3))
    return hipErrorInvalidValue;
  return hipSuccess;
}

}  // namespace

// The first row of the last 256 MB, which is what the large cache holds.
static int64_t kept_from(const LogprobArgs& a) {
  const int64_t rows = (256LL << 20) / (a.vocab * (a.dtype == kBF16 ? 2 : 4));
  return rows < a.rows ? a.rows - rows : 0;
}
// How many segments rows are cut into: where there are too few for the chip and a row is more than 64 KB, as many as keep 4096 elements each, a block of 256 threads to one.
// Up to two blocks of 512 threads to a unit, whole rows of more than 16 KB are one block's of 512 threads, else of 256, of 64 up to 2048 elements, and a
// thread's vectors in a chunk are no more than the row needs (8192 x 4000 bf16, 4 alternatives, 47 with four, 29, now 26.6, with two; 8192 x 100 15.5 with four,
// 10.4 with one).  In us, 20 alternatives:
//                      cut   512   256 threads                            cut   512   256 threads
//   4 x 32768 bf16    11.4  10.3                   64 x 131072 bf16      14.3  24.9
//   4 x 32768 fp32    10.9  12.2                   256 x 131072 bf16     27.8  26.7
//   4 x 131072 fp32   11.2  29.3                   511 x 131072 bf16     40.7  36.7
//   4 x 16384 bf16    11.4   7.9                   511 x 32768 bf16      18.5  14.3
//   4 x 4000 fp32            6.8   6.0             511 x 5000 bf16             10.2   7.7        (600 x 32768 with 256: 19.9)
static int segments_of(int64_t rows, int64_t vocab, int bytes) {
  if (rows < 1 || rows >= 256 || vocab * bytes <= 65536) return 1;
  int64_t n = 1024 / rows;
  if (n > vocab / 4096) n = vocab / 4096;
  return (int)(n < kSegments ? n : kSegments);
}
int64_t logprob_ws_floats(int64_t rows, int64_t vocab, int k) {
  if (rows < 0 || rows > (1LL << 31) - 1 || vocab < 1 || vocab > (1LL << 28) || k < 0 || k > kMaxTop) return -1;
  const int n = segments_of(rows, vocab, 4);             // of either type: bf16 rows are cut in as many or not at all
  return n > 1 ? rows * n * (4 + 2 * k) : 0;
}

hipError_t launch_logprob_fwd(hipStream_t s, const LogprobArgs& a, float* logp, float* entropy, float* stats, int k, int32_t* top_id, float* top_logp,
                              float* ws) {
  if (check(a) != hipSuccess || k < 0 || k > kMaxTop || (k > 0 && (!top_id || !top_logp)) || (k == 0 && (top_id || top_logp)) ||
      (logp && !a.targets) || (!logp && !entropy && !stats && k == 0))
    return hipErrorInvalidValue;
  if (((uintptr_t)logp | (uintptr_t)entropy | (uintptr_t)top_id | (uintptr_t)top_logp) & 3 || (uintptr_t)stats & 7) return hipErrorInvalidValue;
  if (logprob_ws_floats(a.rows, a.vocab, k) > 0 && (!ws || ((uintptr_t)ws & 7))) return hipErrorInvalidValue;
  if (a.rows == 0) return hipSuccess;
  const int bytes = a.dtype == kBF16 ? 2 : 4, n = segments_of(a.rows, a.vocab, bytes);
  auto run = [&](auto t, auto with_top) {
    using T = decltype(t);
    constexpr bool TOP = decltype(with_top)::value;
    const float k2 = a.scale * kLog2e;
    const int64_t most = 1LL << 22;                        // rows of a launch, which takes less than 2^32 threads
    for (int64_t r = 0; r < a.rows; r += most) {
      auto from = [&](auto* p, int64_t per) { return p ? p + r * per : nullptr; };
      const int64_t rows = a.rows - r < most ? a.rows - r : most;
      const LogprobFwdParams p{reinterpret_cast<const T*>(a.z) + r * a.ldz, a.ldz, rows, a.vocab, from(a.targets, 1), a.scale, k2, safe_bound(k2),
                               from(logp, 1), from(entropy, 1), from(stats, 2), k, from(top_id, k), from(top_logp, k), n, (a.vocab + n - 1) / n, ws,
                               kept_from(a) - r};
      const unsigned blocks = (unsigned)(rows * n);
      constexpr int E = Vec<T>::E;
      if (a.vocab <= 64 * E) logprob_fwd_kernel<T, 64, 1, TOP><<<blocks, 64, 0, s>>>(p);
      else if (a.vocab <= 128 * E) logprob_fwd_kernel<T, 64, 2, TOP><<<blocks, 64, 0, s>>>(p);
      else if (a.vocab <= 2048) logprob_fwd_kernel<T, 64, 4, TOP><<<blocks, 64, 0, s>>>(p);
      else if (n == 1 && a.rows <= 512 && a.vocab * bytes > 16384) logprob_fwd_kernel<T, 512, 4, TOP><<<blocks, 512, 0, s>>>(p);
      else if (a.vocab <= 512 * E) logprob_fwd_kernel<T, 256, 2, TOP><<<blocks, 256, 0, s>>>(p);
      else logprob_fwd_kernel<T, 256, 4, TOP><<<blocks, 256, 0, s>>>(p);
      if (n > 1) logprob_join_kernel<T><<<(unsigned)rows, kJoin, 0, s>>>(p);
    }
  };
  auto type = [&](auto t) {
    if (k > 0) run(t, std::true_type{});
    else run(t, std::false_type{});
  };
  if (a.dtype == kF32) type(float{});
  else type(bf16{});
  return hipGetLastError();
}

hipError_t launch_logprob_bwd(hipStream_t s, const LogprobArgs& a, const float* stats, const float* entropy, const float* dlogp, const float* dentropy,
                              void* dz, int64_t lddz) {
  if (check(a) != hipSuccess || !stats || !dz || lddz < a.vocab || (dlogp && !a.targets) || (dentropy && !entropy)) return hipErrorInvalidValue;
  if (((uintptr_t)dlogp | (uintptr_t)entropy | (uintptr_t)dentropy) & 3 || (uintptr_t)stats & 7 || (uintptr_t)dz & (a.dtype == kBF16 ? 1 : 3))
    return hipErrorInvalidValue;
  if (dz == a.z && lddz != a.ldz && a.rows > 1) return hipErrorInvalidValue;   // a row's gradient would lie on other rows' logits
  if (a.rows == 0) return hipSuccess;
  const int64_t seg = (int64_t)kBwdThreads * kBwdVecs * (a.dtype == kBF16 ? 8 : 4), segments = (a.vocab + seg - 1) / seg;
  const float k2 = a.scale * kLog2e;
  const LogprobBwdParams p{a.z, dz, a.ldz, lddz, a.rows, a.vocab, segments, a.targets, a.scale, k2, safe_bound(k2), stats, entropy, dlogp, dentropy, kept_from(a)};
  const int64_t blocks = a.rows * segments, most = 4 * 2048;            // 2048 are on the chip at a time
  const unsigned grid = (unsigned)(blocks < most ? blocks : most);
  if (a.dtype == kF32) logprob_bwd_kernel<float><<<grid, kBwdThreads, 0, s>>>(p);
  else logprob_bwd_kernel<bf16><<<grid, kBwdThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace pw
