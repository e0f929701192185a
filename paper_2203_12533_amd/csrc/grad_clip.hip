// The 2-norm of all gradients together, and the gradients scaled to a largest norm:
//
//   norm = sqrt(sum over tensors and elements g^2),  factor = max_norm / norm where norm > max_norm, else 1;   out = g factor
//
// Squares are formed and added in 64 bits: neither overflows nor vanishes for any fp32 value, and a sum of 10^9 of them keeps 24 bits; it costs two
// operations per element where memory allows for ten.  Two launches for up to kGroup tensors, whose addresses travel with the launch: blocks
// take chunks of tensors in turn and leave a sum each, then every block of the second adds those sums in the same order (16 KB or
// less, from the cache) and scales its chunks.
//
// Bound by memory: two reads and a write of 4 (2) bytes.  The last 256 MB, what the large cache holds, are read so that they stay there, and the
// second launch goes backwards and finds them; all else is read and written past the caches.  336e6 fp32 elements: norm 193 us (6.9 TB/s), all 610
// (6.6 TB/s of three passes over memory); with every access an ordinary one 247 and 765, forwards through the second too and on 1024 blocks. 67e6
// elements 117 us, with nothing kept 132, with ordinary stores 164.  A small set is two launches: 24 tensors of 139e3 elements 9.3 us.
#include "common.hpp"
#include "kernels.hpp"

namespace pw {

namespace {

constexpr int kThreads = 256, kGroup = 96, kParts = 2048, kScaleBlocks = 8 * kParts;
constexpr int64_t kKept = 256LL << 20;       // bytes
constexpr int64_t kChunk = 8192;             // elements

struct Entry {
  const void* g;
  void* out;
  int64_t n;
  uint32_t first;                            // chunk of the launch that it begins with
  uint32_t is_bf16;
};
struct Group {
  Entry t[kGroup];                           // with elements, so that no two begin with the same chunk
  uint32_t count, chunks, kept;              // kept: so many of the last chunks are left in the caches for whoever reads them next
};
static_assert(sizeof(Group) <= 3500, "with the launch");

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));     // wherever an element may be

// The tensor that chunk c of the launch is of: the last one that begins at or before it.  All lanes of a wave look at once.
__device__ __forceinline__ int tensor_of(const Group& a, uint32_t c) {
  int n = 0;
#pragma unroll
  for (int i = 0; i < kGroup; i += 64) {
    const uint32_t at = i + (threadIdx.x & 63);
    n += __popcll(__ballot(at < a.count && a.t[at < kGroup ? at : 0].first <= c));
  }
  return __builtin_amdgcn_readfirstlane(n - 1);
}

// A chunk's vectors of one thread, 16 bytes each: v[i] holds elements (i * kThreads + thread) * E .. of n; zeros behind the end.
constexpr int kVecs = kChunk / 4 / kThreads;
template <class T> struct Piece {
  static constexpr int E = 16 / sizeof(T), kUsed = kChunk / E / kThreads;
  static __device__ __forceinline__ float get(const u32x4& v, int e) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[e]);
    else return __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
  }
  static __device__ __forceinline__ void load(u32x4 (&v)[kVecs], const T* g, int n, bool keep) {
    const u32x4u* const p = reinterpret_cast<const u32x4u*>(g) + threadIdx.x;
    if (n == kChunk && keep) {               // a whole chunk: no question at each vector
#pragma unroll
      for (int i = 0; i < kUsed; ++i) v[i] = p[i * kThreads];
      return;
    }
    if (n == kChunk) {
#pragma unroll
      for (int i = 0; i < kUsed; ++i) v[i] = __builtin_nontemporal_load(p + i * kThreads);
      return;
    }
#pragma unroll
    for (int i = 0; i < kUsed; ++i) {
      const int at = (i * kThreads + threadIdx.x) * E;
      if (at + E <= n) {
        v[i] = *reinterpret_cast<const u32x4u*>(g + at);
      } else {
        v[i] = u32x4{};
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
          if (at + e < n) {
            if constexpr (sizeof(T) == 4) v[i][e] = __builtin_bit_cast(uint32_t, g[at + e]);
            else v[i][e / 2] |= (uint32_t)__builtin_bit_cast(unsigned short, g[at + e]) << (16 * (e & 1));
          }
      }
    }
  }
  static __device__ __forceinline__ u32x4 scaled(const u32x4& v, float f) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(get(v, e) * f);
      else w[e] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)(get(v, 2 * e) * f), (bf16)(get(v, 2 * e + 1) * f)});
    }
    return w;
  }
  static __device__ __forceinline__ void store(const u32x4 (&v)[kVecs], T* o, int n, float f) {
    u32x4u* const p = reinterpret_cast<u32x4u*>(o) + threadIdx.x;
    if (n == kChunk) {
#pragma unroll
      for (int i = 0; i < kUsed; ++i) __builtin_nontemporal_store((u32x4u)scaled(v[i], f), p + i * kThreads);
      return;
    }
#pragma unroll
    for (int i = 0; i < kUsed; ++i) {
      const int at = (i * kThreads + threadIdx.x) * E;
      if (at + E <= n) {
        *reinterpret_cast<u32x4u*>(o + at) = scaled(v[i], f);
      } else {
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
          if (at + e < n) o[at + e] = from_f32<T>(get(v[i], e) * f);
      }
    }
  }
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ double block_sum64(double v) {
  __shared__ double red[kThreads / 64];
  v = wave_sum64(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(Group a, double* part, int add) {
  double s[2] = {0.0, 0.0};
  u32x4 v[kVecs];
  auto squares = [&](auto type) {
    typedef Piece<decltype(type)> P;
#pragma unroll
    for (int i = 0; i < P::kUsed; ++i)
#pragma unroll
      for (int e = 0; e < P::E; ++e) {
        const double x = P::get(v[i], e);
        s[e & 1] = __builtin_fma(x, x, s[e & 1]);
      }
  };
  for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const Entry& k = a.t[tensor_of(a, c)];
    const int64_t from = (int64_t)(c - k.first) * kChunk, left = k.n - from;
    const int n = (int)(left < kChunk ? left : kChunk);
    const bool keep = a.chunks - c <= a.kept;
    if (k.is_bf16) {
      Piece<bf16>::load(v, reinterpret_cast<const bf16*>(k.g) + from, n, keep);
      squares(bf16{});
    } else {
      Piece<float>::load(v, reinterpret_cast<const float*>(k.g) + from, n, keep);
      squares(float{});
    }
  }
  const double t = block_sum64(s[0] + s[1]);
  if (threadIdx.x == 0) part[blockIdx.x] = add ? part[blockIdx.x] + t : t;
}

__global__ __launch_bounds__(kThreads) void grad_scale_kernel(Group a, const double* part, int parts, float max_norm, float* result) {
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kParts / kThreads; ++i) {
    const int at = i * kThreads + threadIdx.x;
    if (at < parts) s += part[at];
  }
  u32x4 v[kVecs];
  float f = 0.f;
  auto factor = [&] {                        // while the first chunk travels
    const double norm = sqrt(block_sum64(s));
    f = norm > (double)max_norm ? (float)((double)max_norm / norm) : norm == norm ? 1.f : __builtin_nanf("");
    if (result && blockIdx.x == 0 && threadIdx.x == 0) {
      result[0] = (float)norm;
      result[1] = f;
    }
  };
  // Backwards: what the first launch read last is in a cache still.
  uint32_t i = blockIdx.x;
  if (i >= a.chunks) factor();
  for (; i < a.chunks; i += gridDim.x) {
    const uint32_t c = a.chunks - 1 - i;
    const Entry& k = a.t[tensor_of(a, c)];
    const int64_t from = (int64_t)(c - k.first) * kChunk, left = k.n - from;
    const int n = (int)(left < kChunk ? left : kChunk);
    const bool first = i == blockIdx.x, keep = i < a.kept;
    if (!first && f == 1.f && k.out == k.g) continue;              // times 1 in place: nothing to do
    if (k.is_bf16) Piece<bf16>::load(v, reinterpret_cast<const bf16*>(k.g) + from, n, keep);
    else Piece<float>::load(v, reinterpret_cast<const float*>(k.g) + from, n, keep);
    if (first) factor();
    if (f == 1.f && k.out == k.g) continue;
    if (k.is_bf16) Piece<bf16>::store(v, reinterpret_cast<bf16*>(k.out) + from, n, f);
    else Piece<float>::store(v, reinterpret_cast<float*>(k.out) + from, n, f);
  }
}

}  // namespace

int64_t grad_clip_ws_floats() { return 2 * kParts; }

hipError_t launch_grad_clip(hipStream_t s, const GradTensor* t, int count, float max_norm, float* result, float* ws) {
  if (count < 0 || count > (1 << 20) || (count > 0 && !t) || !(max_norm >= 0.f) || !result || ((uintptr_t)result & 3) || !ws || ((uintptr_t)ws & 7))
    return hipErrorInvalidValue;
  int64_t total = 0, all_chunks = 0;
  for (int i = 0; i < count; ++i) {
    if ((t[i].dtype != kF32 && t[i].dtype != kBF16) || t[i].n < 0 || t[i].n > (1LL << 40) || (t[i].n > 0 && !t[i].g)) return hipErrorInvalidValue;
    if (((uintptr_t)t[i].g | (uintptr_t)t[i].out) & (t[i].dtype == kBF16 ? 1 : 3)) return hipErrorInvalidValue;
    total += t[i].n;
    all_chunks += (t[i].n + kChunk - 1) / kChunk;
    if (total > (1LL << 40)) return hipErrorInvalidValue;
  }
  double* const part = reinterpret_cast<double*>(ws);
  // Two passes over the groups, the second backwards; the first one's blocks leave their sums in `parts` places, which the first group's launch writes
  // all of.
  const int parts = all_chunks < 1 ? 1 : all_chunks < kParts ? (int)all_chunks : kParts;
  auto bytes_of = [](const GradTensor& x) { return x.n * (x.dtype == kBF16 ? 2 : 4); };
  // The group of tensors begin .. end - 1, behind which `behind` bytes of others follow.
  auto gather = [&](Group& a, int begin, int end, bool outputs, int64_t behind) {
    a.count = a.chunks = a.kept = 0;
    for (int i = begin; i < end; ++i) {
      if (t[i].n == 0 || (outputs && !t[i].out)) continue;
      a.t[a.count++] = Entry{t[i].g, t[i].out, t[i].n, a.chunks, t[i].dtype == kBF16};
      a.chunks += (uint32_t)((t[i].n + kChunk - 1) / kChunk);
    }
    for (uint32_t i = a.count; i-- > 0;) {
      const int64_t chunk = kChunk * (a.t[i].is_bf16 ? 2 : 4), all = (a.t[i].n + kChunk - 1) / kChunk, room = behind < kKept ? (kKept - behind) / chunk : 0;
      a.kept += (uint32_t)(all < room ? all : room);
      if (room < all) break;
      behind += all * chunk;
    }
  };
  auto counts = [&](int i, bool outputs) { return t[i].n > 0 && (!outputs || t[i].out); };
  int64_t behind = 0;
  for (int i = 0; i < count; ++i) behind += bytes_of(t[i]);
  bool done = false;
  for (int i = 0; i < count || !done;) {
    int end = i, n = 0;
    for (; end < count && (n < kGroup || !counts(end, false)); ++end) {
      n += counts(end, false);
      behind -= bytes_of(t[end]);
    }
    Group a;
    gather(a, i, end, false, behind);
    i = end;
    if (a.count == 0 && done) continue;
    grad_norm_kernel<<<done && a.chunks < (uint32_t)parts ? (int)a.chunks : parts, kThreads, 0, s>>>(a, part, done);
    done = true;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  behind = 0;
  done = false;
  for (int end = count; end > 0 || !done;) {
    int i = end, n = 0;
    int64_t bytes = 0;
    for (; i > 0 && (n < kGroup || !counts(i - 1, true)); --i) {
      n += counts(i - 1, true);
      bytes += counts(i - 1, true) ? bytes_of(t[i - 1]) : 0;
    }
    Group a;
    gather(a, i, end, true, behind);
    behind += bytes;
    end = i;
    if (a.count == 0 && done) continue;
    const int blocks = a.chunks < 1 ? 1 : a.chunks < kScaleBlocks ? (int)a.chunks : kScaleBlocks;
    grad_scale_kernel<<<blocks, kThreads, 0, s>>>(a, part, parts, max_norm, done ? nullptr : result);
    done = true;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pw
