// The 2-norm of all gradients together, and the gradients scaled to a largest norm:
//
//   norm = sqrt(sum over tensors and elements g^2),  factor = max_norm / norm where norm > max_norm, else 1;   out = g factor
//
// Squares are formed and added in 64 bits: neither overflows nor vanishes for any fp32 value, and a sum of 10^9 of them keeps 24 bits; it costs two
// operations per element where memory allows for ten.  Two launches for up to kGroup tensors, whose addresses travel with the launch: blocks
// take chunks of tensors in turn and leave a sum each, then every block of the second adds those sums in the same order (4096 or fewer
// bytes, from the cache) and scales its chunks.  Bound by memory: two reads and a write of 4 (2) bytes.
#include "common.hpp"
#include "kernels.hpp"

namespace pw {

namespace {

constexpr int kThreads = 256, kGroup = 96, kParts = 1024;
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
  uint32_t count, chunks;
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
  static __device__ __forceinline__ void load(u32x4 (&v)[kVecs], const T* g, int n) {
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
  static __device__ __forceinline__ void store(const u32x4 (&v)[kVecs], T* o, int n, float f) {
#pragma unroll
    for (int i = 0; i < kUsed; ++i) {
      const int at = (i * kThreads + threadIdx.x) * E;
      if (at + E <= n) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(get(v[i], e) * f);
          else w[e] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)(get(v[i], 2 * e) * f), (bf16)(get(v[i], 2 * e + 1) * f)});
        }
        *reinterpret_cast<u32x4u*>(o + at) = w;
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
    if (k.is_bf16) {
      Piece<bf16>::load(v, reinterpret_cast<const bf16*>(k.g) + from, n);
      squares(bf16{});
    } else {
      Piece<float>::load(v, reinterpret_cast<const float*>(k.g) + from, n);
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
  // Backwards: what the first launch read last is the likeliest to be in a cache still.
  uint32_t i = blockIdx.x;
  if (i >= a.chunks) factor();
  for (; i < a.chunks; i += gridDim.x) {
    const uint32_t c = a.chunks - 1 - i;
    const Entry& k = a.t[tensor_of(a, c)];
    const int64_t from = (int64_t)(c - k.first) * kChunk, left = k.n - from;
    const int n = (int)(left < kChunk ? left : kChunk);
    const bool first = i == blockIdx.x;
    if (!first && f == 1.f && k.out == k.g) continue;              // times 1 in place: nothing to do
    if (k.is_bf16) Piece<bf16>::load(v, reinterpret_cast<const bf16*>(k.g) + from, n);
    else Piece<float>::load(v, reinterpret_cast<const float*>(k.g) + from, n);
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
  // Two passes over the groups; the first one's blocks leave their sums in `parts` places, which the first group's launch writes all of.
  const int parts = all_chunks < 1 ? 1 : all_chunks < kParts ? (int)all_chunks : kParts;
  for (int pass = 0; pass < 2; ++pass) {
    bool done = false;
    for (int i = 0; i < count || !done;) {
      Group a;
      a.count = a.chunks = 0;
      for (; i < count && a.count < kGroup; ++i) {
        if (t[i].n == 0 || (pass == 1 && !t[i].out)) continue;
        a.t[a.count++] = Entry{t[i].g, t[i].out, t[i].n, a.chunks, t[i].dtype == kBF16};
        a.chunks += (uint32_t)((t[i].n + kChunk - 1) / kChunk);
      }
      if (a.count == 0 && done) continue;
      const uint32_t chunks = a.chunks;
      if (pass == 0) {
        const int blocks = done && chunks < (uint32_t)parts ? (int)chunks : parts;
        grad_norm_kernel<<<blocks, kThreads, 0, s>>>(a, part, done);
      } else {
        const int blocks = chunks < 1 ? 1 : chunks < 2 * kParts ? (int)chunks : 2 * kParts;
        grad_scale_kernel<<<blocks, kThreads, 0, s>>>(a, part, parts, max_norm, done ? nullptr : result);
      }
      done = true;
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace pw
