// The 2-norm of all gradients together, and the gradients scaled to a largest norm:
//
//   norm = sqrt(sum over tensors and elements g^2),  factor = max_norm / norm where norm > max_norm, else 1;   out = g factor
//
// Squares are formed and added in 64 bits: neither overflows nor vanishes for any fp32 value, and a sum of 10^9 of them keeps 24 bits; it costs two
// operations per element where memory allows for ten.  Two launches for up to kGroup tensors, whose addresses travel with the launch: blocks
// take chunks of tensors in turn and leave a sum each, then every block of the second adds those sums in the same order (4096 or fewer
// bytes, from the cache) and scales its chunks.  Bound by memory: two reads and a write of 4 (2) bytes.
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"

namespace pw {

namespace {

constexpr int kThreads = 256, kGroup = 96, kParts = 1024;
constexpr int64_t kChunk = 8192;             // elements

struct Group {
  const void* g[kGroup];
  void* out[kGroup];
  int64_t n[kGroup];
  uint32_t first[kGroup + 1];                // chunk of the launch that a tensor begins with
  uint8_t bf16_[kGroup];
  int count;
};
static_assert(sizeof(Group) <= 3500, "with the launch");

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));

// A chunk's vectors of one thread: v[i] holds elements (i * kThreads + thread) * E .. of n; zeros behind the end.
template <class T> struct Piece;
template <> struct Piece<float> {
  static constexpr int E = 4, kVecs = kChunk / E / kThreads;
  f32x4u v[kVecs];
  __device__ __forceinline__ void load(const float* g, int n) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int at = (i * kThreads + threadIdx.x) * E;
      if (at + E <= n) {
        v[i] = *reinterpret_cast<const f32x4u*>(g + at);
      } else {
        v[i] = f32x4u{};
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
          if (at + e < n) v[i][e] = g[at + e];
      }
    }
  }
  __device__ __forceinline__ float get(int i, int e) const { return v[i][e]; }
  __device__ __forceinline__ void store(float* o, int n, float f) const {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int at = (i * kThreads + threadIdx.x) * E;
      if (at + E <= n) {
        *reinterpret_cast<f32x4u*>(o + at) = v[i] * f;
      } else {
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
          if (at + e < n) o[at + e] = v[i][e] * f;
      }
    }
  }
};
template <> struct Piece<bf16> {
  static constexpr int E = 8, kVecs = kChunk / E / kThreads;
  u32x4u v[kVecs];
  __device__ __forceinline__ void load(const bf16* g, int n) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int at = (i * kThreads + threadIdx.x) * E;
      if (at + E <= n) {
        v[i] = *reinterpret_cast<const u32x4u*>(g + at);
      } else {
        v[i] = u32x4u{};
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
          if (at + e < n) v[i][e / 2] |= (uint32_t)__builtin_bit_cast(unsigned short, g[at + e]) << (16 * (e & 1));
      }
    }
  }
  __device__ __forceinline__ float get(int i, int e) const { return __uint_as_float(e & 1 ? v[i][e / 2] & 0xffff0000u : v[i][e / 2] << 16); }
  __device__ __forceinline__ void store(bf16* o, int n, float f) const {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int at = (i * kThreads + threadIdx.x) * E;
      if (at + E <= n) {
        u32x4u w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)(get(i, 2 * e) * f), (bf16)(get(i, 2 * e + 1) * f)});
        *reinterpret_cast<u32x4u*>(o + at) = w;
      } else {
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
          if (at + e < n) o[at + e] = (bf16)(get(i, e) * f);
      }
    }
  }
};

// f(tensor, first element, elements) for the chunks of this block.
template <class F> __device__ __forceinline__ void for_chunks(const Group& a, bool backwards, F&& f) {
  const uint32_t total = a.first[a.count];
  for (uint32_t i = blockIdx.x; i < total; i += gridDim.x) {
    const uint32_t c = backwards ? total - 1 - i : i;
    int lo = 0, hi = a.count - 1;            // the last tensor that begins at or before c and has chunks
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.first[mid] <= c) lo = mid;
      else hi = mid - 1;
    }
    const int64_t from = (int64_t)(c - a.first[lo]) * kChunk, left = a.n[lo] - from;
    f(lo, from, (int)(left < kChunk ? left : kChunk));
  }
}

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
  auto squares = [&](auto&& x) {
    typedef typename std::remove_reference<decltype(x)>::type P;
#pragma unroll
    for (int i = 0; i < P::kVecs; ++i)
#pragma unroll
      for (int e = 0; e < P::E; ++e) {
        const double v = x.get(i, e);
        s[e & 1] = __builtin_fma(v, v, s[e & 1]);
      }
  };
  for_chunks(a, false, [&](int k, int64_t from, int n) {
    if (a.bf16_[k]) {
      Piece<bf16> x;
      x.load(reinterpret_cast<const bf16*>(a.g[k]) + from, n);
      squares(x);
    } else {
      Piece<float> x;
      x.load(reinterpret_cast<const float*>(a.g[k]) + from, n);
      squares(x);
    }
  });
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
  const double norm = sqrt(block_sum64(s));
  const float f = norm > (double)max_norm ? (float)((double)max_norm / norm) : norm == norm ? 1.f : __builtin_nanf("");
  if (result && blockIdx.x == 0 && threadIdx.x == 0) {
    result[0] = (float)norm;
    result[1] = f;
  }
  // Backwards: what the first launch read last is the likeliest to be in a cache still.
  for_chunks(a, true, [&](int k, int64_t from, int n) {
    if (!a.out[k] || (f == 1.f && a.out[k] == a.g[k])) return;     // times 1 in place: nothing to do
    if (a.bf16_[k]) {
      Piece<bf16> x;
      x.load(reinterpret_cast<const bf16*>(a.g[k]) + from, n);
      x.store(reinterpret_cast<bf16*>(a.out[k]) + from, n, f);
    } else {
      Piece<float> x;
      x.load(reinterpret_cast<const float*>(a.g[k]) + from, n);
      x.store(reinterpret_cast<float*>(a.out[k]) + from, n, f);
    }
  });
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
      a.count = 0;
      a.first[0] = 0;
      bool out = false;
      for (; i < count && a.count < kGroup; ++i) {
        if (t[i].n == 0 || (pass == 1 && !t[i].out)) continue;
        const int k = a.count++;
        a.g[k] = t[i].g;
        a.out[k] = t[i].out;
        a.n[k] = t[i].n;
        a.bf16_[k] = t[i].dtype == kBF16;
        a.first[k + 1] = a.first[k] + (uint32_t)((t[i].n + kChunk - 1) / kChunk);
        out = true;
      }
      if (!out && done) continue;
      const uint32_t chunks = a.first[a.count];
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
