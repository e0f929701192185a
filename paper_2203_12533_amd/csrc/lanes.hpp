// Reductions over the lanes of a wave by moves between lanes of the vector unit (no LDS): every lane gets the result, in an order that is
// the same for every launch.
#pragma once
#include "common.hpp"

namespace pw {

namespace lanes {
constexpr int kQuad1 = 0xB1, kQuad2 = 0x4E;               // quad_perm [1,0,3,2], [2,3,0,1]
constexpr int kHalfMirror = 0x141, kMirror = 0x140;       // lane i <- lane 7 - i of 8, 15 - i of 16
template <int CTRL> __device__ __forceinline__ uint32_t move(uint32_t v) { return __builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
// f(own row of 16, neighbouring row) in lanes of rows 0 and 1 (2 and 3) alike; f(own 32 lanes, the others) likewise.
template <class F> __device__ __forceinline__ uint32_t rows16(uint32_t v, F&& f) {
  const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return f(p[0], p[1]);
}
template <class F> __device__ __forceinline__ uint32_t rows32(uint32_t v, F&& f) {
  const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return f(p[0], p[1]);
}
// Over N = 1, 2, 4 .. 64 neighbouring lanes; f is associative and commutative.
template <int N, class F> __device__ __forceinline__ uint32_t all(uint32_t v, F&& f) {
  if constexpr (N >= 2) v = f(v, move<kQuad1>(v));
  if constexpr (N >= 4) v = f(v, move<kQuad2>(v));
  if constexpr (N >= 8) v = f(v, move<kHalfMirror>(v));
  if constexpr (N >= 16) v = f(v, move<kMirror>(v));
  if constexpr (N >= 32) v = rows16(v, f);
  if constexpr (N >= 64) v = rows32(v, f);
  return v;
}
}  // namespace lanes

template <int N = 64> __device__ __forceinline__ float lanes_sum(float v) {
  return __uint_as_float(lanes::all<N>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
template <int N = 64> __device__ __forceinline__ float lanes_max(float v) {
  return __uint_as_float(lanes::all<N>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
template <int N = 64> __device__ __forceinline__ uint32_t lanes_max_bits(uint32_t v) {
  return lanes::all<N>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

}  // namespace pw
