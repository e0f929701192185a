// Operand tiles of the 8- and 4-bit products: direct loads from global memory into LDS, rows of 128 bytes without bank conflicts.
#pragma once
#include "common.hpp"

namespace pw {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

typedef __attribute__((address_space(3))) void* lds_ptr;
constexpr int kRowBytes = 128;            // of an operand in a k tile
constexpr int64_t kMaxLd = 1 << 23;       // rows of a tile are within 32 bits of byte offset

static __device__ __attribute__((aligned(16))) const uint32_t kZeros[4] = {0, 0, 0, 0};

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

// One operand of a group's tile: R rows of 128 bytes, fetched by G waves in pieces of 1 KiB (8 rows); chunk c (16 bytes) of row
// r lies at position c ^ ((r >> 1) & 7) of the row, so that the 16 rows of a fragment read hit all banks.
// HALVES: the first half of a wave's pieces are the first 64 of each 128 rows.
template <int R, int G, bool HALVES>
struct Operand {
  static constexpr int kPer = R / 8 / G;
  static_assert(!HALVES || (G == 8 && kPer == 4), "two times 128 rows");
  __device__ __forceinline__ static int piece(int gw, int j) {
    return HALVES ? (gw >> 2) * 16 + (j >> 1) * 8 + (gw & 3) * 2 + (j & 1) : gw * kPer + j;
  }
  const uint8_t* base;
  uint32_t off[kPer];
  __device__ __forceinline__ static int k_of(int instr, int lane) { return ((lane & 7) ^ (((instr * 8 + (lane >> 3)) >> 1) & 7)) * 16; }
  __device__ __forceinline__ void init(const uint8_t* p, int64_t ld, int64_t row0, int64_t rows, int64_t first, int gw, int lane) {
    base = p + row0 * ld + first * kRowBytes;
    const int last = (int)(rows - row0 < R ? rows - row0 : R) - 1;     // rows past the end are fetched from the last one
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int instr = piece(gw, j), r = instr * 8 + (lane >> 3);
      off[j] = (uint32_t)((r < last ? r : last) * (int)ld + k_of(instr, lane));
    }
  }
  __device__ __forceinline__ void issue_one(int j, uint32_t lds_off, int gw) const { dma16_s(base, off[j], lds_off + piece(gw, j) * 1024); }
  // The next k tile, of which `left` bytes exist (a multiple of 16; whole, partial or none): the rest comes from zeros.
  __device__ __forceinline__ void issue(int64_t left, uint32_t lds_off, int gw, int lane, int from = 0, int to = kPer) const {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (j < from || j >= to) continue;
      const uint8_t* const g = base + off[j];
      dma16(k_of(piece(gw, j), lane) < left ? g : reinterpret_cast<const uint8_t*>(kZeros), lds_off + piece(gw, j) * 1024);
    }
  }
};

}  // namespace pw
