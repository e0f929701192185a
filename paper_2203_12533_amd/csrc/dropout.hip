// Dropout on rows of a branch, with the mask computed from a counter wherever it is needed and stored nowhere.
//
//   forward   y[r, c] = res[r, c] + keep(r, c) (x[r, c] + bias[c]) / (1 - p)
//   backward  dx[r, c] = keep(r, c) dy[r, c] / (1 - p),   dbias[c] = sum_r dx[r, c] (of the unrounded values)
//
// keep(r, c) compares 16 bits of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers, as easy as 1, 2, 3;
// SC 2011) with p in units of 2^-16: key = seed, counter = (c / 8, r, site, step).  Its four words are the eight columns of
// a group, low half first, so a row begins a counter of its own and the mask depends on neither strides nor launch shape.
// p is taken to the nearest 2^-16 and 1 / (1 - p) is of that value: the expectation is exact.  What is dropped is selected
// away, not multiplied: a NaN there leaves no trace.
//
// A thread owns one group of columns and walks down rows, so the bias stays in registers and the bias gradient is summed
// there; threads of a block that share a group meet in LDS in thread order, blocks in a second launch in block order: the
// same bits on every run.
//
// Bound by memory: 8192 x 2048 bf16 into an fp32 residual takes 33 to 34 us forward (168 MB, 5.0 TB/s; a copy reaches 5.15) and 20 to
// 22 backward (101 MB), with 4 to 5 more for the second launch of the bias gradient.  The counter's ten rounds of two products keep the
// vector units busy for a third of that, under the loads of two rows at a time.
#include "common.hpp"
#include "kernels.hpp"

namespace pw {

namespace {

constexpr int kThreads = 256;
constexpr int kOneThreads = 1024;    // of a launch whose blocks take all rows of their columns
constexpr int kGroup = 8;            // columns of one counter

struct Philox { uint32_t w[4]; };
__device__ __forceinline__ Philox philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
    const uint32_t h0 = (uint32_t)(p0 >> 32), h1 = (uint32_t)(p1 >> 32);
    c0 = h1 ^ c1 ^ k0;
    c1 = (uint32_t)p1;
    c2 = h0 ^ c3 ^ k1;
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}

struct Mask {
  uint32_t k0, k1, site, step, threshold;   // kept where the 16 bits are at least the threshold (0 .. 65536)
  // 65536 / (65536 - threshold) in two parts, so that fp32 values are rounded once by it; 0 where everything is dropped.  The
  // second is positive whatever the first: an infinity stays one.
  float scale, rest;
  const uint32_t* step_dev;
};
__device__ __forceinline__ float scaled(const Mask& m, float v) { return __builtin_fmaf(v, m.scale, v * m.rest); }
// Bit j: column j of the group is kept.
__device__ __forceinline__ uint32_t keep_bits(const Mask& m, uint32_t step, uint32_t group, uint32_t row) {
  const Philox r = philox(group, row, m.site, step, m.k0, m.k1);
  uint32_t bits = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    bits |= (uint32_t)((r.w[j] & 0xffffu) >= m.threshold) << (2 * j);
    bits |= (uint32_t)((r.w[j] >> 16) >= m.threshold) << (2 * j + 1);
  }
  return bits;
}

// Eight consecutive elements; rows may start at any element.
template <class T> struct Vec8;
template <> struct Vec8<float> { typedef float type __attribute__((ext_vector_type(8), aligned(4))); };
template <> struct Vec8<bf16> { typedef __bf16 type __attribute__((ext_vector_type(8), aligned(2))); };
template <class T> __device__ __forceinline__ void load8(const T* p, int n, float* v) {
  if (n >= kGroup) {
    const typename Vec8<T>::type u = *reinterpret_cast<const typename Vec8<T>::type*>(p);
#pragma unroll
    for (int j = 0; j < kGroup; ++j) v[j] = (float)u[j];
  } else {
#pragma unroll
    for (int j = 0; j < kGroup; ++j) v[j] = j < n ? to_f32(p[j]) : 0.f;
  }
}
template <class T> __device__ __forceinline__ void store8(T* p, int n, const float* v) {
  if (n >= kGroup) {
    typename Vec8<T>::type u;
#pragma unroll
    for (int j = 0; j < kGroup; ++j) u[j] = from_f32<T>(v[j]);
    *reinterpret_cast<typename Vec8<T>::type*>(p) = u;
  } else {
#pragma unroll
    for (int j = 0; j < kGroup; ++j)
      if (j < n) p[j] = from_f32<T>(v[j]);
  }
}

// Blocks of 2^log_tx groups of columns by threads >> log_tx rows at a time.
struct Shape {
  int log_tx, col_blocks, row_blocks;
  int64_t rows_per;                   // rows of a block
};
Shape shape_of(int64_t rows, int64_t cols, int threads, int64_t most_blocks) {
  const int64_t groups = (cols + kGroup - 1) / kGroup;
  Shape s{};
  while (s.log_tx < 6 && (1 << s.log_tx) < groups) ++s.log_tx;
  const int64_t ty = threads >> s.log_tx;
  const int64_t cb = (groups + (1 << s.log_tx) - 1) >> s.log_tx;
  int64_t rb = (rows + ty - 1) / ty;
  const int64_t most = most_blocks / cb < 1 ? 1 : most_blocks / cb;
  if (rb > most) rb = most;
  if (rb < 1) rb = 1;
  const int64_t per = (rows + rb - 1) / rb;
  s.rows_per = (per + ty - 1) / ty * ty;
  s.row_blocks = (int)((rows + s.rows_per - 1) / s.rows_per);
  if (s.row_blocks < 1) s.row_blocks = 1;
  s.col_blocks = (int)cb;
  return s;
}

template <class T, class TO, bool RES>
__global__ __launch_bounds__(kThreads) void dropout_fwd_kernel(const T* x, const float* __restrict__ bias, const float* res, TO* y,
                                                               int64_t rows, int64_t cols, int64_t ldx, int64_t ldy, int log_tx,
                                                               int64_t rows_per, Mask m) {
  const int tx = 1 << log_tx;
  const int64_t g = (int64_t)blockIdx.x * tx + (threadIdx.x & (tx - 1)), c = g * kGroup;
  if (c >= cols) return;
  const int n = (int)(cols - c < kGroup ? cols - c : kGroup), ty = kThreads >> log_tx;
  const uint32_t step = m.step + (m.step_dev ? *m.step_dev : 0u);
  float b[kGroup] = {};
  if (bias) load8(bias + c, n, b);
  const int64_t r0 = (int64_t)blockIdx.y * rows_per, r1 = r0 + rows_per < rows ? r0 + rows_per : rows;
  auto row = [&](int64_t r, float* v, const float* e) {
    const uint32_t bits = keep_bits(m, step, (uint32_t)g, (uint32_t)r);
#pragma unroll
    for (int j = 0; j < kGroup; ++j) {
      const float k = (bits >> j) & 1u ? scaled(m, v[j] + b[j]) : 0.f;
      v[j] = RES ? e[j] + k : k;
    }
    store8(y + r * ldy + c, n, v);
  };
  int64_t r = r0 + (threadIdx.x >> log_tx);
  for (; r + ty < r1; r += 2 * ty) {            // both rows are read before either is written
    float v[kGroup], e[kGroup], v2[kGroup], e2[kGroup];
    load8(x + r * ldx + c, n, v);
    load8(x + (r + ty) * ldx + c, n, v2);
    if (RES) {
      load8(res + r * ldy + c, n, e);
      load8(res + (r + ty) * ldy + c, n, e2);
    }
    row(r, v, e);
    row(r + ty, v2, e2);
  }
  if (r < r1) {
    float v[kGroup], e[kGroup];
    load8(x + r * ldx + c, n, v);
    if (RES) load8(res + r * ldy + c, n, e);
    row(r, v, e);
  }
}

// sums: null, or [row block][cols] - or, of a single row block, the bias gradient itself.
template <class T, class TO, int NT, bool SUMS>
__global__ __launch_bounds__(NT) void dropout_bwd_kernel(const TO* dy, T* dx, float* __restrict__ sums, int64_t rows, int64_t cols,
                                                         int64_t ldx, int64_t ldy, int log_tx, int64_t rows_per, int add, Mask m) {
  __shared__ __attribute__((aligned(16))) float part[SUMS ? NT : 1][kGroup];
  const int tx = 1 << log_tx, ty = NT >> log_tx;
  const int64_t g = (int64_t)blockIdx.x * tx + (threadIdx.x & (tx - 1)), c = g * kGroup;
  const int n = (int)(cols - c < kGroup ? cols - c : kGroup);
  float sum[kGroup] = {};
  if (c < cols) {
    const uint32_t step = m.step + (m.step_dev ? *m.step_dev : 0u);
    const int64_t r0 = (int64_t)blockIdx.y * rows_per, r1 = r0 + rows_per < rows ? r0 + rows_per : rows;
    auto row = [&](int64_t r, float* v) {
      const uint32_t bits = keep_bits(m, step, (uint32_t)g, (uint32_t)r);
#pragma unroll
      for (int j = 0; j < kGroup; ++j) {
        v[j] = (bits >> j) & 1u ? scaled(m, v[j]) : 0.f;
        if (SUMS) sum[j] += v[j];
      }
      store8(dx + r * ldx + c, n, v);
    };
    int64_t r = r0 + (threadIdx.x >> log_tx);
    for (; r + ty < r1; r += 2 * ty) {          // both rows are read before either is written
      float v[kGroup], u[kGroup];
      load8(dy + r * ldy + c, n, v);
      load8(dy + (r + ty) * ldy + c, n, u);
      row(r, v);
      row(r + ty, u);
    }
    if (r < r1) {
      float v[kGroup];
      load8(dy + r * ldy + c, n, v);
      row(r, v);
    }
  }
  if constexpr (SUMS) {
#pragma unroll
    for (int j = 0; j < kGroup; ++j) part[threadIdx.x][j] = sum[j];
    __syncthreads();
    for (int i = threadIdx.x; i < tx * kGroup; i += NT) {
      const int64_t col = (int64_t)blockIdx.x * tx * kGroup + i;
      if (col < cols) {
        float t = part[i / kGroup][i % kGroup];
        for (int k = 1; k < ty; ++k) t += part[k * tx + i / kGroup][i % kGroup];
        float* const o = sums + (int64_t)blockIdx.y * cols + col;
        *o = add ? *o + t : t;
      }
    }
  }
}

constexpr int64_t kFwdBlocks = 8192, kBwdBlocks = 4096, kMostParts = 256;
// With column sums.  Up to kOneBlock rows a thread of the larger block they are those of one row block, and no second launch is
// needed: 37 x 1003 fp32 5.0 us instead of 7.4, 64 x 2048 5.8 instead of 7.6.  (The larger blocks for all sizes: 8192 x 2048 29 us, 24.)
constexpr int64_t kOneBlock = 8;
Shape sum_shape(int64_t rows, int64_t cols) {
  const Shape s = shape_of(rows, cols, kOneThreads, 1);
  return rows > kOneBlock * (kOneThreads >> s.log_tx) ? shape_of(rows, cols, kThreads, kMostParts * s.col_blocks) : s;
}

bool mask_of(const DropoutArgs& a, Mask& m) {
  if (!(a.p >= 0.f && a.p <= 1.f)) return false;
  m.threshold = (uint32_t)(int)rintf(a.p * 65536.f);
  m.scale = m.rest = 0.f;
  if (m.threshold < 65536) {
    const double whole = 65536.0 / (65536 - (int)m.threshold);
    m.scale = (float)whole;
    if (m.scale > whole) m.scale = nextafterf(m.scale, 0.f);
    m.rest = (float)(whole - m.scale);
    if (m.rest < 0x1p-126f) m.rest = 0x1p-126f;
  }
  m.k0 = (uint32_t)a.seed;
  m.k1 = (uint32_t)(a.seed >> 32);
  m.site = a.site;
  m.step = a.step;
  m.step_dev = a.step_dev;
  return true;
}
bool args_ok(const DropoutArgs& a) {
  if ((a.dtype != kF32 && a.dtype != kBF16) || (a.out_dtype != kF32 && a.out_dtype != kBF16)) return false;
  if (a.dtype == kF32 && a.out_dtype == kBF16) return false;
  if (a.rows < 0 || a.cols < 0 || a.rows > (1LL << 31) || a.cols > (1LL << 24)) return false;
  if (a.ldx < a.cols || a.ldy < a.cols || a.ldx > (1LL << 31) || a.ldy > (1LL << 31)) return false;
  return ((uintptr_t)a.step_dev & 3) == 0;
}
bool aligned_to(const void* p, int dtype) { return ((uintptr_t)p & (dtype == kBF16 ? 1 : 3)) == 0; }

}  // namespace

int64_t dropout_bwd_ws_floats(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0 || rows > (1LL << 31) || cols > (1LL << 24)) return -1;
  if (rows == 0 || cols == 0) return 0;
  const int64_t parts = sum_shape(rows, cols).row_blocks;
  return parts == 1 ? 0 : parts * cols;
}

hipError_t launch_dropout_fwd(hipStream_t s, const DropoutArgs& a, const void* x, const float* bias, const float* res, void* y) {
  Mask m;
  if (!args_ok(a) || !mask_of(a, m) || !x || !y || (res && a.out_dtype != kF32)) return hipErrorInvalidValue;
  if (!aligned_to(x, a.dtype) || !aligned_to(y, a.out_dtype) || !aligned_to(bias, kF32) || !aligned_to(res, kF32)) return hipErrorInvalidValue;
  if (a.rows == 0 || a.cols == 0) return hipSuccess;
  const Shape h = shape_of(a.rows, a.cols, kThreads, kFwdBlocks);
  const dim3 grid((unsigned)h.col_blocks, (unsigned)h.row_blocks);
  auto go = [&](auto t, auto to) {
    using T = decltype(t);
    using TO = decltype(to);
    if constexpr (sizeof(TO) == 4) {
      if (res) {
        dropout_fwd_kernel<T, TO, true><<<grid, kThreads, 0, s>>>((const T*)x, bias, res, (TO*)y, a.rows, a.cols, a.ldx, a.ldy, h.log_tx, h.rows_per, m);
        return;
      }
    }
    dropout_fwd_kernel<T, TO, false><<<grid, kThreads, 0, s>>>((const T*)x, bias, res, (TO*)y, a.rows, a.cols, a.ldx, a.ldy, h.log_tx, h.rows_per, m);
  };
  if (a.dtype == kF32) go(float{}, float{});
  else if (a.out_dtype == kF32) go(bf16{}, float{});
  else go(bf16{}, bf16{});
  return hipGetLastError();
}

hipError_t launch_dropout_bwd(hipStream_t s, const DropoutArgs& a, const void* dy, void* dx, float* dbias, float* ws, int accumulate) {
  Mask m;
  if (!args_ok(a) || !mask_of(a, m) || !dy || !dx) return hipErrorInvalidValue;
  if (!aligned_to(dy, a.out_dtype) || !aligned_to(dx, a.dtype) || !aligned_to(dbias, kF32) || !aligned_to(ws, kF32)) return hipErrorInvalidValue;
  if (a.cols == 0) return hipSuccess;
  if (a.rows == 0) return dbias ? launch_reduce_parts(s, dbias, dbias, 0, a.cols, a.cols, accumulate) : hipSuccess;
  const Shape h = dbias ? sum_shape(a.rows, a.cols) : shape_of(a.rows, a.cols, kThreads, kBwdBlocks);
  const bool one = dbias && h.row_blocks == 1;
  if (dbias && !one && !ws) return hipErrorInvalidValue;
  const dim3 grid((unsigned)h.col_blocks, (unsigned)h.row_blocks);
  auto go = [&](auto t, auto to) {
    using T = decltype(t);
    using TO = decltype(to);
    auto with = [&](auto kernel, int threads, float* sums, int add) {
      kernel<<<grid, threads, 0, s>>>((const TO*)dy, (T*)dx, sums, a.rows, a.cols, a.ldx, a.ldy, h.log_tx, h.rows_per, add, m);
    };
    if (!dbias) with(dropout_bwd_kernel<T, TO, kThreads, false>, kThreads, nullptr, 0);
    else if (one) with(dropout_bwd_kernel<T, TO, kOneThreads, true>, kOneThreads, dbias, accumulate);
    else with(dropout_bwd_kernel<T, TO, kThreads, true>, kThreads, ws, 0);
  };
  if (a.dtype == kF32) go(float{}, float{});
  else if (a.out_dtype == kF32) go(bf16{}, float{});
  else go(bf16{}, bf16{});
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || !dbias || one ? e : launch_reduce_parts(s, ws, dbias, h.row_blocks, a.cols, a.cols, accumulate);
}

}  // namespace pw
