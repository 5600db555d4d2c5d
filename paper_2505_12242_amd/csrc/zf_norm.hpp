// Shared by the kernels of the norms: sums over a block, rows in registers, and
// the joining of columns' partial sums.
#pragma once

#include "zf_layer.hpp"

namespace zf {

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// The block's sum of x, in every thread.  `red` may be used again after the
// next block_sum or barrier (two buffers, alternated by the caller).
template <int NT>
__device__ __forceinline__ float block_sum(float x, float (&red)[NT / 64]) {
  x = wave_sum(x);
  if constexpr (NT == 64) return x;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) s += red[w];
  return s;
}

// Eight elements of a vector of either type.
__device__ __forceinline__ void load_vector(const void* p, int32_t f32, int64_t cols, int64_t c,
                                            float (&g)[8]) {
  if (f32) {
    Vec8<float> v;
    v.load(static_cast<const float*>(p) + c, cols - c);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = v[j];
  } else {
    Vec8<uint16_t> v;
    v.load(static_cast<const uint16_t*>(p) + c, cols - c);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = v[j];
  }
}

template <typename Args>
__device__ __forceinline__ void load_gain(const Args& a, int64_t c, float (&g)[8]) {
  load_vector(a.gain, a.gain_f32, a.cols, c, g);
}

// x + residual, rounded to the storage type.
template <typename T>
__device__ __forceinline__ void add(Vec8<T>& x, const Vec8<T>& r) {
  float s[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) s[j] = x[j] + r[j];
  x.set(s);
}

// Rows [r0, r1) of backward block b of `blocks`.
__device__ __forceinline__ void block_rows(int64_t rows, int64_t blocks, int64_t b, int64_t& r0,
                                           int64_t& r1) {
  r0 = rows * b / blocks;
  r1 = rows * (b + 1) / blocks;
}

constexpr int64_t kMaxGrid = int64_t(1) << 21;  // blocks; a dispatch holds fewer than 2^32 threads
constexpr int64_t kWideCols = 1024 * 8 * 2;  // the widest row kept in registers

// f(threads, pieces a thread) with the fewest threads that hold a row.
template <typename F>
auto with_shape(int64_t cols, F&& f) {
#define ZF_SHAPE(NT, V) \
  if (cols <= NT * V * 8) return f(std::integral_constant<int, NT>(), std::integral_constant<int, V>())
  ZF_SHAPE(64, 1);
  ZF_SHAPE(128, 1);
  ZF_SHAPE(256, 1);
  ZF_SHAPE(384, 1);
  ZF_SHAPE(512, 1);
  ZF_SHAPE(640, 1);
  ZF_SHAPE(768, 1);
  ZF_SHAPE(1024, 1);
  ZF_SHAPE(768, 2);
#undef ZF_SHAPE
  return f(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
}
// out0[j] (and out1[j], of the `parts` x cols partials behind the first; may be
// nullptr) = the sum of column j's `parts` partials, in a fixed order.
void launch_join_columns(const float* part, int64_t parts, int64_t cols, float* out0, float* out1,
                         hipStream_t s);

}  // namespace zf
