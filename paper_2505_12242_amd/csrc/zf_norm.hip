// RMS norm with the residual's addition and an 8-bit output, and its
// gradients (formulas in zf_layer.h).
//
// One block per row, the row in registers between its two uses: every input is
// read once and every output written once.  A thread holds V pieces of 8
// consecutive elements, NT * 8 elements apart; 16 lanes hold one group of the
// 8-bit output.  Sums are fp32: per thread in order, then over the wave, then
// over the block's waves.  Rows too wide for the registers are read twice
// (the *_wide kernels).  Bound by HBM.
//
// The gain's gradient sums over rows.  Backward blocks take a contiguous range
// of rows each and keep their columns' sums in registers; the blocks' partial
// sums are added in block order by a second kernel, so the result does not
// depend on timing.
#include "zf_layer.hpp"

namespace zf {
namespace {

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

__device__ __forceinline__ void load_gain(const NormArgs& a, int64_t c, int64_t valid,
                                          float (&g)[8]) {
  if (a.gain_f32) load8(static_cast<const float*>(a.gain) + c, valid, g);
  else load8(static_cast<const uint16_t*>(a.gain) + c, valid, g);
}
__device__ __forceinline__ void load_gain(const NormBwdArgs& a, int64_t c, int64_t valid,
                                          float (&g)[8]) {
  if (a.gain_f32) load8(static_cast<const float*>(a.gain) + c, valid, g);
  else load8(static_cast<const uint16_t*>(a.gain) + c, valid, g);
}

// h of 8 elements: x, or x + residual rounded to the storage type and kept.
template <typename T>
__device__ __forceinline__ void load_h(const NormArgs& a, int64_t row, int64_t c, int64_t valid,
                                       float (&h)[8]) {
  const T* x = static_cast<const T*>(a.x);
  load8(x + row * a.ld_x + c, valid, h);
  if (a.residual != nullptr) {
    float r[8];
    load8(static_cast<const T*>(a.residual) + row * a.ld_residual + c, valid, r);
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = as_stored(x, h[j] + r[j]);
  }
}
template <typename T>
__device__ __forceinline__ void store_h(const NormArgs& a, int64_t row, int64_t c, int64_t valid,
                                        const float (&h)[8]) {
  if (a.h != nullptr) store8(static_cast<T*>(a.h) + row * a.ld_h + c, valid, h);
}

// y of 8 elements written, in its own type and in 8 bits.  Every lane of a
// 16-lane group calls it (the group's largest magnitude is theirs).
template <typename T>
__device__ __forceinline__ void store_y(const NormArgs& a, int64_t row, int64_t c, int64_t valid,
                                        const float (&h)[8], float rstd, const float (&g)[8]) {
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j)
    y[j] = as_stored(static_cast<const T*>(nullptr), (h[j] * rstd) * g[j]);
  if (a.y != nullptr) store8(static_cast<T*>(a.y) + row * a.ld_y + c, valid, y);
  if (a.q.data != nullptr) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, j < valid ? abs_bits(y[j]) : 0u);
    const uint32_t code = fp8_code(max16(m));
    store_bytes8(a.q.data + row * a.q.ld + c, valid, quant8(y, code));
    if ((threadIdx.x & 15) == 0 && valid > 0)
      a.q.scale[row * a.q.ld_scale + c / kFp8Group] = static_cast<uint8_t>(code);
  }
}

template <typename T, int NT, int V>
__global__ __launch_bounds__(NT) void rmsnorm_kernel(NormArgs a) {
  __shared__ float red[2][NT / 64];
  int flip = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float h[V][8];
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      load_h<T>(a, row, c, a.cols - c, h[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      if (a.residual != nullptr || a.h != a.x) store_h<T>(a, row, c, a.cols - c, h[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) ss += h[i][j] * h[i][j];
    }
    const float mean = block_sum<NT>(ss, red[flip]) / static_cast<float>(a.cols);
    flip ^= 1;
    const float rstd = 1.0f / sqrtf(mean + a.eps);
    if (threadIdx.x == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      float g[8];
      load_gain(a, c, a.cols - c, g);
      store_y<T>(a, row, c, a.cols - c, h[i], rstd, g);
    }
  }
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void rmsnorm_wide_kernel(NormArgs a) {
  __shared__ float red[2][NT / 64];
  int flip = 0;
  const int64_t span = (a.cols + 8 * NT - 1) / (8 * NT) * (8 * NT);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float ss = 0.0f, h[8], g[8];
    for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8 * NT) {
      load_h<T>(a, row, c, a.cols - c, h);
#pragma unroll
      for (int j = 0; j < 8; ++j) ss += h[j] * h[j];
    }
    const float mean = block_sum<NT>(ss, red[flip]) / static_cast<float>(a.cols);
    flip ^= 1;
    const float rstd = 1.0f / sqrtf(mean + a.eps);
    if (threadIdx.x == 0) a.rstd[row] = rstd;
    for (int64_t c = threadIdx.x * 8; c < span; c += 8 * NT) {
      // (h may be x's or the residual's own buffer: read before it is written)
      load_h<T>(a, row, c, a.cols - c, h);
      if (a.residual != nullptr || a.h != a.x) store_h<T>(a, row, c, a.cols - c, h);
      load_gain(a, c, a.cols - c, g);
      store_y<T>(a, row, c, a.cols - c, h, rstd, g);
    }
  }
}

// Rows [r0, r1) of backward block b of `blocks`.
__device__ __forceinline__ void block_rows(int64_t rows, int64_t blocks, int64_t b, int64_t& r0,
                                           int64_t& r1) {
  r0 = rows * b / blocks;
  r1 = rows * (b + 1) / blocks;
}

template <typename T, int NT, int V, bool DGAIN>
__global__ __launch_bounds__(NT) void rmsnorm_backward_kernel(NormBwdArgs a) {
  __shared__ float red[2][NT / 64];
  const T* dy = static_cast<const T*>(a.dy);
  const T* h = static_cast<const T*>(a.h);
  const T* dres = static_cast<const T*>(a.dres);
  float dg[V][8], g[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int64_t c = (threadIdx.x + i * NT) * 8;
    load_gain(a, c, a.cols - c, g[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[i][j] = 0.0f;
  }
  int64_t r0, r1;
  block_rows(a.rows, gridDim.x, blockIdx.x, r0, r1);
  int flip = 0;
  for (int64_t row = r0; row < r1; ++row) {
    const float rstd = a.rstd[row];
    float d[V][8], hh[V][8], r[V][8];
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      load8(dy + row * a.ld_dy + c, a.cols - c, d[i]);
      load8(h + row * a.ld_h + c, a.cols - c, hh[i]);
      if (dres != nullptr) load8(dres + row * a.ld_dres + c, a.cols - c, r[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        hh[i][j] *= rstd;
        if (DGAIN) dg[i][j] += d[i][j] * hh[i][j];
        d[i][j] *= g[i][j];
        s += d[i][j] * hh[i][j];
      }
    const float mean = block_sum<NT>(s, red[flip]) / static_cast<float>(a.cols);
    flip ^= 1;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = rstd * (d[i][j] - hh[i][j] * mean);
        if (dres != nullptr) o[j] += r[i][j];
      }
      store8(static_cast<T*>(a.dx) + row * a.ld_dx + c, a.cols - c, o);
    }
  }
  if constexpr (DGAIN) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      store8(a.part + blockIdx.x * a.cols + c, a.cols - c, dg[i]);
    }
  }
}

// Rows too wide for the registers: the gain's partial sums by column (before
// dx, which may be dy's own buffer, is written), then dx with dy and h read twice.
template <typename T>
__global__ __launch_bounds__(256) void rmsnorm_dgain_wide_kernel(NormBwdArgs a) {
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8;
  if (c >= a.cols) return;
  int64_t r0, r1;
  block_rows(a.rows, gridDim.y, blockIdx.y, r0, r1);
  float dg[8] = {}, d[8], h[8];
  for (int64_t row = r0; row < r1; ++row) {
    load8(static_cast<const T*>(a.dy) + row * a.ld_dy + c, a.cols - c, d);
    load8(static_cast<const T*>(a.h) + row * a.ld_h + c, a.cols - c, h);
    const float rstd = a.rstd[row];
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[j] += d[j] * (h[j] * rstd);
  }
  store8(a.part + blockIdx.y * a.cols + c, a.cols - c, dg);
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void rmsnorm_dx_wide_kernel(NormBwdArgs a) {
  __shared__ float red[2][NT / 64];
  int flip = 0;
  float d[8], h[8], g[8], r[8];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
    const T* hp = static_cast<const T*>(a.h) + row * a.ld_h;
    const float rstd = a.rstd[row];
    float s = 0.0f;
    for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8 * NT) {
      load8(dy + c, a.cols - c, d);
      load8(hp + c, a.cols - c, h);
      load_gain(a, c, a.cols - c, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) s += (d[j] * g[j]) * (h[j] * rstd);
    }
    const float mean = block_sum<NT>(s, red[flip]) / static_cast<float>(a.cols);
    flip ^= 1;
    for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8 * NT) {
      load8(dy + c, a.cols - c, d);
      load8(hp + c, a.cols - c, h);
      load_gain(a, c, a.cols - c, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] = rstd * (d[j] * g[j] - (h[j] * rstd) * mean);
      if (a.dres != nullptr) {
        load8(static_cast<const T*>(a.dres) + row * a.ld_dres + c, a.cols - c, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] += r[j];
      }
      store8(static_cast<T*>(a.dx) + row * a.ld_dx + c, a.cols - c, d);
    }
  }
}

// dgain[j] = the sum of column j's `parts` partials, each of 4 waves a
// contiguous share of them in order, then the waves in order.
__global__ __launch_bounds__(256) void dgain_kernel(const float* __restrict__ part, int64_t parts,
                                                    int64_t cols, float* __restrict__ dgain) {
  __shared__ float red[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 64 + lane;
  const int64_t p0 = parts * wave / 4, p1 = parts * (wave + 1) / 4;
  float s = 0.0f;
  if (c < cols)
    for (int64_t p = p0; p < p1; ++p) s += part[p * cols + c];
  red[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < cols) dgain[c] = ((red[0][lane] + red[1][lane]) + red[2][lane]) + red[3][lane];
}

constexpr int64_t kMaxGrid = int64_t(1) << 22;
constexpr int64_t kWideCols = 1024 * 8 * 4;  // the widest row kept in registers

// Blocks of the backward pass (partial sums of the gain's gradient).
int64_t backward_blocks(int64_t rows) { return rows < 512 ? rows : 512; }

template <typename T>
void norm_forward(const NormArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(a.rows < kMaxGrid ? a.rows : kMaxGrid));
#define ZF_NORM(NT, V) \
  hipLaunchKernelGGL((rmsnorm_kernel<T, NT, V>), grid, dim3(NT), 0, s, a)
  if (a.cols <= 512) ZF_NORM(64, 1);
  else if (a.cols <= 2048) ZF_NORM(256, 1);
  else if (a.cols <= 4096) ZF_NORM(256, 2);
  else if (a.cols <= 8192) ZF_NORM(256, 4);
  else if (a.cols <= 16384) ZF_NORM(1024, 2);
  else if (a.cols <= kWideCols) ZF_NORM(1024, 4);
  else hipLaunchKernelGGL((rmsnorm_wide_kernel<T, 1024>), grid, dim3(1024), 0, s, a);
#undef ZF_NORM
}

template <typename T, bool DGAIN>
void norm_backward(const NormBwdArgs& a, hipStream_t s) {
  const int64_t blocks =
      DGAIN ? backward_blocks(a.rows) : (a.rows < kMaxGrid ? a.rows : kMaxGrid);
  const dim3 grid(static_cast<uint32_t>(blocks));
#define ZF_NORM(NT, V) \
  hipLaunchKernelGGL((rmsnorm_backward_kernel<T, NT, V, DGAIN>), grid, dim3(NT), 0, s, a)
  if (a.cols <= 512) ZF_NORM(64, 1);
  else if (a.cols <= 2048) ZF_NORM(256, 1);
  else if (a.cols <= 4096) ZF_NORM(512, 1);
  else if (a.cols <= 8192) ZF_NORM(1024, 1);
  else if (a.cols <= 16384) ZF_NORM(1024, 2);
  else if (a.cols <= kWideCols) ZF_NORM(1024, 4);
  else {
    if (DGAIN)
      hipLaunchKernelGGL((rmsnorm_dgain_wide_kernel<T>),
                         dim3(static_cast<uint32_t>((a.cols + 2047) / 2048),
                              static_cast<uint32_t>(blocks)),
                         dim3(256), 0, s, a);
    hipLaunchKernelGGL((rmsnorm_dx_wide_kernel<T, 1024>),
                       dim3(static_cast<uint32_t>(a.rows < kMaxGrid ? a.rows : kMaxGrid)),
                       dim3(1024), 0, s, a);
  }
#undef ZF_NORM
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs& a, int32_t dtype, hipStream_t s) {
  (void)hipGetLastError();
  if (dtype == ZF_BF16) norm_forward<uint16_t>(a, s);
  else norm_forward<float>(a, s);
  return hipGetLastError();
}

size_t rmsnorm_backward_workspace(int64_t rows, int64_t cols) {
  return static_cast<size_t>(backward_blocks(rows)) * static_cast<size_t>(cols) * sizeof(float);
}

hipError_t launch_rmsnorm_backward(const NormBwdArgs& a, int32_t dtype, hipStream_t s) {
  (void)hipGetLastError();
  if (a.rows > 0) {
    if (dtype == ZF_BF16) {
      if (a.dgain != nullptr) norm_backward<uint16_t, true>(a, s);
      else norm_backward<uint16_t, false>(a, s);
    } else {
      if (a.dgain != nullptr) norm_backward<float, true>(a, s);
      else norm_backward<float, false>(a, s);
    }
  }
  if (a.dgain != nullptr)  // (no rows: no partials, zeros)
    hipLaunchKernelGGL(dgain_kernel, dim3(static_cast<uint32_t>((a.cols + 63) / 64)), dim3(256), 0,
                       s, a.part, backward_blocks(a.rows), a.cols, a.dgain);
  return hipGetLastError();
}

}  // namespace zf
