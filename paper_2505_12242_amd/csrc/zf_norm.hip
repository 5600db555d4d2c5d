// RMS norm with the residual's addition and an 8-bit output, and its
// gradients (formulas in zf_layer.h).
//
// One block per row, the row in registers between its two uses: every input is
// read once and every output written once.  A thread holds V pieces of 8
// consecutive elements, NT * 8 elements apart, NT the fewest threads that hold
// the row; 16 lanes hold one group of the 8-bit output.  Sums are fp32: per
// thread in order, then over the wave, then over the block's waves.  Rows too
// wide for the registers are read twice (the *_wide kernels).
//
// Bound by HBM.  8192 x 4096 bf16 with residual: forward 46 us (5.8 TB/s) with
// one output, 50 us (6.0 TB/s) with both, backward 53 us (5.1 TB/s) and 5 us for
// the gain's join; one row of 4096, 3.6 us, is latency.  Blocks of fewest
// threads against those of powers of two, two pieces a thread: 8192 x 11008
// forward 121 us, not 147, 8192 x 1000 15, not 19; 8192 x 5120 63, not 59.
//
// The gain's gradient sums over rows.  Backward blocks take a contiguous range
// of rows each and keep their columns' sums in registers; the blocks' partial
// sums are added in block order by a second kernel, so the result does not
// depend on timing.
#include <algorithm>

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

template <typename Args>
__device__ __forceinline__ void load_gain(const Args& a, int64_t c, float (&g)[8]) {
  if (a.gain_f32) {
    Vec8<float> v;
    v.load(static_cast<const float*>(a.gain) + c, a.cols - c);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = v[j];
  } else {
    Vec8<uint16_t> v;
    v.load(static_cast<const uint16_t*>(a.gain) + c, a.cols - c);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = v[j];
  }
}

// x + residual, rounded to the storage type.
template <typename T>
__device__ __forceinline__ void add(Vec8<T>& x, const Vec8<T>& r) {
  float s[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) s[j] = x[j] + r[j];
  x.set(s);
}

// y of 8 elements written, in its own type and in 8 bits.  Every lane of a
// 16-lane group calls it (the group's largest magnitude is theirs); elements
// past the row's end are zeros.
template <typename T>
__device__ __forceinline__ void store_y(const NormArgs& a, int64_t row, int64_t c,
                                        const Vec8<T>& h, float rstd) {
  const int64_t valid = a.cols - c;
  float g[8];
  load_gain(a, c, g);
#pragma unroll
  for (int j = 0; j < 8; ++j) g[j] = j < valid ? (h[j] * rstd) * g[j] : 0.0f;
  Vec8<T> y;
  y.set(g);
  if (a.y != nullptr) y.template store<true>(static_cast<T*>(a.y) + row * a.ld_y + c, valid);
  if (a.q.data != nullptr) {
    const uint32_t code = fp8_code(max16(abs_max(y)));
    store_bytes8(a.q.data + row * a.q.ld + c, valid, quant8(y, code));
    if ((threadIdx.x & 15) == 0 && valid > 0)
      a.q.scale[row * a.q.ld_scale + c / kFp8Group] = static_cast<uint8_t>(code);
  }
}

// The mean of `cols` squares; a row without elements counts as one of zeros.
__device__ __forceinline__ float mean_square(float sum, int64_t cols) {
  return sum / static_cast<float>(cols > 0 ? cols : 1);
}

// RES: a residual is added (and h written); without one h may still be wanted.
// (8 waves to a SIMD, which the scalar registers would else leave at 7: 8192 x 5120
// 64 us, not 73.)
template <typename T, int NT, int V, bool RES>
__global__ __launch_bounds__(NT, V == 1 ? 8 : 1) void rmsnorm_kernel(NormArgs a) {
  __shared__ float red[2][NT / 64];
  int flip = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    Vec8<T> h[V], r[RES ? V : 1];
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      h[i].template fetch<true>(static_cast<const T*>(a.x) + row * a.ld_x + c, a.cols - c);
      if constexpr (RES)
        r[i].template fetch<true>(static_cast<const T*>(a.residual) + row * a.ld_residual + c,
                                  a.cols - c);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      h[i].settle(a.cols - c);
      if constexpr (RES) {
        r[i].settle(a.cols - c);
        add(h[i], r[i]);
      }
      if (RES || (a.h != nullptr && a.h != a.x))
        h[i].template store<true>(static_cast<T*>(a.h) + row * a.ld_h + c, a.cols - c);
#pragma unroll
      for (int j = 0; j < 8; ++j) ss += h[i][j] * h[i][j];
    }
    const float mean = mean_square(block_sum<NT>(ss, red[flip]), a.cols);
    flip ^= 1;
    const float rstd = 1.0f / sqrtf(mean + a.eps);
    if (threadIdx.x == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int i = 0; i < V; ++i) store_y(a, row, (threadIdx.x + i * NT) * 8, h[i], rstd);
  }
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void rmsnorm_wide_kernel(NormArgs a) {
  __shared__ float red[2][NT / 64];
  int flip = 0;
  const int64_t span = (a.cols + 8 * NT - 1) / (8 * NT) * (8 * NT);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    Vec8<T> h, r;
    const auto load_h = [&](int64_t c) {
      h.load(static_cast<const T*>(a.x) + row * a.ld_x + c, a.cols - c);
      if (a.residual != nullptr) {
        r.load(static_cast<const T*>(a.residual) + row * a.ld_residual + c, a.cols - c);
        add(h, r);
      }
    };
    float ss = 0.0f;
    for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8 * NT) {
      load_h(c);
#pragma unroll
      for (int j = 0; j < 8; ++j) ss += h[j] * h[j];
    }
    const float mean = mean_square(block_sum<NT>(ss, red[flip]), a.cols);
    flip ^= 1;
    const float rstd = 1.0f / sqrtf(mean + a.eps);
    if (threadIdx.x == 0) a.rstd[row] = rstd;
    for (int64_t c = threadIdx.x * 8; c < span; c += 8 * NT) {
      load_h(c);  // (before h, which may be x's or the residual's own buffer, is written)
      if (a.residual != nullptr || (a.h != nullptr && a.h != a.x))
        h.store(static_cast<T*>(a.h) + row * a.ld_h + c, a.cols - c);
      store_y(a, row, c, h, rstd);
    }
  }
}

// Rows [r0, r1) of backward block b of `blocks`.
__device__ __forceinline__ void block_rows(int64_t rows, int64_t blocks, int64_t b, int64_t& r0,
                                           int64_t& r1) {
  r0 = rows * b / blocks;
  r1 = rows * (b + 1) / blocks;
}

// The next row is loaded while the present one is reduced, where the registers
// hold both: one piece of each a thread.  (Two pieces spilled: 8192 x 11008 bf16
// 226 us, 153 without the early load.)
template <typename T, int NT, int V, bool DRES, bool DGAIN>
__global__ __launch_bounds__(NT) void rmsnorm_backward_kernel(NormBwdArgs a) {
  __shared__ float red[2][NT / 64];
  float dg[V][8], g[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    load_gain(a, (threadIdx.x + i * NT) * 8, g[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[i][j] = 0.0f;
  }
  int64_t r0, r1;
  block_rows(a.rows, gridDim.x, blockIdx.x, r0, r1);
  struct Row {
    Vec8<T> dy[V], h[V], dres[DRES ? V : 1];
    float rstd;
  };
  const auto load_row = [&](Row& w, int64_t row) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8, valid = a.cols - c;
      w.dy[i].fetch(static_cast<const T*>(a.dy) + row * a.ld_dy + c, valid);
      w.h[i].fetch(static_cast<const T*>(a.h) + row * a.ld_h + c, valid);
      if constexpr (DRES)
        w.dres[i].fetch(static_cast<const T*>(a.dres) + row * a.ld_dres + c, valid);
    }
    w.rstd = a.rstd[row];
  };
  Row next;
  if (V == 1 && r0 < r1) load_row(next, r0);
  int flip = 0;
  for (int64_t row = r0; row < r1; ++row) {
    if (V > 1) load_row(next, row);
    Row w = next;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t valid = a.cols - (threadIdx.x + i * NT) * 8;
      w.dy[i].settle(valid);
      w.h[i].settle(valid);
      if constexpr (DRES) w.dres[i].settle(valid);
    }
    if (V == 1 && row + 1 < r1) load_row(next, row + 1);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float hh = w.h[i][j] * w.rstd;
        if (DGAIN) dg[i][j] += w.dy[i][j] * hh;
        s += (w.dy[i][j] * g[i][j]) * hh;
      }
    const float mean = block_sum<NT>(s, red[flip]) / static_cast<float>(a.cols);
    flip ^= 1;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = w.rstd * (w.dy[i][j] * g[i][j] - (w.h[i][j] * w.rstd) * mean);
        if constexpr (DRES) o[j] += w.dres[i][j];
      }
      Vec8<T> out;
      out.set(o);
      out.template store<true>(static_cast<T*>(a.dx) + row * a.ld_dx + c, a.cols - c);
    }
  }
  if constexpr (DGAIN) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      Vec8<float> out;
      out.set(dg[i]);
      out.store(a.part + blockIdx.x * a.cols + c, a.cols - c);
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
  float dg[8] = {};
  for (int64_t row = r0; row < r1; ++row) {
    Vec8<T> d, h;
    d.load(static_cast<const T*>(a.dy) + row * a.ld_dy + c, a.cols - c);
    h.load(static_cast<const T*>(a.h) + row * a.ld_h + c, a.cols - c);
    const float rstd = a.rstd[row];
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[j] += d[j] * (h[j] * rstd);
  }
  Vec8<float> out;
  out.set(dg);
  out.store(a.part + blockIdx.y * a.cols + c, a.cols - c);
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void rmsnorm_dx_wide_kernel(NormBwdArgs a) {
  __shared__ float red[2][NT / 64];
  int flip = 0;
  Vec8<T> d, h, r;
  float g[8];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
    const T* hp = static_cast<const T*>(a.h) + row * a.ld_h;
    const float rstd = a.rstd[row];
    float s = 0.0f;
    for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8 * NT) {
      d.load(dy + c, a.cols - c);
      h.load(hp + c, a.cols - c);
      load_gain(a, c, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) s += (d[j] * g[j]) * (h[j] * rstd);
    }
    const float mean = block_sum<NT>(s, red[flip]) / static_cast<float>(a.cols);
    flip ^= 1;
    for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8 * NT) {
      d.load(dy + c, a.cols - c);
      h.load(hp + c, a.cols - c);
      load_gain(a, c, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = rstd * (d[j] * g[j] - (h[j] * rstd) * mean);
      if (a.dres != nullptr) {
        r.load(static_cast<const T*>(a.dres) + row * a.ld_dres + c, a.cols - c);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] += r[j];
      }
      d.set(g);
      d.store(static_cast<T*>(a.dx) + row * a.ld_dx + c, a.cols - c);
    }
  }
}

// dgain[j] = the sum of column j's `parts` partials: each of the block's shares a
// contiguous range of them in order, eight loads in flight, then the shares in
// order.  Columns per block: 32 are one line of a partial sum's row; 64 leave a
// join of 384 columns to 6 blocks (8192 x 384: 19 us against 15 with the sums).
constexpr int kJoinCols = 32, kJoinShares = 1024 / kJoinCols;
__global__ __launch_bounds__(1024) void dgain_kernel(const float* __restrict__ part,
                                                     int64_t parts, int64_t cols,
                                                     float* __restrict__ dgain) {
  __shared__ float red[kJoinShares][kJoinCols];
  const int lane = threadIdx.x % kJoinCols, share = threadIdx.x / kJoinCols;
  const int64_t p1 = parts * (share + 1) / kJoinShares;
  for (int64_t c0 = static_cast<int64_t>(blockIdx.x) * kJoinCols; c0 < cols;
       c0 += static_cast<int64_t>(gridDim.x) * kJoinCols) {
    const int64_t c = c0 + lane;
    float s = 0.0f;
    if (c < cols)
      for (int64_t p = parts * share / kJoinShares; p < p1; p += 8) {
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = p + q < p1 ? part[(p + q) * cols + c] : 0.0f;
#pragma unroll
        for (int q = 0; q < 8; ++q) s += v[q];
      }
    red[share][lane] = s;
    __syncthreads();
    if (share == 0 && c < cols) {
#pragma unroll
      for (int w = 1; w < kJoinShares; ++w) s += red[w][lane];
      dgain[c] = s;
    }
    __syncthreads();
  }
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
int backward_threads(int64_t cols) {
  return with_shape(cols, [](auto nt, auto) { return static_cast<int>(nt); });
}
// Blocks of the backward kernel, and partial sums of the gain's gradient: what the
// CUs hold at once, 16 waves each by the kernel's registers, at most 4 blocks a CU
// and at least 2 rows a block (1237 x 384 fp32 8.6 us, one row a block 11.8).  Twice
// that where each still has 8 rows (8192 x 4096 bf16 57 us, not 61; with fewer rows
// the sums cost more: 1237 x 4096 16, not 13).  Equal shares: as many rows to a
// block as the fullest has.
int64_t backward_blocks(int64_t rows, int64_t cols) {
  const int64_t held = 256 * std::min(4, 1024 / backward_threads(cols));
  const int64_t most = rows >= 16 * held ? 2 * held : held;
  const int64_t each = std::max<int64_t>(2, (rows + most - 1) / most);
  return (rows + each - 1) / each;
}

template <typename T, bool RES>
void norm_forward(const NormArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(a.rows < kMaxGrid ? a.rows : kMaxGrid));
  if (a.cols > kWideCols) {
    hipLaunchKernelGGL((rmsnorm_wide_kernel<T, 1024>), grid, dim3(1024), 0, s, a);
    return;
  }
  with_shape(a.cols, [&](auto nt, auto v) {
    hipLaunchKernelGGL((rmsnorm_kernel<T, nt, v, RES>), grid, dim3(nt), 0, s, a);
  });
}

template <typename T, bool DRES, bool DGAIN>
void norm_backward(const NormBwdArgs& a, hipStream_t s) {
  const int64_t blocks =
      DGAIN ? backward_blocks(a.rows, a.cols) : (a.rows < kMaxGrid ? a.rows : kMaxGrid);
  const dim3 grid(static_cast<uint32_t>(blocks));
  if (a.cols <= kWideCols) {
    with_shape(a.cols, [&](auto nt, auto v) {
      hipLaunchKernelGGL((rmsnorm_backward_kernel<T, nt, v, DRES, DGAIN>), grid, dim3(nt), 0, s, a);
    });
  } else {
    if (DGAIN)
      hipLaunchKernelGGL((rmsnorm_dgain_wide_kernel<T>),
                         dim3(static_cast<uint32_t>((a.cols + 2047) / 2048),
                              static_cast<uint32_t>(blocks)),
                         dim3(256), 0, s, a);
    hipLaunchKernelGGL((rmsnorm_dx_wide_kernel<T, 1024>),
                       dim3(static_cast<uint32_t>(a.rows < kMaxGrid ? a.rows : kMaxGrid)),
                       dim3(1024), 0, s, a);
  }
}

template <typename T>
void norm_backward(const NormBwdArgs& a, hipStream_t s) {
  if (a.dres != nullptr) {
    if (a.dgain != nullptr) norm_backward<T, true, true>(a, s);
    else norm_backward<T, true, false>(a, s);
  } else {
    if (a.dgain != nullptr) norm_backward<T, false, true>(a, s);
    else norm_backward<T, false, false>(a, s);
  }
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs& a, int32_t dtype, hipStream_t s) {
  (void)hipGetLastError();
  if (dtype == ZF_BF16) {
    if (a.residual != nullptr) norm_forward<uint16_t, true>(a, s);
    else norm_forward<uint16_t, false>(a, s);
  } else {
    if (a.residual != nullptr) norm_forward<float, true>(a, s);
    else norm_forward<float, false>(a, s);
  }
  return hipGetLastError();
}

size_t rmsnorm_backward_workspace(int64_t rows, int64_t cols) {
  return static_cast<size_t>(backward_blocks(rows, cols)) * static_cast<size_t>(cols) * sizeof(float);
}

hipError_t launch_rmsnorm_backward(const NormBwdArgs& a, int32_t dtype, hipStream_t s) {
  (void)hipGetLastError();
  if (a.rows > 0) {
    if (dtype == ZF_BF16) norm_backward<uint16_t>(a, s);
    else norm_backward<float>(a, s);
  }
  if (a.dgain != nullptr)  // (no rows: no partials, zeros)
    hipLaunchKernelGGL(
        dgain_kernel,
        dim3(static_cast<uint32_t>(std::min<int64_t>((a.cols + kJoinCols - 1) / kJoinCols, kMaxGrid))),
        dim3(1024), 0, s, a.part, backward_blocks(a.rows, a.cols), a.cols, a.dgain);
  return hipGetLastError();
}

}  // namespace zf
