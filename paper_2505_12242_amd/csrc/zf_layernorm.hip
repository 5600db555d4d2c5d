// Layer norm with the residual's addition and an 8-bit output, and its
// gradients (formulas in zf_layer.h).
//
// Rows and blocks as for the RMS norm (zf_norm.hip): one block per row, the row
// in registers, every input read once and every output written once, sums in
// fp32.  The squares are summed about the mean, in a second pass over the
// registers and a second barrier: nothing cancels, as a sum of squares less a
// squared sum would.  (Each wave's squares about its own mean, joined with one
// barrier, cost more than the barrier: 8192 x 5120 bf16 144 us.)  Bound by HBM:
// 8192 x 5120 bf16 with a residual, h, y and 8 bits, 378 MB in 69.5 us, 5.4 TB/s, 0.8
// of a copy's rate.
#include <algorithm>

#include "zf_norm.hpp"

namespace zf {
namespace {

// y of 8 elements written, in its own type and in 8 bits (as the RMS norm's).
template <typename T>
__device__ __forceinline__ void store_y(const LayerNormArgs& a, int64_t row, int64_t c,
                                        const Vec8<T>& h, const float (&g)[8], const float (&b)[8],
                                        float mean, float rstd) {
  const int64_t valid = a.cols - c;
  float o[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = j < valid ? ((h[j] - mean) * rstd) * g[j] + b[j] : 0.0f;
  Vec8<T> y;
  y.set(o);
  if (a.y != nullptr) y.template store<true>(static_cast<T*>(a.y) + row * a.ld_y + c, valid);
  if (a.q.data != nullptr) {
    const uint32_t code = fp8_code(max16(abs_max(y)));
    store_bytes8(a.q.data + row * a.q.ld + c, valid, quant8(y, code));
    if ((threadIdx.x & 15) == 0 && valid > 0)
      a.q.scale[row * a.q.ld_scale + c / kFp8Group] = static_cast<uint8_t>(code);
  }
}

struct Moments {
  float mean, rstd;
};

// Keeps a bf16 row packed from one pass over it to the next: unpacked once for all
// of them, it takes twice the registers.
template <int V>
__device__ __forceinline__ void repack(Vec8<uint16_t> (&h)[V]) {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
  for (int i = 0; i < V; ++i) asm volatile("" : "+v"(h[i].u));
#endif
}
template <int V>
__device__ __forceinline__ void repack(Vec8<float> (&)[V]) {}

// Waits for a vector's, or a value's, loads here.
__device__ __forceinline__ void arrived(float& x) {
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("" : "+v"(x));
#endif
}
__device__ __forceinline__ void arrived(Vec8<uint16_t>& v) {
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("" : "+v"(v.u));
#endif
}
__device__ __forceinline__ void arrived(Vec8<float>& v) {
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("" : "+v"(v.u[0]), "+v"(v.u[1]));
#endif
}

// The row's moments in every thread: piece i of V of the thread's 8 elements
// are columns (threadIdx.x + i * NT) * 8 and on, zeros past the row's end.
// `red`: two of block_sum's.
template <typename T, int NT, int V>
__device__ __forceinline__ Moments moments(Vec8<T> (&h)[V], int64_t cols, float eps,
                                           float (&red)[2][NT / 64]) {
  const float inv = 1.0f / static_cast<float>(cols > 0 ? cols : 1);
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) s += h[i][j];
  const float mean = block_sum<NT>(s, red[0]) * inv;
  repack(h);
  float m2 = 0.0f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int64_t valid = cols - (threadIdx.x + i * NT) * 8;
    if (valid >= 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = h[i][j] - mean;
        m2 += d * d;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = j < valid ? h[i][j] - mean : 0.0f;
        m2 += d * d;
      }
    }
  }
  return Moments{mean, 1.0f / sqrtf(block_sum<NT>(m2, red[1]) * inv + eps)};
}

// G: the gain's and the bias's type.  Beside bf16 rows both are loaded with the row:
// loads behind the stores of h wait for these too (8192 x 5120 69.5 us, not 71.6; 4096
// columns without residual and 8 bits 28.8, not 32.5).  Beside fp32 rows they would
// fill the registers (4096 x 5003 85 us, not 75).
template <typename T, typename G, int NT, int V, bool RES>
__global__ __launch_bounds__(NT, V == 1 ? 8 : 1) void layernorm_kernel(LayerNormArgs a) {
  __shared__ float red[2][2][NT / 64];
  int flip = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    Vec8<T> h[V], r[RES ? V : 1];
    Vec8<G> g[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      h[i].template fetch<true>(static_cast<const T*>(a.x) + row * a.ld_x + c, a.cols - c);
      if constexpr (RES)
        r[i].template fetch<true>(static_cast<const T*>(a.residual) + row * a.ld_residual + c,
                                  a.cols - c);
    }
    const auto fetch = [&](int i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      g[i].fetch(static_cast<const G*>(a.gain) + c, a.cols - c);
      b[i].fetch(static_cast<const G*>(a.bias) + c, a.bias != nullptr ? a.cols - c : 0);
    };
    const auto settle = [&](int i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      g[i].settle(a.cols - c);
      b[i].settle(a.bias != nullptr ? a.cols - c : 0);
    };
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < V; ++i) fetch(i);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      if constexpr (sizeof(T) == 2) settle(i);
      h[i].settle(a.cols - c);
      if constexpr (RES) {
        r[i].settle(a.cols - c);
        add(h[i], r[i]);
      }
      if (RES || (a.h != nullptr && a.h != a.x))
        h[i].template store<true>(static_cast<T*>(a.h) + row * a.ld_h + c, a.cols - c);
    }
    const Moments m = moments<T, NT, V>(h, a.cols, a.eps, red[flip]);
    repack(h);
    flip ^= 1;
    if (threadIdx.x == 0) {
      a.mean[row] = m.mean;
      a.rstd[row] = m.rstd;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if constexpr (sizeof(T) != 2) {
        fetch(i);
        settle(i);
      }
      float gain[8], bias[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        gain[j] = g[i][j];
        bias[j] = b[i][j];
      }
      store_y(a, row, (threadIdx.x + i * NT) * 8, h[i], gain, bias, m.mean, m.rstd);
    }
  }
}

// Rows too wide for the registers: read three times (the sum, the squares about
// the mean, the result).
template <typename T, int NT>
__global__ __launch_bounds__(NT) void layernorm_wide_kernel(LayerNormArgs a) {
  __shared__ float red[2][NT / 64];
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
    float s = 0.0f;
    for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8 * NT) {
      load_h(c);
#pragma unroll
      for (int j = 0; j < 8; ++j) s += h[j];
    }
    const float mean = block_sum<NT>(s, red[0]) / static_cast<float>(a.cols);
    float m2 = 0.0f;
    for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8 * NT) {
      load_h(c);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = c + j < a.cols ? h[j] - mean : 0.0f;
        m2 += d * d;
      }
    }
    const float rstd = 1.0f / sqrtf(block_sum<NT>(m2, red[1]) / static_cast<float>(a.cols) + a.eps);
    if (threadIdx.x == 0) {
      a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
    for (int64_t c = threadIdx.x * 8; c < span; c += 8 * NT) {
      load_h(c);  // (before h, which may be x's or the residual's own buffer, is written)
      if (a.residual != nullptr || (a.h != nullptr && a.h != a.x))
        h.store(static_cast<T*>(a.h) + row * a.ld_h + c, a.cols - c);
      float g[8], b[8] = {};
      load_gain(a, c, g);
      if (a.bias != nullptr) load_vector(a.bias, a.gain_f32, a.cols, c, b);
      store_y(a, row, c, h, g, b, mean, rstd);
    }
  }
}

// Two sums over the block at once.
template <int NT>
__device__ __forceinline__ float2 block_sum2(float x, float y, float2 (&red)[NT / 64]) {
  x = wave_sum(x);
  y = wave_sum(y);
  if constexpr (NT == 64) return float2{x, y};
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = float2{x, y};
  __syncthreads();
  float2 s = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) {
    s.x += red[w].x;
    s.y += red[w].y;
  }
  return s;
}

// A block takes rows one after the other, the next one's loads in flight where a
// thread has one piece, and keeps its columns' sums for both gradients in registers.
// 8192 x 5120 bf16 with a residual: 336 MB in 74 us, of which 5 join the partial sums, 4.9
// TB/s in the first kernel, bound by HBM through few loads in flight (the sums'
// registers leave a CU one block); 56 us where the operands are those of the call
// before, partly in the cache.  GRADS: the gain's and the bias's partial sums are kept (the bias's
// behind all blocks' of the gain).
template <typename T, int NT, int V, bool DRES, bool GRADS>
__global__ __launch_bounds__(NT) void layernorm_backward_kernel(LayerNormBwdArgs a) {
  __shared__ float2 red[2][NT / 64];
  float dg[V][8], db[V][8], g[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    load_gain(a, (threadIdx.x + i * NT) * 8, g[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[i][j] = db[i][j] = 0.0f;
  }
  int64_t r0, r1;
  block_rows(a.rows, gridDim.x, blockIdx.x, r0, r1);
  struct Row {
    Vec8<T> dy[V], h[V], dres[DRES ? V : 1];
    float mean, rstd;
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
    w.mean = a.mean[row];
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
    // (past the row's end dy and the gain are zeros)
    float s = 0.0f, t = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float hh = (w.h[i][j] - w.mean) * w.rstd, u = w.dy[i][j] * g[i][j];
        if (GRADS) {
          dg[i][j] += w.dy[i][j] * hh;
          db[i][j] += w.dy[i][j];
        }
        t += u;
        s += u * hh;
      }
    const float2 sums = block_sum2<NT>(t, s, red[flip]);
    flip ^= 1;
    const float mt = sums.x / static_cast<float>(a.cols), ms = sums.y / static_cast<float>(a.cols);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = w.rstd * ((w.dy[i][j] * g[i][j] - mt) - ((w.h[i][j] - w.mean) * w.rstd) * ms);
        if constexpr (DRES) o[j] += w.dres[i][j];
      }
      Vec8<T> out;
      out.set(o);
      if constexpr (V == 1) {
        // (the next row has to be there before this one is stored: the loop would wait
        // for the store with it)
        arrived(next.dy[0]);
        arrived(next.h[0]);
        if constexpr (DRES) arrived(next.dres[0]);
        arrived(next.mean);
        arrived(next.rstd);
      }
      out.template store<true>(static_cast<T*>(a.dx) + row * a.ld_dx + c, a.cols - c);
    }
  }
  if constexpr (GRADS) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = (threadIdx.x + i * NT) * 8;
      Vec8<float> out;
      out.set(dg[i]);
      out.store(a.part + blockIdx.x * a.cols + c, a.cols - c);
      out.set(db[i]);
      out.store(a.part + (gridDim.x + blockIdx.x) * a.cols + c, a.cols - c);
    }
  }
}

// Rows too wide for the registers: the partial sums by column (before dx, which
// may be dy's own buffer, is written), then dx with dy and h read twice.
template <typename T>
__global__ __launch_bounds__(256) void layernorm_grads_wide_kernel(LayerNormBwdArgs a) {
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8;
  if (c >= a.cols) return;
  int64_t r0, r1;
  block_rows(a.rows, gridDim.y, blockIdx.y, r0, r1);
  float dg[8] = {}, db[8] = {};
  for (int64_t row = r0; row < r1; ++row) {
    Vec8<T> d, h;
    d.load(static_cast<const T*>(a.dy) + row * a.ld_dy + c, a.cols - c);
    h.load(static_cast<const T*>(a.h) + row * a.ld_h + c, a.cols - c);
    const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dg[j] += d[j] * ((h[j] - mean) * rstd);
      db[j] += d[j];
    }
  }
  Vec8<float> out;
  out.set(dg);
  out.store(a.part + blockIdx.y * a.cols + c, a.cols - c);
  out.set(db);
  out.store(a.part + (gridDim.y + blockIdx.y) * a.cols + c, a.cols - c);
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void layernorm_dx_wide_kernel(LayerNormBwdArgs a) {
  __shared__ float2 red[2][NT / 64];
  int flip = 0;
  Vec8<T> d, h, r;
  float g[8];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
    const T* hp = static_cast<const T*>(a.h) + row * a.ld_h;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s = 0.0f, t = 0.0f;
    for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8 * NT) {
      d.load(dy + c, a.cols - c);
      h.load(hp + c, a.cols - c);
      load_gain(a, c, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float u = d[j] * g[j];
        t += u;
        s += u * ((h[j] - mean) * rstd);
      }
    }
    const float2 sums = block_sum2<NT>(t, s, red[flip]);
    flip ^= 1;
    const float mt = sums.x / static_cast<float>(a.cols), ms = sums.y / static_cast<float>(a.cols);
    for (int64_t c = threadIdx.x * 8; c < a.cols; c += 8 * NT) {
      d.load(dy + c, a.cols - c);
      h.load(hp + c, a.cols - c);
      load_gain(a, c, g);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        g[j] = rstd * ((d[j] * g[j] - mt) - ((h[j] - mean) * rstd) * ms);
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

int backward_threads(int64_t cols) {
  return with_shape(cols, [](auto nt, auto) { return static_cast<int>(nt); });
}
// Blocks of the backward kernel, and partial sums of either gradient: what the chip
// holds at once, two rows each at least (8192 x 5120, operands in turn, 74 us, with twice
// the blocks 79: two rounds of them, and twice the sums).
int64_t backward_blocks(int64_t rows, int64_t cols) {
  const int64_t held = 256 * std::min(4, 1024 / backward_threads(cols));
  const int64_t each = std::max<int64_t>(2, (rows + held - 1) / held);
  return (rows + each - 1) / each;
}

// f(threads, pieces a thread) of the forward pass: bf16 rows of more than 2048 columns
// in blocks of 256 threads with more pieces each, which wait for fewer waves at a
// barrier (8192 x 5120 69.5 us, with one piece 78; 8192 x 8192 107, not 110; fp32 81
// us for 4096 x 5003, with one piece 75).
template <typename T, typename F>
auto with_forward_shape(int64_t cols, F&& f) {
  typedef std::integral_constant<int, 256> Threads;
  if constexpr (sizeof(T) == 2) {
    if (cols > 2048 && cols <= 4096) return f(Threads(), std::integral_constant<int, 2>());
    if (cols > 4096 && cols <= 6144) return f(Threads(), std::integral_constant<int, 3>());
    if (cols > 6144 && cols <= 8192) return f(Threads(), std::integral_constant<int, 4>());
  }
  return with_shape(cols, f);
}

template <typename T, bool RES>
void forward(const LayerNormArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(std::min(a.rows, kMaxGrid)));
  if (a.cols > kWideCols) {
    hipLaunchKernelGGL((layernorm_wide_kernel<T, 1024>), grid, dim3(1024), 0, s, a);
    return;
  }
  with_forward_shape<T>(a.cols, [&](auto nt, auto v) {
    if (a.gain_f32) hipLaunchKernelGGL((layernorm_kernel<T, float, nt, v, RES>), grid, dim3(nt), 0, s, a);
    else hipLaunchKernelGGL((layernorm_kernel<T, uint16_t, nt, v, RES>), grid, dim3(nt), 0, s, a);
  });
}

template <typename T, bool DRES, bool GRADS>
void backward(const LayerNormBwdArgs& a, hipStream_t s) {
  const int64_t blocks = GRADS ? backward_blocks(a.rows, a.cols) : std::min(a.rows, kMaxGrid);
  const dim3 grid(static_cast<uint32_t>(blocks));
  if (a.cols <= kWideCols) {
    with_shape(a.cols, [&](auto nt, auto v) {
      hipLaunchKernelGGL((layernorm_backward_kernel<T, nt, v, DRES, GRADS>), grid, dim3(nt), 0, s,
                         a);
    });
  } else {
    if (GRADS)
      hipLaunchKernelGGL((layernorm_grads_wide_kernel<T>),
                         dim3(static_cast<uint32_t>((a.cols + 2047) / 2048),
                              static_cast<uint32_t>(blocks)),
                         dim3(256), 0, s, a);
    hipLaunchKernelGGL((layernorm_dx_wide_kernel<T, 1024>),
                       dim3(static_cast<uint32_t>(std::min(a.rows, kMaxGrid))), dim3(1024), 0, s, a);
  }
}

template <typename T>
void backward(const LayerNormBwdArgs& a, hipStream_t s) {
  const bool grads = a.dgain != nullptr || a.dbias != nullptr;
  if (a.dres != nullptr) {
    if (grads) backward<T, true, true>(a, s);
    else backward<T, true, false>(a, s);
  } else {
    if (grads) backward<T, false, true>(a, s);
    else backward<T, false, false>(a, s);
  }
}

}  // namespace

hipError_t launch_layernorm(const LayerNormArgs& a, int32_t dtype, hipStream_t s) {
  (void)hipGetLastError();
  if (dtype == ZF_BF16) {
    if (a.residual != nullptr) forward<uint16_t, true>(a, s);
    else forward<uint16_t, false>(a, s);
  } else {
    if (a.residual != nullptr) forward<float, true>(a, s);
    else forward<float, false>(a, s);
  }
  return hipGetLastError();
}

size_t layernorm_backward_workspace(int64_t rows, int64_t cols) {
  return 2 * static_cast<size_t>(backward_blocks(rows, cols)) * static_cast<size_t>(cols) *
         sizeof(float);
}

hipError_t launch_layernorm_backward(const LayerNormBwdArgs& a, int32_t dtype, hipStream_t s) {
  (void)hipGetLastError();
  if (a.rows > 0) {
    if (dtype == ZF_BF16) backward<uint16_t>(a, s);
    else backward<float>(a, s);
  }
  // (no rows: no partials, zeros)
  const int64_t parts = backward_blocks(a.rows, a.cols);
  if (a.dgain != nullptr) launch_join_columns(a.part, parts, a.cols, a.dgain, a.dbias, s);
  else if (a.dbias != nullptr)
    launch_join_columns(a.part + parts * a.cols, parts, a.cols, a.dbias, nullptr, s);
  return hipGetLastError();
}

}  // namespace zf
