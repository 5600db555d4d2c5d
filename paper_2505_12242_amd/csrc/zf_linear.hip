// The gradient at a linear layer's product (formulas in zf_layer.h):
// dz = dy act'(z) in 8 bits by rows and by columns, the bias's gradient, and dz
// itself, in one pass over dy and z.
//
// Tiles and blocks as the quantiser's (zf_fp8.hip), whose 8-bit copies these
// are.  The bias's gradient is summed before rounding: over a thread's 8 rows,
// the tile's other 15 units of rows, and, in tile order, by a second kernel.
//
// 4096 x 11008 bf16 with an activation: 271 MB in 62 us, 4.4 TB/s (plus 4 to join the
// bias's sums): as for the quantiser, a tile's loads, reductions and stores follow one
// another and only other blocks overlap them.
#include "zf_activation.hpp"
#include "zf_norm.hpp"
#include "zf_quantize.hpp"

namespace zf {
namespace {

template <typename T, int ACT, bool NT>
__global__ __launch_bounds__(256) void linear_backward_kernel(LinearBwdArgs a) {
  __shared__ TileShared<T> lds;
  __shared__ float sums[4][kTile];
  const int t = threadIdx.x, cg = t & 15, u = t >> 4;
  uint32_t I, J;
  tile_place(blockIdx.x, static_cast<uint32_t>((a.rows + kTile - 1) / kTile),
             static_cast<uint32_t>((a.cols + kTile - 1) / kTile), I, J);
  const int64_t r0 = static_cast<int64_t>(I) * kTile + 8 * u;
  const int64_t c0 = static_cast<int64_t>(J) * kTile + 8 * cg;
  Block<T> x, z;
  const auto valid = [&](int p) { return r0 + p < a.rows ? a.cols - c0 : 0; };
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    x.v[p].template fetch<NT>(static_cast<const T*>(a.dy) + (r0 + p) * a.ld_dy + c0, valid(p));
    if (ACT != ZF_NONE)
      z.v[p].template fetch<NT>(static_cast<const T*>(a.z) + (r0 + p) * a.ld_z + c0, valid(p));
  }
  float sum[8] = {};
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int64_t n = r0 + p < a.rows ? a.cols - c0 : 8;
    x.v[p].settle(n);
    if (ACT != ZF_NONE) z.v[p].settle(n);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = x.v[p][j];
      if (ACT != ZF_NONE) v[j] *= slope<ACT>(z.v[p][j]);
      sum[j] += v[j];
    }
    if (ACT != ZF_NONE) x.v[p].set(v);
    if (a.dz != nullptr)
      x.v[p].template store<true>(static_cast<T*>(a.dz) + (r0 + p) * a.ld_dz + c0, valid(p));
  }
  if (a.dbias != nullptr) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sum[j] += __shfl_xor(sum[j], 16);
      sum[j] += __shfl_xor(sum[j], 32);
      if ((t & 63) < 16) sums[t >> 6][8 * cg + j] = sum[j];
    }
    __syncthreads();
    const int64_t c = static_cast<int64_t>(J) * kTile + t;
    if (t < kTile && c < a.cols)
      a.part[I * a.cols + c] = ((sums[0][t] + sums[1][t]) + sums[2][t]) + sums[3][t];
  }
  write_tile<T, 1>(x, a.rows, a.cols, I, J, a.q, a.qt, lds);
}

int64_t row_tiles(int64_t rows) { return (rows + kTile - 1) / kTile; }

template <typename T>
void launch(const LinearBwdArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(row_tiles(a.rows) * ((a.cols + kTile - 1) / kTile)));
  const auto lines = [](const void* p, int64_t ld) {
    return reinterpret_cast<uintptr_t>(p) % 128 == 0 && ld * sizeof(T) % 128 == 0;
  };
  const bool nt = lines(a.dy, a.ld_dy) && (a.activation == ZF_NONE || lines(a.z, a.ld_z));
  with_activation(a.activation, [&](auto act) {
    if (nt) hipLaunchKernelGGL((linear_backward_kernel<T, act, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((linear_backward_kernel<T, act, false>), grid, dim3(256), 0, s, a);
  });
}

}  // namespace

size_t linear_backward_workspace(int64_t rows, int64_t cols) {
  return static_cast<size_t>(row_tiles(rows)) * static_cast<size_t>(cols) * sizeof(float);
}

hipError_t launch_linear_backward(const LinearBwdArgs& a, int32_t dtype, hipStream_t s) {
  (void)hipGetLastError();
  if (a.rows > 0) {
    if (dtype == ZF_BF16) launch<uint16_t>(a, s);
    else launch<float>(a, s);
  }
  if (a.dbias != nullptr)  // (no rows: no partials, zeros)
    launch_join_columns(a.part, row_tiles(a.rows), a.cols, a.dbias, nullptr, s);
  return hipGetLastError();
}

}  // namespace zf
