// Quantisation to the 8-bit format of zf_layer.h: q = RNE(x * 2^(127 - code)),
// code from the largest magnitude of 128 elements of a row, of a column (the
// transposed copy's groups), or of a 128 x 128 block.
//
// A 256-thread block takes a 128 x 128 tile, whose groups all lie inside it:
// one read of x serves both copies.  A thread holds 8 rows x 8 columns; row
// maxima are taken over 16 lanes, column maxima over the thread's rows, the 4
// lanes of its wave that share its columns and, through LDS, the 4 waves.  The
// transposed copy's 8 x 8 byte blocks pass through LDS so that both copies are
// written in lines of 128 bytes.  Bound by HBM: 2 bytes read and 1 written per
// element and copy.
#include "zf_layer.hpp"

namespace zf {
namespace {

constexpr int kTile = 128;

// Byte offset of the 8 rows `u` (of 16) of column c in the transposed tile.
// 16-byte units are permuted by the column's group so that neither the
// writes (16 column groups at once) nor the reads meet in the same banks.
__device__ __forceinline__ int t_off(int c, int u) {
  return c * kTile + ((((u >> 1) ^ (c >> 3)) & 7) << 4) + ((u & 1) << 3);
}

template <typename T, int GROUP>
__global__ __launch_bounds__(256) void quantize_kernel(QuantArgs a) {
  __shared__ uint32_t cmax[4][kTile];
  __shared__ __align__(16) uint8_t tt[kTile * kTile];
  const T* x = static_cast<const T*>(a.x);
  const int t = threadIdx.x, cg = t & 15, u = t >> 4, wave = t >> 6;
  const int64_t ct = (a.cols + kTile - 1) / kTile, rt = (a.rows + kTile - 1) / kTile;
  for (int64_t b = blockIdx.x; b < rt * ct; b += gridDim.x) {
    const int64_t I = b / ct, J = b - I * ct;
    const int64_t r0 = I * kTile + 8 * u, c0 = J * kTile + 8 * cg;
    float v[8][8];
#pragma unroll
    for (int p = 0; p < 8; ++p)
      load8(x + (r0 + p) * a.ld_x + c0, r0 + p < a.rows ? a.cols - c0 : 0, v[p]);

    uint32_t rm[8], cm[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) cm[j] = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      rm[p] = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t m = abs_bits(v[p][j]);
        rm[p] = max(rm[p], m);
        cm[j] = max(cm[j], m);
      }
    }
    uint32_t block_code = 0;
    if constexpr (GROUP == 1) {
#pragma unroll
      for (int p = 0; p < 8; ++p) rm[p] = fp8_code(max16(rm[p]));
      if (a.qt.data != nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          cm[j] = max(cm[j], static_cast<uint32_t>(__shfl_xor(static_cast<int>(cm[j]), 16)));
          cm[j] = max(cm[j], static_cast<uint32_t>(__shfl_xor(static_cast<int>(cm[j]), 32)));
          if ((t & 63) < 16) cmax[wave][8 * cg + j] = cm[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = 8 * cg + j;
          cm[j] = fp8_code(max(max(cmax[0][c], cmax[1][c]), max(cmax[2][c], cmax[3][c])));
        }
      }
    } else {
      uint32_t m = rm[0];
#pragma unroll
      for (int p = 1; p < 8; ++p) m = max(m, rm[p]);
      m = max16(m);
      m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16)));
      m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32)));
      if ((t & 63) == 0) cmax[wave][0] = m;
      __syncthreads();
      block_code = fp8_code(max(max(cmax[0][0], cmax[1][0]), max(cmax[2][0], cmax[3][0])));
    }

    if (a.q.data != nullptr) {
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        if (r0 + p >= a.rows) break;
        const uint32_t code = GROUP == 1 ? rm[p] : block_code;
        store_bytes8(a.q.data + (r0 + p) * a.q.ld + c0, a.cols - c0, quant8(v[p], code));
        if (GROUP == 1 && cg == 0)
          a.q.scale[(r0 + p) * a.q.ld_scale + J] = static_cast<uint8_t>(code);
      }
      if (GROUP != 1 && t == 0) a.q.scale[I * a.q.ld_scale + J] = static_cast<uint8_t>(block_code);
    }
    if (a.qt.data != nullptr) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t code = GROUP == 1 ? cm[j] : block_code;
        float w[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) w[p] = v[p][j];
        *reinterpret_cast<u32x2*>(tt + t_off(8 * cg + j, u)) = quant8(w, code);
        if (GROUP == 1 && u == 0 && c0 + j < a.cols)
          a.qt.scale[(c0 + j) * a.qt.ld_scale + I] = static_cast<uint8_t>(code);
      }
      if (GROUP != 1 && t == 0)
        a.qt.scale[J * a.qt.ld_scale + I] = static_cast<uint8_t>(block_code);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = 32 * i + (t >> 3), k = t & 7;
        const int64_t col = J * kTile + c, row = I * kTile + 16 * k;
        if (col >= a.cols || row >= a.rows) continue;
        uint8_t* p = a.qt.data + col * a.qt.ld + row;
        const u32x4 w = *reinterpret_cast<const u32x4*>(tt + t_off(c, 2 * k));
        if (row + 16 <= a.rows) {
          *reinterpret_cast<u32x4*>(p) = w;
        } else {
          store_bytes8(p, a.rows - row, u32x2{w.x, w.y});
          store_bytes8(p + 8, a.rows - row - 8, u32x2{w.z, w.w});
        }
      }
    }
    __syncthreads();  // cmax and tt are written again by the next tile
  }
}

}  // namespace

hipError_t launch_quantize(const QuantArgs& a, int32_t dtype, int32_t group, hipStream_t s) {
  (void)hipGetLastError();
  const int64_t tiles =
      ((a.rows + kTile - 1) / kTile) * ((a.cols + kTile - 1) / kTile);
  const dim3 grid(static_cast<uint32_t>(tiles < (1 << 22) ? tiles : (1 << 22)));
  if (dtype == ZF_BF16) {
    if (group == 1) hipLaunchKernelGGL((quantize_kernel<uint16_t, 1>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((quantize_kernel<uint16_t, 128>), grid, dim3(256), 0, s, a);
  } else {
    if (group == 1) hipLaunchKernelGGL((quantize_kernel<float, 1>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((quantize_kernel<float, 128>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace zf
