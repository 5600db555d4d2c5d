// Shared by the kernels that write a 128 x 128 tile in 8 bits, by rows and by
// columns (format in zf_layer.h; see zf_fp8.hip).
#pragma once

#include "zf_layer.hpp"

namespace zf {

constexpr int kTile = 128;

// Byte offset of the 8 rows `u` (of 16) of column c in the transposed tile.
// 16-byte units are permuted by the column's group so that neither the
// writes (16 column groups at once) nor the reads meet in the same banks.
__device__ __forceinline__ int t_off(int c, int u) {
  return c * kTile + ((((u >> 1) ^ (c >> 3)) & 7) << 4) + ((u & 1) << 3);
}

// A thread's 8 x 8 elements.  bf16 ones stay packed in pairs, two columns a word,
// and their magnitudes are compared as 16-bit integers, two at a time.
template <typename T>
struct Block;

template <>
struct Block<uint16_t> {
  static constexpr int kMax = 4;  // words of the 8 columns' maxima
  Vec8<uint16_t> v[8];
  // The largest magnitude of every row (its fp32 bits) and of every column.
  __device__ __forceinline__ void maxima(uint32_t (&rm)[8], uint32_t (&cm)[kMax]) const {
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      uint32_t r = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t m = v[p].u[w] & 0x7fff7fffu;
        r = w == 0 ? m : pk_max(r, m);
        cm[w] = p == 0 ? m : pk_max(cm[w], m);
      }
      rm[p] = max(r << 16, r & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint32_t join_max(uint32_t a, uint32_t b) { return pk_max(a, b); }
  static __device__ __forceinline__ uint32_t column_bits(const uint32_t (&cm)[kMax], int j) {
    return j & 1 ? cm[j >> 1] & 0xffff0000u : cm[j >> 1] << 16;
  }
  __device__ __forceinline__ u32x2 column(int j, uint32_t code) const {
    const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
    uint32_t u[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      u[q] = __builtin_amdgcn_perm(v[2 * q + 1].u[j >> 1], v[2 * q].u[j >> 1], sel);
    return quant8_bf16(u[0], u[1], u[2], u[3], code);
  }
};

template <>
struct Block<float> {
  static constexpr int kMax = 8;
  Vec8<float> v[8];
  __device__ __forceinline__ void maxima(uint32_t (&rm)[8], uint32_t (&cm)[kMax]) const {
#pragma unroll
    for (int p = 0; p < 8; ++p)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t m = abs_bits(v[p][j]);
        rm[p] = j == 0 ? m : max(rm[p], m);
        cm[j] = p == 0 ? m : max(cm[j], m);
      }
  }
  static __device__ __forceinline__ uint32_t join_max(uint32_t a, uint32_t b) { return max(a, b); }
  static __device__ __forceinline__ uint32_t column_bits(const uint32_t (&cm)[kMax], int j) {
    return cm[j];
  }
  __device__ __forceinline__ u32x2 column(int j, uint32_t code) const {
    float w[8];
#pragma unroll
    for (int p = 0; p < 8; ++p) w[p] = v[p][j];
    return quant8(w, code);
  }
};

// Tile b's place among rt x ct tiles: strips of 8 tile rows, walked column by
// column, 64 tiles in a run of one XCD, whose L2 then joins the scales' single
// bytes (of 8 tiles next to each other in either direction).
__device__ __forceinline__ void tile_place(uint32_t b, uint32_t rt, uint32_t ct, uint32_t& I,
                                           uint32_t& J) {
  const uint32_t id = static_cast<uint32_t>(xcd_remap<kOrderScores>(b, rt * ct, 0));
  const uint32_t strip = id / (8 * ct), in = id - strip * 8 * ct;
  const uint32_t left = rt - 8 * strip, h = left < 8 ? left : 8;
  J = in / h;
  I = 8 * strip + in - J * h;
}

// LDS of a block that writes a tile.
template <typename T>
struct TileShared {
  uint32_t cmax[4][16][Block<T>::kMax];
  __align__(16) uint8_t tt[kTile * kTile];
};

// Tile (I, J) of rows x cols in 8 bits: thread t of 256 holds rows r0 .. r0 + 7
// of columns c0 .. c0 + 7, t / 16 and t % 16 units of 8 into the tile; elements
// outside are zeros.  Every thread of the block calls it.
template <typename T, int GROUP>
__device__ __forceinline__ void write_tile(const Block<T>& x, int64_t rows, int64_t cols, uint32_t I,
                                           uint32_t J, const Fp8Out& q, const Fp8Out& qt,
                                           TileShared<T>& lds) {
  typedef Block<T> B;
  auto& cmax = lds.cmax;
  auto& tt = lds.tt;
  const int t = threadIdx.x, cg = t & 15, u = t >> 4, wave = t >> 6;
  const int64_t r0 = static_cast<int64_t>(I) * kTile + 8 * u;
  const int64_t c0 = static_cast<int64_t>(J) * kTile + 8 * cg;
  uint32_t rm[8], cm[B::kMax];
  x.maxima(rm, cm);
  uint32_t block_code = 0;
  if constexpr (GROUP == 1) {
#pragma unroll
    for (int p = 0; p < 8; ++p) rm[p] = fp8_code(max16(rm[p]));
    if (qt.data != nullptr) {
#pragma unroll
      for (int w = 0; w < B::kMax; ++w) {
        cm[w] = B::join_max(cm[w], __shfl_xor(cm[w], 16));
        cm[w] = B::join_max(cm[w], __shfl_xor(cm[w], 32));
        if ((t & 63) < 16) cmax[wave][cg][w] = cm[w];
      }
      __syncthreads();
#pragma unroll
      for (int w = 0; w < B::kMax; ++w)
        cm[w] = B::join_max(B::join_max(cmax[0][cg][w], cmax[1][cg][w]),
                            B::join_max(cmax[2][cg][w], cmax[3][cg][w]));
    }
  } else {
    uint32_t m = rm[0];
#pragma unroll
    for (int p = 1; p < 8; ++p) m = max(m, rm[p]);
    m = max16(m);
    m = max(m, __shfl_xor(m, 16));
    m = max(m, __shfl_xor(m, 32));
    if ((t & 63) == 0) cmax[wave][0][0] = m;
    __syncthreads();
    block_code = fp8_code(max(max(cmax[0][0][0], cmax[1][0][0]), max(cmax[2][0][0], cmax[3][0][0])));
  }

  if (q.data != nullptr) {
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      if (r0 + p >= rows) break;
      const uint32_t code = GROUP == 1 ? rm[p] : block_code;
      store_bytes8(q.data + (r0 + p) * q.ld + c0, cols - c0, quant8(x.v[p], code));
      if (GROUP == 1 && cg == 0)
        q.scale[(r0 + p) * q.ld_scale + J] = static_cast<uint8_t>(code);
    }
    if (GROUP != 1 && t == 0) q.scale[I * q.ld_scale + J] = static_cast<uint8_t>(block_code);
  }
  if (qt.data != nullptr) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t code = GROUP == 1 ? fp8_code(B::column_bits(cm, j)) : block_code;
      *reinterpret_cast<u32x2*>(tt + t_off(8 * cg + j, u)) = x.column(j, code);
      if (GROUP == 1 && u == 0 && c0 + j < cols)
        qt.scale[(c0 + j) * qt.ld_scale + I] = static_cast<uint8_t>(code);
    }
    if (GROUP != 1 && t == 0) qt.scale[J * qt.ld_scale + I] = static_cast<uint8_t>(block_code);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = 32 * i + (t >> 3), k = t & 7;
      const int64_t col = static_cast<int64_t>(J) * kTile + c;
      const int64_t row = static_cast<int64_t>(I) * kTile + 16 * k;
      if (col >= cols || row >= rows) continue;
      uint8_t* p = qt.data + col * qt.ld + row;
      const u32x4 w = *reinterpret_cast<const u32x4*>(tt + t_off(c, 2 * k));
      if (row + 16 <= rows) {
        *reinterpret_cast<u32x4*>(p) = w;
      } else {
        store_bytes8(p, rows - row, u32x2{w.x, w.y});
        store_bytes8(p + 8, rows - row - 8, u32x2{w.z, w.w});
      }
    }
  }
}

}  // namespace zf
