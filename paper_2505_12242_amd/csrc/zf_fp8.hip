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
// element and copy (bf16, both copies: 8192 x 11008 68 us, 5.3 TB/s; 4096 x 11008
// 37 us, 4.9; 4099 x 5003, whose rows begin anywhere in a line, 16 us with one scale
// a block).  Four blocks a CU: with six (lane offsets in 32 bits) 4096 x 11008 takes
// 38.7 us, not 37.6.
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

// NT: x's rows are whole lines, each read by one block (nontemporal: 4096 x 11008
// both ways 44 -> 38 us; rows that share lines 19 -> 28 us, so not those).
template <typename T, int GROUP, bool NT>
__global__ __launch_bounds__(256) void quantize_kernel(QuantArgs a) {
  typedef Block<T> B;
  __shared__ uint32_t cmax[4][16][B::kMax];
  __shared__ __align__(16) uint8_t tt[kTile * kTile];
  const int t = threadIdx.x, cg = t & 15, u = t >> 4, wave = t >> 6;
  uint32_t I, J;
  tile_place(blockIdx.x, static_cast<uint32_t>((a.rows + kTile - 1) / kTile),
             static_cast<uint32_t>((a.cols + kTile - 1) / kTile), I, J);
  const int64_t r0 = static_cast<int64_t>(I) * kTile + 8 * u;
  const int64_t c0 = static_cast<int64_t>(J) * kTile + 8 * cg;
  B x;
#pragma unroll
  for (int p = 0; p < 8; ++p)
    x.v[p].template fetch<NT>(static_cast<const T*>(a.x) + (r0 + p) * a.ld_x + c0,
                             r0 + p < a.rows ? a.cols - c0 : 0);
#pragma unroll
  for (int p = 0; p < 8; ++p) x.v[p].settle(r0 + p < a.rows ? a.cols - c0 : 8);

  uint32_t rm[8], cm[B::kMax];
  x.maxima(rm, cm);
  uint32_t block_code = 0;
  if constexpr (GROUP == 1) {
#pragma unroll
    for (int p = 0; p < 8; ++p) rm[p] = fp8_code(max16(rm[p]));
    if (a.qt.data != nullptr) {
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

  if (a.q.data != nullptr) {
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      if (r0 + p >= a.rows) break;
      const uint32_t code = GROUP == 1 ? rm[p] : block_code;
      store_bytes8(a.q.data + (r0 + p) * a.q.ld + c0, a.cols - c0, quant8(x.v[p], code));
      if (GROUP == 1 && cg == 0)
        a.q.scale[(r0 + p) * a.q.ld_scale + J] = static_cast<uint8_t>(code);
    }
    if (GROUP != 1 && t == 0) a.q.scale[I * a.q.ld_scale + J] = static_cast<uint8_t>(block_code);
  }
  if (a.qt.data != nullptr) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t code = GROUP == 1 ? fp8_code(B::column_bits(cm, j)) : block_code;
      *reinterpret_cast<u32x2*>(tt + t_off(8 * cg + j, u)) = x.column(j, code);
      if (GROUP == 1 && u == 0 && c0 + j < a.cols)
        a.qt.scale[(c0 + j) * a.qt.ld_scale + I] = static_cast<uint8_t>(code);
    }
    if (GROUP != 1 && t == 0) a.qt.scale[J * a.qt.ld_scale + I] = static_cast<uint8_t>(block_code);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = 32 * i + (t >> 3), k = t & 7;
      const int64_t col = static_cast<int64_t>(J) * kTile + c;
      const int64_t row = static_cast<int64_t>(I) * kTile + 16 * k;
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
}

}  // namespace

hipError_t launch_quantize(const QuantArgs& a, int32_t dtype, int32_t group, hipStream_t s) {
  (void)hipGetLastError();
  const dim3 grid(
      static_cast<uint32_t>(((a.rows + kTile - 1) / kTile) * ((a.cols + kTile - 1) / kTile)));
  const bool lines = reinterpret_cast<uintptr_t>(a.x) % 128 == 0 &&
                     a.ld_x * (dtype == ZF_BF16 ? 2 : 4) % 128 == 0;
#define ZF_QUANT(T, G)                                                                        \
  if (lines) hipLaunchKernelGGL((quantize_kernel<T, G, true>), grid, dim3(256), 0, s, a);     \
  else hipLaunchKernelGGL((quantize_kernel<T, G, false>), grid, dim3(256), 0, s, a)
  if (dtype == ZF_BF16) {
    if (group == 1) { ZF_QUANT(uint16_t, 1); }
    else { ZF_QUANT(uint16_t, 128); }
  } else {
    if (group == 1) { ZF_QUANT(float, 1); }
    else { ZF_QUANT(float, 128); }
  }
#undef ZF_QUANT
  return hipGetLastError();
}

}  // namespace zf
