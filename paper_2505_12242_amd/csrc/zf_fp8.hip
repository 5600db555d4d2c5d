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
#include "zf_quantize.hpp"

namespace zf {
namespace {

// NT: x's rows are whole lines, each read by one block (nontemporal: 4096 x 11008
// both ways 44 -> 38 us; rows that share lines 19 -> 28 us, so not those).
template <typename T, int GROUP, bool NT>
__global__ __launch_bounds__(256) void quantize_kernel(QuantArgs a) {
  typedef Block<T> B;
  __shared__ TileShared<T> lds;
  const int t = threadIdx.x, cg = t & 15, u = t >> 4;
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
  write_tile<T, GROUP>(x, a.rows, a.cols, I, J, a.q, a.qt, lds);
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
