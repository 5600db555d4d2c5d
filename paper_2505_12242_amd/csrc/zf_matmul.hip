// Matrix product of two 8-bit operands with a scale for each 128 elements of
// the reduction (formulas and format in zf_layer.h).
//
// out[i][j] = sum over groups g of 2^(ca[i][g] + cb[j][g] - 254) * sum over
// the group of a * b.
#include "zf_layer.hpp"

namespace zf {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

constexpr int kBK = 128;  // reduction per step: one scale group

// Tiles in units of 16 bytes: unit c of row r lies at this byte of the tile.
// 16 consecutive rows reading one unit meet all 64 banks once.
__device__ __forceinline__ int tile_off(int r, int c) {
  return r * kBK + ((c ^ ((r >> 1) & 7)) << 4);
}

// One 32 x 32 tile of the accumulator: += x y^T over 64 elements of the
// reduction, of which a lane holds 32 of row lane % 32 (x: the tile's
// registers, y: its lanes).  Two forms:
//   fast     the scaled 8-bit instruction.  It aligns 64 products to the
//            largest of them and cuts what lies below 2^-13 of it (measured:
//            1.3e-5 relative on normal data), far below the 2^-4 that e4m3
//            itself cut and the 2^-9 of a bf16 result.
//   precise  elements and scale to bf16 (exact), products and sums in fp32
//            (7e-9 relative), at 0.42 of the rate.  Taken for fp32 results.
template <bool PRECISE>
struct Operand;
template <>
struct Operand<false> {
  v8i v;
  __device__ __forceinline__ void set(u32x4 x, u32x4 y, int) {
    v = v8i{(int)x.x, (int)x.y, (int)x.z, (int)x.w, (int)y.x, (int)y.y, (int)y.z, (int)y.w};
  }
};
template <>
struct Operand<true> {
  v8b v[4];
  __device__ __forceinline__ void set(u32x4 x, u32x4 y, int scale) {
    const float s = __uint_as_float(static_cast<uint32_t>(scale & 255) << 23);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t lo = q < 2 ? x[2 * q] : y[2 * q - 4], hi = q < 2 ? x[2 * q + 1] : y[2 * q - 3];
      const v2b a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false);
      const v2b b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true);
      const v2b c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false);
      const v2b d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true);
      v[q] = v8b{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
  }
};
__device__ __forceinline__ v16f mma(const Operand<false>& x, int sx, const Operand<false>& y, int sy,
                                    v16f acc) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x.v, y.v, acc, 0, 0, 0, sx, 0, sy);
}
__device__ __forceinline__ v16f mma(const Operand<true>& x, int, const Operand<true>& y, int,
                                    v16f acc) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.v[q], y.v[q], acc, 0, 0, 0);
  return acc;
}

// Stores 8 results of a row.
__device__ __forceinline__ void put8(void* out, int64_t at, int64_t valid, bool f32,
                                     const float (&v)[8]) {
  if (f32) store8(static_cast<float*>(out) + at, valid, v);
  else store8(static_cast<uint16_t*>(out) + at, valid, v);
}

// A 256-thread block computes a BM x BN tile, each wave a quarter of it, with
// two stages of 128 elements of the reduction in LDS.  Rows past an operand's
// end repeat its last row (their results are not stored); the units past the
// reduction's end repeat the row's last one and are cleared in LDS.
template <int BM, int BN, bool PRECISE>
__global__ __launch_bounds__(256, 1) void matmul_tile_kernel(MatmulArgs p) {
  constexpr int WM = BM / 2, WN = BN / 2, TM = WM / 32, TN = WN / 32;
  constexpr int kStage = (BM + BN) * kBK;
  constexpr int UA = BM / 32, UB = BN / 32;  // loads of 8 rows a wave issues per stage
  __shared__ __align__(1024) uint8_t lds[2 * kStage];
  const int t = threadIdx.x, lane = t & 63, wave = uniform_i32(t >> 6);
  const int wm = (wave & 1) * WM, wn = (wave >> 1) * WN;
  const uint32_t nt = static_cast<uint32_t>((p.n + BN - 1) / BN);
  const uint32_t mi = uniform_i32(blockIdx.x / nt);
  const int64_t m0 = static_cast<int64_t>(mi) * BM;
  const int64_t n0 = static_cast<int64_t>(blockIdx.x - mi * nt) * BN;
  const int steps = static_cast<int>((p.k + kBK - 1) / kBK);
  const int tail = static_cast<int>(p.k % kBK);

  const rsrc_t ra = make_rsrc(p.a.data + m0 * p.a.ld, -1), rb = make_rsrc(p.b.data + n0 * p.b.ld, -1);
  uint32_t row_a[UA], row_b[UB];
#pragma unroll
  for (int i = 0; i < UA; ++i)
    row_a[i] = static_cast<uint32_t>(min<int64_t>(8 * (wave + 4 * i) + (lane >> 3), p.m - 1 - m0)) *
               static_cast<uint32_t>(p.a.ld);
#pragma unroll
  for (int i = 0; i < UB; ++i)
    row_b[i] = static_cast<uint32_t>(min<int64_t>(8 * (wave + 4 * i) + (lane >> 3), p.n - 1 - n0)) *
               static_cast<uint32_t>(p.b.ld);

  // One stage from memory to LDS, 16 bytes a lane: the lane's place in LDS is
  // fixed, so it loads the unit that tile_off puts there.
  const auto load_stage = [&](int kt) {
    const int soff = kt * kBK;
    const uint32_t last = kt + 1 == steps && tail ? ((tail + 15) / 16 - 1) * 16u : 112u;
    uint8_t* const s = lds + (kt & 1) * kStage;
#pragma unroll
    for (int i = 0; i < UA + UB; ++i) {
      const bool a = i < UA;
      const int unit = wave + 4 * (a ? i : i - UA);
      const uint32_t c = ((lane & 7) ^ ((4 * unit + (lane >> 4)) & 7)) << 4;
      const uint32_t voff = (a ? row_a[a ? i : 0] : row_b[a ? 0 : i - UA]) + min(c, last);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          a ? ra : rb,
          (__attribute__((address_space(3))) void*)(s + (a ? 0 : BM * kBK) + unit * 1024), 16, voff,
          soff, 0, 0);
    }
  };
  // The stage's bytes past the reduction's end cleared (its last step only).
  const auto clear_stage = [&](int kt) {
    uint8_t* const s = lds + (kt & 1) * kStage;
    for (int r = t; r < BM + BN; r += 256) {
      const int rr = r < BM ? r : r - BM;
      uint8_t* const base = s + (r < BM ? 0 : BM * kBK);
      for (int c = tail / 16; c < 8; ++c) {
        u32x4* const u = reinterpret_cast<u32x4*>(base + tile_off(rr, c));
        u32x4 v = *u;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int n = tail - 16 * c - 4 * w;  // bytes of this word that count
          v[w] = n >= 4 ? v[w] : n <= 0 ? 0u : v[w] & ((1u << (8 * n)) - 1u);
        }
        *u = v;
      }
    }
    __syncthreads();
  };

  // Codes of four steps at a time, one word a row.
  const uint8_t* sa_row[TM];
  const uint8_t* sb_row[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t r = min<int64_t>(m0 + wm + 32 * i + (lane & 31), p.m - 1);
    sa_row[i] = p.a.scale + (r >> p.a.shift) * p.a.ld_scale;
  }
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int64_t r = min<int64_t>(n0 + wn + 32 * j + (lane & 31), p.n - 1);
    sb_row[j] = p.b.scale + (r >> p.b.shift) * p.b.ld_scale;
  }
  uint32_t wa[TM], wb[TN];
  const auto load_codes = [&](int kt) {
#pragma unroll
    for (int i = 0; i < TM; ++i) wa[i] = *reinterpret_cast<const uint32_t*>(sa_row[i] + (kt & ~3));
#pragma unroll
    for (int j = 0; j < TN; ++j) wb[j] = *reinterpret_cast<const uint32_t*>(sb_row[j] + (kt & ~3));
  };

  v16f acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

  if (steps > 0) {
    load_codes(0);
    load_stage(0);
  }
  for (int kt = 0; kt < steps; ++kt) {
    __syncthreads();
    if (kt + 1 == steps && tail) clear_stage(kt);
    if (kt > 0 && (kt & 3) == 0) load_codes(kt);
    if (kt + 1 < steps) load_stage(kt + 1);
    const int sh = 8 * (kt & 3);
    const uint8_t* const s = lds + (kt & 1) * kStage;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = 4 * h + 2 * (lane >> 5);
      Operand<PRECISE> fa[TM], fb[TN];
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int r = wm + 32 * i + (lane & 31);
        fa[i].set(*reinterpret_cast<const u32x4*>(s + tile_off(r, c)),
                  *reinterpret_cast<const u32x4*>(s + tile_off(r, c + 1)), wa[i] >> sh);
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int r = wn + 32 * j + (lane & 31);
        fb[j].set(*reinterpret_cast<const u32x4*>(s + BM * kBK + tile_off(r, c)),
                  *reinterpret_cast<const u32x4*>(s + BM * kBK + tile_off(r, c + 1)), wb[j] >> sh);
      }
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = mma(fb[j], wb[j] >> sh, fa[i], wa[i] >> sh, acc[i][j]);
    }
  }

  // A lane holds 4 consecutive columns of a row at a time; through LDS, 32
  // rows of the wave's tile at a time, the rows become contiguous.
  __syncthreads();
  constexpr int kPitch = WN + 4;  // floats
  static_assert(4 * 32 * kPitch * 4 <= 2 * kStage, "the waves' slabs fit the stages");
  float* const slab = reinterpret_cast<float*>(lds) + wave * 32 * kPitch;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int col = 32 * j + 2 * e + 4 * (lane >> 5);
        *reinterpret_cast<float4*>(slab + (lane & 31) * kPitch + col) =
            float4{acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int u = lane; u < 32 * (WN / 8); u += 64) {
      const int r = u / (WN / 8), c = u % (WN / 8) * 8;
      float v[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = slab[r * kPitch + c + q];
      const int64_t row = m0 + wm + 32 * i + r, col = n0 + wn + c;
      if (row < p.m) put8(p.out, row * p.ld_out + col, p.n - col, p.out_f32, v);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace

size_t matmul_workspace(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_matmul(const MatmulArgs& a, void*, hipStream_t s) {
  (void)hipGetLastError();
  const auto tiles = [&](int bm, int bn) {
    return dim3(static_cast<uint32_t>(((a.m + bm - 1) / bm) * ((a.n + bn - 1) / bn)));
  };
  if (a.out_f32)
    hipLaunchKernelGGL((matmul_tile_kernel<128, 128, true>), tiles(128, 128), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((matmul_tile_kernel<128, 128, false>), tiles(128, 128), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace zf
