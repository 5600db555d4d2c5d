// Internal types of the operators of include/zf_layer.h, shared by their host
// entry points (zf_layer_api.hip) and kernels.
#pragma once

#include "zf_device.hpp"
#include "zf_layer.h"

namespace zf {

zf_status hip_fail(hipError_t e);  // keeps the code for zf_last_hip_error

constexpr int kFp8Group = 128;  // elements that share a scale along a row

// An 8-bit operand as the kernels see it; data == nullptr: not wanted.
struct Fp8Out {
  uint8_t* data;
  int64_t ld;
  uint8_t* scale;
  int64_t ld_scale;
};

struct QuantArgs {
  const void* x;
  int64_t rows, cols, ld_x;
  Fp8Out q, qt;
};
hipError_t launch_quantize(const QuantArgs& a, int32_t dtype, int32_t group, hipStream_t s);

struct MatmulOperand {
  const uint8_t* data;
  int64_t ld;
  const uint8_t* scale;
  int64_t ld_scale;
  int32_t shift;  // row >> shift is the scale's row (0 or 7)
};
struct MatmulArgs {
  MatmulOperand a, b;
  int64_t m, n, k;
  void* out;
  int64_t ld_out;
  int32_t out_f32;
  int32_t share;  // steps of one share of the reduction, where it is split
};
size_t matmul_workspace(int64_t m, int64_t n, int64_t k);
hipError_t launch_matmul(const MatmulArgs& a, void* ws, hipStream_t s);

struct NormArgs {
  const void* x;
  int64_t ld_x;
  const void* residual;
  int64_t ld_residual;
  int64_t rows, cols;
  const void* gain;
  int32_t gain_f32;
  float eps;
  void* h;
  int64_t ld_h;
  void* y;
  int64_t ld_y;
  Fp8Out q;
  float* rstd;
};
hipError_t launch_rmsnorm(const NormArgs& a, int32_t dtype, hipStream_t s);

struct NormBwdArgs {
  const void* dy;
  int64_t ld_dy;
  const void* h;
  int64_t ld_h;
  int64_t rows, cols;
  const void* gain;
  int32_t gain_f32;
  const float* rstd;
  const void* dres;
  int64_t ld_dres;
  void* dx;
  int64_t ld_dx;
  float* dgain;
  float* part;
};
size_t rmsnorm_backward_workspace(int64_t rows, int64_t cols);
hipError_t launch_rmsnorm_backward(const NormBwdArgs& a, int32_t dtype, hipStream_t s);

// AdamW: one tensor of a plan's device table.
struct AdamTensor {
  int64_t n;
  const void* grad;
  float* master;
  uint16_t* weight;
  void* m;
  void* v;
  float* ms;  // nullptr: 32-bit states
  float* vs;
  int32_t grad_f32;
  int32_t pad;
};
constexpr int kAdamwChunk = 4096;  // elements per block
hipError_t launch_adamw(const AdamTensor* tensors, const int64_t* off, int32_t count,
                        int64_t blocks, const AdamK& c, const float* grad_scale, hipStream_t s);


// ---- device helpers --------------------------------------------------------

// fp32 elements at any 4-byte alignment, 16 bytes a lane (see u32x4_h for bf16).
typedef u32x4 u32x4_f __attribute__((aligned(4)));

// Elements p[0 .. 8) as fp32; those at and past `valid` are 0 and not read.
__device__ __forceinline__ void load8(const uint16_t* p, int64_t valid, float (&v)[8]) {
  if (valid >= 8) {
    const u32x4 u = *reinterpret_cast<const u32x4_h*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < valid ? widen_bf16(p[i]) : 0.0f;
  }
}
__device__ __forceinline__ void load8(const float* p, int64_t valid, float (&v)[8]) {
  if (valid >= 8) {
    const u32x4 a = *reinterpret_cast<const u32x4_f*>(p);
    const u32x4 b = *reinterpret_cast<const u32x4_f*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = __uint_as_float(a[i]);
      v[4 + i] = __uint_as_float(b[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < valid ? p[i] : 0.0f;
  }
}

// v rounded to the type of p and stored at p[0 .. min(valid, 8)).
__device__ __forceinline__ void store8(uint16_t* p, int64_t valid, const float (&v)[8]) {
  if (valid >= 8) {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      u[i] = round_bf16(v[2 * i]) | (static_cast<uint32_t>(round_bf16(v[2 * i + 1])) << 16);
    *reinterpret_cast<u32x4_h*>(p) = u;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < valid) p[i] = round_bf16(v[i]);
  }
}
__device__ __forceinline__ void store8(float* p, int64_t valid, const float (&v)[8]) {
  if (valid >= 8) {
    u32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = __float_as_uint(v[i]);
      b[i] = __float_as_uint(v[4 + i]);
    }
    *reinterpret_cast<u32x4_f*>(p) = a;
    *reinterpret_cast<u32x4_f*>(p + 4) = b;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < valid) p[i] = v[i];
  }
}

// A value as its storage type holds it.
__device__ __forceinline__ float as_stored(const uint16_t*, float v) {
  return widen_bf16(round_bf16(v));
}
__device__ __forceinline__ float as_stored(const float*, float v) { return v; }

// The largest x of the calling lane's 16 (lanes 16i .. 16i + 15), in each of
// them.  Magnitudes are compared as bit patterns, in which a NaN is largest.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return __builtin_amdgcn_update_dpp(0u, x, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ uint32_t max16(uint32_t x) {
  x = max(x, dpp<0x128>(x));  // row_ror 8, 4, 2, 1
  x = max(x, dpp<0x124>(x));
  x = max(x, dpp<0x122>(x));
  return max(x, dpp<0x121>(x));
}
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// The e8m0 code of a group whose largest magnitude has these bits: the least
// code with magnitude <= 448 * 2^(code - 127).  448 = 1.75 * 2^8: the sum
// carries into the exponent iff the mantissa is above 1.75.
__device__ __forceinline__ uint32_t fp8_code(uint32_t bits) {
  if (bits >= 0x7f800000u) return 255u;
  const uint32_t e = (bits + 0x1fffffu) >> 23;
  return e > 8u ? e - 8u : 0u;
}
// What a group's elements are multiplied by: 2^(127 - code), an exact
// operation but for results below 2^-126, which round to code 0 either way.
__device__ __forceinline__ float fp8_mult(uint32_t code) {
  return __uint_as_float((254u - (code < 255u ? code : 254u)) << 23);
}

// Four values of magnitude <= 448 (plus rounding) to e4m3, ties to even.
__device__ __forceinline__ uint32_t pack_fp8(float a, float b, float c, float d) {
  int u = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, u, true));
}

// Eight values of a group to e4m3 codes.
__device__ __forceinline__ u32x2 quant8(const float (&v)[8], uint32_t code) {
  const float f = fp8_mult(code);
  u32x2 u;
  u.x = pack_fp8(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
  u.y = pack_fp8(v[4] * f, v[5] * f, v[6] * f, v[7] * f);
  if (code == 255u) u = u32x2{0u, 0u};
  return u;
}

// Bytes p[0 .. min(valid, 8)); p is 8-byte aligned.
__device__ __forceinline__ void store_bytes8(uint8_t* p, int64_t valid, u32x2 u) {
  if (valid >= 8) {
    *reinterpret_cast<u32x2*>(p) = u;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < valid) p[i] = static_cast<uint8_t>((i < 4 ? u.x : u.y) >> (8 * (i & 3)));
  }
}

}  // namespace zf
