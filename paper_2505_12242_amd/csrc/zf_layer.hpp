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
constexpr int kAdamwChunk = 1024;  // elements per block
hipError_t launch_adamw(const AdamTensor* tensors, const int64_t* off, int32_t count,
                        int64_t blocks, const AdamK& c, const float* grad_scale, hipStream_t s);


// ---- device helpers --------------------------------------------------------

// fp32 elements at any 4-byte alignment, 16 bytes a lane (see u32x4_h for bf16).
typedef u32x4 u32x4_f __attribute__((aligned(4)));

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Two values to bf16, to nearest, ties to even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// Eight elements as they are stored: loaded and stored with as few accesses as
// any element alignment allows, widened where they are used.  Elements at and
// past `valid` are zeros, neither read nor written.  NT: read or written once.
//
// A row's last, partial piece is read as 4, 2 and 1 elements, as the bits of
// `valid` say, and put in order by settle(), which is where they are waited for:
// load() is fetch() and settle().  (Element by element, each load waited for the
// one before: 8192 rows of 5004 bf16 columns took 91 us, of 5120 columns 62.)
template <typename T>
struct Vec8;

typedef uint32_t u32_h __attribute__((aligned(2)));
typedef u32x2 u32x2_f __attribute__((aligned(4)));
template <>
struct Vec8<uint16_t> {
  u32x4 u;
  template <bool NT = false>
  __device__ __forceinline__ void fetch(const uint16_t* p, int64_t valid) {
    if (valid >= 8) {
      u = NT ? load8_bf16(p) : *reinterpret_cast<const u32x4_h*>(p);
    } else {
      u = u32x4{0, 0, 0, 0};
      if (valid <= 0) return;
      if (valid & 4) {
        const u32x2 t = *reinterpret_cast<const u32x2_h*>(p);
        u.x = t.x;
        u.y = t.y;
      }
      if (valid & 2) u.z = *reinterpret_cast<const u32_h*>(p + (valid & 4));
      if (valid & 1) u.w = p[valid - 1];
    }
  }
  __device__ __forceinline__ void settle(int64_t valid) {
    if (valid >= 8) return;
    const uint32_t t0 = valid & 2 ? u.z : u.w, t1 = valid & 2 ? u.w : 0u;
    u = valid & 4 ? u32x4{u.x, u.y, t0, t1} : u32x4{t0, t1, 0u, 0u};
  }
  template <bool NT = false>
  __device__ __forceinline__ void load(const uint16_t* p, int64_t valid) {
    fetch<NT>(p, valid);
    settle(valid);
  }
  template <bool NT = false>
  __device__ __forceinline__ void store(uint16_t* p, int64_t valid) const {
    if (valid >= 8) {
      if (NT) store8_bf16(p, u);
      else *reinterpret_cast<u32x4_h*>(p) = u;
    } else if (valid > 0) {
      if (valid & 4) *reinterpret_cast<u32x2_h*>(p) = u32x2{u.x, u.y};
      const uint32_t t0 = valid & 4 ? u.z : u.x, t1 = valid & 4 ? u.w : u.y;
      if (valid & 2) *reinterpret_cast<u32_h*>(p + (valid & 4)) = t0;
      if (valid & 1) p[valid - 1] = static_cast<uint16_t>(valid & 2 ? t1 : t0);
    }
  }
  __device__ __forceinline__ float operator[](int j) const {
    return __uint_as_float(j & 1 ? u[j >> 1] & 0xffff0000u : u[j >> 1] << 16);
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {  // rounded
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
  }
};

template <>
struct Vec8<float> {
  u32x4 u[2];
  template <bool NT = false>
  __device__ __forceinline__ void fetch(const float* p, int64_t valid) {
    if (valid >= 8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const u32x4_f* const q = reinterpret_cast<const u32x4_f*>(p + 4 * i);
        u[i] = NT ? __builtin_nontemporal_load(q) : *q;
      }
    } else {
      u[0] = u[1] = u32x4{0, 0, 0, 0};
      if (valid <= 0) return;
      if (valid & 4) u[0] = *reinterpret_cast<const u32x4_f*>(p);
      if (valid & 2) {
        const u32x2 t = *reinterpret_cast<const u32x2_f*>(p + (valid & 4));
        u[1].x = t.x;
        u[1].y = t.y;
      }
      if (valid & 1) u[1].z = __float_as_uint(p[valid - 1]);
    }
  }
  __device__ __forceinline__ void settle(int64_t valid) {
    if (valid >= 8) return;
    const bool four = (valid & 4) != 0, two = (valid & 2) != 0;
    const uint32_t t[4] = {two ? u[1].x : u[1].z, two ? u[1].y : 0u, two ? u[1].z : 0u, 0u};
#pragma unroll
    for (int j = 0; j < 4; ++j) {  // (element by element: whole vectors go through memory)
      const uint32_t a = u[0][j];
      u[0][j] = four ? a : t[j];
      u[1][j] = four ? t[j] : 0u;
    }
  }
  template <bool NT = false>
  __device__ __forceinline__ void load(const float* p, int64_t valid) {
    fetch<NT>(p, valid);
    settle(valid);
  }
  template <bool NT = false>
  __device__ __forceinline__ void store(float* p, int64_t valid) const {
    if (valid >= 8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        u32x4_f* const q = reinterpret_cast<u32x4_f*>(p + 4 * i);
        if (NT) __builtin_nontemporal_store(u[i], q);
        else *q = u[i];
      }
    } else if (valid > 0) {
      if (valid & 4) *reinterpret_cast<u32x4_f*>(p) = u[0];
      const bool four = (valid & 4) != 0;
      const uint32_t t0 = four ? u[1].x : u[0].x, t1 = four ? u[1].y : u[0].y,
                     t2 = four ? u[1].z : u[0].z;
      if (valid & 2) *reinterpret_cast<u32x2_f*>(p + (valid & 4)) = u32x2{t0, t1};
      if (valid & 1) p[valid - 1] = __uint_as_float(valid & 2 ? t2 : t0);
    }
  }
  __device__ __forceinline__ float operator[](int j) const {
    return __uint_as_float(u[j >> 2][j & 3]);
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j >> 2][j & 3] = __float_as_uint(v[j]);
  }
};

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
// The larger 16-bit integers of each pair.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                __builtin_bit_cast(u16x2, b)));
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
// Four values of magnitude <= 448 (plus rounding) to e4m3, ties to even.
__device__ __forceinline__ uint32_t pack_fp8(float a, float b, float c, float d) {
  const int u = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, u, true));
}

// The scale of a code, as the conversions below take it (its exponent bits).
__device__ __forceinline__ float fp8_scale(uint32_t code) { return __uint_as_float(code << 23); }

// Eight values of a group over its scale to e4m3, to nearest, ties to even;
// zeros where the group holds an infinity or a NaN.
typedef short i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 quant8(const float (&v)[8], uint32_t code) {
  const float s = fp8_scale(code);
  u32x2 u;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    i16x2 q = {0, 0};
    q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, v[4 * i], v[4 * i + 1], s, false);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, v[4 * i + 2], v[4 * i + 3], s, true);
    u[i] = __builtin_bit_cast(uint32_t, q);
  }
  return code == 255u ? u32x2{0u, 0u} : u;
}
// The same of bf16 values, two a word.
__device__ __forceinline__ u32x2 quant8_bf16(uint32_t a, uint32_t b, uint32_t c, uint32_t d,
                                             uint32_t code) {
  const float s = fp8_scale(code);
  i16x2 q = {0, 0}, r = {0, 0};
  q = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q, __builtin_bit_cast(bf16x2, a), s, false);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q, __builtin_bit_cast(bf16x2, b), s, true);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, c), s, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, d), s, true);
  const u32x2 u = {__builtin_bit_cast(uint32_t, q), __builtin_bit_cast(uint32_t, r)};
  return code == 255u ? u32x2{0u, 0u} : u;
}

// A group's magnitudes, and its elements in 8 bits.
template <typename T>
__device__ __forceinline__ uint32_t abs_max(const Vec8<T>& v) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, abs_bits(v[j]));
  return m;
}
__device__ __forceinline__ u32x2 quant8(const Vec8<uint16_t>& v, uint32_t code) {
  return quant8_bf16(v.u[0], v.u[1], v.u[2], v.u[3], code);
}
__device__ __forceinline__ u32x2 quant8(const Vec8<float>& v, uint32_t code) {
  const float w[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
  return quant8(w, code);
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
