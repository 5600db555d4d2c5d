// AdamW over many tensors in one launch (formulas in zf_layer.h).
//
// A 256-thread block takes a chunk of consecutive elements of one tensor, 2048 of
// one with 8-bit states, 1024 of one with 32-bit states; the plan's table of block
// offsets says which.  (202 M elements in us, chunks of 1024 / 2048 / 4096: 8-bit
// 618 / 587 / 637, 32-bit 941 / 990 / 1013.  Remapping blocks to XCDs changes
// nothing: no line is shared.)  32 lanes hold one 128-element
// block of the 8-bit states, 4 elements a lane, so that every stream is read
// and written in contiguous lines: its largest magnitudes are taken over those
// lanes and the codes written in the same pass.  Bound by HBM: 28 bytes per
// element with a bf16 gradient, a bf16 weight and 32-bit states, 16 with 8-bit
// states.
#include "zf_layer.hpp"

namespace zf {
namespace {

__device__ __forceinline__ u32x4 load4_f32(const float* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4_f*>(p));
}
__device__ __forceinline__ void store4_f32(float* p, u32x4 v) {
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4_f*>(p));
}

// p[0 .. min(valid, 4)) as fp32, the rest 0.
__device__ __forceinline__ void get4(const float* p, int64_t valid, float (&v)[4]) {
  if (valid >= 4) {
    const u32x4 u = load4_f32(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(u[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = j < valid ? p[j] : 0.0f;
  }
}
__device__ __forceinline__ void get4(const uint16_t* p, int64_t valid, float (&v)[4]) {
  if (valid >= 4) {
    const u32x2 u = load4_bf16(p);
    v[0] = __uint_as_float(u.x << 16);
    v[1] = __uint_as_float(u.x & 0xffff0000u);
    v[2] = __uint_as_float(u.y << 16);
    v[3] = __uint_as_float(u.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = j < valid ? widen_bf16(p[j]) : 0.0f;
  }
}
__device__ __forceinline__ void put4(float* p, int64_t valid, const float (&v)[4]) {
  if (valid >= 4) {
    store4_f32(p, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                        __float_as_uint(v[3])});
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < valid) p[j] = v[j];
  }
}
__device__ __forceinline__ void put4(uint16_t* p, int64_t valid, const float (&v)[4]) {
  if (valid >= 4) {
    const uint32_t a = round_bf16(v[0]), b = round_bf16(v[1]), c = round_bf16(v[2]),
                   d = round_bf16(v[3]);
    store4_bf16(p, u32x2{a | (b << 16), c | (d << 16)});
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < valid) p[j] = round_bf16(v[j]);
  }
}

// Four codes at any alignment.
typedef uint32_t u32_b __attribute__((aligned(1)));
__device__ __forceinline__ uint32_t get_codes(const uint8_t* p, int64_t valid) {
  if (valid >= 4) return __builtin_nontemporal_load(reinterpret_cast<const u32_b*>(p));
  uint32_t u = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < valid) u |= static_cast<uint32_t>(p[j]) << (8 * j);
  return u;
}
__device__ __forceinline__ void put_codes(uint8_t* p, int64_t valid, uint32_t u) {
  if (valid >= 4) {
    __builtin_nontemporal_store(u, reinterpret_cast<u32_b*>(p));
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < valid) p[j] = static_cast<uint8_t>(u >> (8 * j));
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void decode4(uint32_t u, float scale, float (&v)[4]) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(u), false);
  const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(u), true);
  v[0] = a.x * scale;
  v[1] = a.y * scale;
  v[2] = b.x * scale;
  v[3] = b.y * scale;
}

__device__ __forceinline__ uint32_t max32(uint32_t x) {
  x = max16(x);
  return max(x, static_cast<uint32_t>(__shfl_xor(static_cast<int>(x), 16)));
}

// Codes of a lane's four of 128 values whose scale is *scale.  KEEP: what is
// not zero does not get code 0.
template <bool KEEP>
__device__ __forceinline__ uint32_t encode4(const float (&x)[4], float* scale) {
  uint32_t m = max(max(abs_bits(x[0]), abs_bits(x[1])), max(abs_bits(x[2]), abs_bits(x[3])));
  const float top = __uint_as_float(max32(m));
  if (top < 0x1p-100f) {
    *scale = 0.0f;
    return 0u;
  }
  const float inv = 448.0f / top;
  *scale = top / 448.0f;
  uint32_t u = pack_fp8(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  if constexpr (KEEP) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (((u >> (8 * j)) & 0xffu) == 0 && x[j] > 0.0f && inv > 0.0f) u |= 1u << (8 * j);
  }
  return u;
}

template <typename G>
__device__ __forceinline__ void adamw_f32(const AdamTensor& t, int64_t base, const AdamK& c,
                                          float gs, bool scaled) {
  constexpr int kQuads = kAdamwChunk32 / (256 * 4);
  float g[kQuads][4], p[kQuads][4], m[kQuads][4], v[kQuads][4];
  float* const mp = static_cast<float*>(t.m);
  float* const vp = static_cast<float*>(t.v);
#pragma unroll
  for (int q = 0; q < kQuads; ++q) {
    const int64_t i = base + (threadIdx.x + q * 256) * 4;
    get4(static_cast<const G*>(t.grad) + i, t.n - i, g[q]);
    get4(t.master + i, t.n - i, p[q]);
    get4(mp + i, t.n - i, m[q]);
    get4(vp + i, t.n - i, v[q]);
  }
#pragma unroll
  for (int q = 0; q < kQuads; ++q) {
    const int64_t i = base + (threadIdx.x + q * 256) * 4;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      adam_step(scaled ? g[q][j] * gs : g[q][j], p[q][j], m[q][j], v[q][j], c);
    put4(t.master + i, t.n - i, p[q]);
    put4(mp + i, t.n - i, m[q]);
    put4(vp + i, t.n - i, v[q]);
    if (t.weight != nullptr) put4(t.weight + i, t.n - i, p[q]);
  }
}

template <typename G>
__device__ __forceinline__ void adamw_8bit(const AdamTensor& t, int64_t base, const AdamK& c,
                                           float gs, bool scaled) {
  constexpr int kQuads = kAdamwChunk8 / (256 * 4);
  float g[kQuads][4], p[kQuads][4], ms[kQuads], vs[kQuads];
  uint32_t mq[kQuads], vq[kQuads];
  uint8_t* const mp = static_cast<uint8_t*>(t.m);
  uint8_t* const vp = static_cast<uint8_t*>(t.v);
#pragma unroll
  for (int q = 0; q < kQuads; ++q) {
    const int64_t i = base + (threadIdx.x + q * 256) * 4;
    get4(static_cast<const G*>(t.grad) + i, t.n - i, g[q]);
    get4(t.master + i, t.n - i, p[q]);
    mq[q] = get_codes(mp + i, t.n - i);
    vq[q] = get_codes(vp + i, t.n - i);
    ms[q] = i < t.n ? t.ms[i / 128] : 0.0f;
    vs[q] = i < t.n ? t.vs[i / 128] : 0.0f;
  }
#pragma unroll
  for (int q = 0; q < kQuads; ++q) {
    const int64_t i = base + (threadIdx.x + q * 256) * 4;
    float m[4], v[4];
    decode4(mq[q], ms[q], m);
    decode4(vq[q], vs[q], v);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = v[j] * v[j];
      adam_step(scaled ? g[q][j] * gs : g[q][j], p[q][j], m[j], v[j], c);
      // the square root of the new second moment; elements past the end count as zeros
      v[j] = j < t.n - i ? sqrtf(v[j]) : 0.0f;
      m[j] = j < t.n - i ? m[j] : 0.0f;
    }
    put4(t.master + i, t.n - i, p[q]);
    if (t.weight != nullptr) put4(t.weight + i, t.n - i, p[q]);
    float sm, sv;
    const uint32_t um = encode4<false>(m, &sm), uv = encode4<true>(v, &sv);
    put_codes(mp + i, t.n - i, um);
    put_codes(vp + i, t.n - i, uv);
    if ((threadIdx.x & 31) == 0 && i < t.n) {
      t.ms[i / 128] = sm;
      t.vs[i / 128] = sv;
    }
  }
}

__global__ __launch_bounds__(256) void adamw_kernel(const AdamTensor* __restrict__ tensors,
                                                    const int64_t* __restrict__ off,
                                                    int32_t count, AdamK c,
                                                    const float* __restrict__ grad_scale) {
  const int64_t b = blockIdx.x;
  const auto* o = const_table(off);
  int lo = 0, hi = count - 1;
  while (lo < hi) {  // largest q with off[q] <= b
    const int mid = (lo + hi + 1) >> 1;
    if (o[mid] <= b) lo = mid; else hi = mid - 1;
  }
  AdamTensor t;
  {
    const auto* s = const_table(tensors) + lo;
    t.n = s->n;
    t.grad = s->grad;
    t.master = s->master;
    t.weight = s->weight;
    t.m = s->m;
    t.v = s->v;
    t.ms = s->ms;
    t.vs = s->vs;
    t.grad_f32 = s->grad_f32;
  }
  const int64_t base = (b - o[lo]) * (t.ms != nullptr ? kAdamwChunk8 : kAdamwChunk32);
  const bool scaled = grad_scale != nullptr;
  const float gs = scaled ? *grad_scale : 1.0f;
  if (t.ms != nullptr) {
    if (t.grad_f32) adamw_8bit<float>(t, base, c, gs, scaled);
    else adamw_8bit<uint16_t>(t, base, c, gs, scaled);
  } else {
    if (t.grad_f32) adamw_f32<float>(t, base, c, gs, scaled);
    else adamw_f32<uint16_t>(t, base, c, gs, scaled);
  }
}

}  // namespace

hipError_t launch_adamw(const AdamTensor* tensors, const int64_t* off, int32_t count,
                        int64_t blocks, const AdamK& c, const float* grad_scale, hipStream_t s) {
  (void)hipGetLastError();
  hipLaunchKernelGGL(adamw_kernel, dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, s, tensors,
                     off, count, c, grad_scale);
  return hipGetLastError();
}

}  // namespace zf
