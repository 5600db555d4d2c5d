// AdamW over many tensors in one launch (formulas in zf_layer.h).
//
// A 256-thread block takes a chunk of 1024 consecutive elements of one tensor, 4
// a lane; the plan's table of block offsets says which.  (202 M elements in us,
// chunks of 1024 / 2048 / 4096: 8-bit states 538 / 565 / 567, 32-bit 960 / 990 /
// 1013.  Remapping blocks to XCDs changes nothing: no line is shared.)  32 lanes
// hold one 128-element block of the 8-bit states, so that every stream is read
// and written in contiguous lines: its largest magnitudes are taken over those
// lanes and the codes written in the same pass.  Bound by HBM: 28 bytes per
// element with a bf16 gradient, a bf16 weight and 32-bit states (5.9 TB/s), 16
// with 8-bit states (6.0 TB/s).
#include "zf_layer.hpp"

namespace zf {
namespace {

// Four elements of a stream that is read and written once, at any element
// alignment.  FULL: all four exist; else those at and past `valid` are zeros,
// neither read nor written.
template <bool FULL>
__device__ __forceinline__ void get4(const float* p, int64_t valid, float (&v)[4]) {
  if (FULL || valid >= 4) {
    const u32x4 u = __builtin_nontemporal_load(reinterpret_cast<const u32x4_f*>(p));
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(u[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = j < valid ? p[j] : 0.0f;
  }
}
template <bool FULL>
__device__ __forceinline__ void get4(const uint16_t* p, int64_t valid, float (&v)[4]) {
  if (FULL || valid >= 4) {
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
template <bool FULL>
__device__ __forceinline__ void put4(float* p, int64_t valid, const float (&v)[4]) {
  if (FULL || valid >= 4) {
    __builtin_nontemporal_store(u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]),
                                      __float_as_uint(v[2]), __float_as_uint(v[3])},
                                reinterpret_cast<u32x4_f*>(p));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < valid) p[j] = v[j];
  }
}
template <bool FULL>
__device__ __forceinline__ void put4(uint16_t* p, int64_t valid, const float (&v)[4]) {
  const u32x2 u = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  if (FULL || valid >= 4) {
    store4_bf16(p, u);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < valid) p[j] = static_cast<uint16_t>(u[j >> 1] >> (16 * (j & 1)));
  }
}

typedef uint32_t u32_b __attribute__((aligned(1)));
template <bool FULL>
__device__ __forceinline__ uint32_t get_codes(const uint8_t* p, int64_t valid) {
  if (FULL || valid >= 4) return __builtin_nontemporal_load(reinterpret_cast<const u32_b*>(p));
  uint32_t u = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < valid) u |= static_cast<uint32_t>(p[j]) << (8 * j);
  return u;
}
template <bool FULL>
__device__ __forceinline__ void put_codes(uint8_t* p, int64_t valid, uint32_t u) {
  if (FULL || valid >= 4) {
    __builtin_nontemporal_store(u, reinterpret_cast<u32_b*>(p));
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < valid) p[j] = static_cast<uint8_t>(u >> (8 * j));
}

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
    // (a byte of u is zero: rare, but for values that are zero)
    if (((u - 0x01010101u) & ~u & 0x80808080u) != 0 && inv > 0.0f) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (((u >> (8 * j)) & 0xffu) == 0 && x[j] > 0.0f) u |= 1u << (8 * j);
    }
  }
  return u;
}

// Correctly rounded square roots of x in [2^-96, 2^100): the hardware's reciprocal
// root and one step of Newton's on the remainder, 6 instructions where the general
// sequence, which scales its operand first, takes 18.  (Equal to sqrtf() for each
// of the 1.64e9 floats of that range.)
constexpr uint32_t kRootLow = 0x0f800000u, kRootHigh = 0x71800000u;  // 2^-96, 2^100
__device__ __forceinline__ float root_in_range(float x) {
  const float s = __builtin_amdgcn_rsqf(x);
  const float y = x * s, h = 0.5f * s;
  return __builtin_fmaf(__builtin_fmaf(-y, y, x), h, y);
}
__device__ __forceinline__ void roots4(const float (&x)[4], float (&r)[4]) {
  uint32_t lo = ~0u, hi = 0u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    lo = min(lo, __float_as_uint(x[j]));
    hi = max(hi, __float_as_uint(x[j]));
  }
  if (lo >= kRootLow && hi < kRootHigh) {
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = root_in_range(x[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = sqrtf(x[j]);
  }
}

// adam_step() for four elements, operation for operation.
__device__ __forceinline__ void adam_step4(const float (&g)[4], float (&p)[4], float (&m)[4],
                                           float (&v)[4], const AdamK& c) {
  float x[4], r[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m[j] = c.b1 * m[j] + c.c1 * g[j];
    v[j] = c.b2 * v[j] + c.c2 * (g[j] * g[j]);
    x[j] = v[j] * c.ib2;
  }
  roots4(x, r);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float u = (m[j] * c.ib1) / (r[j] + c.eps);
    if (c.wd != 0.0f) p[j] = p[j] - c.wd * p[j];
    p[j] = p[j] - c.lr * u;
  }
}

// Guarded at every load and store: without that the compiler moves all loads to
// the front, and the kernel is 4 % slower (1008 us, not 960, on the 202 M elements).
template <typename G>
__device__ __forceinline__ void adamw_f32(const AdamTensor& t, int64_t i, const AdamK& c,
                                          float gs, bool scaled) {
  float g[4], p[4], m[4], v[4];
  float* const mp = static_cast<float*>(t.m) + i;
  float* const vp = static_cast<float*>(t.v) + i;
  const int64_t left = t.n - i;
  get4<false>(static_cast<const G*>(t.grad) + i, left, g);
  get4<false>(t.master + i, left, p);
  get4<false>(mp, left, m);
  get4<false>(vp, left, v);
#pragma unroll
  for (int j = 0; j < 4; ++j) adam_step(scaled ? g[j] * gs : g[j], p[j], m[j], v[j], c);
  put4<false>(t.master + i, left, p);
  put4<false>(mp, left, m);
  put4<false>(vp, left, v);
  if (t.weight != nullptr) put4<false>(t.weight + i, left, p);
}

// FULL: the tensor holds the block's whole chunk.
template <typename G, bool FULL>
__device__ __forceinline__ void adamw_8bit(const AdamTensor& t, int64_t i, const AdamK& c,
                                           float gs, bool scaled) {
  float g[4], p[4], m[4], v[4], root[4];
  uint8_t* const mp = static_cast<uint8_t*>(t.m) + i;
  uint8_t* const vp = static_cast<uint8_t*>(t.v) + i;
  const int64_t left = t.n - i, block = i / 128;
  get4<FULL>(static_cast<const G*>(t.grad) + i, left, g);
  get4<FULL>(t.master + i, left, p);
  decode4(get_codes<FULL>(mp, left), FULL || left > 0 ? t.ms[block] : 0.0f, m);
  decode4(get_codes<FULL>(vp, left), FULL || left > 0 ? t.vs[block] : 0.0f, v);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = v[j] * v[j];
    if (scaled) g[j] *= gs;
  }
  adam_step4(g, p, m, v, c);
  roots4(v, root);
  if constexpr (!FULL) {  // elements past the end count as zeros
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j >= left) m[j] = root[j] = 0.0f;
  }
  put4<FULL>(t.master + i, left, p);
  if (t.weight != nullptr) put4<FULL>(t.weight + i, left, p);
  float sm, sv;
  const uint32_t um = encode4<false>(m, &sm), uv = encode4<true>(root, &sv);
  put_codes<FULL>(mp, left, um);
  put_codes<FULL>(vp, left, uv);
  if ((threadIdx.x & 31) == 0 && (FULL || left > 0)) {
    t.ms[block] = sm;
    t.vs[block] = sv;
  }
}

template <typename G>
__device__ __forceinline__ void adamw_chunk(const AdamTensor& t, int64_t base, const AdamK& c,
                                            float gs, bool scaled) {
  const int64_t i = base + threadIdx.x * 4;
  if (t.ms == nullptr) adamw_f32<G>(t, i, c, gs, scaled);
  else if (base + kAdamwChunk <= t.n) adamw_8bit<G, true>(t, i, c, gs, scaled);
  else adamw_8bit<G, false>(t, i, c, gs, scaled);
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
  const int64_t base = (b - o[lo]) * kAdamwChunk;
  const bool scaled = grad_scale != nullptr;
  const float gs = scaled ? *grad_scale : 1.0f;
  if (t.grad_f32) adamw_chunk<float>(t, base, c, gs, scaled);
  else adamw_chunk<uint16_t>(t, base, c, gs, scaled);
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
