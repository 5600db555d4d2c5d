// Shared by the attention kernels (formulas in zf_layer.h).
//
// Rows.  The query heads of one key head are rows of the same products: row r
// of a sequence is query token r / group, head r % group of the key head's
// `group` query heads.  A single token of a model with 8 query heads to a key
// head is 8 rows over one read of the cache, and the gradients of k and v sum
// over the heads inside the products.
//
// Products.  32 x 32 x 16 bf16 products with fp32 sums.  A lane holds 8
// consecutive elements of row lane % 32 of either operand, half = lane / 32
// saying which 8 of the 16; of the result it holds column lane % 32, rows
// 8 (r / 4) + 4 half + r % 4 in registers r = 0 .. 15.  So the result's
// registers 8 c .. 8 c + 7, rounded to bf16, are one operand of a product that
// sums over the rows 16 c .. 16 c + 15, taken in the order
// 4 half + {0 .. 3}, 8 + 4 half + {0 .. 3}: scores become weights of the next
// product where they stand.  The other operand has to come in the same order,
// transposed: two transposing reads of LDS, 4 rows each, give it (frag_t).
#pragma once

#include "zf_layer.hpp"

namespace zf {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v4b __attribute__((ext_vector_type(4)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

constexpr float kLog2E = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Rows of 8-element units (16 bytes) in LDS, as frag and frag_t read them.
// DP: the head's width rounded up to one of 64, 96, 128.
template <int DP>
struct Heads {
  static constexpr int kPitch = DP <= 64 ? 128 : 256;  // bytes of a row
  static constexpr int kUnits = kPitch / 16;
  static constexpr int kChunks = DP / 16;  // of a sum over the head's width
  static constexpr int kTiles = DP / 32;   // of a result that wide
  static constexpr int kPer = 1024 / kPitch;  // rows that a wave loads at once

  // The unit's place in row r: 16 consecutive rows reading one unit, and 4 rows
  // reading 4 consecutive units, meet every bank once.
  static __device__ __forceinline__ int swizzle(int r) {
    return kUnits == 16 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
  }

  // The lane's part of frag's and frag_t's addresses: what chunk, tile and row add
  // are exclusive ors and sums of constants, so that a slot's start is added once.
  static __device__ __forceinline__ uint32_t lane_rows() {
    const int lane = threadIdx.x & 63, r = lane & 31;
    return r * kPitch + (((lane >> 5) ^ swizzle(r)) << 4);
  }
  static __device__ __forceinline__ uint32_t lane_columns() {
    const int lane = threadIdx.x & 63, i = lane & 15, r = 4 * (lane >> 5) + (i >> 2);
    return r * kPitch + ((((lane >> 3 & 2) | (i >> 1 & 1)) ^ swizzle(r)) << 4) + 8 * (i & 1);
  }
  // Chunk c of rows r0 .. r0 + 31 (r0 a multiple of 16), a row a lane; `at`: byte of
  // the tile in LDS plus lane_rows().
  static __device__ __forceinline__ v8b frag(uint32_t at, int r0, int c) {
    return *(const __attribute__((address_space(3))) v8b*)((at ^ (c << 5)) + r0 * kPitch);
  }
  // Columns 32 t .. 32 t + 31, a column a lane, of rows r0 .. r0 + 15 (r0 a
  // multiple of 16) in the order above; `at`: with lane_columns().
  static __device__ __forceinline__ v8b frag_t(uint32_t at, int r0, int t) {
    v4s x[2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
      x[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(
          (at ^ (t << 6 | e << 5)) + (r0 + 8 * e) * kPitch));
    return __builtin_bit_cast(
        v8b, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// A product of 32 rows of a and of b: b's rows along the lanes of the result.
__device__ __forceinline__ v16f mma(v8b a, v8b b, v16f c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ v16f zero16() {
  v16f z;
#pragma unroll
  for (int e = 0; e < 16; ++e) z[e] = 0.0f;
  return z;
}
// The result's row in register r, of the lane's half.
__device__ __forceinline__ int reg_row(int r) { return 8 * (r >> 2) + (r & 3); }

// Registers 8 c .. 8 c + 7 rounded to bf16.
__device__ __forceinline__ v8b pack8(const v16f& s, int c) {
  u32x4 u;
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = pack_bf16(s[8 * c + 2 * i], s[8 * c + 2 * i + 1]);
  return __builtin_bit_cast(v8b, u);
}

// x of the lane with the same lane % 32 in the other half joined with the lane's.
__device__ __forceinline__ float other_half(float x) {
  const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float((threadIdx.x & 32) ? t[0] : t[1]);
}

struct HeadsArg {
  uint16_t* p;
  int64_t ld_token, ld_head;
};
struct AttentionArgs {
  HeadsArg q, k, v;
  uint16_t* out;
  int64_t ld_out_token, ld_out_head;
  float* lse;
  const int32_t* seq_q;
  const int32_t* seq_k;
  const int32_t* len_k;
  int64_t tokens_q, tokens_k;
  int32_t sequences, heads, kv_heads, group, dim, causal;
  int32_t tiles;   // of rows, of one key head (an upper bound)
  int32_t splits;  // of the keys, the most; piece: keys of one, the least (128 n)
  int32_t piece;
  float scale;
  float* part_out;  // [splits][heads][tokens_q][dim]
  float* part_lse;  // [splits][heads][tokens_q]
};

// A sequence, and where one of its tiles (of rows, or of keys) begins.
struct Sequence {
  int32_t q0, lq, k0, lk;
  int32_t rows, first;
};

__device__ __forceinline__ int32_t clamp_token(int32_t x, int64_t tokens) {
  return x < 0 ? 0 : x > tokens ? static_cast<int32_t>(tokens) : x;
}

// The last of `count` sequences for which before(i) holds (it does up to some i),
// or -1.  The wave searches 64 at a time.
template <typename F>
__device__ __forceinline__ int32_t find_sequence(int32_t count, const F& before) {
  const int lane = threadIdx.x & 63;
  int32_t s = 0;
  do {
    const int32_t step = (count + 63) / 64;
    const int64_t at = static_cast<int64_t>(lane) * step;
    const uint64_t found = __ballot(at < count && before(s + static_cast<int32_t>(at)));
    if (found == 0) return -1;
    const int32_t last = 63 - __builtin_clzll(found);
    s += last * step;
    count = min(step, count - last * step);
  } while (count > 1);
  return uniform_i32(s);
}

template <typename Args>
__device__ __forceinline__ void read_sequence(const Args& a, int32_t s, Sequence& w) {
  if (a.seq_q != nullptr) {
    w.q0 = clamp_token(a.seq_q[s], a.tokens_q);
    w.lq = max(clamp_token(a.seq_q[s + 1], a.tokens_q) - w.q0, 0);
    w.k0 = clamp_token(a.seq_k[s], a.tokens_k);
    w.lk = max(clamp_token(a.seq_k[s + 1], a.tokens_k) - w.k0, 0);
    if (a.len_k != nullptr) w.lk = min(w.lk, max(a.len_k[s], 0));
  } else {
    w.q0 = w.k0 = 0;
    w.lq = static_cast<int32_t>(a.tokens_q);
    w.lk = static_cast<int32_t>(a.tokens_k);
  }
  w.q0 = uniform_i32(w.q0);
  w.lq = uniform_i32(w.lq);
  w.k0 = uniform_i32(w.k0);
  w.lk = uniform_i32(w.lk);
  w.rows = w.lq * a.group;
}

// Tile `g` of the tiles of 2^lg rows (KEYS: of keys): sequence s has the tiles
// from (start * group >> lg) + s on, which are at least as many as it needs
// before the next one's.  So no list of tiles is built, and a captured call
// follows the lengths.  False: no such tile.
template <bool KEYS, typename Args>
__device__ __forceinline__ bool find_tile(const Args& a, int64_t g, int lg, Sequence& w) {
  const int64_t group = KEYS ? 1 : a.group;
  int32_t s = 0;
  if (a.seq_q != nullptr) {
    const int32_t* const starts = KEYS ? a.seq_k : a.seq_q;
    const int64_t tokens = KEYS ? a.tokens_k : a.tokens_q;
    s = find_sequence(a.sequences, [&](int32_t i) {
      return (clamp_token(starts[i], tokens) * group >> lg) + i <= g;
    });
    if (s < 0) return false;
  }
  read_sequence(a, s, w);
  const int64_t first = (g - (((KEYS ? w.k0 : w.q0) * group >> lg) + s)) << lg;
  if (first >= (KEYS ? w.lk : w.rows)) return false;
  w.first = static_cast<int32_t>(first);
  return true;
}

// Keys that query token i of a sequence sees.
template <typename Args>
__device__ __forceinline__ int32_t keys_of(const Args& a, const Sequence& w, int32_t i) {
  return a.causal ? max(min(w.lk, i + w.lk - w.lq + 1), 0) : w.lk;
}

// 16 or 4 bytes a lane from memory to LDS, at byte `lds` + lane * 16 or 4 (`lds` the
// same in every lane).  Written out because the compiler would wait for all of them
// before the next transposing read of any part of LDS: the kernels wait
// themselves, where a tile is needed.  Nothing is loaded to a register.
__device__ __forceinline__ uint32_t lds_offset(const uint8_t* lds) {
  return static_cast<uint32_t>(uniform_i32(static_cast<int32_t>(reinterpret_cast<uintptr_t>(
      (const __attribute__((address_space(3))) uint8_t*)lds))));
}
template <bool NT = false>
__device__ __forceinline__ void dma16(rsrc_t r, uint32_t lds, uint32_t voff) {
#ifdef __HIP_DEVICE_COMPILE__
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(
                     lds),
                 "v"(voff), "s"(r)
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(
                     lds),
                 "v"(voff), "s"(r)
                 : "memory", "m0");
#endif
}
__device__ __forceinline__ void dma4(rsrc_t r, uint32_t lds, uint32_t voff) {
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(
                   lds),
               "v"(voff), "s"(r)
               : "memory", "m0");
#endif
}
// Waits for a vector's loads here, in front of a loop, so that the loop does not
// wait for loads at their first use (and with them for its own, one tile ahead).
template <int N>
__device__ __forceinline__ void settle(v8b (&x)[N]) {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
  for (int c = 0; c < N; ++c) asm volatile("" : "+v"(x[c]));
#endif
}
// Holds sums in their registers at a loop's end: without it the compiler copies all
// of them in every pass, for their use behind the loop (4% of 16384 tokens).
template <int N>
__device__ __forceinline__ void pin(v16f (&x)[N]) {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
  for (int t = 0; t < N; ++t) asm volatile("" : "+v"(x[t]));
#endif
}
// Waits until at most N of the wave's loads are in flight and its reads of LDS are
// done (the other waves may load where it read), then for the block's other waves.
template <int N>
__device__ __forceinline__ void wait_dma() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The same without the other waves.
template <int N>
__device__ __forceinline__ void wait_own_dma() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Waits until the wave's reads of LDS are done: what they read may be overwritten.
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Loads tiles of N keys of k and v: the wave's part of each (`waves` of them load
// together), rows past the last key repeating it, units past the head's width as
// zeros: their offsets lie beyond the resource, and such loads write zeros.  (The
// other operand is zero there, but 0 x infinity, were they copies of other units,
// is not: a key whose score is -infinity would have none.)  NT: each is read by one
// block (nontemporal).
template <int DP, int N, int WAVES, bool NT = false>
struct KeyLoader {
  typedef Heads<DP> H;
  static constexpr int kLoads = N / H::kPer / WAVES;  // of a wave, of either
  static constexpr int kTile = N * H::kPitch;
  static constexpr uint32_t kBeyond = 0x80000000u;  // (a tile's offsets are below half of it)
  const uint16_t *k, *v;
  int64_t ldk, ldv;
  uint32_t at[2][kLoads], unit[kLoads];
  int32_t keys, row[kLoads];

  template <typename Args>
  __device__ __forceinline__ KeyLoader(const Args& a, const Sequence& w, int32_t kvh, int wave) {
    const int lane = threadIdx.x & 63;
    ldk = a.k.ld_token;
    ldv = a.v.ld_token;
    k = a.k.p + kvh * a.k.ld_head + w.k0 * ldk;
    v = a.v.p + kvh * a.v.ld_head + w.k0 * ldv;
    keys = w.lk;
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
      row[n] = (wave * kLoads + n) * H::kPer + lane / H::kUnits;
      const int u = (lane % H::kUnits) ^ H::swizzle(row[n]);
      unit[n] = u < a.dim / 8 ? 16 * u : kBeyond;
      at[0][n] = offset(row[n], ldk) + unit[n];
      at[1][n] = offset(row[n], ldv) + unit[n];
    }
  }
  static __device__ __forceinline__ uint32_t offset(int32_t row, int64_t ld) {
    return static_cast<uint32_t>(row) * (static_cast<uint32_t>(ld) * 2);
  }
  // Keys kb .. kb + N - 1 of k, of v, or of both (v's kTile behind k's), to byte
  // `lds`.  kb < keys.
  template <bool K, bool V>
  __device__ __forceinline__ void load(int32_t kb, uint32_t lds, int wave) const {
    const rsrc_t rk = make_rsrc(k + kb * ldk, kBeyond), rv = make_rsrc(v + kb * ldv, kBeyond);
    lds += wave * kLoads * 1024;
    const uint32_t to_v = K ? lds + kTile : lds;
    if (kb + N <= keys) {
#pragma unroll
      for (int n = 0; n < kLoads; ++n)
        if (K) dma16<NT>(rk, lds + n * 1024, at[0][n]);
#pragma unroll
      for (int n = 0; n < kLoads; ++n)
        if (V) dma16<NT>(rv, to_v + n * 1024, at[1][n]);
    } else {
#pragma unroll
      for (int n = 0; n < kLoads; ++n)
        if (K) dma16<NT>(rk, lds + n * 1024, offset(min(row[n], keys - 1 - kb), ldk) + unit[n]);
#pragma unroll
      for (int n = 0; n < kLoads; ++n)
        if (V) dma16<NT>(rv, to_v + n * 1024, offset(min(row[n], keys - 1 - kb), ldv) + unit[n]);
    }
  }
};

size_t attention_workspace(const AttentionArgs& a);
hipError_t launch_attention(AttentionArgs a, void* ws, hipStream_t s);

struct AttentionBwdArgs {
  HeadsArg q, k, v, out, dout;
  HeadsArg dq, dk, dv;  // (written)
  const float* lse;
  float* delta;  // [heads][tokens_q]
  const int32_t* seq_q;
  const int32_t* seq_k;
  const int32_t* len_k;  // nullptr
  int64_t tokens_q, tokens_k;
  int32_t sequences, heads, kv_heads, group, dim, causal;
  int32_t tiles, key_tiles;
  float scale;
};
size_t attention_backward_workspace(const AttentionBwdArgs& a);
hipError_t launch_attention_backward(AttentionBwdArgs a, void* ws, hipStream_t s);

}  // namespace zf
