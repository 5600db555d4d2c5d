// Matrix product of two 8-bit operands with a scale for each 128 elements of
// the reduction (formulas and format in zf_layer.h).
//
// out[i][j] = sum over groups g of 2^(ca[i][g] + cb[j][g] - 254) * sum over
// the group of a * b, products and sums in fp32 (to_bf16 below says on which
// instruction, and why).
//
// Three forms.  Many rows: tiles of 128 x 128 (matmul_tile_kernel), bound by the
// bf16 instruction's rate and the conversions before it: 1.15-1.20 PFLOP/s at 8192 x
// 11008 x 4096, 8192 x 4096 x 11008, 4096 x 11008 x 8192 and 2048 x 4096 x 11008.  Few
// tiles: the reduction is split over blocks and the shares' results joined in order
// (64 x 11008 x 4096: 22 + 4 us).  Up to 16 rows: the second operand's bytes are all
// that counts (matmul_rows_kernel; 1 x 11008 x 4096: 45 MB in 11.8 us, 3.8 TB/s).
#include <algorithm>

#include "zf_layer.hpp"

namespace zf {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

constexpr int kBK = 128;  // reduction per step: one scale group
// A block's tile, a wave's quarter of it, that in 32 x 32 tiles, and fragments of
// half a step (64 rows of the block's tile each).
constexpr int kBM = 128, kBN = 128, kWM = kBM / 2, kWN = kBN / 2, kTM = kWM / 32, kTN = kWN / 32;
constexpr int kParts = kTM + kTN;

// A step's rows in LDS: 16-byte unit c (of 8) of row r lies at this byte.  16
// consecutive rows reading one unit meet all 64 banks once.
__device__ __forceinline__ int tile_off(int r, int c) {
  return r * kBK + ((c ^ ((r >> 1) & 7)) << 4);
}

// The 8-bit matrix instruction aligns every 8 products to the largest of them and
// cuts what lies 2^-15 below it (1.3e-5 relative on normal data, any share of a
// result that cancels).  So elements times scale go to bf16, which holds them
// exactly, and products and sums are the bf16 instruction's, in fp32 (7e-9), at
// 0.42 of the 8-bit rate.  s: the scale; an infinity's bits stand for a NaN's code.
__device__ __forceinline__ void to_bf16(v8i x, float s, v8b (&out)[4]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const v2b a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 * q], s, false);
    const v2b b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 * q], s, true);
    const v2b c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 * q + 1], s, false);
    const v2b d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 * q + 1], s, true);
    out[q] = v8b{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
}

// One phase of a wave: acc[i][j] += y_j x_i^T (32 x 32 tiles) over 64 elements of
// the reduction, of which a lane holds 32 of row lane % 32 of each tile.  y's
// rows run along the accumulator's registers, x's along its lanes.  Tiles
// [G TM TN / (TM + TN), (G + 1) TM TN / (TM + TN)) of it (row by row of acc); cvt
// holds the phase's y in bf16, and its x of the row at hand.
struct Converted {
  v8b x[4], y[kTN][4];
};
template <int G>
__device__ __forceinline__ void mma(const v8i (&x)[kTM], const float (&sx)[kTM],
                                    const v8i (&y)[kTN], const float (&sy)[kTN],
                                    v16f (&acc)[kTM][kTN], Converted& cvt) {
  if constexpr (G == 0)
#pragma unroll
    for (int j = 0; j < kTN; ++j) to_bf16(y[j], sy[j], cvt.y[j]);
#pragma unroll
  for (int t = G * kTM * kTN / kParts; t < (G + 1) * kTM * kTN / kParts; ++t) {
    const int i = t / kTN, j = t % kTN;
    if (j == 0) to_bf16(x[i], sx[i], cvt.x);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cvt.y[j][q], cvt.x[q], acc[i][j], 0, 0, 0);
#ifdef __HIP_DEVICE_COMPILE__  // (the host's pass does not know the registers)
    // (keeps the product from being moved behind what follows)
    asm volatile("" : "+a"(acc[i][j]));
#endif
  }
}
__device__ __forceinline__ v8i join(u32x4 x, u32x4 y) {
  return v8i{(int)x.x, (int)x.y, (int)x.z, (int)x.w, (int)y.x, (int)y.y, (int)y.z, (int)y.w};
}

// A 16-byte unit of an operand row with the bytes at and past `valid` cleared.
__device__ __forceinline__ u32x4 clear_tail(u32x4 v, int valid) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int n = valid - 4 * w;  // bytes of this word that count
    v[w] = n >= 4 ? v[w] : n <= 0 ? 0u : v[w] & ((1u << (8 * n)) - 1u);
  }
  return v;
}

// Tile of block b in a grid of mt x nt.  Each XCD takes a contiguous range of
// the order; within it 4 tile rows are walked together, so that the tiles an
// XCD works on at once share rows of both operands in its L2.
__device__ __forceinline__ void tile_of(uint32_t b, uint32_t mt, uint32_t nt, uint32_t& mi,
                                        uint32_t& ni) {
  constexpr uint32_t kRows = 4;
  const uint32_t B = mt * nt, q = B / kXcds, r = B % kXcds, x = b % kXcds, i = b / kXcds;
  const uint32_t id = (x < r ? x * (q + 1) : r * (q + 1) + (x - r) * q) + i;
  const uint32_t g = id / (kRows * nt), left = mt - g * kRows, h = left < kRows ? left : kRows;
  const uint32_t in = id - g * kRows * nt;
  mi = uniform_i32(g * kRows + in % h);
  ni = uniform_i32(in / h);
}

// 16 or 4 bytes a lane from memory to LDS, at lds + lane * 16 or 4 (`lds` the
// same in every lane).
__device__ __forceinline__ void load_lds16(rsrc_t r, uint8_t* lds, uint32_t voff, int soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 16,
                                           voff, soff, 0, 0);
}
__device__ __forceinline__ void load_lds4(rsrc_t r, uint8_t* lds, uint32_t voff, int soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 4, voff,
                                           soff, 0, 0);
}

template <int I>
struct Part {
  static constexpr int value = I;
};
// f(Part<0>), ..., f(Part<N - 1>).
template <int N, int I = 0, typename F>
__device__ __forceinline__ void for_parts(const F& f) {
  if constexpr (I < N) {
    f(Part<I>{});
    for_parts<N, I + 1>(f);
  }
}

// Waits until at most N of the wave's loads from memory are in flight, or until
// its LDS reads are done, then for the block's other waves.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_reads() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The first `valid` of a 16-byte unit's elements.
__device__ __forceinline__ void store_units(uint16_t* out, u32x4 v, int64_t valid) {
  Vec8<uint16_t> u;
  u.u = v;
  u.store(out, valid);
}
__device__ __forceinline__ void store_units(float* out, u32x4 v, int64_t valid) {
  uint32_t* const q = reinterpret_cast<uint32_t*>(out);
  if (valid >= 4) {
    *reinterpret_cast<u32x4_f*>(q) = v;
  } else if (valid > 0) {
    if (valid & 2) *reinterpret_cast<u32x2_f*>(q) = u32x2{v.x, v.y};
    if (valid & 1) q[valid - 1] = valid & 2 ? v.z : v.x;
  }
}

// A 256-thread block computes a 128 x 128 tile, each wave a quarter of it, from two
// slots of 128 elements of the reduction in LDS.  Each half of a step multiplies
// 64 elements from registers while the next 64 are read from LDS.  Memory is
// loaded straight to LDS, in whole 128-byte lines, spread evenly over the
// products: a wave issues in order, and a load that waits for room in the
// memory pipeline holds up the products behind it.  Rows past an operand's end
// repeat its last row (their results are not stored); the units past the
// reduction's end repeat the row's last one and are cleared in LDS.
// Scales are taken relative to the largest of their row (of this share of the
// reduction), and the results multiplied by both rows' largest at the end: what
// bf16 and the sums can hold does not depend on where the scales lie.  PART: the
// results are a share's, in fp32.
template <typename Out, bool PART>
__global__ __launch_bounds__(256, 1) void matmul_tile_kernel(MatmulArgs p) {
  constexpr int kRows = kBM + kBN;
  constexpr int kSlot = kRows * kBK;
  constexpr int kLoads = 2 * kParts + 1;  // of a wave per step: 8 rows each, and 64 rows' codes
  constexpr int kCodes = 2 * kSlot;       // a word (four steps) a row, two groups of steps
  constexpr int kTops = kCodes + 2 * kRows * 4;  // a row's exponent of its largest scale
  // A step's 2 kParts groups of products.  Groups kOpen .. issue its loads.
  constexpr int kOpen = kTM / 2, kOpenB = kParts / 2, kIssue = 2 * kParts - kOpen;
  static_assert(kTM % 2 == 0 && kTN % 2 == 0, "two fragments are read at a time");
  static_assert(kRows == 256, "a row of either operand a thread");
  static_assert((kOpenB - kOpen) * kLoads / kIssue <= 2 * kTM, "rows of x alone until y's are read");
  __shared__ __align__(1024) uint8_t lds[kTops + kRows * 4];
  const int t = threadIdx.x, lane = t & 63, wave = uniform_i32(t >> 6);
  const int wm = (wave & 1) * kWM, wn = (wave >> 1) * kWN;
  uint32_t mi, ni;
  tile_of(blockIdx.x, static_cast<uint32_t>((p.m + kBM - 1) / kBM),
          static_cast<uint32_t>((p.n + kBN - 1) / kBN), mi, ni);
  const int64_t m0 = static_cast<int64_t>(mi) * kBM, n0 = static_cast<int64_t>(ni) * kBN;
  // this share's steps [first, steps), the first a multiple of four
  const int all = static_cast<int>((p.k + kBK - 1) / kBK);
  const int first = PART ? static_cast<int>(blockIdx.y) * p.share : 0;
  const int steps = PART ? min(all, first + p.share) : all;
  // elements of a last step that is not whole, or 0
  const int tail = steps == all ? static_cast<int>(p.k % kBK) : 0;

  const rsrc_t ra = make_rsrc(p.a.data + m0 * p.a.ld, -1), rb = make_rsrc(p.b.data + n0 * p.b.ld, -1);
  const rsrc_t rca = make_rsrc(p.a.scale + (m0 >> p.a.shift) * p.a.ld_scale, -1);
  const rsrc_t rcb = make_rsrc(p.b.scale + (n0 >> p.b.shift) * p.b.ld_scale, -1);
  const int last_a = static_cast<int>(min<int64_t>(kBM, p.m - m0)) - 1;
  const int last_b = static_cast<int>(min<int64_t>(kBN, p.n - n0)) - 1;
  // Load i < 2 kParts covers 8 rows of every wave: together 32 of part i / 2's 64.
  uint32_t row[2 * kParts];
#pragma unroll
  for (int i = 0; i < 2 * kParts; ++i) {
    const int r = 8 * (wave + 4 * i) + (lane >> 3);
    row[i] = 32 * i < kBM ? static_cast<uint32_t>(min(r, last_a)) * static_cast<uint32_t>(p.a.ld)
                         : static_cast<uint32_t>(min(r - kBM, last_b)) * static_cast<uint32_t>(p.b.ld);
  }
  const uint32_t code_row =
      t < kBM ? static_cast<uint32_t>(min(t, last_a) >> p.a.shift) * static_cast<uint32_t>(p.a.ld_scale)
              : static_cast<uint32_t>(min(t - kBM, last_b) >> p.b.shift) *
                    static_cast<uint32_t>(p.b.ld_scale);

  // Step kt from memory to a slot, 16 bytes a lane: the lane's place in LDS is
  // fixed, so it loads the unit that tile_off puts there (past the reduction's
  // end the last unit that holds anything).
  const uint32_t unit = ((lane & 7) ^ ((4 * wave + (lane >> 4)) & 7)) << 4;
  const uint32_t last_unit = tail ? ((tail + 15) / 16 - 1) * 16 : 112;
  const auto load_rows = [&](int kt, int slot, int i) {
    load_lds16(32 * i < kBM ? ra : rb, lds + slot * kSlot + wave * 1024 + i * 4096,
               row[i] + min(unit, kt + 1 == steps ? last_unit : 112u), kt * kBK);
  };
  const auto load_step = [&](int kt, int slot) {
#pragma unroll
    for (int i = 0; i < 2 * kParts; ++i) load_rows(kt, slot, i);
  };
  // The last step's bytes past the reduction's end cleared, once it has landed.
  const auto clear_slot = [&](int slot) {
    wait_loads<0>();
    for (int r = t; r < kRows; r += 256)
      for (int c = tail / 16; c < 8; ++c) {
        u32x4* const u = reinterpret_cast<u32x4*>(
            lds + slot * kSlot + (r < kBM ? tile_off(r, c) : kBM * kBK + tile_off(r - kBM, c)));
        *u = clear_tail(*u, tail - 16 * c);
      }
    __syncthreads();
  };
  // The codes of the four steps of group g.
  const auto load_codes = [&](int g) {
    load_lds4(64 * wave < kBM ? rca : rcb, lds + kCodes + (g & 1) * kRows * 4 + wave * 256, code_row,
              4 * g);
  };

  v16f acc[kTM][kTN];
#pragma unroll
  for (int i = 0; i < kTM; ++i)
#pragma unroll
    for (int j = 0; j < kTN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

  v8i xa[2][kTM], yb[2][kTN];
  float sa[kTM], sb[kTN];
  int top_a[kTM], top_b[kTN];
  Converted cvt;
  const auto read_part = [&](int slot, int h, int i) {
    const uint8_t* const s = lds + slot * kSlot;
    const int c = 4 * h + 2 * (lane >> 5);
    const int r = (i < kTM ? wm + 32 * i : wn + 32 * (i - kTM)) + (lane & 31);
    const uint8_t* const q = s + (i < kTM ? 0 : kBM * kBK);
    const v8i v = join(*reinterpret_cast<const u32x4*>(q + tile_off(r, c)),
                       *reinterpret_cast<const u32x4*>(q + tile_off(r, c + 1)));
    if (i < kTM) xa[h][i < kTM ? i : 0] = v;
    else yb[h][i < kTM ? 0 : i - kTM] = v;
  };
  int* const tops = reinterpret_cast<int*>(lds + kTops);
  const auto read_scales = [&](int kt, float(&sa)[kTM], float(&sb)[kTN]) {
    const uint32_t* const w =
        reinterpret_cast<const uint32_t*>(lds + kCodes + ((kt >> 2) & 1) * kRows * 4) + (lane & 31);
    const auto scale = [&](uint32_t word, int top) {
      const int code = static_cast<int>(word >> (8 * (kt & 3)) & 255u) - top;
      return __uint_as_float(static_cast<uint32_t>(max(code, 0)) << 23);
    };
#pragma unroll
    for (int i = 0; i < kTM; ++i) sa[i] = scale(w[wm + 32 * i], top_a[i]);
#pragma unroll
    for (int j = 0; j < kTN; ++j) sb[j] = scale(w[kBM + wn + 32 * j], top_b[j]);
  };

  // Step kt, in 2 kParts groups of products, of its first half and then of its
  // second.  During the first half's groups its second half is read, two
  // fragments a group, x's first: when every wave has them, the slot's rows of
  // x, then those of y, take step kt + 2.  During the second half's groups step
  // kt + 1's first half is read, a fragment a group: its rows of x have landed
  // at the half's start (behind them, y's and what kt + 2 has issued may still
  // be in flight), those of y where it reaches them.  Past the last step the
  // last one is loaded and read again, into a slot that nothing uses: the loop
  // has no branch.  The codes of the next four steps are loaded with each step.
  const int last_group = (steps - 1) >> 2;
  if (first < steps) {
    load_codes(first >> 2);
    load_step(first, 0);
    load_step(min(first + 1, steps - 1), 1);
    load_codes(min((first >> 2) + 1, last_group));
    // The thread's row's largest code less 127 (what follows the last step's in its
    // word may be anything).  With a NaN's among them, 0: it stays one.
    const uint32_t* const codes = reinterpret_cast<const uint32_t*>(
        t < kBM ? p.a.scale + (m0 >> p.a.shift) * p.a.ld_scale + code_row
                : p.b.scale + (n0 >> p.b.shift) * p.b.ld_scale + code_row);
    uint32_t most = 0;  // of even and of odd codes
    const uint32_t whole = steps & 3 ? (1u << (8 * (steps & 3))) - 1u : ~0u;  // of the last word
#pragma unroll 8
    for (int g = first >> 2; g <= last_group; ++g) {
      const uint32_t w = codes[g] & (g == last_group ? whole : ~0u);
      most = pk_max(most, pk_max(w & 0x00ff00ffu, w >> 8 & 0x00ff00ffu));
    }
    const int top = static_cast<int>(max(most & 0xffffu, most >> 16));
    tops[t] = top == 255 ? 0 : top - 127;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTM; ++i) top_a[i] = tops[wm + 32 * i + (lane & 31)];
#pragma unroll
    for (int j = 0; j < kTN; ++j) top_b[j] = tops[kBM + wn + 32 * j + (lane & 31)];
    wait_loads<kLoads>();
    if (tail && first + 1 == steps) clear_slot(0);
    read_scales(first, sa, sb);
#pragma unroll
    for (int i = 0; i < kParts; ++i) read_part(0, 0, i);
  }
  int slot = 0;
  for (int kt = first; kt < steps; ++kt) {
    const int next = slot ^ 1, ahead = min(kt + 2, steps - 1);
    // loads [g kLoads / kIssue, (g + 1) kLoads / kIssue) of step kt + 2
    const auto issue = [&](auto g) {
      if constexpr (g.value >= 0)
#pragma unroll
        for (int i = g.value * kLoads / kIssue; i < (g.value + 1) * kLoads / kIssue; ++i) {
          if (i < 2 * kParts) load_rows(ahead, slot, i);
          else load_codes(min((kt >> 2) + 1, last_group));
        }
    };
    for_parts<kParts>([&](auto g) {
      if constexpr (2 * g.value < kParts) {
        read_part(slot, 1, 2 * g.value);
        read_part(slot, 1, 2 * g.value + 1);
      }
      if constexpr (g.value == kOpen || g.value == kOpenB) wait_reads();
      issue(Part<g.value - kOpen>{});
      mma<g.value>(xa[0], sa, yb[0], sb, acc, cvt);
      __builtin_amdgcn_sched_barrier(0);
    });
    float na[kTM], nb[kTN];
    for_parts<kParts>([&](auto g) {
      // loads of step kt + 2 issued before this group
      constexpr int issued = (kParts + g.value - kOpen) * kLoads / kIssue;
      if constexpr (g.value == 0) {
        wait_loads<kLoads - 2 * kTM + issued>();
        if (tail && kt + 2 == steps) clear_slot(next);
        read_scales(kt + 1, na, nb);
      }
      if constexpr (g.value == kTM) wait_loads<issued>();
      read_part(next, 0, g.value);
      issue(Part<kParts + g.value - kOpen>{});
      mma<g.value>(xa[1], sa, yb[1], sb, acc, cvt);
      __builtin_amdgcn_sched_barrier(0);
    });
#pragma unroll
    for (int i = 0; i < kTM; ++i) sa[i] = na[i];
#pragma unroll
    for (int j = 0; j < kTN; ++j) sb[j] = nb[j];
    slot = next;
  }
  wait_loads<0>();  // nothing lands in LDS from here on

  // A lane holds 4 consecutive columns of a row at a time; through LDS, 32
  // rows of the wave's tile at a time, the rows become contiguous.  (Scaled on their
  // way out, in a loop: as they are written, each of 64 results in code of its own,
  // 256 x 4096 x 4096 took 23.2 us, not 22.2.)
  constexpr int kPitch = kWN + 4;
  static_assert(4 * 32 * kPitch * 4 <= 2 * kSlot, "the waves' slabs fit the slots");
  float* const slab = reinterpret_cast<float*>(lds) + wave * 32 * kPitch;
  constexpr int kPer = 16 / sizeof(Out), kRun = kWN / kPer;  // elements of a store, lanes of a row
  const int c = lane % kRun * kPer;
  Out* const out = static_cast<Out*>(p.out) + (PART ? blockIdx.y * p.m * p.ld_out : 0) +
                   (m0 + wm) * p.ld_out + n0 + wn + c;
  const int64_t rows = p.m - m0 - wm, cols = p.n - n0 - wn - c;
  int top[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) top[e] = tops[kBM + wn + c + e];
#pragma unroll
  for (int i = 0; i < kTM; ++i) {
#pragma unroll
    for (int j = 0; j < kTN; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<v4f*>(slab + (lane & 31) * kPitch + 32 * j + 2 * e + 4 * (lane >> 5)) =
            v4f{acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int r = lane / kRun; r < 32; r += 64 / kRun) {
      if (32 * i + r >= rows) break;
      const int row_top = tops[wm + 32 * i + r];
      float v[kPer];
#pragma unroll
      for (int e = 0; e < kPer; e += 4) {
        const v4f w = *reinterpret_cast<const v4f*>(slab + r * kPitch + c + e);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[e + q] = __builtin_ldexpf(w[q], row_top + top[e + q]);
      }
      u32x4 u;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if constexpr (sizeof(Out) == 4) u[q] = __float_as_uint(v[q]);
        else u[q] = pack_bf16(v[2 * q], v[2 * q + 1]);
      }
      Out* const o = out + (32 * i + r) * p.ld_out;
      if (cols >= kPer) __builtin_nontemporal_store(u, reinterpret_cast<u32x4_h*>(o));
      else store_units(o, u, cols);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// out = the sum of `shares` partial results, in order (row by row of n, which
// the partial results are stored in without padding).
template <typename Out>
__global__ __launch_bounds__(256) void matmul_join_kernel(const float* __restrict__ part,
                                                          int32_t shares, int64_t m, int64_t n,
                                                          Out* __restrict__ out, int64_t ld_out) {
  const int64_t size = m * n;
  for (int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8; i < size;
       i += static_cast<int64_t>(gridDim.x) * 256 * 8) {
    float v[8] = {};
    for (int32_t q = 0; q < shares; ++q) {
      Vec8<float> w;
      w.load(part + q * size + i, size - i);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = q == 0 ? w[j] : v[j] + w[j];
    }
    int64_t row = i / n, col = i - row * n;
    Vec8<Out> o;
    o.set(v);
    if (col + 8 <= n) {
      o.store(out + row * ld_out + col, 8);
    } else {  // the run ends in a later row
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (i + j < size) {
          const float one[8] = {v[j]};
          o.set(one);
          o.store(out + row * ld_out + col, 1);
        }
        if (++col == n) {
          col = 0;
          ++row;
        }
      }
    }
  }
}

// Up to 16 rows of a (tokens): every element of b is read once, straight to
// registers, and little else counts.  A block takes 16 rows of b; its waves take
// shares of the reduction, each with the loads of U steps in flight, and their
// sums are added in order.  a's rows past its end repeat the last one.  16 x 16
// products: b's rows along the accumulator's registers, a's along its lanes.  Each
// group's sum is multiplied by its scales, in fp32.
template <int W, int U, typename Out>
__global__ __launch_bounds__(64 * W) void matmul_rows_kernel(MatmulArgs p) {
  __shared__ float sums[W][4][64];
  const int lane = threadIdx.x & 63, wave = uniform_i32(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * 16;
  const int steps = static_cast<int>((p.k + kBK - 1) / kBK), tail = static_cast<int>(p.k % kBK);
  const int per = (steps + W - 1) / W;
  const int k0 = wave * per, k1 = min(steps, k0 + per);

  const rsrc_t rb = make_rsrc(p.b.data + n0 * p.b.ld, -1), ra = make_rsrc(p.a.data, -1);
  const int64_t qa = min<int64_t>(r, p.m - 1), qb = min<int64_t>(n0 + r, p.n - 1);
  const uint32_t row_a = static_cast<uint32_t>(qa) * static_cast<uint32_t>(p.a.ld);
  const uint32_t row_b = static_cast<uint32_t>(qb - n0) * static_cast<uint32_t>(p.b.ld);
  const uint8_t* const code_a = p.a.scale + (qa >> p.a.shift) * p.a.ld_scale;
  const uint8_t* const code_b = p.b.scale + (qb >> p.b.shift) * p.b.ld_scale;
  v4f acc = {0, 0, 0, 0};
  for (int kt = k0; kt < k1; kt += U) {
    u32x4 a[U][2], b[U][2];
    int ca[U], cb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {  // (steps past the share's end repeat its last one, unused)
      const int ks = min(kt + u, k1 - 1);
      const uint32_t last = tail && ks + 1 == steps ? ((tail + 15) / 16 - 1) * 16u : 112u;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t c = min<uint32_t>(32 * g + 16 * h, last);
        b[u][h] = buf_b128(rb, row_b + c, ks * kBK);
        a[u][h] = buf_b128(ra, row_a + c, ks * kBK);
      }
      cb[u] = code_b[ks];
      ca[u] = code_a[ks];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (kt + u >= k1) break;
      if (tail && kt + u + 1 == steps) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          b[u][h] = clear_tail(b[u][h], tail - 32 * g - 16 * h);
          a[u][h] = clear_tail(a[u][h], tail - 32 * g - 16 * h);
        }
      }
      const v8i x = join(a[u][0], a[u][1]), y = join(b[u][0], b[u][1]);
      v8b xb[4], yb[4];
      to_bf16(x, ca[u] == 255 ? __uint_as_float(255u << 23) : 1.0f, xb);
      to_bf16(y, cb[u] == 255 ? __uint_as_float(255u << 23) : 1.0f, yb);
      v4f sum = {0, 0, 0, 0};
#pragma unroll
      for (int q = 0; q < 4; ++q)
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(yb[q], xb[q], sum, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        acc[e] += __builtin_ldexpf(sum[e], ca[u] + __shfl(cb[u], 4 * g + e) - 254);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sums[wave][e][lane] = acc[e];
  __syncthreads();
  // result (row, col): row = lane % 16, col = 4 (lane / 16) + e
  for (int q = threadIdx.x; q < 256; q += 64 * W) {
    const int col = q & 15, row = q >> 4, e = col & 3, l = row + 16 * (col >> 2);
    float v = sums[0][e][l];
#pragma unroll
    for (int w = 1; w < W; ++w) v += sums[w][e][l];
    if (row < p.m && n0 + col < p.n) {
      const int64_t at = row * p.ld_out + n0 + col;
      if constexpr (sizeof(Out) == 4) static_cast<float*>(p.out)[at] = v;
      else static_cast<uint16_t*>(p.out)[at] = round_bf16(v);
    }
  }
}

// ---- choice of a form --------------------------------------------------------

// Rows of a up to which matmul_rows_kernel is taken, and rows of b that its blocks
// of 16 still reach in one dispatch (of fewer than 2^32 threads).
constexpr int64_t kRowsMax = 16;
constexpr int64_t kRowsReach = int64_t(1) << 27;
bool takes_rows(int64_t m, int64_t n) { return m <= kRowsMax && n <= kRowsReach; }

int64_t tiles(int64_t m, int64_t n) { return ((m + kBM - 1) / kBM) * ((n + kBN - 1) / kBN); }

// Shares of the reduction where the tiles do not fill the 256 CUs: the number for
// which this estimate in us is least.  A step takes 0.95 us on a CU of its own and
// 1.75 as one of two; a share's partial result is written and read at some 6 TB/s,
// the joining launch costs 3.
int shares(int64_t m, int64_t n, int64_t k) {
  if (takes_rows(m, n)) return 1;
  const int64_t t = tiles(m, n), steps = (k + kBK - 1) / kBK;
  if (t > 160) return 1;
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= 16 && s * t <= 512; ++s) {
    const int64_t per = ((steps + s - 1) / s + 3) / 4 * 4;  // (codes come four steps at a time)
    if (s > 1 && (s - 1) * per >= steps) continue;
    const double us = per * (s * t > 256 ? 1.75 : 0.95) + (s > 1 ? 3.0 + 8.0 * s * m * n / 6e6 : 0.0);
    if (us < least) {
      least = us;
      best = s;
    }
  }
  return best;
}

template <typename Out>
void launch_rows(const MatmulArgs& a, hipStream_t s) {
#define ZF_ROWS(W, U)                                                                   \
  hipLaunchKernelGGL((matmul_rows_kernel<W, U, Out>), dim3(static_cast<uint32_t>(blocks)), \
                     dim3(64 * W), 0, s, a)
  const int64_t blocks = (a.n + 15) / 16;
  if (blocks >= 512) ZF_ROWS(4, 8);
  else if (blocks >= 128) ZF_ROWS(8, 4);
  else ZF_ROWS(16, 4);
#undef ZF_ROWS
}

template <typename Out>
void launch_tiles(const MatmulArgs& a, void* ws, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(tiles(a.m, a.n)));
  const int q = shares(a.m, a.n, a.k);
  if (q == 1) {
    hipLaunchKernelGGL((matmul_tile_kernel<Out, false>), grid, dim3(256), 0, s, a);
    return;
  }
  MatmulArgs b = a;
  b.out = ws;
  b.ld_out = a.n;
  const int64_t steps = (a.k + kBK - 1) / kBK;
  b.share = static_cast<int32_t>(((steps + q - 1) / q + 3) / 4 * 4);
  hipLaunchKernelGGL((matmul_tile_kernel<float, true>), dim3(grid.x, q), dim3(256), 0, s, b);
  const int64_t blocks = (a.m * a.n + 2047) / 2048;
  hipLaunchKernelGGL((matmul_join_kernel<Out>), dim3(static_cast<uint32_t>(std::min<int64_t>(blocks, 2048))),
                     dim3(256), 0, s, static_cast<const float*>(ws), q, a.m, a.n,
                     static_cast<Out*>(a.out), a.ld_out);
}

}  // namespace

size_t matmul_workspace(int64_t m, int64_t n, int64_t k) {
  const int q = shares(m, n, k);
  return q > 1 ? static_cast<size_t>(q) * m * n * sizeof(float) : 0;
}

hipError_t launch_matmul(const MatmulArgs& a, void* ws, hipStream_t s) {
  (void)hipGetLastError();
  if (takes_rows(a.m, a.n)) {
    if (a.out_f32) launch_rows<float>(a, s);
    else launch_rows<uint16_t>(a, s);
  } else {
    if (a.out_f32) launch_tiles<float>(a, ws, s);
    else launch_tiles<uint16_t>(a, ws, s);
  }
  return hipGetLastError();
}

}  // namespace zf
