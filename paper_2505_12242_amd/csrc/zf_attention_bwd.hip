// Attention's gradients (formulas and contract in zf_layer.h; rows, products and
// the layout of LDS in zf_attention.hpp).
//
// Two kernels.  The first takes 128 rows a block, as the forward pass does (or 32,
// where there are few), and walks their keys: scores again, dP, dS, dq; before that
// it forms d = dout . out of its rows, which the second needs too.  The second takes 128 keys a block and
// walks the rows that see them, over all query heads of the key head: scores, dP,
// dk and dv.  Seven products in place of the five that one kernel needs, but no
// gradient is summed across blocks: no atomics, no partial results in memory, and
// the same bits on every run.  2 x 4096 tokens x 32 heads of 128, causal: 400 us and
// 550, 1.0 PFLOP/s of these products either (the library's 8192^3 bf16 product 1.26).
// P and dS are rounded to bf16, as the instruction takes them: against 64 bits the
// gradients' relative error (2-norm) is 2.35e-3 where one rounding of the results makes
// 1.66e-3.  With a second operand for what the rounding leaves it would be the latter,
// for three more products.
//
// In either, the operand that a wave keeps (rows, or keys) stays in registers and
// runs along the lanes of the scores; what is walked runs along their registers,
// so that P and dS, rounded to bf16, are operands of the second products where
// they stand.
#include <algorithm>

#include "zf_attention.hpp"

namespace zf {
namespace {

constexpr int kLg = 7, kBlock = 1 << kLg;  // rows, or keys, of a block
constexpr int kKeys = 64;                  // keys of a tile (dq)
constexpr int kRows = 32;                  // rows of a tile (dk, dv)

// A vector as the lane's part of an operand: 8 elements of each chunk of 16,
// zeros past the head's width.
template <int DP>
__device__ __forceinline__ void load_vector(const uint16_t* p, int dim, v8b (&x)[DP / 16]) {
#pragma unroll
  for (int c = 0; c < DP / 16; ++c) {
    const int e = 16 * c + 8 * (threadIdx.x >> 5 & 1);
    u32x4 u = {0, 0, 0, 0};
    if (e < dim) u = *reinterpret_cast<const u32x4*>(p + e);
    x[c] = __builtin_bit_cast(v8b, u);
  }
}

// Tells the compiler to issue `reads` LDS reads and `products` products of the
// region evenly, the reads `ahead` in front.
template <int READS, int PRODUCTS, int AHEAD, int I = 0>
__device__ __forceinline__ void reads_ahead() {
  if constexpr (I == 0) __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
  if constexpr (I < PRODUCTS) {
    constexpr int kRest = READS - AHEAD;
    constexpr int kReads = (I + 1) * kRest / PRODUCTS - I * kRest / PRODUCTS;
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if constexpr (kReads > 0) __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
    reads_ahead<READS, PRODUCTS, AHEAD, I + 1>();
  }
}

// 32 elements (tile t) of a gradient's vector, along the lane's registers of a result.
__device__ __forceinline__ void store_tile(uint16_t* p, int dim, int t, const v16f& x, float scale) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int d = 32 * t + 8 * g + 4 * (threadIdx.x >> 5 & 1);
    if (d < dim)
      *reinterpret_cast<u32x2*>(p + d) = u32x2{pack_bf16(x[4 * g] * scale, x[4 * g + 1] * scale),
                                               pack_bf16(x[4 * g + 2] * scale, x[4 * g + 3] * scale)};
  }
}
template <int DP>
__device__ __forceinline__ void store_vector(uint16_t* p, int dim, const v16f (&x)[DP / 32],
                                             float scale) {
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) store_tile(p, dim, t, x[t], scale);
}

// A wave's 32 rows, a row a lane.
template <int DP>
struct Rows {
  v8b q[DP / 16], dout[DP / 16];
  v16f dq[DP / 32];
  float delta, lse;  // (lse in powers of two)
};
template <int DP>
__device__ __forceinline__ void load_rows(const AttentionBwdArgs& a, int64_t token, int64_t head,
                                          Rows<DP>& x) {
  load_vector<DP>(a.q.p + token * a.q.ld_token + head * a.q.ld_head, a.dim, x.q);
  load_vector<DP>(a.dout.p + token * a.dout.ld_token + head * a.dout.ld_head, a.dim, x.dout);
  v8b out[DP / 16];
  load_vector<DP>(a.out.p + token * a.out.ld_token + head * a.out.ld_head, a.dim, out);
  x.lse = a.lse[head * a.tokens_q + token] * kLog2E;
  x.delta = 0.0f;
#pragma unroll
  for (int c = 0; c < DP / 16; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      x.delta = fmaf(static_cast<float>(x.dout[c][e]), static_cast<float>(out[c][e]), x.delta);
  x.delta += other_half(x.delta);
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) x.dq[t] = zero16();
  settle(x.q);
  settle(x.dout);
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("" : "+v"(x.lse));  // (see settle)
#endif
}

template <int DP>
__global__ __launch_bounds__(256, 2) void attention_dq_kernel(AttentionBwdArgs a) {
  typedef Heads<DP> H;
  constexpr int kTile = kKeys * H::kPitch;
  __shared__ __align__(1024) uint8_t lds[4 * kTile];  // two slots of k and v
  const int lane = threadIdx.x & 63, wave = uniform_i32(threadIdx.x >> 6), half = lane >> 5;
  const int32_t kvh = blockIdx.x % a.kv_heads;
  Sequence w;
  if (!find_tile<false>(a, a.tiles - 1 - static_cast<int64_t>(blockIdx.x / a.kv_heads), kLg, w))
    return;
  const int32_t row = w.first + 32 * wave + (lane & 31);
  const bool valid = row < w.rows;
  const int32_t i = min(row, w.rows - 1) / a.group;
  const int64_t head = kvh * a.group + min(row, w.rows - 1) - i * a.group;
  const int64_t token = w.q0 + i;
  const float c = a.scale * kLog2E;
  const int32_t lim = keys_of(a, w, i);

  const auto token_of = [&](int32_t row) { return min(row, w.rows - 1) / a.group; };
  const int32_t least = uniform_i32(keys_of(a, w, token_of(w.first + 32 * wave)));
  const int32_t most =
      uniform_i32(w.first + 32 * wave < w.rows ? keys_of(a, w, token_of(w.first + 32 * wave + 31)) : 0);
  const int32_t end = uniform_i32(keys_of(a, w, token_of(w.first + kBlock - 1)));
  const KeyLoader<DP, kKeys, 4> keys(a, w, kvh, wave);
  const uint32_t base = lds_offset(lds), rows = H::lane_rows(), columns = H::lane_columns();
  if (end > 0) keys.template load<true, true>(0, base, wave);
  Rows<DP> x;
  load_rows(a, token, head, x);
  if (valid && lane < 32) a.delta[head * a.tokens_q + token] = x.delta;
  int slot = 0;
  for (int32_t kb = 0; kb < end; kb += kKeys) {
    wait_dma<0>();
    if (kb + kKeys < end) keys.template load<true, true>(kb + kKeys, base + (slot ^ 1) * 2 * kTile, wave);
    const uint32_t at = base + slot * 2 * kTile;
    const uint32_t k = at + rows, kt = at + columns, v = at + kTile + rows;
    if (kb < most) {
      const bool mask = kb + kKeys > least;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        v16f s = zero16(), dp = zero16();
#pragma unroll
        for (int j = 0; j < H::kChunks; ++j) s = mma(H::frag(k, 32 * t, j), x.q[j], s);
#pragma unroll
        for (int j = 0; j < H::kChunks; ++j) dp = mma(H::frag(v, 32 * t, j), x.dout[j], dp);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -x.lse)) * (dp[r] - x.delta);
        if (mask) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (kb + 32 * t + reg_row(r) + 4 * half >= lim) s[r] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const v8b ds = pack8(s, j);
#pragma unroll
          for (int u = 0; u < H::kTiles; ++u)
            x.dq[u] = mma(H::frag_t(kt, 32 * t + 16 * j, u), ds, x.dq[u]);
        }
      }
    }
    slot ^= 1;
  }
  if (valid)
    store_vector<DP>(a.dq.p + token * a.dq.ld_token + head * a.dq.ld_head, a.dim, x.dq, a.scale);
}

// The same for few rows: 32 of them a block, which all of its waves keep, and every
// fourth tile of 32 keys a wave, loaded by it for itself; their sums are added in LDS,
// in the waves' order.  v's slot is filled again as soon as dP is done, k's after dq.
constexpr int kDqWaves = 4, kDqStep = 32 * kDqWaves;
template <int DP>
__global__ __launch_bounds__(64 * kDqWaves, 2) void attention_dq_narrow_kernel(AttentionBwdArgs a) {
  typedef Heads<DP> H;
  typedef KeyLoader<DP, 32, 1> Loader;
  constexpr int kTile = 32 * H::kPitch, kN = Loader::kLoads;
  static_assert(kDqWaves * 2 * kTile >= (kDqWaves - 1) * H::kTiles * 4096, "the sums fit the tiles");
  __shared__ __align__(1024) uint8_t lds[kDqWaves * 2 * kTile];
  const int lane = threadIdx.x & 63, wave = uniform_i32(threadIdx.x >> 6), half = lane >> 5;
  const int32_t kvh = blockIdx.x % a.kv_heads;
  Sequence w;
  if (!find_tile<false>(a, a.tiles - 1 - static_cast<int64_t>(blockIdx.x / a.kv_heads), 5, w)) return;
  const int32_t row = w.first + (lane & 31);
  const bool valid = row < w.rows;
  const int32_t i = min(row, w.rows - 1) / a.group;
  const int64_t head = kvh * a.group + min(row, w.rows - 1) - i * a.group;
  const int64_t token = w.q0 + i;
  const int32_t lim = keys_of(a, w, i);
  const int32_t least = uniform_i32(keys_of(a, w, w.first / a.group));
  const int32_t end = uniform_i32(keys_of(a, w, min(w.first + 31, w.rows - 1) / a.group));
  const Loader keys(a, w, kvh, 0);
  const uint32_t base = lds_offset(lds) + wave * 2 * kTile;
  const int32_t first = 32 * wave;
  if (first < end) {
    keys.template load<false, true>(first, base + kTile, 0);
    keys.template load<true, false>(first, base, 0);
  }
  Rows<DP> x;
  load_rows(a, token, head, x);
  if (valid && wave == 0 && lane < 32) a.delta[head * a.tokens_q + token] = x.delta;
  const float c = a.scale * kLog2E;
  const uint32_t k = base + H::lane_rows(), kt = base + H::lane_columns(), v = k + kTile;
  for (int32_t kb = first; kb < end; kb += kDqStep) {
    const bool next = kb + kDqStep < end;
    wait_own_dma<kN>();  // (this k is behind this v)
    v16f s = zero16(), dp = zero16();
#pragma unroll
    for (int j = 0; j < H::kChunks; ++j) dp = mma(H::frag(v, 0, j), x.dout[j], dp);
    wait_reads();
    if (next) {
      keys.template load<false, true>(kb + kDqStep, base + kTile, 0);
      wait_own_dma<kN>();
    } else {
      wait_own_dma<0>();
    }
#pragma unroll
    for (int j = 0; j < H::kChunks; ++j) s = mma(H::frag(k, 0, j), x.q[j], s);
#pragma unroll
    for (int r = 0; r < 16; ++r)
      s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -x.lse)) * (dp[r] - x.delta);
    if (kb + 32 > least) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (kb + reg_row(r) + 4 * half >= lim) s[r] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const v8b ds = pack8(s, j);
#pragma unroll
      for (int u = 0; u < H::kTiles; ++u) x.dq[u] = mma(H::frag_t(kt, 16 * j, u), ds, x.dq[u]);
    }
    wait_reads();
    if (next) keys.template load<true, false>(kb + kDqStep, base, 0);
    pin(x.dq);
  }
  // (a wave waits for its last tile's loads)
  float* const sums = reinterpret_cast<float*>(lds);
  const auto place = [&](int wave, int t, int r) {
    return sums + (((wave - 1) * H::kTiles + t) * 16 + r) * 64 + lane;
  };
  __syncthreads();
  if (wave > 0)
#pragma unroll
    for (int t = 0; t < H::kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) *place(wave, t, r) = x.dq[t][r];
  __syncthreads();
  if (wave > 0 || !valid) return;
#pragma unroll
  for (int g = 1; g < kDqWaves; ++g)
#pragma unroll
    for (int t = 0; t < H::kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) x.dq[t][r] += *place(g, t, r);
  store_vector<DP>(a.dq.p + token * a.dq.ld_token + head * a.dq.ld_head, a.dim, x.dq, a.scale);
}

// 32 WK keys a block, of which a wave keeps 32: k in registers, v in LDS.  WR groups
// of WK waves have the same keys and every WR-th tile of rows each, which the
// group's waves load together and share; the groups' sums are added in LDS, in
// their order.
// (LDS of the launch's own size: told that one block fills a CU's LDS, the compiler
// takes twice the registers and copies sums between their two halves, 224 copies a
// tile of rows.)
template <int DP, int WK, int WR>
struct Shared {
  typedef Heads<DP> H;
  static constexpr int kTile = kRows * H::kPitch;
  static constexpr int kSlot = 2 * kTile + 1024;  // q, dout, lse and delta (256 bytes a wave)
  static constexpr int kOwn = (WK == 1 ? 1 : 2) * kSlot;  // of a group
  static constexpr int kValues = WR * kOwn;       // the block's v
  static constexpr int kAll = kValues + 32 * WK * H::kPitch;
  static constexpr int kSums = (WR - 1) * WK * H::kTiles * 4096;
  static constexpr int kBytes = kAll > kSums ? kAll : kSums;
};
template <int DP, int WK, int WR>
__global__ __launch_bounds__(64 * WK * WR, 2) void attention_dkv_kernel(AttentionBwdArgs a) {
  typedef Heads<DP> H;
  typedef Shared<DP, WK, WR> S;
  constexpr int kTile = S::kTile, kSlot = S::kSlot, kOwn = S::kOwn, kValues = S::kValues;
  constexpr int kLoads = kRows / H::kPer / WK;
  constexpr int kStep = WR * kRows;  // from a group's tile to its next
  extern __shared__ __align__(1024) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = uniform_i32(threadIdx.x >> 6), half = lane >> 5;
  const int part = wave % WK, own = wave / WK;  // of the block's keys, the group
  const int32_t kvh = blockIdx.x % a.kv_heads;
  Sequence w;
  if (!find_tile<true>(a, blockIdx.x / a.kv_heads, WK == 4 ? kLg : 5, w)) return;
  const int32_t key0 = w.first + 32 * part, key = key0 + (lane & 31);
  const bool valid = key < w.lk;
  const int64_t token = w.k0 + min(key, w.lk - 1);
  const uint32_t base = lds_offset(lds);
  v8b k[H::kChunks];
  load_vector<DP>(a.k.p + token * a.k.ld_token + kvh * a.k.ld_head, a.dim, k);
  {
    const rsrc_t rv = make_rsrc(
        a.v.p + (static_cast<int64_t>(w.k0) + w.first) * a.v.ld_token + kvh * a.v.ld_head, -1);
    constexpr int kN = 32 / H::kPer / WR > 0 ? 32 / H::kPer / WR : 1;
    if (wave * kN * H::kPer < 32 * WK)
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      const int r = (wave * kN + n) * H::kPer + lane / H::kUnits;
      const int unit = min((lane % H::kUnits) ^ H::swizzle(r), a.dim / 8 - 1);
      dma16(rv, base + kValues + (wave * kN + n) * 1024,
            static_cast<uint32_t>(min(r, w.lk - 1 - w.first)) *
                    (static_cast<uint32_t>(a.v.ld_token) * 2) + unit * 16);
    }
  }
  v16f dk[H::kTiles], dv[H::kTiles];
#pragma unroll
  for (int t = 0; t < H::kTiles; ++t) dk[t] = dv[t] = zero16();
  // the first row that sees a key (of any query head)
  const auto first_row = [&](int32_t key) {
    return a.causal ? max(key - (w.lk - w.lq), 0) * a.group : 0;
  };
  const int32_t from = first_row(min(key, w.lk - 1));
  const int32_t most = uniform_i32(first_row(min(key0 + 31, w.lk - 1)));
  const int32_t least = uniform_i32(key0 < w.lk ? first_row(key0) : w.rows);
  const int32_t begin = uniform_i32(first_row(w.first)) / kRows * kRows + own * kRows;

  const uint32_t ldq = static_cast<uint32_t>(a.q.ld_token) * 2, ldo = static_cast<uint32_t>(a.dout.ld_token) * 2;
  const uint32_t lhq = static_cast<uint32_t>(a.q.ld_head) * 2, lho = static_cast<uint32_t>(a.dout.ld_head) * 2;
  const int64_t head0 = static_cast<int64_t>(kvh) * a.group;
  const rsrc_t rl = make_rsrc(a.lse + head0 * a.tokens_q + w.q0, -1);
  const rsrc_t rd = make_rsrc(a.delta + head0 * a.tokens_q + w.q0, -1);
  const uint32_t magic = 0xffffffffu / static_cast<uint32_t>(a.group) + 1;  // (0: a group of one)
  const auto load = [&](int32_t r0, int slot) {
    const int32_t t0 = uniform_i32(r0 / a.group);
    const uint32_t in = static_cast<uint32_t>(r0 - t0 * a.group);
    const int64_t tok = static_cast<int64_t>(w.q0) + t0;
    const rsrc_t rq = make_rsrc(a.q.p + tok * a.q.ld_token + head0 * a.q.ld_head, -1);
    const rsrc_t ro = make_rsrc(a.dout.p + tok * a.dout.ld_token + head0 * a.dout.ld_head, -1);
    const int last = w.rows - 1 - r0;
    const uint32_t to = base + own * kOwn + slot * kSlot;
    const auto split = [&](int r, uint32_t& tok, uint32_t& g) {  // row r0 + r
      const uint32_t x = in + static_cast<uint32_t>(min(r, last));
      tok = magic ? __umulhi(x, magic) : x;
      g = x - tok * static_cast<uint32_t>(a.group);
    };
    uint32_t tk, g;
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
      const int r = (part * kLoads + n) * H::kPer + lane / H::kUnits;
      const int unit = min((lane % H::kUnits) ^ H::swizzle(r), a.dim / 8 - 1);
      split(r, tk, g);
      const uint32_t p = to + (part * kLoads + n) * 1024;
      dma16(rq, p, tk * ldq + g * lhq + unit * 16);
      dma16(ro, p + kTile, tk * ldo + g * lho + unit * 16);
    }
    // (lanes 32 and up repeat the rows, behind them; parts 2 and 3 the first two)
    split(lane & 31, tk, g);
    const uint32_t at = (g * static_cast<uint32_t>(a.tokens_q) + static_cast<uint32_t>(t0) + tk) * 4;
    if constexpr (WK == 4) {
      dma4(part & 1 ? rd : rl, to + 2 * kTile + part * 256, at);
    } else {
      dma4(rl, to + 2 * kTile, at);
      dma4(rd, to + 2 * kTile + 256, at);
    }
  };
  const float c = a.scale * kLog2E;
  if (begin < w.rows) load(begin, 0);
  settle(k);
  const uint32_t lane_r = base + H::lane_rows(), lane_c = base + H::lane_columns();
  if (WK == 1 || a.dim < DP) wait_dma<0>();  // (every wave's part of v)
  if (a.dim < DP) {  // dout's units past the head's width hold anything: v's are zeros
    const int first = a.dim / 8, n = DP / 8 - first;
    for (int i = threadIdx.x; i < 32 * WK * n; i += 64 * WK * WR) {
      const int r = i / n, unit = first + i - r * n;
      *reinterpret_cast<u32x4*>(lds + kValues + r * H::kPitch + ((unit ^ H::swizzle(r)) << 4)) =
          u32x4{0, 0, 0, 0};
    }
    __syncthreads();
  }
  int slot = 0;
  // (groups that share barriers walk as many tiles, the last one perhaps of none)
  const int32_t end = WK == 1 ? w.rows : w.rows + own * kRows;
  for (int32_t r0 = begin; r0 < end; r0 += kStep) {
    if (WK == 1) wait_own_dma<0>();
    else wait_dma<0>();
    if (WK != 1 && r0 + kStep < w.rows) load(r0 + kStep, slot ^ 1);
    const uint32_t q = lane_r + own * kOwn + slot * kSlot, qt = lane_c + own * kOwn + slot * kSlot;
    const uint32_t dout = q + kTile, dout_t = qt + kTile, v = lane_r + kValues + part * 32 * H::kPitch;
    const float* const stats =
        reinterpret_cast<const float*>(lds + own * kOwn + slot * kSlot + 2 * kTile);
    if (r0 + kRows > least && r0 < w.rows) {
      v16f s = zero16(), dp = zero16();
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int j = 0; j < H::kChunks; ++j) s = mma(H::frag(q, 0, j), k[j], s);
#pragma unroll
      for (int j = 0; j < H::kChunks; ++j) dp = mma(H::frag(dout, 0, j), H::frag(v, 0, j), dp);
      reads_ahead<3 * H::kChunks, 2 * H::kChunks, 5>();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int at = 8 * g + 4 * half;
        const u32x4 l = *reinterpret_cast<const u32x4*>(stats + at);
        const u32x4 d = *reinterpret_cast<const u32x4*>(stats + 64 + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * g + e;
          s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -(__uint_as_float(l[e]) * kLog2E)));
          dp[r] = s[r] * (dp[r] - __uint_as_float(d[e]));
        }
      }
      if (r0 < most || r0 + kRows > w.rows) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int32_t row = r0 + reg_row(r) + 4 * half;
          if (row < from || row >= w.rows) s[r] = dp[r] = 0.0f;
        }
      }
      const v8b p[2] = {pack8(s, 0), pack8(s, 1)}, ds[2] = {pack8(dp, 0), pack8(dp, 1)};
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int t = 0; t < H::kTiles; ++t) {
          dv[t] = mma(H::frag_t(dout_t, 16 * j, t), p[j], dv[t]);
          dk[t] = mma(H::frag_t(qt, 16 * j, t), ds[j], dk[t]);
        }
      }
      reads_ahead<8 * H::kTiles, 4 * H::kTiles, 6>();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(0);
    }
    if (WK == 1) {
      wait_reads();
      if (r0 + kStep < w.rows) load(r0 + kStep, 0);
    } else {
      slot ^= 1;
    }
  }
  uint16_t* const to_k = a.dk.p + token * a.dk.ld_token + kvh * a.dk.ld_head;
  uint16_t* const to_v = a.dv.p + token * a.dv.ld_token + kvh * a.dv.ld_head;
  // (all loads have landed: a wave waits for its last tile's)
  float* const sums = reinterpret_cast<float*>(lds);
  const auto join = [&](v16f(&x)[H::kTiles]) {
    const auto place = [&](int group, int t, int r) {
      return sums + ((((group - 1) * WK + part) * H::kTiles + t) * 16 + r) * 64 + lane;
    };
    __syncthreads();
    if (own > 0)
#pragma unroll
      for (int t = 0; t < H::kTiles; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) *place(own, t, r) = x[t][r];
    __syncthreads();
    if (own == 0)
#pragma unroll
      for (int g = 1; g < WR; ++g)
#pragma unroll
        for (int t = 0; t < H::kTiles; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) x[t][r] += *place(g, t, r);
  };
  if (WR > 1) {
    join(dk);
    join(dv);
  }
  if (own == 0 && valid) {
    store_vector<DP>(to_k, a.dim, dk, a.scale);
    store_vector<DP>(to_v, a.dim, dv, 1.0f);
  }
}

// Forms by the number of blocks of 128 keys (of 512 that the chip holds at once).
// (All gradients of a call, causal, heads 128 wide where no width is said.)
// Few: blocks of 32 keys, whose waves share the walk.  Of these eight waves a block
// where walks are long and the blocks at most 512, else four.  A CU holds one block of
// eight waves, or two of heads up to 64 wide, by LDS, and two of four waves: 512 are up
// to two rounds of the chip, but the last block's walk is what counts (504 blocks, 11
// sequences of 1 to 1003 x 4 key heads x 5, 80 wide: 88 us, with four waves 106; 257,
// 8192 x 1 key head x 8: 930 and 1209; 312 with short walks, 2 x 600 x 8 heads: 46 and
// 35; 784, 2 x 1536 x 8 key heads x 4: 203 and 185; 1032, 4096 x 8 key heads x 4: 550
// and 529.  Over a single key head with very long walks eight would win beyond the limit
// too: 513, 16384 x 8: 2881 and 3454.)  128 keys a block and one group of waves take 221
// us for the first.  Causal, up to two rounds: the first keys' blocks would be the last
// to end, so two groups of waves share a walk (8192 x 8 key heads x 4 1840 us, one group
// 2335; not causal 3451 and 3416).  Else one group, without the second one's barriers (2
// x 4096 x 32 heads 955, with two 1000).
enum { kNarrow, kNarrowLong, kTwoGroups, kWide };
constexpr int64_t kFewBlocks = 448, kTwoRounds = 1024, kLongRows = 1536;
int32_t form_of(const AttentionBwdArgs& a) {
  const int64_t blocks = ((a.tokens_k >> kLg) + a.sequences) * a.kv_heads;
  if (blocks < kFewBlocks)
    return ((a.tokens_k >> 5) + a.sequences) * a.kv_heads <= 512 &&
                   a.tokens_q * a.group >= kLongRows * a.sequences
               ? kNarrowLong
               : kNarrow;
  return a.causal && blocks < kTwoRounds ? kTwoGroups : kWide;
}

int64_t row_tiles(const AttentionBwdArgs& a, int lg) { return (a.tokens_q * a.group >> lg) + a.sequences; }
// dq by blocks of 32 rows where those of 128 are fewer than the CUs, and a walk's length is
// what counts (all gradients, 132 blocks: 4096 tokens x 4 heads 113 us, with 128 rows
// 174; 144: 1024 x 16 heads 42, 56; 260: 2 x 2048 x 2 key heads x 4 143, 162; 288: 1024 x
// 32 heads 72.7, 73.8; 272: 2 x 512 x 8 key heads x 4 57.8, 53.9; 620: the first of the
// above 96, 91).
bool dq_narrow(const AttentionBwdArgs& a) { return row_tiles(a, kLg) * a.kv_heads <= 256; }

template <int DP, int WK, int WR>
void launch_dkv(const AttentionBwdArgs& a, hipStream_t s) {
  constexpr int kBytes = Shared<DP, WK, WR>::kBytes;
  hipLaunchKernelGGL((attention_dkv_kernel<DP, WK, WR>),
                     dim3(static_cast<uint32_t>(a.key_tiles) * a.kv_heads), dim3(64 * WK * WR),
                     kBytes, s, a);
}

template <int DP>
void launch(const AttentionBwdArgs& a, hipStream_t s) {
  if (a.tokens_q > 0 && dq_narrow(a))
    hipLaunchKernelGGL((attention_dq_narrow_kernel<DP>),
                       dim3(static_cast<uint32_t>(a.tiles) * a.kv_heads), dim3(64 * kDqWaves), 0, s, a);
  else if (a.tokens_q > 0)
    hipLaunchKernelGGL((attention_dq_kernel<DP>), dim3(static_cast<uint32_t>(a.tiles) * a.kv_heads),
                       dim3(256), 0, s, a);
  if (a.tokens_k == 0) return;
  const int32_t form = form_of(a);
  if (form == kNarrow) launch_dkv<DP, 1, 4>(a, s);
  else if (form == kNarrowLong) launch_dkv<DP, 1, 8>(a, s);
  else if (form == kTwoGroups) launch_dkv<DP, 4, 2>(a, s);
  else launch_dkv<DP, 4, 1>(a, s);
}

}  // namespace

size_t attention_backward_workspace(const AttentionBwdArgs& a) {
  return static_cast<size_t>(a.heads) * a.tokens_q * sizeof(float);
}

hipError_t launch_attention_backward(AttentionBwdArgs a, void* ws, hipStream_t s) {
  (void)hipGetLastError();
  a.delta = static_cast<float*>(ws);
  a.tiles = static_cast<int32_t>(row_tiles(a, dq_narrow(a) ? 5 : kLg));
  a.key_tiles =
      static_cast<int32_t>((a.tokens_k >> (form_of(a) <= kNarrowLong ? 5 : kLg)) + a.sequences);
  if (a.dim <= 64) launch<64>(a, s);
  else if (a.dim <= 96) launch<96>(a, s);
  else launch<128>(a, s);
  return hipGetLastError();
}

}  // namespace zf
