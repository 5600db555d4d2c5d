// Attention's forward pass (formulas and contract in zf_layer.h; rows, products
// and the layout of LDS in zf_attention.hpp).
//
// A block takes 128 rows, a wave 32 of them, and walks the keys that its last
// row sees in tiles of 64, which are loaded straight to LDS one tile ahead.
// Scores are computed transposed, keys along the registers and rows along the
// lanes: a row's maximum and sum are a lane's own (and its other half's), and
// the weights are an operand of the second product where they stand.  One pass
// with the running maximum and sum; the sums are scaled down only when the
// maximum has grown by more than 2^8, so that most tiles leave them alone.
// (The weights are rounded to bf16, as the instruction takes them, whatever power of two
// the maximum lags by: the rounding is relative.  The sum that divides them is of the
// unrounded ones.  Against 64 bits the result's relative error, 2-norm, is 2.0e-3 to
// 2.2e-3 where its own rounding makes 1.6e-3; with a second operand for what the rounding
// leaves it would be the latter, for half as many products again.)
//
// Bound by the matrix instructions and, between them, the exponentials: 16384
// tokens x 32 heads of 128, causal, 2.2e12 operations in 2.08 ms, 1.06 PFLOP/s,
// 0.84 of what the library's 8192^3 bf16 product reaches on the same card (1.26;
// the clock falls under either).  32 keys a tile and three waves a SIMD take as long;
// 256 rows a block take 3 to 5% longer where all keys are seen or heads are 64
// wide, as long elsewhere.
#include <algorithm>

#include "zf_attention.hpp"

namespace zf {
namespace {

constexpr int kRowsLg = 7, kRows = 1 << kRowsLg;  // rows of a block
constexpr int kKeys = 64;                         // keys of a tile

// A wave's 32 rows.
template <int DP>
struct Rows {
  typedef Heads<DP> H;
  v8b q[H::kChunks];
  v16f o[H::kTiles];
  float m, l;    // the running maximum (of the scores themselves), and the lane's part of the sum
  int32_t lim;   // keys that the lane's row sees
};

// A weight of 0 hides no infinity and no NaN from a product.  So in the tiles with
// weights of 0, where some row does not see keys that others do, or behind the last
// key, such elements of v become zeros in LDS, before the product, and are added
// behind the loop, to the rows that see them (add_odd).

// The halves of a word whose exponent is all ones, as 0x8000 each.
__device__ __forceinline__ uint32_t odd_halves(uint32_t x) {
  return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}
// Clears them in N KB of LDS from byte `at` on.  Whether there were any.
template <int N>
__device__ __forceinline__ bool scrub(uint32_t at) {
  uint32_t any = 0;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    auto* const p = (__attribute__((address_space(3))) u32x4*)(at + n * 1024 + 16 * (threadIdx.x & 63));
    u32x4 x = *p;
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) odd |= odd_halves(x[i]);
    if (odd != 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] &= ~((odd_halves(x[i]) >> 15) * 0xffffu);
      *p = x;
    }
    any |= odd;
  }
  return any != 0;
}
// Adds what scrub cleared of keys [from, to).
template <int DP>
__device__ __noinline__ void add_odd(const uint16_t* v, int64_t ld, int32_t dim, int32_t from,
                                     int32_t to, int32_t lim, float* o) {
  for (int32_t key = from; key < min(to, lim); ++key)
    for (int d = 4 * (threadIdx.x >> 5 & 1); d < dim; d += 8) {
      const u32x2 x = *reinterpret_cast<const u32x2*>(v + key * ld + d);
      if ((odd_halves(x.x) | odd_halves(x.y)) == 0) continue;
      for (int e = 0; e < 4; ++e) {
        const float f = widen_bf16(static_cast<uint16_t>((e & 2 ? x.y : x.x) >> (16 * (e & 1))));
        if (!(fabsf(f) < INFINITY)) o[d / 8 * 4 + e] += f;
      }
    }
}
template <int DP>
__device__ __forceinline__ void add_odd(const AttentionArgs& a, const Sequence& w, int32_t kvh,
                                        int32_t from, int32_t to, Rows<DP>& x) {
  float o[DP / 2];
#pragma unroll
  for (int i = 0; i < DP / 2; ++i) o[i] = x.o[i / 16][i % 16];
  add_odd<DP>(a.v.p + kvh * a.v.ld_head + w.k0 * a.v.ld_token, a.v.ld_token, a.dim, from, to, x.lim, o);
#pragma unroll
  for (int i = 0; i < DP / 2; ++i) x.o[i / 16][i % 16] = o[i];
}

// One tile of KEYS keys, from key kb of the sequence on.  MASK: some row may see only
// some of them.  k is read before after_scores, v behind before_values.
template <int DP, int KEYS, bool MASK, typename F, typename G>
__device__ __forceinline__ void tile_step(Rows<DP>& w, uint32_t k, uint32_t v, int32_t kb, float c,
                                          const F& after_scores,
                                          const G& before_values) {
  typedef Heads<DP> H;
  const int half = threadIdx.x >> 5 & 1;
  v16f s[KEYS / 32];
#pragma unroll
  for (int t = 0; t < KEYS / 32; ++t) {
    s[t] = zero16();
#pragma unroll
    for (int j = 0; j < H::kChunks; ++j) s[t] = mma(H::frag(k, 32 * t, j), w.q[j], s[t]);
  }
  __builtin_amdgcn_sched_barrier(0);
  after_scores();
  if (MASK) {
#pragma unroll
    for (int t = 0; t < KEYS / 32; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (kb + 32 * t + reg_row(r) + 4 * half >= w.lim) s[t][r] = -INFINITY;
  }
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < KEYS / 32; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
  top = fmaxf(top, other_half(top));
  // (The first tile that a row sees anything of has m = -infinity.  Each row by its own
  // scores: what others see is not to change its roundings.)
  const bool up = top * c > w.m * c + 8.0f;
  if (__any(up)) {
    const float f = up ? __builtin_amdgcn_exp2f((w.m - top) * c) : 1.0f;
    w.m = up ? top : w.m;
    w.l *= f;
#pragma unroll
    for (int t = 0; t < H::kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) w.o[t][r] *= f;
  }
  const float mc = w.m == -INFINITY ? 0.0f : w.m * c;
  v8b p[KEYS / 16];
#pragma unroll
  for (int t = 0; t < KEYS / 32; ++t) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], c, -mc));
      w.l += s[t][r];
    }
    p[2 * t] = pack8(s[t], 0);
    p[2 * t + 1] = pack8(s[t], 1);
  }
  before_values();
#pragma unroll
  for (int j = 0; j < KEYS / 16; ++j)
#pragma unroll
    for (int t = 0; t < H::kTiles; ++t) w.o[t] = mma(H::frag_t(v, 16 * j, t), p[j], w.o[t]);
}

// The lane's row: row `row` of the sequence, or its last where there are fewer
// (`valid`: it is the row itself).
struct Place {
  bool valid;
  int32_t token;  // of the sequence
  int64_t head;
};
__device__ __forceinline__ Place place_row(const AttentionArgs& a, const Sequence& w, int32_t kvh,
                                           int32_t row) {
  Place p;
  p.valid = row < w.rows;
  row = min(row, w.rows - 1);
  p.token = row / a.group;
  p.head = static_cast<int64_t>(kvh) * a.group + (row - p.token * a.group);
  return p;
}

template <int DP>
__device__ __forceinline__ void start_rows(const AttentionArgs& a, const Sequence& w,
                                           const Place& at, Rows<DP>& x) {
  typedef Heads<DP> H;
  x.lim = keys_of(a, w, at.token);
  x.m = -INFINITY;
  x.l = 0.0f;
  const uint16_t* const q = a.q.p + static_cast<int64_t>(w.q0 + at.token) * a.q.ld_token + at.head * a.q.ld_head;
#pragma unroll
  for (int c = 0; c < H::kChunks; ++c) {
    const int e = 16 * c + 8 * (threadIdx.x >> 5 & 1);
    u32x4 u = {0, 0, 0, 0};
    if (e < a.dim) u = *reinterpret_cast<const u32x4*>(q + e);
    x.q[c] = __builtin_bit_cast(v8b, u);
  }
#pragma unroll
  for (int t = 0; t < H::kTiles; ++t) x.o[t] = zero16();
}

// 32 elements (tile t) of a row's result, `part` < 0: of out itself.
__device__ __forceinline__ void store_out(const AttentionArgs& a, const Sequence& w, const Place& at,
                                          int32_t part, int t, const v16f& o, float inv) {
  const int64_t token = w.q0 + at.token;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int d = 32 * t + 8 * g + 4 * (threadIdx.x >> 5 & 1);
    if (d >= a.dim) continue;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = o[4 * g + e] * inv;
    if (part >= 0) {
      const int64_t row = (part * static_cast<int64_t>(a.heads) + at.head) * a.tokens_q + token;
      *reinterpret_cast<u32x4*>(a.part_out + row * a.dim + d) =
          u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    } else {
      *reinterpret_cast<u32x2*>(a.out + token * a.ld_out_token + at.head * a.ld_out_head + d) =
          u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    }
  }
}
// A row's 1 / sum and its lse, stored; zero and -infinity where it sees no key.
__device__ __forceinline__ float finish_row(const AttentionArgs& a, const Sequence& w, const Place& at,
                                            int32_t part, float m, float sum, bool store) {
  const bool any = sum > 0.0f || sum != sum;
  const float lse = any ? fmaf(m, a.scale, kLn2 * __log2f(sum)) : -INFINITY;
  if (at.valid && store) {
    const int64_t row = at.head * a.tokens_q + w.q0 + at.token;
    if (part >= 0) a.part_lse[static_cast<int64_t>(part) * a.heads * a.tokens_q + row] = lse;
    else if (a.lse != nullptr) a.lse[row] = lse;
  }
  return any ? 1.0f / sum : 0.0f;
}

// The most pieces of a sequence's keys, of either form: the join holds one a lane.
constexpr int kMaxPieces = 64;

// Keys of a piece of a sequence of lk keys, and how many pieces it has.
__device__ __forceinline__ int32_t piece_of(const AttentionArgs& a, int32_t lk) {
  return max(a.piece, ((lk + a.splits - 1) / a.splits + 127) / 128 * 128);
}
__device__ __forceinline__ int32_t pieces_of(const AttentionArgs& a, int32_t lk) {
  const int32_t piece = piece_of(a, lk);
  return max((lk + piece - 1) / piece, 1);
}

template <int DP, bool SPLIT>
__global__ __launch_bounds__(256, 2) void attention_kernel(AttentionArgs a) {
  typedef Heads<DP> H;
  constexpr int kTile = kKeys * H::kPitch;
  __shared__ __align__(1024) uint8_t lds[4 * kTile];  // two slots of k and v
  const int lane = threadIdx.x & 63, wave = uniform_i32(threadIdx.x >> 6);
  // the key head is the fastest: with a multiple of 8 of them an XCD's blocks
  // share heads in its L2.  Long tiles first.
  const int32_t kvh = blockIdx.x % a.kv_heads;
  Sequence w;
  if (!find_tile<false>(a, a.tiles - 1 - static_cast<int64_t>(blockIdx.x / a.kv_heads), kRowsLg, w)) return;
  int32_t part = -1, begin = 0;
  if (SPLIT) {
    const int32_t pieces = pieces_of(a, w.lk);
    if (static_cast<int32_t>(blockIdx.y) >= pieces) return;
    if (pieces > 1) part = blockIdx.y;
    begin = static_cast<int32_t>(blockIdx.y) * piece_of(a, w.lk);
  }
  const int32_t row0 = w.first + 32 * wave;
  const Place at = place_row(a, w, kvh, row0 + (lane & 31));
  Rows<DP> x;
  start_rows<DP>(a, w, at, x);

  // keys: the wave's first and last row's, the block's last row's
  const auto keys_at = [&](int32_t row) {
    return uniform_i32(keys_of(a, w, min(row, w.rows - 1) / a.group));
  };
  const int32_t most = row0 < w.rows ? keys_at(row0 + 31) : 0;
  int32_t end = keys_at(w.first + kRows - 1);
  if (SPLIT) end = min(end, begin + piece_of(a, w.lk));

  const KeyLoader<DP, kKeys, 4> keys(a, w, kvh, wave);
  const uint32_t base = lds_offset(lds), rows = H::lane_rows(), columns = H::lane_columns();
  if (begin < end) keys.template load<true, true>(begin, base, wave);
  settle(x.q);
  // the tiles that every row sees whole, then the others
  const int32_t whole = keys_at(w.first);
  int slot = 0, odd = 0;
  int32_t kb = begin;
  const auto step = [&](auto mask) {
    wait_dma<0>();
    if (kb + kKeys < end)
      keys.template load<true, true>(kb + kKeys, base + (slot ^ 1) * 2 * kTile, wave);
    const uint32_t in = base + slot * 2 * kTile;
    if (mask.value)
      odd |= __syncthreads_or(scrub<kTile / 4096>(in + kTile + wave * (kTile / 4)));
    if (kb < most)
      tile_step<DP, kKeys, mask.value>(x, in + rows, in + kTile + columns, kb, a.scale * kLog2E,
                                       [] {}, [] {});
    pin(x.o);
    slot ^= 1;
  };
  for (; kb < end && kb + kKeys <= whole; kb += kKeys) step(std::false_type());
  for (; kb < end; kb += kKeys) step(std::true_type());
  if (odd) add_odd<DP>(a, w, kvh, max(begin, whole / kKeys * kKeys), end, x);
  const float sum = x.l + other_half(x.l);
  const float inv = finish_row(a, w, at, part, x.m, sum, lane < 32);
  if (!at.valid) return;
#pragma unroll
  for (int t = 0; t < H::kTiles; ++t) store_out(a, w, at, part, t, x.o[t], inv);
}

// Few rows (single tokens over a cache): a block takes a piece of a sequence's keys
// for 32 of its rows at a time, and its four waves every fourth tile of 32 keys, loaded
// by the wave for itself: no barrier until the waves' results are joined in LDS.
// Bound by HBM while enough loads are in flight: k's slot is filled again as soon as
// the scores are done, v's after its product, eight waves a CU.  48 tokens x 64 heads
// over 8 key heads and 1 to 8000 keys, 832 MB: 147 us, 5.66 TB/s, 0.95 of a large
// read's rate.  (The whole call 153; where the loads are not marked as read once 171;
// with products of 16 rows, k from memory straight to registers and twice the waves, 251:
// an instruction of theirs reads 64 bytes each of 16 keys.)
constexpr int kFewWaves = 4, kFewStep = 32 * kFewWaves;  // keys of all waves' tiles
template <int DP>
struct FewRows {
  typedef Heads<DP> H;
  static constexpr int kTile = 32 * H::kPitch;
  static constexpr int kOwn = 2 * kTile;  // of a wave
  static constexpr int kStats = kFewWaves * kOwn;
  static constexpr int kBytes = kStats + 2 * kFewWaves * 32 * 4;
};
template <int DP>
__global__ __launch_bounds__(64 * kFewWaves, 2) void attention_few_kernel(AttentionArgs a) {
  typedef Heads<DP> H;
  typedef FewRows<DP> S;
  typedef KeyLoader<DP, 32, 1, true> Loader;
  constexpr int kTile = S::kTile, kN = Loader::kLoads;
  extern __shared__ __align__(1024) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = uniform_i32(threadIdx.x >> 6);
  const int32_t kvh = blockIdx.x % a.kv_heads;
  const int32_t s = static_cast<int32_t>(blockIdx.x) / a.kv_heads;
  Sequence w;
  read_sequence(a, s, w);
  const int32_t pieces = pieces_of(a, w.lk), piece = piece_of(a, w.lk);
  if (static_cast<int32_t>(blockIdx.y) >= pieces) return;
  const int32_t part = pieces > 1 ? static_cast<int32_t>(blockIdx.y) : -1;
  const int32_t begin = static_cast<int32_t>(blockIdx.y) * piece;
  const Loader keys(a, w, kvh, 0);
  const uint32_t base = lds_offset(lds) + wave * S::kOwn;
  const uint32_t rows = base + H::lane_rows(), columns = base + kTile + H::lane_columns();
  float* const stats = reinterpret_cast<float*>(lds + S::kStats);

  for (int32_t row0 = 0; row0 < w.rows; row0 += 32) {
    const Place at = place_row(a, w, kvh, row0 + (lane & 31));
    Rows<DP> x;
    start_rows<DP>(a, w, at, x);
    const int32_t least = uniform_i32(keys_of(a, w, row0 / a.group));
    const int32_t end = min(begin + piece,
                            uniform_i32(keys_of(a, w, min(row0 + 31, w.rows - 1) / a.group)));
    // the wave's tiles: from `first` on, every kFewStep keys
    const int32_t first = begin + 32 * wave;
    if (first < end) keys.template load<true, true>(first, base, 0);
    settle(x.q);
    int32_t kb = first;
    bool odd = false;
    const auto step = [&](auto mask) {
      const bool next = kb + kFewStep < end;
      wait_own_dma<kN>();  // (this v is behind this k)
      tile_step<DP, 32, mask.value>(
          x, rows, columns, kb, a.scale * kLog2E,
          [&] {
            wait_reads();
            if (next) keys.template load<true, false>(kb + kFewStep, base, 0);
          },
          [&] {
            if (next) wait_own_dma<kN>();
            else wait_own_dma<0>();
            if (mask.value) odd |= scrub<S::kTile / 1024>(base + kTile);
          });
      wait_reads();
      if (next) keys.template load<false, true>(kb + kFewStep, base + kTile, 0);
      pin(x.o);
    };
    for (; kb < end && kb + 32 <= least; kb += kFewStep) step(std::false_type());
    const int32_t from = kb;
    for (; kb < end; kb += kFewStep) step(std::true_type());
    if (__any(odd))
      for (int32_t t = from; t < end; t += kFewStep) add_odd<DP>(a, w, kvh, t, min(t + 32, end), x);
    // the waves' results: the largest maximum, then the sums with their factors
    const float sum = x.l + other_half(x.l);
    __syncthreads();
    if (lane < 32) {
      stats[wave * 32 + lane] = x.m;
      stats[(kFewWaves + wave) * 32 + lane] = sum;
    }
    float* const sums = reinterpret_cast<float*>(lds);
    const auto place = [&](int wave, int t, int r) {
      return sums + ((wave * H::kTiles + t) * 16 + r) * 64 + lane;
    };
#pragma unroll
    for (int t = 0; t < H::kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) *place(wave, t, r) = x.o[t][r];
    __syncthreads();
    float m = -INFINITY, f[kFewWaves], all = 0.0f;
#pragma unroll
    for (int v = 0; v < kFewWaves; ++v) m = fmaxf(m, stats[v * 32 + (lane & 31)]);
    const float c = a.scale * kLog2E;
#pragma unroll
    for (int v = 0; v < kFewWaves; ++v) {
      const float n = stats[v * 32 + (lane & 31)], l = stats[(kFewWaves + v) * 32 + (lane & 31)];
      // (a wave that saw nothing has no part, but a NaN has)
      f[v] = n == -INFINITY && l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((n - (m == -INFINITY ? 0.0f : m)) * c);
      all += f[v] * l;
    }
    const float inv = finish_row(a, w, at, part, m, all, lane < 32 && wave == 0);
#pragma unroll 1
    for (int t = wave; t < H::kTiles; t += kFewWaves) {
      v16f o;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        o[r] = 0.0f;
#pragma unroll
        for (int v = 0; v < kFewWaves; ++v)
          if (f[v] != 0.0f) o[r] = fmaf(f[v], *place(v, t, r), o[r]);
      }
      if (at.valid) store_out(a, w, at, part, t, o, inv);
    }
    wait_own_dma<0>();  // (the stores: the next rows' loads are counted alone)
    __syncthreads();
  }
}

// The pieces' results of one token and head joined by W waves: weights exp(lse of the
// piece - lse of all) (a piece a lane, at most kMaxPieces); wave w adds pieces w, w + W, ...
// in order, and the waves' sums are added in order.  W 4 where there are many pieces, 1
// where many rows (512 tokens x 32 heads in 4 pieces: the whole call 58 us, with 4
// waves 75).
template <int W>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a) {
  static_assert(kMaxPieces <= 64, "a piece a lane");
  __shared__ float sums[W > 1 ? W - 1 : 1][128];
  const int lane = threadIdx.x & 63, index = uniform_i32(threadIdx.x >> 6);
  const int wave = W == 1 ? 0 : index;
  const int64_t n = static_cast<int64_t>(a.heads) * a.tokens_q;
  const int64_t at = W == 1 ? static_cast<int64_t>(blockIdx.x) * 4 + index : blockIdx.x;
  if (at >= n) return;
  const int64_t head = at / a.tokens_q, token = at - head * a.tokens_q;
  int32_t s = 0;
  if (a.seq_q != nullptr) {
    s = find_sequence(a.sequences,
                      [&](int32_t i) { return clamp_token(a.seq_q[i], a.tokens_q) <= token; });
    if (s < 0) return;
  }
  Sequence w;
  read_sequence(a, s, w);
  if (token >= w.q0 + w.lq) return;
  const int32_t pieces = pieces_of(a, w.lk);
  if (pieces == 1) return;  // (written already)
  const float lse = lane < pieces ? a.part_lse[lane * n + at] : -INFINITY;
  float top = lse;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float f = expf(lse - (top == -INFINITY ? 0.0f : top));  // (a NaN stays one)
  float sum = f;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  const int e = 2 * lane;
  float o[2] = {0.0f, 0.0f};
#pragma unroll 4
  for (int32_t p = wave; p < pieces; p += W) {
    const float g = __shfl(f, p);
    float2 v = {0.0f, 0.0f};
    if (e < a.dim) v = *reinterpret_cast<const float2*>(a.part_out + (p * n + at) * a.dim + e);
    o[0] = fmaf(g, v.x, o[0]);
    o[1] = fmaf(g, v.y, o[1]);
  }
  if constexpr (W > 1) {
    if (wave > 0) {
      sums[wave - 1][e] = o[0];
      sums[wave - 1][e + 1] = o[1];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int v = 0; v < W - 1; ++v) {
      o[0] += sums[v][e];
      o[1] += sums[v][e + 1];
    }
  }
  const bool any = sum > 0.0f || sum != sum;
  const float inv = any ? 1.0f / sum : 0.0f;
  if (a.lse != nullptr && lane == 0) a.lse[at] = any ? top + logf(sum) : -INFINITY;
  if (e < a.dim)
    *reinterpret_cast<uint32_t*>(a.out + token * a.ld_out_token + head * a.ld_out_head + e) =
        pack_bf16(o[0] * inv, o[1] * inv);
}

// Tiles of rows (an upper bound, see find_tile).
int64_t row_tiles(const AttentionArgs& a, int lg) {
  return (a.tokens_q * a.group >> lg) + a.sequences;
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int32_t pieces_within(int64_t splits) {
  return static_cast<int32_t>(std::min<int64_t>(kMaxPieces, std::max<int64_t>(1, splits)));
}

// How a call is done.  Up to 8 rows a sequence (on average: the lengths are on the
// device): by sequences and pieces of keys (48 tokens of 8 rows over 1 to 8000 keys 153
// us, by tiles 194; 8 tokens x 32 key heads over 4096 keys 93, not 98; with 16 rows, 16
// sequences x 8 key heads over 4096 keys, 55, by tiles 52.7; with 32 rows 61 and 54.4).
// A block walks all rows of its sequence, 32 at a time, so that one long prompt among
// many tokens sets the call's time (4096 tokens among 1024 single ones, 32 heads: 4.08 ms,
// in two calls 0.70; 8 heads 3.55 and 0.22).
// Else by tiles of 128 rows, and by pieces of keys as often as the 512 blocks that the
// chip holds allow (512 tokens x 32 heads over 4096 keys 60 us, whole 76; 1024 x 32
// heads, 288 blocks, 25, in 3 pieces 42).
struct Form {
  bool few;
  int32_t splits, piece;
};
Form form_of(const AttentionArgs& a) {
  const int64_t rows = a.tokens_q * a.group, most = ceil_div(a.tokens_k, 128);
  if (rows <= 8 * static_cast<int64_t>(a.sequences)) {
    // pieces of 128 to 1024 keys, so that there are some 256 of them, a CU each (512
    // leave more to join: one token x 8 key heads over 32768 keys 32.3 us, not 36.9), and
    // so many of a sequence that one of more than the average length has them too
    const int64_t blocks = static_cast<int64_t>(a.sequences) * a.kv_heads;
    const int64_t piece = 128 * std::min<int64_t>(8, std::max<int64_t>(1, a.tokens_k * a.kv_heads / (256 * 128)));
    const int64_t splits = std::min(ceil_div(a.tokens_k, piece),
                                    std::max(ceil_div(a.tokens_k, piece * a.sequences), 2048 / blocks));
    return Form{true, pieces_within(splits), static_cast<int32_t>(piece)};
  }
  const int64_t blocks = row_tiles(a, kRowsLg) * a.kv_heads;
  return Form{false, pieces_within(std::min(512 / blocks, most / 2)), 256};
}

template <int DP>
void launch(const AttentionArgs& a, bool few, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(few ? a.sequences : a.tiles) * a.kv_heads, a.splits);
  constexpr int kFewBytes = FewRows<DP>::kBytes;
  if (few) hipLaunchKernelGGL((attention_few_kernel<DP>), grid, dim3(64 * kFewWaves), kFewBytes, s, a);
  else if (a.splits > 1) hipLaunchKernelGGL((attention_kernel<DP, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((attention_kernel<DP, false>), grid, dim3(256), 0, s, a);
  if (a.splits == 1) return;
  const int64_t n = static_cast<int64_t>(a.heads) * a.tokens_q;
  if (a.splits > 8)
    hipLaunchKernelGGL(attention_join_kernel<4>, dim3(static_cast<uint32_t>(n)), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(attention_join_kernel<1>, dim3(static_cast<uint32_t>((n + 3) / 4)), dim3(256),
                       0, s, a);
}

}  // namespace

size_t attention_workspace(const AttentionArgs& a) {
  const int64_t n = form_of(a).splits;
  return n == 1 ? 0 : static_cast<size_t>(n * a.heads * a.tokens_q * (a.dim + 1)) * sizeof(float);
}

hipError_t launch_attention(AttentionArgs a, void* ws, hipStream_t s) {
  (void)hipGetLastError();
  a.tiles = static_cast<int32_t>(row_tiles(a, kRowsLg));
  const Form form = form_of(a);
  a.splits = form.splits;
  a.piece = form.piece;
  a.part_out = static_cast<float*>(ws);
  a.part_lse = a.part_out + static_cast<int64_t>(a.splits) * a.heads * a.tokens_q * a.dim;
  if (a.dim <= 64) launch<64>(a, form.few, s);
  else if (a.dim <= 96) launch<96>(a, form.few, s);
  else launch<128>(a, form.few, s);
  return hipGetLastError();
}

}  // namespace zf
