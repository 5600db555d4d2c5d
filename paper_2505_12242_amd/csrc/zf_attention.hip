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

// One tile of keys, from key kb of the sequence on.  mask: some row sees only
// some of them.
template <int DP>
__device__ __forceinline__ void tile_step(Rows<DP>& w, uint32_t k, uint32_t v, int32_t kb,
                                          bool mask, float c) {
  typedef Heads<DP> H;
  const int half = threadIdx.x >> 5 & 1;
  v16f s[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    s[t] = zero16();
#pragma unroll
    for (int j = 0; j < H::kChunks; ++j) s[t] = mma(H::frag(k, 32 * t, j), w.q[j], s[t]);
  }
  __builtin_amdgcn_sched_barrier(0);
  if (mask) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (kb + 32 * t + reg_row(r) + 4 * half >= w.lim) s[t][r] = -INFINITY;
  }
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
  top = fmaxf(top, other_half(top));
  // (the first tile that a row sees anything of has m = -infinity)
  if (__any(top * c > w.m * c + 8.0f)) {
    const float m = fmaxf(w.m, top);
    const float f = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((w.m - m) * c);
    w.m = m;
    w.l *= f;
#pragma unroll
    for (int t = 0; t < H::kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) w.o[t][r] *= f;
  }
  const float mc = w.m == -INFINITY ? 0.0f : w.m * c;
  v8b p[4];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], c, -mc));
      w.l += s[t][r];
    }
    p[2 * t] = pack8(s[t], 0);
    p[2 * t + 1] = pack8(s[t], 1);
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int t = 0; t < H::kTiles; ++t) w.o[t] = mma(H::frag_t(v, 16 * j, t), p[j], w.o[t]);
  __builtin_amdgcn_sched_barrier(0);
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

  // the lane's row; rows past the last repeat it, and are not stored
  const int32_t row = w.first + 32 * wave + (lane & 31);
  const bool valid = row < w.rows;
  const int32_t i = min(row, w.rows - 1) / a.group;
  const int64_t head = kvh * a.group + min(row, w.rows - 1) - i * a.group;
  Rows<DP> x;
  x.lim = keys_of(a, w, i);
  x.m = -INFINITY;
  x.l = 0.0f;
  const uint16_t* const q = a.q.p + static_cast<int64_t>(w.q0 + i) * a.q.ld_token + head * a.q.ld_head;
#pragma unroll
  for (int c = 0; c < H::kChunks; ++c) {
    const int e = 16 * c + 8 * (lane >> 5);
    u32x4 u = {0, 0, 0, 0};
    if (e < a.dim) u = *reinterpret_cast<const u32x4*>(q + e);
    x.q[c] = __builtin_bit_cast(v8b, u);
  }
#pragma unroll
  for (int t = 0; t < H::kTiles; ++t) x.o[t] = zero16();

  // keys: the wave's first and last row's, the block's last row's
  const auto token = [&](int32_t row) { return min(row, w.rows - 1) / a.group; };
  const int32_t least = uniform_i32(keys_of(a, w, token(w.first + 32 * wave)));
  const int32_t most = uniform_i32(
      w.first + 32 * wave < w.rows ? keys_of(a, w, token(w.first + 32 * wave + 31)) : 0);
  int32_t begin = 0, end = uniform_i32(keys_of(a, w, token(w.first + kRows - 1)));
  if (SPLIT) {
    const int32_t per = ((w.lk + kKeys - 1) / kKeys + a.splits - 1) / a.splits * kKeys;
    begin = static_cast<int32_t>(blockIdx.y) * per;
    end = min(end, begin + per);
  }

  const KeyLoader<DP, kKeys, 4> keys(a, w, kvh, wave);
  const uint32_t base = lds_offset(lds), rows = H::lane_rows(), columns = H::lane_columns();
  if (begin < end) keys.load(begin, base, wave);
  settle(x.q);
  int slot = 0;
  for (int32_t kb = begin; kb < end; kb += kKeys) {
    wait_dma<0>();
    if (kb + kKeys < end) keys.load(kb + kKeys, base + (slot ^ 1) * 2 * kTile, wave);
    const uint32_t at = base + slot * 2 * kTile;
    if (kb < most) tile_step<DP>(x, at + rows, at + kTile + columns, kb, kb + kKeys > least, a.scale * kLog2E);
    slot ^= 1;
  }

  const float sum = x.l + other_half(x.l);
  const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
  const float lse = sum > 0.0f || sum != sum ? fmaf(x.m, a.scale, kLn2 * __log2f(sum)) : -INFINITY;
  if (!valid) return;
  if (SPLIT) {
    const int64_t at = (static_cast<int64_t>(blockIdx.y) * a.heads + head) * a.tokens_q + w.q0 + i;
    if (lane < 32) a.part_lse[at] = lse;
    float* const o = a.part_out + at * a.dim;
#pragma unroll
    for (int t = 0; t < H::kTiles; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d = 32 * t + 8 * g + 4 * (lane >> 5);
        if (d < a.dim)
          *reinterpret_cast<u32x4*>(o + d) =
              u32x4{__float_as_uint(x.o[t][4 * g] * inv), __float_as_uint(x.o[t][4 * g + 1] * inv),
                    __float_as_uint(x.o[t][4 * g + 2] * inv), __float_as_uint(x.o[t][4 * g + 3] * inv)};
      }
  } else {
    if (a.lse != nullptr && lane < 32) a.lse[head * a.tokens_q + w.q0 + i] = lse;
    uint16_t* const o = a.out + static_cast<int64_t>(w.q0 + i) * a.ld_out_token + head * a.ld_out_head;
#pragma unroll
    for (int t = 0; t < H::kTiles; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d = 32 * t + 8 * g + 4 * (lane >> 5);
        if (d < a.dim)
          *reinterpret_cast<u32x2*>(o + d) =
              u32x2{pack_bf16(x.o[t][4 * g] * inv, x.o[t][4 * g + 1] * inv),
                    pack_bf16(x.o[t][4 * g + 2] * inv, x.o[t][4 * g + 3] * inv)};
      }
  }
}

// The splits' results of one token and head joined by a wave: weights
// exp(lse of the split - lse of all), in the splits' order.
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t n = static_cast<int64_t>(a.heads) * a.tokens_q;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (at >= n) return;
  const int64_t head = at / a.tokens_q, token = at - head * a.tokens_q;
  if (a.seq_q != nullptr && (token < a.seq_q[0] || token >= a.seq_q[a.sequences])) return;
  float top = -INFINITY;
  bool bad = false;
  for (int32_t s = 0; s < a.splits; ++s) {
    const float l = a.part_lse[s * n + at];
    bad |= l != l;
    top = fmaxf(top, l);
  }
  float sum = 0.0f, o[2] = {0.0f, 0.0f};
  const float base = top == -INFINITY ? 0.0f : top;
  for (int32_t s = 0; s < a.splits; ++s) {
    const float f = expf(a.part_lse[s * n + at] - base);
    if (f == 0.0f) continue;
    sum += f;
    const float* const p = a.part_out + (s * n + at) * a.dim;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (lane + 64 * e < a.dim) o[e] = fmaf(f, p[lane + 64 * e], o[e]);
  }
  const float inv = sum > 0.0f || bad ? 1.0f / sum : 0.0f;
  if (a.lse != nullptr && lane == 0)
    a.lse[at] = sum > 0.0f || bad ? top + logf(sum) : -INFINITY;
  uint16_t* const out = a.out + token * a.ld_out_token + head * a.ld_out_head;
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (lane + 64 * e < a.dim) out[lane + 64 * e] = round_bf16(o[e] * inv);
}

// Tiles of rows (an upper bound, see find_tile).
int64_t row_tiles(const AttentionArgs& a, int lg) {
  return (a.tokens_q * a.group >> lg) + a.sequences;
}

// Splits of the keys: where the tiles do not fill the chip, so many that they do,
// of at least 256 keys each on average.
int splits_of(const AttentionArgs& a) {
  const int64_t blocks = row_tiles(a, kRowsLg) * a.kv_heads;
  if (blocks >= 384) return 1;
  const int64_t keys = a.tokens_k / a.sequences;
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(512 / blocks, keys / 256)));
}

template <int DP>
void launch(const AttentionArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(a.tiles) * a.kv_heads, a.splits);
  if (a.splits > 1) {
    hipLaunchKernelGGL((attention_kernel<DP, true>), grid, dim3(256), 0, s, a);
    const int64_t n = static_cast<int64_t>(a.heads) * a.tokens_q;
    hipLaunchKernelGGL(attention_join_kernel, dim3(static_cast<uint32_t>((n + 3) / 4)), dim3(256), 0,
                       s, a);
  } else {
    hipLaunchKernelGGL((attention_kernel<DP, false>), grid, dim3(256), 0, s, a);
  }
}

}  // namespace

size_t attention_workspace(const AttentionArgs& a) {
  const int n = splits_of(a);
  if (n == 1) return 0;
  return static_cast<size_t>(n) * a.heads * a.tokens_q * (a.dim + 1) * sizeof(float);
}

hipError_t launch_attention(AttentionArgs a, void* ws, hipStream_t s) {
  (void)hipGetLastError();
  a.tiles = static_cast<int32_t>(row_tiles(a, kRowsLg));
  a.splits = splits_of(a);
  a.part_out = static_cast<float*>(ws);
  a.part_lse = a.part_out + static_cast<int64_t>(a.splits) * a.heads * a.tokens_q * a.dim;
  if (a.dim <= 64) launch<64>(a, s);
  else if (a.dim <= 96) launch<96>(a, s);
  else launch<128>(a, s);
  return hipGetLastError();
}

}  // namespace zf
