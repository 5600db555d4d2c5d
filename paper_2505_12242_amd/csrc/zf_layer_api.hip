// Host entry points of include/zf_layer.h: argument validation, Adam constants
// and the AdamW plan.  Every check runs before the first HIP call.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <new>
#include <vector>

#include "zf_attention.hpp"
#include "zf_layer.hpp"

namespace {

using zf::hip_fail;

constexpr int64_t kSizeLimit = int64_t(1) << 30;
constexpr int64_t kStrideLimit = int64_t(1) << 23;
constexpr int64_t kGridLimit = int64_t(1) << 24;  // blocks of 256 threads in a dispatch

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool size_ok(int64_t x) { return x >= 0 && x < kSizeLimit; }
bool dtype_ok(int32_t t) { return t == ZF_BF16 || t == ZF_F32; }
size_t dtype_size(int32_t t) { return t == ZF_F32 ? 4 : 2; }
hipStream_t as_stream(zf_stream s) { return static_cast<hipStream_t>(s); }

// A [rows][ld] buffer's bytes, lo == hi where it holds nothing.  `ok` is
// cleared when it is missing, misaligned or its stride too small or so large
// that its end passes 2^62 bytes.
struct Span {
  uintptr_t lo = 0, hi = 0;
};

Span span(const void* p, int64_t rows, int64_t width, int64_t ld, size_t elem, bool& ok) {
  Span s;
  if (ld < width) ok = false;
  if (rows <= 0 || width <= 0 || !ok) return s;
  if (p == nullptr || !aligned(p, elem) || ld > (int64_t(1) << 31)) {
    ok = false;
    return s;
  }
  s.lo = reinterpret_cast<uintptr_t>(p);
  s.hi = s.lo + (static_cast<uintptr_t>(rows - 1) * static_cast<uintptr_t>(ld) +
                 static_cast<uintptr_t>(width)) * elem;
  return s;
}

bool overlaps(const Span& a, const Span& b) {
  return a.hi > a.lo && b.hi > b.lo && a.lo < b.hi && b.lo < a.hi;
}

// No span of `out` meets another of `out` or one of `in`.
bool disjoint(const std::initializer_list<Span>& out, const std::initializer_list<Span>& in) {
  for (auto a = out.begin(); a != out.end(); ++a) {
    for (auto b = a + 1; b != out.end(); ++b)
      if (overlaps(*a, *b)) return false;
    for (const Span& b : in)
      if (overlaps(*a, b)) return false;
  }
  return true;
}

struct Fp8Spans {
  Span data, scale;
};

// Validates an 8-bit operand of rows x cols.
Fp8Spans fp8_spans(const zf_fp8* f, int64_t rows, int64_t cols, bool& ok) {
  Fp8Spans s;
  if (f->group != 1 && f->group != zf::kFp8Group) ok = false;
  if (f->ld_data % 16 != 0 || f->ld_scale % 4 != 0) ok = false;
  if (!ok || rows == 0 || cols == 0) return s;
  s.data = span(f->data, rows, cols, f->ld_data, 1, ok);
  s.scale = span(f->scale, ceil_div(rows, f->group), ceil_div(cols, zf::kFp8Group), f->ld_scale, 1,
                 ok);
  if (!aligned(f->data, 16) || !aligned(f->scale, 4)) ok = false;
  return s;
}

zf::Fp8Out fp8_out(const zf_fp8* f) {
  if (f == nullptr) return zf::Fp8Out{nullptr, 0, nullptr, 0};
  return zf::Fp8Out{f->data, f->ld_data, f->scale, f->ld_scale};
}

zf::MatmulOperand operand(const zf_fp8* f) {
  return zf::MatmulOperand{f->data, f->ld_data, f->scale, f->ld_scale, f->group == 1 ? 0 : 7};
}

zf_status done(hipError_t e) { return e == hipSuccess ? ZF_OK : hip_fail(e); }

// An output in place of an input: the same elements, or apart from it.
bool apart_or_same(const Span& so, const void* out, int64_t ld_out, const Span& si, const void* in,
                   int64_t ld_in, int64_t rows) {
  return !overlaps(so, si) || (out == in && (rows <= 1 || ld_out == ld_in));
}

// A workspace of `need` bytes, 16-byte aligned, as a span.
zf_status workspace_span(void* ws, size_t ws_bytes, size_t need, bool ok, Span& s) {
  if (!ok) return ZF_EINVAL;
  if (need == 0) return ZF_OK;
  if (ws_bytes < need) return ZF_EWORKSPACE;
  if (ws == nullptr || !aligned(ws, 16)) return ZF_EINVAL;
  s.lo = reinterpret_cast<uintptr_t>(ws);
  s.hi = s.lo + need;
  return ZF_OK;
}

bool activation_ok(int32_t a) { return a >= ZF_NONE && a <= ZF_SILU; }

// What a product's tiles can address (32-bit offsets inside one) and a launch hold.
bool product_ok(const zf_fp8* a, const zf_fp8* b, int64_t m, int64_t n, int64_t k) {
  return k < kStrideLimit &&
         (m <= 1 || k == 0 || (a->ld_data < kStrideLimit && a->ld_scale < kStrideLimit)) &&
         (n <= 1 || k == 0 || (b->ld_data < kStrideLimit && b->ld_scale < kStrideLimit)) &&
         ceil_div(m, 128) * ceil_div(n, 128) < kGridLimit;
}

// ---- attention ----

bool attention_ok(const zf_attention* a) {
  if (a == nullptr || !size_ok(a->tokens_q) || !size_ok(a->tokens_k) || a->sequences < 1 ||
      a->kv_heads < 1 || a->heads < 1 || a->heads > (1 << 16) || a->heads % a->kv_heads != 0 ||
      a->dim < 8 || a->dim > 128 || a->dim % 8 != 0 || !std::isfinite(a->scale) || !(a->scale > 0.0f))
    return false;
  if ((a->seq_q == nullptr) != (a->seq_k == nullptr)) return false;
  if (a->seq_q == nullptr && (a->sequences != 1 || a->len_k != nullptr)) return false;
  if (!aligned(a->seq_q, 4) || !aligned(a->seq_k, 4) || !aligned(a->len_k, 4)) return false;
  // rows and keys, of all heads, that a launch's blocks (of 512 threads) still
  // reach, and that 32 bits count
  return (std::max(a->tokens_q * a->heads, a->tokens_k * a->kv_heads) / 16 +
          static_cast<int64_t>(a->sequences) * a->kv_heads) < kGridLimit / 2;
}

// Bytes from the first to past the last element.  `ok` is cleared where the
// tensor is missing, misaligned or its strides outside their limits.
Span heads_span(const zf_heads* t, int64_t tokens, int64_t heads, int64_t dim, bool& ok) {
  Span s;
  if (t == nullptr) ok = false;
  if (!ok || tokens == 0) return s;
  if (t->data == nullptr || !aligned(t->data, 16) || t->ld_token < 0 || t->ld_head < 0 ||
      t->ld_token % 8 != 0 || t->ld_head % 8 != 0 || t->ld_token >= kStrideLimit ||
      t->ld_head >= (int64_t(1) << 40)) {
    ok = false;
    return s;
  }
  s.lo = reinterpret_cast<uintptr_t>(t->data);
  s.hi = s.lo + static_cast<uintptr_t>((tokens - 1) * t->ld_token + (heads - 1) * t->ld_head + dim) * 2;
  return s;
}

// No two vectors of a tensor share an element: tokens and heads are nested one
// way or the other.
bool rows_apart(const zf_heads* t, int64_t tokens, int64_t heads, int64_t dim) {
  if (tokens <= 1 && heads <= 1) return true;
  const int64_t lt = t->ld_token, lh = t->ld_head;
  if (tokens <= 1) return lh >= dim;
  if (heads <= 1) return lt >= dim;
  return (lh >= dim && lt >= (heads - 1) * lh + dim) || (lt >= dim && lh >= (tokens - 1) * lt + dim);
}

// Two tensors share no element: their bytes lie apart, or both are columns of
// rows of one length.
bool heads_apart(const zf_heads* a, int64_t tokens_a, int64_t heads_a, const zf_heads* b,
                 int64_t tokens_b, int64_t heads_b, int64_t dim) {
  bool ok = true;
  const Span sa = heads_span(a, tokens_a, heads_a, dim, ok);
  const Span sb = heads_span(b, tokens_b, heads_b, dim, ok);
  if (!overlaps(sa, sb)) return true;
  const uintptr_t row = static_cast<uintptr_t>(a->ld_token) * 2;
  if (a->ld_token != b->ld_token || row == 0) return false;
  const uintptr_t wa = static_cast<uintptr_t>((heads_a - 1) * a->ld_head + dim) * 2;
  const uintptr_t wb = static_cast<uintptr_t>((heads_b - 1) * b->ld_head + dim) * 2;
  // b's first column among a's rows
  const uintptr_t at = sb.lo >= sa.lo ? (sb.lo - sa.lo) % row : (row - (sa.lo - sb.lo) % row) % row;
  return at >= wa && at + wb <= row;
}

struct SequenceSpans {
  Span q, k, len;
};
SequenceSpans sequence_spans(const zf_attention& a) {
  const auto ints = [](const int32_t* p, int64_t n) {
    Span s;
    if (p != nullptr) {
      s.lo = reinterpret_cast<uintptr_t>(p);
      s.hi = s.lo + static_cast<uintptr_t>(n) * 4;
    }
    return s;
  };
  return {ints(a.seq_q, a.sequences + int64_t(1)), ints(a.seq_k, a.sequences + int64_t(1)),
          ints(a.len_k, a.sequences)};
}

zf::HeadsArg heads_arg(const zf_heads* t) {
  return zf::HeadsArg{static_cast<uint16_t*>(t->data), t->ld_token, t->ld_head};
}

zf::AttentionArgs attention_args(const zf_attention& a) {
  zf::AttentionArgs r{};
  r.seq_q = a.seq_q;
  r.seq_k = a.seq_k;
  r.len_k = a.len_k;
  r.tokens_q = a.tokens_q;
  r.tokens_k = a.tokens_k;
  r.sequences = a.sequences;
  r.heads = a.heads;
  r.kv_heads = a.kv_heads;
  r.group = a.heads / a.kv_heads;
  r.dim = a.dim;
  r.causal = a.causal != 0;
  r.scale = a.scale;
  return r;
}

zf::AttentionBwdArgs attention_bwd_args(const zf_attention& a) {
  zf::AttentionBwdArgs r{};
  r.seq_q = a.seq_q;
  r.seq_k = a.seq_k;
  r.tokens_q = a.tokens_q;
  r.tokens_k = a.tokens_k;
  r.sequences = a.sequences;
  r.heads = a.heads;
  r.kv_heads = a.kv_heads;
  r.group = a.heads / a.kv_heads;
  r.dim = a.dim;
  r.causal = a.causal != 0;
  r.scale = a.scale;
  return r;
}

}  // namespace

extern "C" {

zf_status zf_quantize_fp8(const void* x, int32_t x_dtype, int64_t rows, int64_t cols,
                          int64_t ld_x, const zf_fp8* out, const zf_fp8* out_t,
                          zf_stream stream) {
  if (!dtype_ok(x_dtype) || !size_ok(rows) || !size_ok(cols) ||
      (out == nullptr && out_t == nullptr) ||
      (out != nullptr && out_t != nullptr && out->group != out_t->group))
    return ZF_EINVAL;
  bool ok = true;
  const Span sx = span(x, rows, cols, ld_x, dtype_size(x_dtype), ok);
  Fp8Spans q, qt;
  if (out != nullptr) q = fp8_spans(out, rows, cols, ok);
  if (out_t != nullptr) qt = fp8_spans(out_t, cols, rows, ok);
  if (!ok || ceil_div(rows, 128) * ceil_div(cols, 128) >= kGridLimit ||
      !disjoint({q.data, q.scale, qt.data, qt.scale}, {sx}))
    return ZF_EINVAL;
  if (rows == 0 || cols == 0) return ZF_OK;
  const zf::QuantArgs a{x, rows, cols, ld_x, fp8_out(out), fp8_out(out_t)};
  return done(zf::launch_quantize(a, x_dtype, (out != nullptr ? out : out_t)->group,
                                  as_stream(stream)));
}

size_t zf_matmul_fp8_workspace_bytes(int64_t m, int64_t n, int64_t k) {
  if (!size_ok(m) || !size_ok(n) || !size_ok(k) || m == 0 || n == 0) return 0;
  return zf::matmul_workspace(m, n, k);
}

zf_status zf_matmul_fp8(const zf_fp8* a, const zf_fp8* b, int64_t m, int64_t n, int64_t k,
                        void* out, int32_t out_dtype, int64_t ld_out, void* ws, size_t ws_bytes,
                        zf_stream stream) {
  if (a == nullptr || b == nullptr || !dtype_ok(out_dtype) || !size_ok(m) || !size_ok(n) ||
      !size_ok(k))
    return ZF_EINVAL;
  bool ok = true;
  const Fp8Spans sa = fp8_spans(a, m, k, ok), sb = fp8_spans(b, n, k, ok);
  const Span so = span(out, m, n, ld_out, dtype_size(out_dtype), ok);
  // a tile's rows are addressed through 32-bit offsets
  if (k >= kStrideLimit ||
      (m > 1 && k > 0 && (a->ld_data >= kStrideLimit || a->ld_scale >= kStrideLimit)) ||
      (n > 1 && k > 0 && (b->ld_data >= kStrideLimit || b->ld_scale >= kStrideLimit)))
    ok = false;
  if (!ok || ceil_div(m, 128) * ceil_div(n, 128) >= kGridLimit) return ZF_EINVAL;
  const size_t need = zf_matmul_fp8_workspace_bytes(m, n, k);
  Span sw;
  if (need > 0) {
    if (ws_bytes < need) return ZF_EWORKSPACE;
    if (ws == nullptr || !aligned(ws, 16)) return ZF_EINVAL;
    sw.lo = reinterpret_cast<uintptr_t>(ws);
    sw.hi = sw.lo + need;
  }
  if (!disjoint({so, sw}, {sa.data, sa.scale, sb.data, sb.scale})) return ZF_EINVAL;
  if (m == 0 || n == 0) return ZF_OK;
  const zf::MatmulArgs args{operand(a), operand(b), m, n, k, out, ld_out,
                            out_dtype == ZF_F32 ? 1 : 0, 0};
  return done(zf::launch_matmul(args, ws, as_stream(stream)));
}

zf_status zf_rmsnorm_forward(const void* x, int64_t ld_x, const void* residual,
                             int64_t ld_residual, int32_t dtype, int64_t rows, int64_t cols,
                             const void* gain, int32_t gain_dtype, double eps, void* h,
                             int64_t ld_h, void* y, int64_t ld_y, const zf_fp8* q, float* rstd,
                             zf_stream stream) {
  if (!dtype_ok(dtype) || !dtype_ok(gain_dtype) || !size_ok(rows) || !size_ok(cols) ||
      !std::isfinite(eps) || !(eps >= 0.0))
    return ZF_EINVAL;
  const size_t e = dtype_size(dtype);
  bool ok = true;
  Span sr, sh, sy;
  Fp8Spans sq;
  const Span sx = span(x, rows, cols, ld_x, e, ok);
  const Span sg = span(gain, rows == 0 ? 0 : 1, cols, cols, dtype_size(gain_dtype), ok);
  const Span st = span(rstd, 1, rows, rows, 4, ok);
  if (residual != nullptr) {
    sr = span(residual, rows, cols, ld_residual, e, ok);
    if (h == nullptr && rows > 0 && cols > 0) ok = false;
  }
  if (h != nullptr) sh = span(h, rows, cols, ld_h, e, ok);
  if (y != nullptr) sy = span(y, rows, cols, ld_y, e, ok);
  if (q != nullptr) {
    if (q->group != 1) ok = false;
    sq = fp8_spans(q, rows, cols, ok);
  }
  if (!ok || !disjoint({sh, sy, sq.data, sq.scale, st}, {sg}) ||
      !disjoint({sy, sq.data, sq.scale, st}, {sx, sr}))
    return ZF_EINVAL;
  // h in place of an input: the same elements, or apart from it
  if ((overlaps(sh, sx) && (h != x || (rows > 1 && ld_h != ld_x))) ||
      (overlaps(sh, sr) && (h != residual || (rows > 1 && ld_h != ld_residual))))
    return ZF_EINVAL;
  if (rows == 0) return ZF_OK;
  const zf::NormArgs a{x, ld_x, residual, ld_residual, rows, cols, gain, gain_dtype == ZF_F32,
                       static_cast<float>(eps), h, ld_h, y, ld_y, fp8_out(q), rstd};
  return done(zf::launch_rmsnorm(a, dtype, as_stream(stream)));
}

size_t zf_rmsnorm_backward_workspace_bytes(int64_t rows, int64_t cols) {
  if (!size_ok(rows) || !size_ok(cols)) return 0;
  return zf::rmsnorm_backward_workspace(rows, cols);
}

zf_status zf_rmsnorm_backward(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h,
                              int32_t dtype, int64_t rows, int64_t cols, const void* gain,
                              int32_t gain_dtype, const float* rstd, const void* dresidual,
                              int64_t ld_dresidual, void* dx, int64_t ld_dx, float* dgain,
                              void* ws, size_t ws_bytes, zf_stream stream) {
  if (!dtype_ok(dtype) || !dtype_ok(gain_dtype) || !size_ok(rows) || !size_ok(cols))
    return ZF_EINVAL;
  const size_t e = dtype_size(dtype);
  bool ok = true;
  Span sr, sd, sw;
  const Span sy = span(dy, rows, cols, ld_dy, e, ok);
  const Span sh = span(h, rows, cols, ld_h, e, ok);
  const Span sx = span(dx, rows, cols, ld_dx, e, ok);
  const Span sg = span(gain, rows == 0 ? 0 : 1, cols, cols, dtype_size(gain_dtype), ok);
  const Span st = span(rstd, cols == 0 ? 0 : 1, rows, rows, 4, ok);
  if (dresidual != nullptr) sr = span(dresidual, rows, cols, ld_dresidual, e, ok);
  if (dgain != nullptr) {
    sd = span(dgain, 1, cols, cols, 4, ok);
    const size_t need = zf_rmsnorm_backward_workspace_bytes(rows, cols);
    if (ok && need > 0) {
      if (ws_bytes < need) return ZF_EWORKSPACE;
      if (ws == nullptr || !aligned(ws, 16)) return ZF_EINVAL;
      sw.lo = reinterpret_cast<uintptr_t>(ws);
      sw.hi = sw.lo + need;
    }
  }
  if (!ok || !disjoint({sx, sd, sw}, {sh, sg, st}) || !disjoint({sd, sw}, {sy, sr}))
    return ZF_EINVAL;
  if ((overlaps(sx, sy) && (dx != dy || (rows > 1 && ld_dx != ld_dy))) ||
      (overlaps(sx, sr) && (dx != dresidual || (rows > 1 && ld_dx != ld_dresidual))))
    return ZF_EINVAL;
  if (cols == 0 || (rows == 0 && dgain == nullptr)) return ZF_OK;
  const zf::NormBwdArgs a{dy, ld_dy, h, ld_h, rows, cols, gain, gain_dtype == ZF_F32, rstd,
                          dresidual, ld_dresidual, dx, ld_dx, dgain, static_cast<float*>(ws)};
  return done(zf::launch_rmsnorm_backward(a, dtype, as_stream(stream)));
}

zf_status zf_layernorm_forward(const void* x, int64_t ld_x, const void* residual,
                               int64_t ld_residual, int32_t dtype, int64_t rows, int64_t cols,
                               const void* gain, const void* bias, int32_t gain_dtype, double eps,
                               void* h, int64_t ld_h, void* y, int64_t ld_y, const zf_fp8* q,
                               float* mean, float* rstd, zf_stream stream) {
  if (!dtype_ok(dtype) || !dtype_ok(gain_dtype) || !size_ok(rows) || !size_ok(cols) ||
      !std::isfinite(eps) || !(eps >= 0.0))
    return ZF_EINVAL;
  const size_t e = dtype_size(dtype);
  bool ok = true;
  Span sr, sh, sy, sb;
  Fp8Spans sq;
  const Span sx = span(x, rows, cols, ld_x, e, ok);
  const Span sg = span(gain, rows == 0 ? 0 : 1, cols, cols, dtype_size(gain_dtype), ok);
  if (bias != nullptr) sb = span(bias, rows == 0 ? 0 : 1, cols, cols, dtype_size(gain_dtype), ok);
  const Span sm = span(mean, 1, rows, rows, 4, ok);
  const Span st = span(rstd, 1, rows, rows, 4, ok);
  if (residual != nullptr) {
    sr = span(residual, rows, cols, ld_residual, e, ok);
    if (h == nullptr && rows > 0 && cols > 0) ok = false;
  }
  if (h != nullptr) sh = span(h, rows, cols, ld_h, e, ok);
  if (y != nullptr) sy = span(y, rows, cols, ld_y, e, ok);
  if (q != nullptr) {
    if (q->group != 1) ok = false;
    sq = fp8_spans(q, rows, cols, ok);
  }
  if (!ok || !disjoint({sh, sy, sq.data, sq.scale, sm, st}, {sg, sb}) ||
      !disjoint({sy, sq.data, sq.scale, sm, st}, {sx, sr}))
    return ZF_EINVAL;
  // h in place of an input: the same elements, or apart from it
  if (!apart_or_same(sh, h, ld_h, sx, x, ld_x, rows) ||
      !apart_or_same(sh, h, ld_h, sr, residual, ld_residual, rows))
    return ZF_EINVAL;
  if (rows == 0) return ZF_OK;
  const zf::LayerNormArgs a{x, ld_x, residual, ld_residual, rows, cols, gain, bias,
                            gain_dtype == ZF_F32, static_cast<float>(eps), h, ld_h, y, ld_y,
                            fp8_out(q), mean, rstd};
  return done(zf::launch_layernorm(a, dtype, as_stream(stream)));
}

size_t zf_layernorm_backward_workspace_bytes(int64_t rows, int64_t cols) {
  if (!size_ok(rows) || !size_ok(cols)) return 0;
  return zf::layernorm_backward_workspace(rows, cols);
}

zf_status zf_layernorm_backward(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h,
                                int32_t dtype, int64_t rows, int64_t cols, const void* gain,
                                int32_t gain_dtype, const float* mean, const float* rstd,
                                const void* dresidual, int64_t ld_dresidual, void* dx,
                                int64_t ld_dx, float* dgain, float* dbias, void* ws,
                                size_t ws_bytes, zf_stream stream) {
  if (!dtype_ok(dtype) || !dtype_ok(gain_dtype) || !size_ok(rows) || !size_ok(cols))
    return ZF_EINVAL;
  const size_t e = dtype_size(dtype);
  bool ok = true;
  Span sr, sd, sb, sw;
  const Span sy = span(dy, rows, cols, ld_dy, e, ok);
  const Span sh = span(h, rows, cols, ld_h, e, ok);
  const Span sx = span(dx, rows, cols, ld_dx, e, ok);
  const Span sg = span(gain, rows == 0 ? 0 : 1, cols, cols, dtype_size(gain_dtype), ok);
  const Span sm = span(mean, cols == 0 ? 0 : 1, rows, rows, 4, ok);
  const Span st = span(rstd, cols == 0 ? 0 : 1, rows, rows, 4, ok);
  if (dresidual != nullptr) sr = span(dresidual, rows, cols, ld_dresidual, e, ok);
  if (dgain != nullptr) sd = span(dgain, 1, cols, cols, 4, ok);
  if (dbias != nullptr) sb = span(dbias, 1, cols, cols, 4, ok);
  if (dgain != nullptr || dbias != nullptr) {
    const zf_status st_ws = workspace_span(ws, ws_bytes,
                                           zf_layernorm_backward_workspace_bytes(rows, cols), ok, sw);
    if (st_ws != ZF_OK) return st_ws;
  }
  if (!ok || !disjoint({sx, sd, sb, sw}, {sh, sg, sm, st}) || !disjoint({sd, sb, sw}, {sy, sr}))
    return ZF_EINVAL;
  if (!apart_or_same(sx, dx, ld_dx, sy, dy, ld_dy, rows) ||
      !apart_or_same(sx, dx, ld_dx, sr, dresidual, ld_dresidual, rows))
    return ZF_EINVAL;
  if (cols == 0 || (rows == 0 && dgain == nullptr && dbias == nullptr)) return ZF_OK;
  const zf::LayerNormBwdArgs a{dy, ld_dy, h, ld_h, rows, cols, gain, gain_dtype == ZF_F32, mean, rstd,
                               dresidual, ld_dresidual, dx, ld_dx, dgain, dbias,
                               static_cast<float*>(ws)};
  return done(zf::launch_layernorm_backward(a, dtype, as_stream(stream)));
}

size_t zf_linear_fp8_workspace_bytes(int64_t m, int64_t n, int64_t k, int32_t q) {
  if (!size_ok(m) || !size_ok(n) || !size_ok(k) || m == 0 || n == 0) return 0;
  return zf::linear_workspace(m, n, k, q != 0);
}

zf_status zf_linear_fp8(const zf_fp8* a, const zf_fp8* b, int64_t m, int64_t n, int64_t k,
                        const zf_epilogue* e, void* ws, size_t ws_bytes, zf_stream stream) {
  if (a == nullptr || b == nullptr || e == nullptr || !dtype_ok(e->dtype) ||
      !dtype_ok(e->bias_dtype) || !activation_ok(e->activation) || !size_ok(m) || !size_ok(n) ||
      !size_ok(k) || (e->z == nullptr && e->y == nullptr && e->q == nullptr))
    return ZF_EINVAL;
  bool ok = true;
  const size_t size = dtype_size(e->dtype);
  const Fp8Spans sa = fp8_spans(a, m, k, ok), sb = fp8_spans(b, n, k, ok);
  Span si, sr, sz, sy, sw;
  Fp8Spans sq;
  if (e->bias != nullptr) si = span(e->bias, m == 0 ? 0 : 1, n, n, dtype_size(e->bias_dtype), ok);
  if (e->residual != nullptr) sr = span(e->residual, m, n, e->ld_residual, size, ok);
  if (e->z != nullptr) sz = span(e->z, m, n, e->ld_z, size, ok);
  if (e->y != nullptr) sy = span(e->y, m, n, e->ld_y, size, ok);
  if (e->q != nullptr) {
    if (e->q->group != 1) ok = false;
    sq = fp8_spans(e->q, m, n, ok);
  }
  if (!product_ok(a, b, m, n, k)) ok = false;
  if (!ok) return ZF_EINVAL;
  const zf_status st_ws =
      workspace_span(ws, ws_bytes, zf_linear_fp8_workspace_bytes(m, n, k, e->q != nullptr), ok, sw);
  if (st_ws != ZF_OK) return st_ws;
  if (!disjoint({sz, sy, sq.data, sq.scale, sw},
                {sa.data, sa.scale, sb.data, sb.scale, si}) ||
      !disjoint({sz, sq.data, sq.scale, sw}, {sr}) ||
      !apart_or_same(sy, e->y, e->ld_y, sr, e->residual, e->ld_residual, m))
    return ZF_EINVAL;
  if (m == 0 || n == 0) return ZF_OK;
  const zf::MatmulArgs args{operand(a), operand(b), m, n, k, nullptr, 0, 0, 0};
  const zf::Epilogue ep{e->bias, e->bias_dtype == ZF_F32, e->activation, e->residual, e->ld_residual,
                        e->z, e->ld_z, e->y, e->ld_y, fp8_out(e->q)};
  return done(zf::launch_linear(args, ep, e->dtype, ws, as_stream(stream)));
}

size_t zf_linear_fp8_backward_workspace_bytes(int64_t rows, int64_t cols) {
  if (!size_ok(rows) || !size_ok(cols)) return 0;
  return zf::linear_backward_workspace(rows, cols);
}

zf_status zf_linear_fp8_backward(const void* dy, int64_t ld_dy, const void* z, int64_t ld_z,
                                 int32_t dtype, int64_t rows, int64_t cols, int32_t activation,
                                 void* dz, int64_t ld_dz, const zf_fp8* q, const zf_fp8* q_t,
                                 float* dbias, void* ws, size_t ws_bytes, zf_stream stream) {
  if (!dtype_ok(dtype) || !size_ok(rows) || !size_ok(cols) || !activation_ok(activation) ||
      (dz == nullptr && q == nullptr && q_t == nullptr && dbias == nullptr))
    return ZF_EINVAL;
  const size_t e = dtype_size(dtype);
  bool ok = true;
  Span sz, sd, sb, sw;
  Fp8Spans sq, st;
  const Span sy = span(dy, rows, cols, ld_dy, e, ok);
  if (activation != ZF_NONE) sz = span(z, rows, cols, ld_z, e, ok);
  if (dz != nullptr) sd = span(dz, rows, cols, ld_dz, e, ok);
  if (q != nullptr) {
    if (q->group != 1) ok = false;
    sq = fp8_spans(q, rows, cols, ok);
  }
  if (q_t != nullptr) {
    if (q_t->group != 1) ok = false;
    st = fp8_spans(q_t, cols, rows, ok);
  }
  if (dbias != nullptr) {
    sb = span(dbias, 1, cols, cols, 4, ok);
    const zf_status st_ws = workspace_span(
        ws, ws_bytes, zf_linear_fp8_backward_workspace_bytes(rows, cols), ok, sw);
    if (st_ws != ZF_OK) return st_ws;
  }
  if (!ok || ceil_div(rows, 128) * ceil_div(cols, 128) >= kGridLimit ||
      !disjoint({sd, sq.data, sq.scale, st.data, st.scale, sb, sw}, {}) ||
      !disjoint({sq.data, sq.scale, st.data, st.scale, sb, sw}, {sy, sz}) ||
      !apart_or_same(sd, dz, ld_dz, sy, dy, ld_dy, rows) ||
      !apart_or_same(sd, dz, ld_dz, sz, z, ld_z, rows))
    return ZF_EINVAL;
  if (cols == 0 || (rows == 0 && dbias == nullptr)) return ZF_OK;
  const zf::LinearBwdArgs a{dy, ld_dy, z, ld_z, rows, cols, activation, dz, ld_dz, fp8_out(q),
                            fp8_out(q_t), dbias, static_cast<float*>(ws)};
  return done(zf::launch_linear_backward(a, dtype, as_stream(stream)));
}

// ---- attention ---------------------------------------------------------------

size_t zf_attention_forward_workspace_bytes(const zf_attention* a) {
  if (!attention_ok(a)) return 0;
  return zf::attention_workspace(attention_args(*a));
}

zf_status zf_attention_forward(const zf_attention* a, const zf_heads* q, const zf_heads* k,
                               const zf_heads* v, const zf_heads* out, float* lse, void* ws,
                               size_t ws_bytes, zf_stream stream) {
  if (!attention_ok(a)) return ZF_EINVAL;
  bool ok = true;
  const Span sq = heads_span(q, a->tokens_q, a->heads, a->dim, ok);
  const Span sk = heads_span(k, a->tokens_k, a->kv_heads, a->dim, ok);
  const Span sv = heads_span(v, a->tokens_k, a->kv_heads, a->dim, ok);
  const Span so = heads_span(out, a->tokens_q, a->heads, a->dim, ok);
  if (!ok || !rows_apart(out, a->tokens_q, a->heads, a->dim)) return ZF_EINVAL;
  Span sl, sw;
  if (lse != nullptr) sl = span(lse, a->heads, a->tokens_q, a->tokens_q, 4, ok);
  const SequenceSpans ss = sequence_spans(*a);
  const zf_status st_ws =
      workspace_span(ws, ws_bytes, zf_attention_forward_workspace_bytes(a), ok, sw);
  if (st_ws != ZF_OK) return st_ws;
  if (!disjoint({so, sl, sw}, {sq, sk, sv, ss.q, ss.k, ss.len})) return ZF_EINVAL;
  if (a->tokens_q == 0) return ZF_OK;
  zf::AttentionArgs args = attention_args(*a);
  args.q = heads_arg(q);
  args.k = heads_arg(k);
  args.v = heads_arg(v);
  args.out = static_cast<uint16_t*>(out->data);
  args.ld_out_token = out->ld_token;
  args.ld_out_head = out->ld_head;
  args.lse = lse;
  return done(zf::launch_attention(args, ws, as_stream(stream)));
}

size_t zf_attention_backward_workspace_bytes(const zf_attention* a) {
  if (!attention_ok(a) || a->len_k != nullptr) return 0;
  return zf::attention_backward_workspace(attention_bwd_args(*a));
}

zf_status zf_attention_backward(const zf_attention* a, const zf_heads* q, const zf_heads* k,
                                const zf_heads* v, const zf_heads* out, const float* lse,
                                const zf_heads* dout, const zf_heads* dq, const zf_heads* dk,
                                const zf_heads* dv, void* ws, size_t ws_bytes, zf_stream stream) {
  if (!attention_ok(a) || a->len_k != nullptr) return ZF_EINVAL;
  const int64_t tq = a->tokens_q, tk = a->tokens_k;
  const int32_t h = a->heads, kv = a->kv_heads, d = a->dim;
  bool ok = true;
  const Span sq = heads_span(q, tq, h, d, ok), sk = heads_span(k, tk, kv, d, ok),
             sv = heads_span(v, tk, kv, d, ok), so = heads_span(out, tq, h, d, ok),
             sdo = heads_span(dout, tq, h, d, ok), sdq = heads_span(dq, tq, h, d, ok),
             sdk = heads_span(dk, tk, kv, d, ok), sdv = heads_span(dv, tk, kv, d, ok);
  if (!ok || !rows_apart(dq, tq, h, d) || !rows_apart(dk, tk, kv, d) || !rows_apart(dv, tk, kv, d))
    return ZF_EINVAL;
  // (a tile's rows are addressed through 32-bit offsets, over a key head's query heads)
  const int64_t group = h / kv;
  if (tq > 0 && group > 1 && (q->ld_head >= (int64_t(1) << 30) / group ||
                              dout->ld_head >= (int64_t(1) << 30) / group))
    return ZF_EINVAL;
  const Span sl = span(lse, h, tq, tq, 4, ok);
  Span sw;
  const SequenceSpans ss = sequence_spans(*a);
  const zf_status st_ws =
      workspace_span(ws, ws_bytes, zf_attention_backward_workspace_bytes(a), ok, sw);
  if (st_ws != ZF_OK) return st_ws;
  // (the gradients may be columns of one buffer: apart from each other element by element)
  if (!disjoint({sdq, sw}, {sq, sk, sv, so, sdo, sl, ss.q, ss.k}) ||
      !disjoint({sdk, sw}, {sq, sk, sv, so, sdo, sl, ss.q, ss.k}) ||
      !disjoint({sdv, sw}, {sq, sk, sv, so, sdo, sl, ss.q, ss.k}) ||
      !heads_apart(dq, tq, h, dk, tk, kv, d) || !heads_apart(dq, tq, h, dv, tk, kv, d) ||
      !heads_apart(dk, tk, kv, dv, tk, kv, d))
    return ZF_EINVAL;
  if (tq == 0 && tk == 0) return ZF_OK;
  zf::AttentionBwdArgs args = attention_bwd_args(*a);
  args.q = heads_arg(q);
  args.k = heads_arg(k);
  args.v = heads_arg(v);
  args.out = heads_arg(out);
  args.dout = heads_arg(dout);
  args.dq = heads_arg(dq);
  args.dk = heads_arg(dk);
  args.dv = heads_arg(dv);
  args.lse = lse;
  return done(zf::launch_attention_backward(args, ws, as_stream(stream)));
}

}  // extern "C"

// ---- AdamW over many tensors -------------------------------------------------

struct zf_adamw_plan {
  std::vector<unsigned char> image;  // offsets, then tensors: uploaded as they are
  int32_t count = 0;
  int64_t blocks = 0;
  const int64_t* d_off = nullptr;
  const zf::AdamTensor* d_tensors = nullptr;
};

namespace {

size_t adamw_bytes(int32_t count) {
  return static_cast<size_t>(count) * (sizeof(zf::AdamTensor) + sizeof(int64_t));
}

int64_t adamw_chunks(const zf_adamw_tensor& t) {
  return ceil_div(t.n, zf::kAdamwChunk);
}

bool adamw_tensor_ok(const zf_adamw_tensor& t) {
  if (t.n < 0 || !dtype_ok(t.grad_dtype)) return false;
  const bool eight = t.exp_avg_scale != nullptr;
  if (eight != (t.exp_avg_sq_scale != nullptr) && t.n > 0) return false;
  if (t.n == 0) return true;
  if (t.n >= kGridLimit * zf::kAdamwChunk) return false;
  const size_t state = eight ? 1 : 4;
  return t.grad != nullptr && aligned(t.grad, dtype_size(t.grad_dtype)) && t.master != nullptr &&
         aligned(t.master, 4) && aligned(t.weight, 2) && t.exp_avg != nullptr &&
         aligned(t.exp_avg, state) && t.exp_avg_sq != nullptr && aligned(t.exp_avg_sq, state) &&
         aligned(t.exp_avg_scale, 4) && aligned(t.exp_avg_sq_scale, 4);
}

// Blocks of the launch, or -1 when a descriptor is invalid or buffers overlap.
int64_t adamw_blocks(const zf_adamw_tensor* tensors, int32_t count) {
  if (tensors == nullptr || count < 1) return -1;
  struct Use {
    uintptr_t lo, hi;
  };
  std::vector<Use> used;
  used.reserve(static_cast<size_t>(count) * 7);
  int64_t blocks = 0;
  for (int32_t i = 0; i < count; ++i) {
    const zf_adamw_tensor& t = tensors[i];
    if (!adamw_tensor_ok(t)) return -1;
    blocks += adamw_chunks(t);
    if (blocks >= kGridLimit) return -1;
    if (t.n == 0) continue;
    const bool eight = t.exp_avg_scale != nullptr;
    const size_t n = static_cast<size_t>(t.n);
    const auto add = [&](const void* p, size_t bytes) {
      const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
      if (p != nullptr) used.push_back({lo, lo + bytes});
    };
    add(t.grad, n * dtype_size(t.grad_dtype));
    add(t.master, n * 4);
    add(t.weight, n * 2);
    add(t.exp_avg, n * (eight ? 1 : 4));
    add(t.exp_avg_sq, n * (eight ? 1 : 4));
    add(t.exp_avg_scale, (n + 127) / 128 * 4);
    add(t.exp_avg_sq_scale, (n + 127) / 128 * 4);
  }
  std::sort(used.begin(), used.end(), [](const Use& a, const Use& b) { return a.lo < b.lo; });
  for (size_t i = 1; i < used.size(); ++i)
    if (used[i].lo < used[i - 1].hi) return -1;
  return blocks;
}

}  // namespace

extern "C" {

zf_status zf_adamw_plan_query(const zf_adamw_tensor* tensors, int32_t count,
                              size_t* device_bytes) {
  if (device_bytes == nullptr) return ZF_EINVAL;
  try {
    if (adamw_blocks(tensors, count) < 0) return ZF_EINVAL;
  } catch (const std::bad_alloc&) {
    return ZF_ENOMEM;
  }
  *device_bytes = adamw_bytes(count);
  return ZF_OK;
}

zf_status zf_adamw_plan_create(const zf_adamw_tensor* tensors, int32_t count, void* device_mem,
                               size_t device_bytes, zf_stream stream, zf_adamw_plan** out) {
  if (out == nullptr || device_mem == nullptr || !aligned(device_mem, 256)) return ZF_EINVAL;
  zf_adamw_plan* p = nullptr;
  try {
    const int64_t blocks = adamw_blocks(tensors, count);
    if (blocks < 0) return ZF_EINVAL;
    const size_t bytes = adamw_bytes(count);
    if (device_bytes < bytes) return ZF_EWORKSPACE;
    p = new zf_adamw_plan();
    p->image.resize(bytes);
    p->count = count;
    p->blocks = blocks;
  } catch (const std::bad_alloc&) {
    delete p;
    return ZF_ENOMEM;
  }
  int64_t* const off = reinterpret_cast<int64_t*>(p->image.data());
  zf::AdamTensor* const dev = reinterpret_cast<zf::AdamTensor*>(off + count);
  int64_t at = 0;
  for (int32_t i = 0; i < count; ++i) {
    const zf_adamw_tensor& t = tensors[i];
    off[i] = at;
    at += adamw_chunks(t);
    dev[i] = zf::AdamTensor{t.n, t.grad, t.master, t.weight, t.exp_avg, t.exp_avg_sq,
                            t.exp_avg_scale, t.exp_avg_sq_scale, t.grad_dtype == ZF_F32 ? 1 : 0,
                            0};
  }
  p->d_off = static_cast<const int64_t*>(device_mem);
  p->d_tensors = reinterpret_cast<const zf::AdamTensor*>(p->d_off + count);
  // stream-ordered upload of the tables; the host image stays with the plan
  const hipError_t e = hipMemcpyAsync(device_mem, p->image.data(), p->image.size(),
                                      hipMemcpyHostToDevice, as_stream(stream));
  if (e != hipSuccess) {
    delete p;
    return hip_fail(e);
  }
  *out = p;
  return ZF_OK;
}

void zf_adamw_plan_destroy(zf_adamw_plan* plan) { delete plan; }

zf_status zf_adamw_step(zf_adamw_plan* plan, const zf_adam_hparams* hp, int64_t step,
                        const float* grad_scale, zf_stream stream) {
  if (plan == nullptr || !zf::hparams_ok(hp) || step < 1 || !aligned(grad_scale, 4))
    return ZF_EINVAL;
  if (plan->blocks == 0) return ZF_OK;
  return done(zf::launch_adamw(plan->d_tensors, plan->d_off, plan->count, plan->blocks,
                               zf::adam_consts(*hp, step), grad_scale, as_stream(stream)));
}

}  // extern "C"
