// Host entry points of include/zf_layer.h: argument validation, Adam constants
// and the AdamW plan.  Every check runs before the first HIP call.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <new>
#include <vector>

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
