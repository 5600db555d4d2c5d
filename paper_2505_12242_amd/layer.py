"""Binding of include/zf_layer.h: the operators around the weights that the
selective update serves.

Argument marshalling only, as in _lib.py: tensors are checked for dtype,
device, shape and stride, outputs that are not given are allocated, and every
operator runs in the HIP kernels of libzf.so.

`stream` is the torch stream a call is launched on (None: the current one).  What
the call allocates, outputs and workspaces, belongs to that stream; the inputs
must be ready there, and an output that is used on another stream is the
caller's to order, as any tensor's.
"""

from __future__ import annotations

import ctypes
from dataclasses import dataclass
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from ._lib import (LIB, AdamHparams, ZfAdamwTensor, ZfFp8, _check, _empty, _mat, _ptr, _stream,
                   _vec, _workspace, c_sz, c_vp)

DTYPES = {torch.bfloat16: 0, torch.float32: 1}  # zf_dtype
DATA, SCALE = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _dtype(t: torch.Tensor, name: str) -> int:
    code = DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: expected bfloat16 or float32, got {t.dtype}")
    return code


def _up(x: int, unit: int) -> int:
    return -(-x // unit) * unit


# ---- 8-bit operands -----------------------------------------------------------

class Fp8:
    """A matrix in 8 bits: `data` [rows, cols] torch.float8_e4m3fn (row stride a
    multiple of 16) and `scale` [ceil(rows / group), ceil(cols / 128)]
    torch.float8_e8m0fnu (row stride a multiple of 4).  group is 1 (128
    elements of a row share a scale) or 128 (a block of 128 x 128 does).
    alloc_fp8 allocates one."""

    __slots__ = ("data", "scale", "group")

    def __init__(self, data: torch.Tensor, scale: torch.Tensor, group: int = 1):
        self.data, self.scale, self.group = data, scale, group

    @property
    def shape(self):
        return self.data.shape

    def dequantize(self) -> torch.Tensor:
        """The values it stands for, fp32 (elementary torch operations)."""
        rows, cols = self.data.shape
        code = self.scale.view(torch.uint8).to(torch.int32)
        s = torch.where(code == 0, 2.0 ** -127, (code << 23).view(torch.float32))
        s = torch.where(code == 255, float("nan"), s)
        s = s.repeat_interleave(128, 1)[:, :cols].repeat_interleave(self.group, 0)[:rows]
        return self.data.float() * s

    def as_c(self, name: str, rows: Optional[int] = None, cols: Optional[int] = None) -> ZfFp8:
        data, scale, group = self.data, self.scale, self.group
        if group not in (1, 128):
            raise ValueError(f"{name}: group is 1 or 128, got {group}")
        ld = _mat(data, DATA, name, rows, cols)
        r, c = data.shape
        sr, sc = -(-r // group), -(-c // 128)
        ld_scale = _mat(scale, SCALE, name, sr, sc)
        if r <= 1 or not c:  # (a single row's stride is its width, as in _mat)
            ld = _up(c, 16)
        if sr <= 1 or not c:
            ld_scale = _up(sc, 4)
        if r and c:
            if ld % 16 or ld_scale % 4:
                raise ValueError(f"{name}: row strides must be multiples of 16 (data) and 4 "
                                 f"(scale), got {ld} and {ld_scale}")
            # rows are read in whole units of 16 bytes, their scales of 4
            if c % 16:
                self._room(name, data, ld, _up(c, 16))
            if sc % 4:
                self._room(name, scale, ld_scale, _up(sc, 4))
        return ZfFp8(data.data_ptr() or None, ld, scale.data_ptr() or None, ld_scale, group)

    @staticmethod
    def _room(name: str, t: torch.Tensor, ld: int, width: int) -> None:
        end = t.storage_offset() + (t.shape[0] - 1) * ld + width
        if t.untyped_storage().nbytes() < end:
            raise ValueError(f"{name}: the last row's storage ends inside a unit (alloc_fp8 pads "
                             f"rows)")


def _alloc_fp8(rows: int, cols: int, group: int, device, stream=None) -> Tuple[Fp8, ZfFp8]:
    """A new Fp8 and its C struct."""
    sr, sc = -(-rows // group), -(-cols // 128)
    ld, ld_scale = _up(cols, 16), _up(sc, 4)
    data = _empty((rows, ld), DATA, device, stream)
    scale = _empty((sr, ld_scale), SCALE, device, stream)
    c = ZfFp8(data.data_ptr() or None, ld, scale.data_ptr() or None, ld_scale, group)
    if ld != cols:
        data = data[:, :cols]
    if ld_scale != sc:
        scale = scale[:, :sc]
    return Fp8(data, scale, group), c


def alloc_fp8(rows: int, cols: int, group: int = 1, device="cuda") -> Fp8:
    """Uninitialised storage of a rows x cols matrix in 8 bits, rows padded to
    multiples of 16 bytes (data) and 4 (scale)."""
    return _alloc_fp8(rows, cols, group, device)[0]


def quantize_fp8(x: torch.Tensor, group: int = 1, rows: bool = True, transposed: bool = False,
                 out: Optional[Fp8] = None, out_t: Optional[Fp8] = None, stream=None
                 ) -> Tuple[Optional[Fp8], Optional[Fp8]]:
    """x (bf16 or fp32 [r, c]) in 8 bits (zf_quantize_fp8): (x, x's transpose),
    each where asked for (`rows`, `transposed`, or its output given)."""
    dt = _dtype(x, "x")
    ld = _mat(x, x.dtype, "x")
    r, c = x.shape
    c_out = c_out_t = None
    if out is not None:
        c_out = out.as_c("out", r, c)
    elif rows:
        out, c_out = _alloc_fp8(r, c, group, x.device, stream)
    if out_t is not None:
        c_out_t = out_t.as_c("out_t", c, r)
    elif transposed:
        out_t, c_out_t = _alloc_fp8(c, r, group, x.device, stream)
    if out is None and out_t is None:
        raise ValueError("neither output is wanted")
    _check("zf_quantize_fp8", LIB.zf_quantize_fp8(
        _ptr(x), dt, r, c, ld, ctypes.byref(c_out) if c_out is not None else None,
        ctypes.byref(c_out_t) if c_out_t is not None else None, _stream(stream)))
    return out, out_t


def matmul_fp8_workspace_bytes(m: int, n: int, k: int) -> int:
    return LIB.zf_matmul_fp8_workspace_bytes(m, n, k)


def matmul_fp8(a: Fp8, b: Fp8, out: Optional[torch.Tensor] = None, dtype=torch.bfloat16,
               workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """a @ b.T of two 8-bit operands of the same width (zf_matmul_fp8), summed in
    fp32, in bf16 or fp32 (out's type where it is given).  A linear layer of weight w [n, k]:
    forward matmul_fp8(x, w), input gradient matmul_fp8(dy, wt), weight
    gradient matmul_fp8(dyt, xt) in ROW_MAJOR or matmul_fp8(xt, dyt) in
    CHANNEL_MAJOR, with *t the transposed copies of quantize_fp8."""
    m, k = a.data.shape
    n = b.data.shape[0]
    c_a, c_b = a.as_c("a"), b.as_c("b", None, k)
    if out is None:
        out, ld = _empty((m, n), dtype, a.data.device, stream), n
    else:
        ld = _mat(out, out.dtype, "out", m, n)
    dt = _dtype(out, "out")
    need = LIB.zf_matmul_fp8_workspace_bytes(m, n, k)
    if workspace is None and need:
        workspace = _empty(need, torch.uint8, out.device, stream)
    _check("zf_matmul_fp8", LIB.zf_matmul_fp8(
        ctypes.byref(c_a), ctypes.byref(c_b), m, n, k, _ptr(out), dt, ld, _ptr(workspace),
        _workspace(workspace), _stream(stream)))
    return out


# ---- RMS norm ---------------------------------------------------------------------

class RmsNorm(NamedTuple):
    """What rmsnorm returns; y, q: None where not wanted; h: x itself without a
    residual."""
    y: Optional[torch.Tensor]
    h: torch.Tensor
    rstd: torch.Tensor
    q: Optional[Fp8]


def rmsnorm(x: torch.Tensor, gain: torch.Tensor, residual: Optional[torch.Tensor] = None,
            eps: float = 1e-6, want_y: bool = True, want_q: bool = False,
            h: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
            q: Optional[Fp8] = None, rstd: Optional[torch.Tensor] = None,
            stream=None) -> RmsNorm:
    """h = x + residual, y = h / rms(h) * gain, in x's type and/or in 8 bits
    (zf_rmsnorm_forward).  x, residual [rows, cols] bf16 or fp32, gain [cols]
    bf16 or fp32.  h may be the residual's (or x's) own tensor; outputs that
    are not given are allocated."""
    dt = _dtype(x, "x")
    ld = _mat(x, x.dtype, "x")
    r, c = x.shape
    gdt = _dtype(gain, "gain")
    _vec(gain, gain.dtype, "gain", c)
    dtype, dev = x.dtype, x.device
    if rstd is None:
        rstd = _empty(r, torch.float32, dev, stream)
    else:
        _vec(rstd, torch.float32, "rstd", r)
    ld_res, ld_h, ld_y, c_q = 0, c, c, None
    if residual is not None:
        ld_res = _mat(residual, dtype, "residual", r, c)
    if h is not None:
        ld_h = _mat(h, dtype, "h", r, c)
    elif residual is not None:
        h = _empty((r, c), dtype, dev, stream)
    if y is not None:
        ld_y = _mat(y, dtype, "y", r, c)
    elif want_y:
        y = _empty((r, c), dtype, dev, stream)
    if q is not None:
        c_q = q.as_c("q", r, c)
    elif want_q:
        q, c_q = _alloc_fp8(r, c, 1, dev, stream)
    _check("zf_rmsnorm_forward", LIB.zf_rmsnorm_forward(
        _ptr(x), ld, _ptr(residual), ld_res, dt, r, c, _ptr(gain), gdt, float(eps), _ptr(h), ld_h,
        _ptr(y), ld_y, ctypes.byref(c_q) if c_q is not None else None, _ptr(rstd),
        _stream(stream)))
    return RmsNorm(y, x if h is None else h, rstd, q)


def rmsnorm_backward_workspace_bytes(rows: int, cols: int) -> int:
    return LIB.zf_rmsnorm_backward_workspace_bytes(rows, cols)


def rmsnorm_backward(dy: torch.Tensor, h: torch.Tensor, gain: torch.Tensor, rstd: torch.Tensor,
                     dresidual: Optional[torch.Tensor] = None,
                     dx: Optional[torch.Tensor] = None, dgain: Optional[torch.Tensor] = None,
                     want_dgain: bool = True, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(dx, dgain) of rmsnorm, from its h and rstd (zf_rmsnorm_backward).  dx is
    the gradient of x and of the residual; dresidual, the gradient that
    reaches h from elsewhere, is added to it.  dx may be dy's or dresidual's
    own tensor.  dgain is fp32 [cols]."""
    dt = _dtype(dy, "dy")
    ld_dy = _mat(dy, dy.dtype, "dy")
    r, c = dy.shape
    ld_h = _mat(h, dy.dtype, "h", r, c)
    gdt = _dtype(gain, "gain")
    _vec(gain, gain.dtype, "gain", c)
    _vec(rstd, torch.float32, "rstd", r)
    ld_res = 0
    if dresidual is not None:
        ld_res = _mat(dresidual, dy.dtype, "dresidual", r, c)
    if dx is None:
        dx, ld_dx = _empty((r, c), dy.dtype, dy.device, stream), c
    else:
        ld_dx = _mat(dx, dy.dtype, "dx", r, c)
    if dgain is not None:
        _vec(dgain, torch.float32, "dgain", c)
    elif want_dgain:
        dgain = _empty(c, torch.float32, dy.device, stream)
    if dgain is not None:
        if workspace is None:
            need = LIB.zf_rmsnorm_backward_workspace_bytes(r, c)
            workspace = _empty(need, torch.uint8, dy.device, stream) if need else None
    _check("zf_rmsnorm_backward", LIB.zf_rmsnorm_backward(
        _ptr(dy), ld_dy, _ptr(h), ld_h, dt, r, c, _ptr(gain), gdt, _ptr(rstd), _ptr(dresidual),
        ld_res, _ptr(dx), ld_dx, _ptr(dgain), _ptr(workspace),
        _workspace(workspace), _stream(stream)))
    return dx, dgain


# ---- AdamW over many tensors -----------------------------------------------------------

@dataclass
class AdamWBuffers:
    """Device tensors of one parameter, each contiguous and of the same number
    of elements (any shape).  grad bf16 or fp32; master fp32; weight its bf16
    copy, or None.  exp_avg and exp_avg_sq fp32, or, with the two scales ([ceil(n
    / 128)] fp32) given, torch.float8_e4m3fn codes (zf_layer.h).  Zeros are the
    states of a fresh parameter either way."""
    grad: torch.Tensor
    master: torch.Tensor
    exp_avg: torch.Tensor
    exp_avg_sq: torch.Tensor
    weight: Optional[torch.Tensor] = None
    exp_avg_scale: Optional[torch.Tensor] = None
    exp_avg_sq_scale: Optional[torch.Tensor] = None

    @staticmethod
    def fresh(grad: torch.Tensor, master: torch.Tensor, weight: Optional[torch.Tensor] = None,
              bits: int = 32) -> "AdamWBuffers":
        """With new zero states in 32 or 8 bits."""
        if bits not in (32, 8):
            raise ValueError(f"bits is 32 or 8, got {bits}")
        n, dev = master.numel(), master.device

        def zeros():
            if bits == 32:
                return torch.zeros(n, dtype=torch.float32, device=dev)
            return torch.zeros(n, dtype=torch.uint8, device=dev).view(DATA)

        def scale():
            return torch.zeros(-(-n // 128), dtype=torch.float32, device=dev) if bits == 8 else None

        return AdamWBuffers(grad, master, zeros(), zeros(), weight, scale(), scale())

    def as_c(self) -> ZfAdamwTensor:
        n = self.master.numel()
        if (self.exp_avg_scale is None) != (self.exp_avg_sq_scale is None):
            raise ValueError("8-bit states take both scales, 32-bit states none")
        eight = self.exp_avg_scale is not None
        state = DATA if eight else torch.float32
        for name, t, dtype, count in (
                ("grad", self.grad, self.grad.dtype, n),
                ("master", self.master, torch.float32, n),
                ("weight", self.weight, torch.bfloat16, n),
                ("exp_avg", self.exp_avg, state, n), ("exp_avg_sq", self.exp_avg_sq, state, n),
                ("exp_avg_scale", self.exp_avg_scale, torch.float32, -(-n // 128)),
                ("exp_avg_sq_scale", self.exp_avg_sq_scale, torch.float32, -(-n // 128))):
            if t is None:
                continue
            if t.dtype != dtype:
                raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
            if t.numel() != count or not t.is_contiguous():
                raise ValueError(f"{name}: expected {count} contiguous elements, got shape "
                                 f"{tuple(t.shape)}")
            if count and not t.is_cuda:
                raise ValueError(f"{name}: must live on a GPU")
        return ZfAdamwTensor(n, _ptr(self.grad), _dtype(self.grad, "grad"), _ptr(self.master),
                             _ptr(self.weight), _ptr(self.exp_avg), _ptr(self.exp_avg_sq),
                             _ptr(self.exp_avg_scale), _ptr(self.exp_avg_sq_scale))


class AdamWPlan:
    """A set of parameters stepped by one launch (zf_adamw_*): those that are
    not split by channel, such as norm gains, biases and embeddings.  32- and
    8-bit states may be mixed.  The gradients are read where the buffers given
    here hold them.  Streams and lifetime as for Plan."""

    def __init__(self, tensors: Sequence[AdamWBuffers], stream=None):
        self._h = None
        self.tensors = list(tensors)  # keeps the tensors alive
        if not self.tensors:
            raise ValueError("a plan needs at least one tensor")
        arr = (ZfAdamwTensor * len(self.tensors))(*[b.as_c() for b in self.tensors])
        nbytes = c_sz()
        _check("zf_adamw_plan_query",
               LIB.zf_adamw_plan_query(arr, len(self.tensors), ctypes.byref(nbytes)))
        self.device = self.tensors[0].master.device
        self._mem = _empty(nbytes.value + 256, torch.uint8, self.device, stream)
        aligned = (self._mem.data_ptr() + 255) & ~255
        st = stream if stream is not None else torch.cuda.current_stream(self.device)
        h = c_vp()
        _check("zf_adamw_plan_create", LIB.zf_adamw_plan_create(
            arr, len(self.tensors), aligned, nbytes.value, st.cuda_stream, ctypes.byref(h)))
        self._h = h
        st.synchronize()

    def step(self, hp: AdamHparams, step: int, grad_scale: Optional[torch.Tensor] = None,
             stream=None) -> None:
        """One AdamW step of every tensor.  grad_scale: a one-element fp32 GPU
        tensor the gradients are multiplied by (clipping, loss scaling)."""
        if grad_scale is not None:
            if grad_scale.numel() != 1:
                raise ValueError("grad_scale: expected one element")
            if grad_scale.dtype != torch.float32 or not grad_scale.is_cuda:
                raise TypeError("grad_scale: expected a float32 GPU tensor")
        c_hp = hp.as_c()
        _check("zf_adamw_step", LIB.zf_adamw_step(self._h, ctypes.byref(c_hp), step,
                                                  _ptr(grad_scale), _stream(stream)))

    def close(self) -> None:
        if getattr(self, "_h", None):
            torch.cuda.synchronize(self.device)  # launches may still read the tables
            LIB.zf_adamw_plan_destroy(self._h)
            self._h = None
            self._mem = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
