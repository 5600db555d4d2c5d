"""What the operators of include/zf_layer.h refuse, on the host and before any
HIP call (fake device addresses are never dereferenced), and what the binding
refuses."""
import ctypes

import pytest
import torch

zf = pytest.importorskip("paper_2505_12242_amd")
from paper_2505_12242_amd import _lib  # noqa: E402

LIB = _lib.LIB
OK, EINVAL, EWS = _lib.ZF_OK, _lib.ZF_EINVAL, _lib.ZF_EWORKSPACE
BASE = 0x7F0000000000


def addr(i):
    return BASE + (i << 36)


def fp8(i, ld, lds, group=1, off=0):
    return _lib.ZfFp8(addr(i) + off, ld, addr(i + 1), lds, group)


def ref(x):
    return ctypes.byref(x) if x is not None else None


def quantize(x=addr(0), dt=0, rows=100, cols=200, ld=200, out=None, out_t=None):
    return LIB.zf_quantize_fp8(x, dt, rows, cols, ld, ref(out), ref(out_t), None)


def test_quantize():
    q, t = fp8(1, 208, 4), fp8(3, 112, 4)
    assert quantize() == EINVAL  # no output
    for kw in (dict(x=None), dict(dt=2), dict(rows=-1), dict(cols=1 << 30), dict(ld=199),
               dict(x=addr(0) + 1), dict(dt=1, x=addr(0) + 2), dict(out=fp8(1, 207, 4)),
               dict(out=fp8(1, 192, 4)), dict(out=fp8(1, 208, 3)), dict(out=fp8(1, 208, 0)),
               dict(out=fp8(1, 208, 4, group=64)), dict(out=fp8(1, 208, 4, off=8)),
               dict(out_t=fp8(3, 96, 4)), dict(out_t=fp8(3, 112, 4, group=128)),
               dict(out=_lib.ZfFp8(None, 208, addr(2), 4, 1)),
               dict(out=_lib.ZfFp8(addr(1), 208, None, 4, 1)),
               dict(out=_lib.ZfFp8(addr(1), 208, addr(2) + 2, 4, 1)),
               dict(out=fp8(0, 208, 4)),  # x's own memory
               dict(out_t=fp8(1, 112, 4)),  # the other output's
               dict(out=_lib.ZfFp8(addr(1), 208, addr(1) + 64, 4, 1))):
        assert quantize(**{**dict(out=q, out_t=t), **kw}) == EINVAL, kw
    assert quantize(rows=0, out=q) == OK and quantize(cols=0, x=None, out=q, out_t=t) == OK


def matmul(a=None, b=None, m=100, n=60, k=200, out=addr(9), dt=0, ld=60, ws=addr(12), wsb=1 << 34):
    a = a if a is not None else fp8(1, 208, 4)
    b = b if b is not None else fp8(3, 208, 4, 128)
    return LIB.zf_matmul_fp8(ref(a), ref(b), m, n, k, out, dt, ld, ws, wsb, None)


def test_matmul():
    for kw in (dict(dt=3), dict(m=-1), dict(n=1 << 30), dict(k=1 << 30), dict(k=1 << 23),
               dict(ld=59), dict(out=None), dict(out=addr(9) + 1), dict(dt=1, out=addr(9) + 2),
               dict(a=fp8(1, 192, 4)), dict(a=fp8(1, 200, 4)), dict(b=fp8(3, 208, 2)),
               dict(b=fp8(3, 208, 4, 2)), dict(a=fp8(1, 1 << 23, 4)), dict(b=fp8(3, 1 << 24, 4)),
               dict(a=fp8(1, 208, 1 << 23)), dict(b=fp8(3, 208, 1 << 23)),
               dict(a=_lib.ZfFp8(None, 208, addr(2), 4, 1)), dict(out=addr(1)), dict(out=addr(4)),
               dict(m=1 << 29, n=1 << 29)):
        if kw.get("n") == 1 << 30 or kw.get("n") == 1 << 29:
            kw = {**kw, "ld": 1 << 30}
        assert matmul(**kw) == EINVAL, kw
    assert LIB.zf_matmul_fp8(None, ref(fp8(3, 208, 4)), 1, 1, 1, addr(9), 0, 1, None, 0,
                             None) == EINVAL
    assert matmul(m=0) == OK and matmul(n=0, ld=0) == OK
    assert LIB.zf_matmul_fp8_workspace_bytes(-1, 5, 5) == 0
    sizes = [(m, n, k) for m in (1, 64, 200, 1000) for n in (64, 4096) for k in (64, 11008)]
    needy = [s for s in sizes if LIB.zf_matmul_fp8_workspace_bytes(*s)]
    for m, n, k in needy:
        need = LIB.zf_matmul_fp8_workspace_bytes(m, n, k)
        kw = dict(a=fp8(1, 11008, 88), b=fp8(3, 11008, 88), m=m, n=n, k=k, ld=n)
        assert matmul(**kw, wsb=need - 1) == EWS
        assert matmul(**kw, ws=None, wsb=need) == EINVAL
        assert matmul(**kw, ws=addr(12) + 8) == EINVAL
        assert matmul(**kw, ws=addr(9)) == EINVAL


def forward(x=addr(0), ldx=300, res=addr(1), ldr=300, dt=0, rows=10, cols=300, gain=addr(2), gdt=0,
            eps=1e-6, h=addr(3), ldh=300, y=addr(4), ldy=300, q=None, rstd=addr(8)):
    return LIB.zf_rmsnorm_forward(x, ldx, res, ldr, dt, rows, cols, gain, gdt, eps, h, ldh, y, ldy,
                                  ref(q), rstd, None)


def test_rmsnorm_forward():
    for kw in (dict(x=None), dict(ldx=299), dict(ldr=299), dict(dt=5), dict(gdt=-1), dict(rows=-1),
               dict(cols=1 << 30), dict(gain=None), dict(eps=-1.0), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(h=None), dict(ldh=4), dict(ldy=299), dict(rstd=None),
               dict(rstd=addr(8) + 2), dict(x=addr(0) + 1), dict(dt=1, y=addr(4) + 2),
               dict(q=fp8(5, 304, 4, 128)), dict(q=fp8(5, 300, 4)), dict(q=fp8(4, 304, 4)),
               dict(y=addr(0)), dict(y=addr(1)), dict(y=addr(3)), dict(rstd=addr(2)),
               dict(h=addr(0) + 2), dict(h=addr(1), ldh=304), dict(h=addr(2))):
        assert forward(**kw) == EINVAL, kw
    assert forward(rows=0, x=None, res=None, gain=None, h=None, y=None, rstd=None) == OK


def backward(dy=addr(0), ldy=300, h=addr(1), ldh=300, dt=0, rows=10, cols=300, gain=addr(2), gdt=0,
             rstd=addr(3), res=addr(4), ldr=300, dx=addr(5), ldx=300, dg=addr(6), ws=addr(7),
             wsb=1 << 30):
    return LIB.zf_rmsnorm_backward(dy, ldy, h, ldh, dt, rows, cols, gain, gdt, rstd, res, ldr, dx,
                                   ldx, dg, ws, wsb, None)


def test_rmsnorm_backward():
    need = LIB.zf_rmsnorm_backward_workspace_bytes(10, 300)
    assert need > 0
    for kw in (dict(dy=None), dict(ldy=299), dict(h=None), dict(ldh=9), dict(dt=2), dict(rows=-5),
               dict(gain=None), dict(rstd=None), dict(rstd=addr(3) + 1), dict(ldr=1), dict(dx=None),
               dict(ldx=299), dict(dg=addr(6) + 2), dict(ws=None), dict(ws=addr(7) + 4),
               dict(dx=addr(1)), dict(dx=addr(0) + 2), dict(dx=addr(4), ldx=304), dict(dg=addr(5)),
               dict(ws=addr(0)), dict(dg=addr(3))):
        assert backward(**kw) == EINVAL, kw
    assert backward(wsb=need - 1) == EWS
    assert backward(rows=0, dy=None, h=None, dx=None, dg=None, gain=None, rstd=None, res=None) == OK
    assert backward(cols=0, ldy=0, ldh=0, ldr=0, ldx=0) == OK


def tensor(i=1, n=1000, eight=False, **kw):
    a = dict(n=n, grad=addr(i), grad_dtype=0, master=addr(i + 1), weight=addr(i + 2),
             exp_avg=addr(i + 3), exp_avg_sq=addr(i + 4),
             exp_avg_scale=addr(i + 5) if eight else None,
             exp_avg_sq_scale=addr(i + 6) if eight else None)
    a.update(kw)
    return _lib.ZfAdamwTensor(**a)


def query(*ts):
    arr = (_lib.ZfAdamwTensor * len(ts))(*ts)
    need = ctypes.c_size_t()
    return LIB.zf_adamw_plan_query(arr, len(ts), ctypes.byref(need)), need.value


def test_adamw_plan():
    st, need = query(tensor(1), tensor(11, eight=True), tensor(21, n=0, grad=None, master=None))
    assert st == OK and need > 0
    for t in (tensor(n=-1), tensor(grad=None), tensor(master=None), tensor(exp_avg=None),
              tensor(exp_avg_sq=None), tensor(grad_dtype=2), tensor(grad=addr(1) + 1),
              tensor(master=addr(2) + 2), tensor(weight=addr(3) + 1), tensor(exp_avg=addr(4) + 1),
              tensor(exp_avg_scale=addr(6)), tensor(exp_avg_sq_scale=addr(6)),
              tensor(eight=True, exp_avg_scale=addr(6) + 2), tensor(exp_avg=addr(2)),
              tensor(weight=addr(1)), tensor(n=1 << 36)):
        assert query(t)[0] == EINVAL
    assert query(tensor(1), tensor(1))[0] == EINVAL  # one buffer in two tensors
    assert query(*[tensor(1 + 10 * i, n=1 << 34) for i in range(5)])[0] == EINVAL
    assert LIB.zf_adamw_plan_query(None, 1, ctypes.byref(ctypes.c_size_t())) == EINVAL
    arr = (_lib.ZfAdamwTensor * 1)(tensor())
    assert LIB.zf_adamw_plan_query(arr, 0, ctypes.byref(ctypes.c_size_t())) == EINVAL
    assert LIB.zf_adamw_plan_query(arr, 1, None) == EINVAL
    h, (_, need) = ctypes.c_void_p(), query(tensor())
    for mem, size, out, want in ((None, need, h, EINVAL), (addr(30) + 16, need, h, EINVAL),
                                 (addr(30), need - 1, h, EWS), (addr(30), need, None, EINVAL)):
        assert LIB.zf_adamw_plan_create(arr, 1, mem, size, None, ref(out)) == want
    hp = _lib.ZfAdamHparams(1e-3, 0.9, 0.999, 1e-8, 0.0)
    assert LIB.zf_adamw_step(None, ctypes.byref(hp), 1, None, None) == EINVAL
    LIB.zf_adamw_plan_destroy(None)


def test_binding():
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # a host tensor
        zf.quantize_fp8(x)
    with pytest.raises(TypeError):
        zf.quantize_fp8(x.half())
    with pytest.raises(ValueError):
        zf.quantize_fp8(x[0])
    with pytest.raises(TypeError):
        zf.rmsnorm(x.double(), x[0])
    f = zf.alloc_fp8(4, 8, device="cpu")
    assert f.data.stride(0) == 16 and f.scale.shape == (4, 1) and f.scale.stride(0) == 4
    with pytest.raises(ValueError):
        zf.matmul_fp8(f, f)
    with pytest.raises(ValueError):
        zf.AdamWPlan([])
    with pytest.raises(ValueError):
        zf.AdamWBuffers.fresh(x, x.float(), bits=16)
    b = zf.AdamWBuffers.fresh(x, x.float())
    with pytest.raises(ValueError):
        b.as_c()
    b.exp_avg_scale = torch.zeros(1)
    with pytest.raises(ValueError):
        b.as_c()
