"""What the attention, the layer norm and the linear layer of include/zf_layer.h
refuse, on the host and before any HIP call (fake device addresses are never
dereferenced), and what the binding refuses."""
import ctypes

import pytest
import torch

zf = pytest.importorskip("paper_2505_12242_amd")
from paper_2505_12242_amd import _lib  # noqa: E402

LIB = _lib.LIB
OK, EINVAL, EWS = _lib.ZF_OK, _lib.ZF_EINVAL, _lib.ZF_EWORKSPACE
BASE = 0x7F0000000000
ref = ctypes.byref


def addr(i):
    return BASE + (i << 36)


def shape(tq=100, tk=200, n=1, heads=8, kv=2, dim=64, causal=1, scale=0.1, sq=None, sk=None, ln=None):
    return _lib.ZfAttention(tq, tk, n, heads, kv, dim, causal, scale, sq, sk, ln)


def heads(i, n=8, dim=64, lt=None, lh=None, off=0):
    return _lib.ZfHeads(addr(i) + off if i is not None else None, n * dim if lt is None else lt,
                        dim if lh is None else lh)


def forward(a=None, q=None, k=None, v=None, out=None, lse=addr(5), ws=addr(6), wsb=1 << 34):
    a = a or shape()
    return LIB.zf_attention_forward(ref(a), ref(q or heads(1)), ref(k or heads(2, 2)),
                                    ref(v or heads(3, 2)), ref(out or heads(4)), lse, ws, wsb, None)


BAD_SHAPES = [dict(tq=-1), dict(tk=1 << 30), dict(n=0), dict(heads=0), dict(kv=0), dict(heads=9),
              dict(dim=0), dict(dim=60), dict(dim=136), dict(scale=0.0), dict(scale=-1.0),
              dict(scale=float("nan")), dict(scale=float("inf")), dict(sq=addr(8)), dict(n=2),
              dict(sk=addr(8)), dict(ln=addr(8)), dict(sq=addr(8) + 2, sk=addr(9)),
              dict(sq=addr(8), sk=addr(9), ln=addr(10) + 1), dict(heads=1 << 17, kv=1 << 17),
              dict(tq=(1 << 30) - 1, heads=64, kv=64), dict(sq=addr(8), sk=addr(9), n=1 << 24)]
BAD_HEADS = [dict(i=None), dict(off=8), dict(lt=516), dict(lh=60), dict(lt=1 << 23), dict(lt=-8)]


def test_attention_forward():
    for kw in BAD_SHAPES:
        assert forward(shape(**kw)) == EINVAL, kw
        assert LIB.zf_attention_forward_workspace_bytes(ref(shape(**kw))) == 0
    assert LIB.zf_attention_forward(None, None, None, None, None, None, None, 0, None) == EINVAL
    for name, i, n in (("q", 1, 8), ("k", 2, 2), ("v", 3, 2), ("out", 4, 8)):
        for kw in BAD_HEADS:
            assert forward(**{name: heads(**{**dict(i=i, n=n), **kw})}) == EINVAL, (name, kw)
    # an output's vectors share elements, or an input's
    for o in (heads(4, lt=0), heads(4, lh=0), heads(4, lt=64), heads(1), heads(2), heads(3, off=16)):
        assert forward(out=o) == EINVAL
    assert forward(lse=addr(5) + 2) == EINVAL and forward(lse=addr(1)) == EINVAL
    assert forward(shape(sq=addr(8), sk=addr(9)), lse=addr(8)) == EINVAL
    one = shape(tq=1, tk=1 << 16)
    need = LIB.zf_attention_forward_workspace_bytes(ref(one))
    assert need > 0
    assert forward(one, wsb=need - 1) == EWS and forward(one, ws=None) == EINVAL
    assert forward(one, ws=addr(6) + 8) == EINVAL and forward(one, ws=addr(4)) == EINVAL
    none = heads(None)
    assert forward(shape(tq=0, tk=0), q=none, k=none, v=none, out=none, lse=None) == OK


def backward(a=None, ws=addr(20), wsb=1 << 30, lse=addr(5), **kw):
    t = dict(q=heads(1), k=heads(2, 2), v=heads(3, 2), out=heads(4), dout=heads(7), dq=heads(11),
             dk=heads(12, 2), dv=heads(13, 2))
    t.update(kw)
    return LIB.zf_attention_backward(ref(a or shape()), ref(t["q"]), ref(t["k"]), ref(t["v"]),
                                     ref(t["out"]), lse, ref(t["dout"]), ref(t["dq"]), ref(t["dk"]),
                                     ref(t["dv"]), ws, wsb, None)


def test_attention_backward():
    for kw in BAD_SHAPES + [dict(sq=addr(8), sk=addr(9), ln=addr(10))]:
        assert backward(shape(**kw)) == EINVAL, kw
    for name, i, n in (("q", 1, 8), ("k", 2, 2), ("v", 3, 2), ("out", 4, 8), ("dout", 7, 8),
                       ("dq", 11, 8), ("dk", 12, 2), ("dv", 13, 2)):
        for kw in BAD_HEADS:
            assert backward(**{name: heads(**{**dict(i=i, n=n), **kw})}) == EINVAL, (name, kw)
    # broadcast gradients, gradients on inputs or on each other
    for kw in (dict(dq=heads(11, lt=0)), dict(dk=heads(12, 2, lh=0)), dict(dv=heads(13, 2, lt=64)),
               dict(dq=heads(1)), dict(dk=heads(2, 2)), dict(dv=heads(7)), dict(dk=heads(13, 2)),
               dict(dq=heads(12)), dict(lse=addr(11)), dict(ws=addr(5)), dict(ws=addr(11)),
               dict(lse=None), dict(q=heads(1, lh=1 << 28)), dict(dout=heads(7, lh=1 << 28))):
        assert backward(**kw) == EINVAL, kw
    need = LIB.zf_attention_backward_workspace_bytes(ref(shape()))
    assert need > 0 and backward(wsb=need - 1) == EWS and backward(ws=None) == EINVAL
    # columns of one buffer that meet
    a = shape(tk=100)
    wide = dict(dq=heads(11, lt=768), dk=heads(11, 2, lt=768, off=1024))
    assert backward(a, dv=heads(11, 2, lt=768, off=1024 + 128), **wide) == EINVAL
    assert backward(a, dv=heads(11, 2, lt=776, off=1024 + 256), **wide) == EINVAL
    none = heads(None)
    assert backward(shape(tq=0, tk=0), lse=None, ws=None, **{n: none for n in (
        "q", "k", "v", "out", "dout", "dq", "dk", "dv")}) == OK


def test_binding_attention():
    q = torch.zeros(4, 2, 16, dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # host tensors
        zf.attention(q, q, q)
    with pytest.raises(TypeError):
        zf.attention(q.float(), q, q)
    for bad in (q[0], q[:, :, :12]):
        with pytest.raises(ValueError):
            zf.attention(bad, bad, bad)
    empty = torch.zeros(0, 2, 16, dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # 2 heads over 3
        zf.attention(empty, torch.zeros(0, 3, 16, dtype=torch.bfloat16),
                     torch.zeros(0, 3, 16, dtype=torch.bfloat16))
    with pytest.raises(ValueError):  # v's shape
        zf.attention(empty, empty, empty[:, :1])
    with pytest.raises(ValueError):
        zf.attention(empty, empty, empty, seq_k=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        zf.attention(empty, empty, empty, seq_q=torch.zeros(2))
    with pytest.raises(ValueError):
        zf.attention(empty, empty, empty, seq_q=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        zf.attention(empty, empty, empty, lse=torch.zeros(3, 0))


def fp8(i, ld, lds, group=1, off=0):
    return _lib.ZfFp8(addr(i) + off, ld, addr(i + 1), lds, group)


def ln_forward(x=addr(0), ldx=300, res=addr(1), ldr=300, dt=0, rows=10, cols=300, gain=addr(2),
               bias=addr(9), gdt=0, eps=1e-6, h=addr(3), ldh=300, y=addr(4), ldy=300, q=None,
               mean=addr(7), rstd=addr(8)):
    return LIB.zf_layernorm_forward(x, ldx, res, ldr, dt, rows, cols, gain, bias, gdt, eps, h, ldh, y,
                                    ldy, ref(q) if q else None, mean, rstd, None)


def test_layernorm_forward():
    for kw in (dict(x=None), dict(ldx=299), dict(ldr=299), dict(dt=5), dict(gdt=-1), dict(rows=-1),
               dict(cols=1 << 30), dict(gain=None), dict(bias=addr(9) + 1), dict(eps=-1.0),
               dict(eps=float("nan")), dict(eps=float("inf")), dict(h=None), dict(ldh=4),
               dict(ldy=299), dict(rstd=None), dict(mean=None), dict(mean=addr(8)),
               dict(rstd=addr(8) + 2), dict(x=addr(0) + 1), dict(dt=1, y=addr(4) + 2),
               dict(q=fp8(5, 304, 4, 128)), dict(q=fp8(5, 300, 4)), dict(q=fp8(4, 304, 4)),
               dict(y=addr(0)), dict(y=addr(1)), dict(y=addr(3)), dict(rstd=addr(2)),
               dict(mean=addr(9)), dict(h=addr(0) + 2), dict(h=addr(1), ldh=304), dict(h=addr(2))):
        assert ln_forward(**kw) == EINVAL, kw
    assert ln_forward(rows=0, x=None, res=None, gain=None, bias=None, h=None, y=None, mean=None,
                      rstd=None) == OK


def ln_backward(dy=addr(0), ldy=300, h=addr(1), ldh=300, dt=0, rows=10, cols=300, gain=addr(2), gdt=0,
                mean=addr(9), rstd=addr(3), res=addr(4), ldr=300, dx=addr(5), ldx=300, dg=addr(6),
                db=addr(8), ws=addr(7), wsb=1 << 30):
    return LIB.zf_layernorm_backward(dy, ldy, h, ldh, dt, rows, cols, gain, gdt, mean, rstd, res, ldr,
                                     dx, ldx, dg, db, ws, wsb, None)


def test_layernorm_backward():
    need = LIB.zf_layernorm_backward_workspace_bytes(10, 300)
    assert need > 0
    for kw in (dict(dy=None), dict(ldy=299), dict(h=None), dict(ldh=9), dict(dt=2), dict(rows=-5),
               dict(gain=None), dict(rstd=None), dict(mean=None), dict(rstd=addr(3) + 1), dict(ldr=1),
               dict(dx=None), dict(ldx=299), dict(dg=addr(6) + 2), dict(db=addr(6)), dict(ws=None),
               dict(ws=addr(7) + 4), dict(dx=addr(1)), dict(dx=addr(0) + 2), dict(dx=addr(4), ldx=304),
               dict(dg=addr(5)), dict(ws=addr(0)), dict(dg=addr(3)), dict(db=addr(9)),
               dict(db=addr(0))):
        assert ln_backward(**kw) == EINVAL, kw
    assert ln_backward(wsb=need - 1) == EWS
    assert ln_backward(dg=None, wsb=need - 1) == EWS
    none = dict(dy=None, h=None, dx=None, gain=None, mean=None, rstd=None, res=None)
    assert ln_backward(rows=0, dg=None, db=None, **none) == OK
    assert ln_backward(cols=0, ldy=0, ldh=0, ldr=0, ldx=0) == OK


def epilogue(**kw):
    a = dict(bias=addr(14), bias_dtype=0, activation=2, dtype=0, residual=addr(15), ld_residual=60,
             z=addr(16), ld_z=60, y=addr(17), ld_y=60, q=None)
    a.update(kw)
    q = a.pop("q")
    e = _lib.ZfEpilogue(**a)
    if q is not None:
        e.q = ctypes.pointer(q)
    return e


def linear(a=None, b=None, m=100, n=60, k=200, e=None, ws=addr(12), wsb=1 << 34):
    return LIB.zf_linear_fp8(ref(a or fp8(1, 208, 4)), ref(b or fp8(3, 208, 4, 128)), m, n, k,
                             ref(e or epilogue()), ws, wsb, None)


def test_linear():
    for kw in (dict(m=-1), dict(n=1 << 30), dict(k=1 << 23), dict(a=fp8(1, 192, 4)),
               dict(b=fp8(3, 208, 4, 2)), dict(a=fp8(1, 1 << 23, 4)), dict(b=fp8(3, 208, 1 << 23))):
        assert linear(**kw) == EINVAL, kw
    for kw in (dict(dtype=2), dict(bias_dtype=2), dict(activation=5), dict(activation=-1),
               dict(bias=addr(14) + 1), dict(bias_dtype=1, bias=addr(14) + 2), dict(ld_residual=59),
               dict(ld_z=59), dict(ld_y=1), dict(z=None, y=None), dict(z=addr(16) + 1),
               dict(dtype=1, y=addr(17) + 2), dict(q=fp8(18, 64, 4, 128)), dict(q=fp8(18, 60, 4)),
               dict(q=fp8(17, 64, 4)), dict(z=addr(17)), dict(z=addr(15)), dict(y=addr(15) + 2),
               dict(y=addr(15), ld_y=64), dict(y=addr(1)), dict(z=addr(4)), dict(y=addr(14)),
               dict(q=fp8(15, 64, 4))):
        assert linear(e=epilogue(**kw)) == EINVAL, kw
    assert LIB.zf_linear_fp8(ref(fp8(1, 208, 4)), ref(fp8(3, 208, 4)), 1, 1, 1, None, None, 0,
                             None) == EINVAL
    assert linear(m=0) == OK and linear(n=0) == OK
    need = LIB.zf_linear_fp8_workspace_bytes(8, 60, 200, 1)
    assert need > 0 and LIB.zf_linear_fp8_workspace_bytes(-1, 60, 200, 1) == 0
    e = epilogue(q=fp8(18, 64, 4))
    assert linear(m=8, e=e, wsb=need - 1) == EWS and linear(m=8, e=e, ws=None) == EINVAL
    assert linear(m=8, e=e, ws=addr(17)) == EINVAL


def linear_backward(dy=addr(0), ldy=300, z=addr(1), ldz=300, dt=0, rows=10, cols=300, act=2,
                    dz=addr(2), lddz=300, q=None, qt=None, db=addr(7), ws=addr(8), wsb=1 << 30):
    return LIB.zf_linear_fp8_backward(dy, ldy, z, ldz, dt, rows, cols, act, dz, lddz,
                                      ref(q) if q else None, ref(qt) if qt else None, db, ws, wsb,
                                      None)


def test_linear_backward():
    need = LIB.zf_linear_fp8_backward_workspace_bytes(10, 300)
    for kw in (dict(dy=None), dict(ldy=299), dict(z=None), dict(ldz=3), dict(dt=2), dict(rows=-1),
               dict(cols=1 << 30), dict(act=5), dict(act=-1), dict(dz=None, db=None),
               dict(dz=addr(0) + 2), dict(dz=addr(1), lddz=304), dict(q=fp8(3, 304, 4, 128)),
               dict(qt=fp8(3, 16, 4, 128)), dict(q=fp8(3, 304, 4), qt=fp8(3, 16, 4)),
               dict(q=fp8(0, 304, 4)), dict(qt=fp8(1, 16, 4)), dict(db=addr(0)), dict(db=addr(7) + 1),
               dict(ws=None), dict(ws=addr(8) + 4), dict(ws=addr(1)), dict(ws=addr(2))):
        assert linear_backward(**kw) == EINVAL, kw
    assert need > 0 and linear_backward(wsb=need - 1) == EWS
    assert linear_backward(rows=0, dy=None, z=None, dz=addr(2), db=None) == OK
    assert linear_backward(cols=0, ldy=0, ldz=0, lddz=0) == OK


def test_binding_layer():
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        zf.layernorm(x, x[0])
    with pytest.raises(TypeError):
        zf.layernorm(x.double(), x[0])
    with pytest.raises(ValueError):
        zf.layernorm_backward(x, x, x[0], x[:, 0].float(), x[:, 0].float())
    f = zf.alloc_fp8(4, 8, device="cpu")
    with pytest.raises(ValueError):
        zf.linear_fp8(f, f)
    e = zf.Fp8(f.data[:0], f.scale[:0])
    with pytest.raises(ValueError):
        zf.linear_fp8(e, e, activation="tanh")
    with pytest.raises(TypeError):
        zf.linear_fp8(e, e, dtype=torch.float16)
    with pytest.raises(ValueError):
        zf.linear_fp8(e, e, want_y=False)
    with pytest.raises(ValueError):
        zf.linear_fp8_backward(x)
    with pytest.raises(ValueError):
        zf.linear_fp8_backward(x[:0], None, "gelu")
    with pytest.raises(ValueError):
        zf.linear_fp8_backward(x[:0], rows=False, transposed=False, want_dbias=False)


def test_tensors_of_other_gpus():
    """With more than one GPU: all tensors on the launch's."""
    class On:
        is_cuda = True

        def __init__(self, i):
            self.index = i

        def get_device(self):
            return self.index

    class Stream:
        def __init__(self, i):
            self.device = torch.device("cuda", i)

    host = torch.zeros(1)
    _lib._same_device(Stream(1), q=On(1), k=None, v=host, out=On(1))
    with pytest.raises(ValueError, match="^k: lives on GPU 0, other arguments on GPU 1"):
        _lib._same_device(Stream(1), q=On(1), k=On(0))
    with pytest.raises(ValueError, match="^k: lives on GPU 1, the call is launched on GPU 0"):
        _lib._same_device(Stream(0), q=None, k=On(1))
