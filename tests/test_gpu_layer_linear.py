"""zf_linear_fp8 and zf_linear_fp8_backward against 64 bits.

E, H: half a step of fp32 and of bf16, relative.  The activations' exponentials
and reciprocals are good to 2^-22, the normal integral's polynomial to 2^-20;
an exponential's argument x is off by a few E |x|, relative to the result."""
import math

import pytest
import torch

from _layer import F64, fp8_buffers, quantize, random_fp8, strided

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")

BF16, F32 = torch.bfloat16, torch.float32
E, H = 2.0 ** -24, 2.0 ** -8
ACTS = [None, "relu", "gelu", "gelu_tanh", "silu"]


def half(dtype):
    return H if dtype == BF16 else E


def phi(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def act(z, name):
    """(value, slope, relative error of the factor that multiplies z, the largest slope)"""
    one = torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).to(F64), 0 * one, 1.0
    if name == "gelu":
        return (z * phi(z), phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi),
                2.0 ** -20 + 4 * E * z * z, 1.13)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        u = c * (z + 0.044715 * z ** 3)
        p = torch.sigmoid(2 * u)
        return (z * p, p + z * p * (1 - p) * 2 * c * (1 + 0.134145 * z * z),
                2.0 ** -20 + 16 * E * u.abs(), 1.13)
    if name == "silu":
        p = torch.sigmoid(z)
        return z * p, p * (1 + z * (1 - p)), 2.0 ** -20 + 4 * E * z.abs(), 1.1
    return z, one, 0 * one, 1.0


# rows of the second operand reach every form: one row, up to 16, tiles, split tiles
SHAPES = [(1, 40, 70), (1, 1000, 256), (3, 129, 384), (8, 515, 1000), (16, 256, 128), (17, 130, 520),
          (40, 256, 6000), (128, 128, 128), (129, 257, 385), (300, 500, 256), (64, 128, 0),
          (1700, 1664, 136)]


@pytest.mark.parametrize("activation", ACTS)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_forward(m, n, k, activation):
    gen = torch.Generator().manual_seed(m + n + k)
    dtype = BF16 if (m + k) % 2 == 0 else F32
    a, av = random_fp8(zf, m, k, 1, gen, spread=1)
    b, bv = random_fp8(zf, n, k, 128, gen, spread=1)
    # (elements of 448 and fewer: results of a few units)
    unit = 2.0 ** -8 / max(1.0, k) ** 0.5
    b.scale.view(torch.uint8)[:] = (b.scale.view(torch.uint8).int() + round(math.log2(unit)) - 8).to(
        torch.uint8)
    bv = bv * 2.0 ** (round(math.log2(unit)) - 8)
    bias = torch.randn(n, generator=gen).to(F32 if n % 2 else BF16)
    res = torch.randn(m, n, generator=gen).to(dtype)
    y, z = strided(torch.zeros(m, n, dtype=dtype), 5, 1), strided(torch.zeros(m, n, dtype=dtype), 2, 3)
    q, qd, qs = fp8_buffers(zf, m, n, 1)
    zf.linear_fp8(a, b, bias.cuda(), activation, strided(res, 3, 2), y=y, z=z, q=q)
    t = av @ bv.t() + bias.to(F64)
    dt = (k + 8) * E * (av.abs() @ bv.abs().t()) + 2 * E * t.abs()
    assert ((z.cpu().to(F64) - t).abs() <= dt + half(dtype) * (t.abs() + dt)).all()
    value, _, rel, most = act(t, activation)
    want = value + res.to(F64)
    tol = most * 1.01 * dt + (rel + 4 * E) * value.abs() + 2 * E * want.abs() + 1e-30
    tol = tol + half(dtype) * (want.abs() + tol)
    err = (y.cpu().to(F64) - want).abs()
    assert (err <= tol).all(), (err / tol).max().item()
    codes, scale = quantize(y.cpu().to(F64), 1)
    assert torch.equal(q.data.cpu().float(), codes.float())
    assert torch.equal(q.scale.view(torch.uint8).cpu(), scale)
    assert (qd[:m, n:] == 0x7F).all() and (qd[m:] == 0x7F).all()
    assert (qs[:m, scale.shape[1]:] == 0xFF).all() and (qs[m:] == 0xFF).all()


@pytest.mark.parametrize("m,n,k", [(1, 300, 256), (16, 300, 256), (40, 256, 6000), (200, 300, 256)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_forms(m, n, k, dtype):
    """Parts of the epilogue and of the outputs; without any, matmul_fp8's bits."""
    gen = torch.Generator().manual_seed(1)
    a, _ = random_fp8(zf, m, k, 1, gen)
    b, _ = random_fp8(zf, n, k, 1, gen)
    plain = zf.matmul_fp8(a, b, dtype=dtype)
    got = zf.linear_fp8(a, b, want_z=True, dtype=dtype)
    assert torch.equal(got.y, plain) and torch.equal(got.z, plain) and got.q is None
    bias, res = torch.randn(n, generator=gen).cuda(), torch.randn(m, n, generator=gen).to(dtype).cuda()
    full = zf.linear_fp8(a, b, bias, "silu", res, want_z=True, want_q=True, dtype=dtype)
    for kw in (dict(want_y=False, want_q=True), dict(want_y=False, want_z=True), dict()):
        part = zf.linear_fp8(a, b, bias, "silu", res, dtype=dtype, **kw)
        for x, w in zip(part, full):
            if x is not None and not isinstance(x, zf.Fp8):
                assert torch.equal(x, w)
            elif x is not None:
                assert torch.equal(x.data.view(torch.uint8), w.data.view(torch.uint8))
                assert torch.equal(x.scale.view(torch.uint8), w.scale.view(torch.uint8))
    own = res.clone()
    assert torch.equal(zf.linear_fp8(a, b, bias, "silu", own, y=own).y, full.y)


def test_empty_and_nan():
    gen = torch.Generator().manual_seed(1)
    a, _ = random_fp8(zf, 20, 256, 1, gen)
    b, _ = random_fp8(zf, 130, 256, 1, gen)
    assert zf.linear_fp8(zf.Fp8(a.data[:0], a.scale[:0]), b, want_q=True).y.shape == (0, 130)
    for m in (20, 5):
        f = zf.Fp8(a.data[:m], a.scale[:m])
        bias = torch.zeros(130, device="cuda")
        want = zf.linear_fp8(f, b, bias, "gelu", want_q=True)
        bias[129] = float("inf")
        got = zf.linear_fp8(f, b, bias, "gelu", want_q=True)
        assert torch.equal(got.y[:, :129], want.y[:, :129])
        assert (got.q.scale.view(torch.uint8)[:, 1] == 255).all()
        assert torch.equal(got.q.data.view(torch.uint8)[:, :128], want.q.data.view(torch.uint8)[:, :128])


@pytest.mark.parametrize("name", ACTS[1:])
def test_activation_over_its_range(name):
    """Every bf16 number of magnitude up to 2^12 through the backward pass, and
    through the forward as a bias."""
    bits = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16)
    z = bits.view(BF16)
    z = z[torch.isfinite(z.float()) & (z.float().abs() <= 4096)]
    n = z.numel()
    gen = torch.Generator().manual_seed(1)
    a, _ = random_fp8(zf, 1, 0, 1, gen)
    b = zf.alloc_fp8(n, 0)
    y = zf.linear_fp8(a, b, z.cuda(), name, dtype=F32).y[0].cpu().to(F64)
    value, slope, rel, _ = act(z.to(F64), name)
    # a factor of z below 2^-126 may be flushed to 0; it is that small only between z = -88,
    # where exp(-z) passes 2^126, and -128 at the most (exp(-89) is infinite): what is lost
    # is less than 2^-126 * 128
    assert ((y - value).abs() <= (rel + 4 * E) * value.abs() + 2.0 ** -119).all()
    got = zf.linear_fp8_backward(torch.ones(1, n, device="cuda"), z.float()[None].cuda(), name,
                                 rows=False, transposed=False, want_dz=True)
    # a slope is a factor (off by rel) plus a term of at most 0.6 of the same kind, times z
    # to some power that the exponential outweighs
    tol = (2 * rel + 8 * E) * (slope.abs() + (slope - value / torch.where(z == 0, 1.0, z.to(F64))).abs()
                               + (value / torch.where(z == 0, 1.0, z.to(F64))).abs()) + 2.0 ** -119
    assert ((got.dz[0].cpu().to(F64) - slope).abs() <= tol).all()
    assert torch.equal(got.dz[0], got.dbias)


@pytest.mark.parametrize("name", ACTS[1:])
def test_activation_of_large_values(name):
    """Every finite bf16 number beyond 2^12: value and slope are z and 1, or 0 (the
    exponentials there are 0 in 32 bits and their complements 1)."""
    z = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16).view(BF16).float()
    z = z[torch.isfinite(z) & (z.abs() > 4096)]
    n = z.numel()
    a, _ = random_fp8(zf, 1, 0, 1, torch.Generator().manual_seed(1))
    y = zf.linear_fp8(a, zf.alloc_fp8(n, 0), z.cuda(), name, dtype=F32).y[0].cpu()
    assert torch.equal(y, z.clamp(min=0))
    got = zf.linear_fp8_backward(torch.ones(1, n, device="cuda"), z[None].cuda(), name, rows=False,
                                 transposed=False, want_dz=True)
    assert torch.equal(got.dz[0].cpu(), (z > 0).float())


BACK = [(1, 1), (5, 300), (16, 128), (127, 129), (128, 256), (300, 515), (1000, 264), (129, 2048)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("activation", ACTS)
@pytest.mark.parametrize("rows,cols", BACK)
def test_backward(rows, cols, activation, dtype):
    gen = torch.Generator().manual_seed(rows + cols)
    dy, z = torch.randn(rows, cols, generator=gen).to(dtype), torch.randn(rows, cols, generator=gen)
    z = (2 * z).to(dtype)
    q, qd, qs = fp8_buffers(zf, rows, cols, 1)
    qt, td, ts = fp8_buffers(zf, cols, rows, 1)
    dz = strided(torch.zeros_like(dy), 3, 1)
    got = zf.linear_fp8_backward(strided(dy, 2, 3), strided(z, 1, 2), activation, dz=dz, q=q, qt=qt)
    zz = z.to(F64)
    value, slope, rel, _ = act(zz, activation)
    factor = value / torch.where(zz == 0, 1.0, zz)
    err = (2 * rel + 8 * E) * (slope.abs() + (slope - factor).abs() + factor.abs())
    want = dy.to(F64) * slope
    tol = dy.to(F64).abs() * err + 2 * E * want.abs() + 2.0 ** -119
    assert ((dz.cpu().to(F64) - want).abs() <= tol + half(dtype) * (want.abs() + tol)).all()
    chain = (8 + 20 + rows // 128) * E
    assert ((got.dbias.cpu().to(F64) - want.sum(0)).abs()
            <= tol.sum(0) * 1.01 + chain * want.abs().sum(0)).all()
    for f, d, s, x in ((q, qd, qs, dz.cpu()), (qt, td, ts, dz.cpu().t())):
        codes, scale = quantize(x.to(F64).contiguous(), 1)
        r, c = codes.shape
        assert torch.equal(f.data.cpu().float(), codes.float())
        assert torch.equal(f.scale.view(torch.uint8).cpu(), scale)
        assert (d[:r, c:] == 0x7F).all() and (d[r:] == 0x7F).all()
        assert (s[:r, scale.shape[1]:] == 0xFF).all() and (s[r:] == 0xFF).all()


def test_backward_forms():
    gen = torch.Generator().manual_seed(3)
    dy, z = (torch.randn(200, 300, generator=gen).to(BF16).cuda() for _ in range(2))
    full = zf.linear_fp8_backward(dy, z, "gelu", want_dz=True)
    for kw in (dict(rows=False), dict(transposed=False, want_dbias=False),
               dict(rows=False, transposed=False)):
        part = zf.linear_fp8_backward(dy, z, "gelu", **kw)
        for x, w in zip(part, full):
            if isinstance(x, zf.Fp8):
                assert torch.equal(x.data.view(torch.uint8), w.data.view(torch.uint8))
            elif x is not None:
                assert torch.equal(x, w)
    for i in range(2):
        args = [dy.clone(), z.clone()]
        zf.linear_fp8_backward(args[0], args[1], "gelu", dz=args[i])
        assert torch.equal(args[i], full.dz)
    # without an activation: the quantiser's bits, and the column sums
    none = zf.linear_fp8_backward(dy)
    q, qt = zf.quantize_fp8(dy, transposed=True)
    assert torch.equal(none.q.data.view(torch.uint8), q.data.view(torch.uint8))
    assert torch.equal(none.qt.scale.view(torch.uint8), qt.scale.view(torch.uint8))
    empty = zf.linear_fp8_backward(dy[:0], z[:0], "gelu")
    assert (empty.dbias == 0).all() and empty.qt.shape == (300, 0)


def test_captured():
    gen = torch.Generator().manual_seed(4)
    a, _ = random_fp8(zf, 40, 6000, 1, gen, spread=1)
    b, _ = random_fp8(zf, 256, 6000, 128, gen, spread=1)
    bias, dy = torch.randn(256, generator=gen).cuda(), torch.randn(40, 256, generator=gen).to(BF16).cuda()

    def step():
        f = zf.linear_fp8(a, b, bias, "gelu", want_z=True, want_q=True)
        g = zf.linear_fp8_backward(dy, f.z, "gelu")
        return [f.y, f.z, f.q.data.view(torch.uint8), g.q.data.view(torch.uint8),
                g.qt.data.view(torch.uint8), g.dbias]

    step()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = step()
    for i in range(3):
        bias.mul_(-1.5)
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
