"""zf_layernorm_forward and zf_layernorm_backward against 64 bits.

E, H: half a step of fp32 and of bf16, relative.  A sum of n terms is taken to
be off by at most d E times the sum of magnitudes, d the longest chain of
additions: a thread's elements (16, or n / 1024 of rows read in pieces), 6 over
a wave, 16 over a block."""
import pytest
import torch

from _layer import F64, fp8_buffers, quantize, strided

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")

BF16, F32 = torch.bfloat16, torch.float32
E, H = 2.0 ** -24, 2.0 ** -8


def half(dtype):
    return H if dtype == BF16 else E


def depth(cols):
    return 40 + cols // 1024


def data(gen, rows, cols, dtype, mean=0.3, std=1.0):
    return (torch.randn(rows, cols, generator=gen) * std + mean).to(dtype)


SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 127), (4, 128), (7, 129), (64, 500), (33, 1003), (17, 2048),
          (9, 3001), (5, 5120), (3, 8192), (2, 8200), (3, 12000), (2, 16384), (2, 16385), (3, 20001)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward(rows, cols, dtype):
    gen = torch.Generator().manual_seed(rows * 7 + cols)
    x, r = data(gen, rows, cols, dtype, mean=2.0), data(gen, rows, cols, dtype)
    gdt = F32 if cols % 2 else dtype
    gain, bias = data(gen, 1, cols, gdt, 1.0, 0.2)[0], data(gen, 1, cols, gdt, 0.0, 0.5)[0]
    gx, gr = strided(x, 5, 1), strided(r, 3, 2)
    y = strided(torch.zeros_like(x), 7, 3)
    q, qd, qs = fp8_buffers(zf, rows, cols, 1)
    got = zf.layernorm(gx, gain.cuda(), bias.cuda(), residual=gr, eps=1e-5, y=y, q=q)
    h = (x.to(F64) + r.to(F64)).to(dtype)
    assert torch.equal(got.h.cpu(), (x.float() + r.float()).to(dtype))
    h = got.h.cpu().to(F64)
    d = depth(cols)
    mean = h.mean(1)
    a = h.abs().mean(1)
    var = (h - mean[:, None]).square().mean(1)
    rstd = (var + 1e-5) ** -0.5
    dm = d * E * a + E * mean.abs()
    dv = 8 * d * E * var + 4 * var.sqrt() * d * E * a + (d * E * a) ** 2
    dr = 0.5 * dv / (var + 1e-5) * 1.1 + 4 * E
    assert ((got.mean.cpu().to(F64) - mean).abs() <= dm).all()
    assert ((got.rstd.cpu().to(F64) / rstd - 1).abs() <= dr).all()
    hh = (h - mean[:, None]) * rstd[:, None]
    g, b = gain.to(F64), bias.to(F64)
    want = hh * g + b
    tol = (((dm + E * mean.abs()) * rstd)[:, None] + hh.abs() * (dr + 4 * E)[:, None]) * g.abs() \
        + E * want.abs()
    tol = tol * 1.01 + half(dtype) * (want.abs() + tol)
    assert ((y.cpu().to(F64) - want).abs() <= tol).all()
    # the 8-bit output is y's, and nothing else of its buffers is written
    codes, scale = quantize(y.cpu().to(F64), 1)
    assert torch.equal(q.data.cpu().float(), codes.float())
    assert torch.equal(q.scale.view(torch.uint8).cpu(), scale)
    assert (qd[:rows, cols:] == 0x7F).all() and (qd[rows:] == 0x7F).all()
    assert (qs[:rows, scale.shape[1]:] == 0xFF).all() and (qs[rows:] == 0xFF).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_forward_forms(dtype):
    """Without residual or bias, in place, parts of the outputs alone."""
    gen = torch.Generator().manual_seed(3)
    x, r = data(gen, 40, 700, dtype).cuda(), data(gen, 40, 700, dtype).cuda()
    gain, bias = data(gen, 1, 700, dtype, 1.0)[0].cuda(), data(gen, 1, 700, dtype)[0].cuda()
    full = zf.layernorm(x, gain, bias, r, want_q=True)
    plain = zf.layernorm(full.h, gain, bias)
    assert plain.h is full.h and torch.equal(plain.y, full.y) and torch.equal(plain.rstd, full.rstd)
    assert torch.equal(zf.layernorm(x, gain, residual=r).y,
                       zf.layernorm(x, gain, torch.zeros_like(bias), r).y)
    only = zf.layernorm(x, gain, bias, r, want_y=False, want_q=True)
    assert only.y is None
    assert torch.equal(only.q.data.view(torch.uint8), full.q.data.view(torch.uint8))
    r2, x2 = r.clone(), x.clone()
    assert torch.equal(zf.layernorm(x, gain, bias, r2, h=r2).y, full.y) and torch.equal(r2, full.h)
    assert torch.equal(zf.layernorm(x2, gain, bias, r, h=x2).y, full.y) and torch.equal(x2, full.h)
    copy = torch.empty_like(x)
    zf.layernorm(x, gain, bias, h=copy)
    assert torch.equal(copy, x)


def test_rows_about_a_large_mean():
    """Squares about the mean do not cancel, as sum(h^2) - n mean^2 would."""
    gen = torch.Generator().manual_seed(1)
    for cols in (384, 5000, 20000):
        h = (torch.randn(6, cols, generator=gen, dtype=F64) + 4096.0).float()
        got = zf.layernorm(h.cuda(), torch.ones(cols, device="cuda"), eps=0.0)
        x = h.to(F64)
        std = (x - x.mean(1, keepdim=True)).square().mean(1).sqrt()
        # the mean is off by depth E 4096; the variance by four times that and its own sums'
        d = depth(cols) * E
        tol = 4 * d * 4096 / std + 8 * d + (d * 4096 / std) ** 2
        assert ((got.rstd.cpu().to(F64) * std - 1).abs() <= tol).all()


def test_constant_rows_and_no_columns():
    x = torch.full((3, 1000), 0.5, device="cuda")
    got = zf.layernorm(x, torch.ones(1000, device="cuda"), torch.full((1000,), 2.0, device="cuda"),
                       eps=1e-4)
    assert (got.mean == 0.5).all() and (got.y == 2).all()
    assert ((got.rstd - 100).abs() <= 100 * 4 * E).all()
    got = zf.layernorm(x[:, :0], torch.ones(0, device="cuda"), eps=0.25)
    assert (got.mean == 0).all() and (got.rstd == 2).all()
    assert zf.layernorm(x[:0], torch.ones(1000, device="cuda")).y.shape == (0, 1000)


@pytest.mark.parametrize("cols", [128, 1000, 20000])
def test_nan_stays_in_its_row(cols):
    x = torch.randn(4, cols, device="cuda")
    g = torch.ones(cols, device="cuda")
    want = zf.layernorm(x, g, want_q=True)
    x[2, cols // 2] = float("nan")
    got = zf.layernorm(x, g, want_q=True)
    keep = [0, 1, 3]
    assert torch.equal(got.y[keep], want.y[keep]) and got.y[2].isnan().all()
    assert (got.q.scale.view(torch.uint8)[2] == 255).all()


BACK = [(1, 1), (2, 130), (16, 384), (33, 1003), (300, 515), (1237, 640), (64, 5120), (5, 8192),
        (9, 12000), (7, 16385), (3000, 264)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", BACK)
def test_backward(rows, cols, dtype):
    gen = torch.Generator().manual_seed(rows + cols)
    h, dy = data(gen, rows, cols, dtype, 1.0), data(gen, rows, cols, dtype, 0.0)
    res = data(gen, rows, cols, dtype) if rows % 2 else None
    gain = data(gen, 1, cols, dtype, 1.0, 0.2)[0]
    hm = h.to(F64)
    mean = hm.mean(1).float()
    rstd = ((hm - mean.to(F64)[:, None]).square().mean(1) + 1e-5).pow(-0.5).float()
    dx = strided(torch.zeros_like(h), 3, 1)
    out = zf.layernorm_backward(strided(dy, 2, 1), strided(h, 4, 3), gain.cuda(), mean.cuda(),
                                rstd.cuda(), None if res is None else strided(res, 1, 0), dx=dx)
    m, rs = mean.to(F64)[:, None], rstd.to(F64)[:, None]
    hh, t = (hm - m) * rs, dy.to(F64) * gain.to(F64)
    mt, ms = t.mean(1, keepdim=True), (t * hh).mean(1, keepdim=True)
    want = rs * (t - mt - hh * ms)
    d = depth(cols)
    # hh: a difference and a product; its share of (h - mean) rounds relative to it
    dhh = 3 * E * hh.abs()
    dmt = (d + 2) * E * t.abs().mean(1, keepdim=True)
    dms = (d + 6) * E * (t * hh).abs().mean(1, keepdim=True)
    tol = rs * (4 * E * (t.abs() + mt.abs() + 2 * (hh * ms).abs()) + dmt + hh.abs() * dms
                + dhh * ms.abs()) * 1.01 + 2 * E * want.abs()
    if res is not None:
        want = want + res.to(F64)
        tol = tol + E * want.abs()
    tol = tol + half(dtype) * (want.abs() + tol) + 1e-37
    assert ((out[0].cpu().to(F64) - want).abs() <= tol).all()
    chain = (64 + rows // 64) * E
    for got, terms in ((out[1], dy.to(F64) * hh), (out[2], dy.to(F64))):
        assert ((got.cpu().to(F64) - terms.sum(0)).abs() <= (chain + 4 * E) * terms.abs().sum(0)).all()


def test_backward_forms():
    gen = torch.Generator().manual_seed(2)
    h, dy, res = (data(gen, 70, 520, BF16).cuda() for _ in range(3))
    gain = data(gen, 1, 520, F32, 1.0)[0].cuda()
    f = zf.layernorm(h, gain)
    dx, dg, db = zf.layernorm_backward(dy, h, gain, f.mean, f.rstd, res)
    for kw, want in ((dict(want_dbias=False), (dx, dg, None)), (dict(want_dgain=False), (dx, None, db)),
                     (dict(want_dgain=False, want_dbias=False), (dx, None, None))):
        got = zf.layernorm_backward(dy, h, gain, f.mean, f.rstd, res, **kw)
        for a, b in zip(got, want):
            assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    for own in (dy.clone(), res.clone()):
        args = (own, h, gain, f.mean, f.rstd, res) if torch.equal(own, dy) else \
            (dy, h, gain, f.mean, f.rstd, own)
        got = zf.layernorm_backward(*args, dx=own)
        assert torch.equal(got[0], dx) and torch.equal(got[1], dg) and torch.equal(got[2], db)
    none = zf.layernorm_backward(dy[:0], h[:0], gain, f.mean[:0], f.rstd[:0])
    assert (none[1] == 0).all() and (none[2] == 0).all()


def test_gradients_against_differences():
    gen = torch.Generator().manual_seed(9)
    x = torch.randn(5, 40, generator=gen, dtype=F64)
    gain, bias, do = (torch.randn(n, generator=gen, dtype=F64) for n in ((40,), (40,), (5, 40)))
    f = zf.layernorm(x.float().cuda(), gain.float().cuda(), bias.float().cuda())
    got = zf.layernorm_backward(do.float().cuda(), x.float().cuda(), gain.float().cuda(), f.mean, f.rstd)
    inputs = [x.float().to(F64), gain.float().to(F64), bias.float().to(F64)]

    def loss(x, gain, bias):
        c = x - x.mean(1, keepdim=True)
        return ((c * (c.square().mean(1, keepdim=True) + 1e-5) ** -0.5 * gain + bias)
                * do.float().to(F64)).sum()

    for i in range(3):
        d = torch.randn(inputs[i].shape, generator=gen, dtype=F64)
        ends = [loss(*[b + s * 1e-5 * d if j == i else b for j, b in enumerate(inputs)])
                for s in (1, -1)]
        slope = (ends[0] - ends[1]) / 2e-5
        g = got[i].cpu().to(F64)
        # fp32 (100 E per element covers the bounds above), and a difference's 1e-8
        assert abs(slope - (g * d).sum()) <= 100 * E * (g * d).abs().sum() + 1e-7


def test_captured():
    gen = torch.Generator().manual_seed(4)
    x, r, dy = (data(gen, 600, 512, BF16).cuda() for _ in range(3))
    gain, bias = data(gen, 1, 512, BF16, 1.0)[0].cuda(), data(gen, 1, 512, BF16)[0].cuda()

    def step():
        f = zf.layernorm(x, gain, bias, r, want_q=True)
        return [f.y, f.mean, f.rstd, f.q.data.view(torch.uint8),
                *zf.layernorm_backward(dy, f.h, gain, f.mean, f.rstd)]

    step()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = step()
    for i in range(3):
        x.add_(0.25)
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
