"""zf_rmsnorm_forward and zf_rmsnorm_backward against 64 bits.

A sum of n terms in fp32, taken in pieces, errs by at most `terms(n)` roundings
(2^-24 each) of the sum of magnitudes: the longest chain of additions is a
thread's share plus the wave's 6 and the block's 16."""
import pytest
import torch

from tests import _layer as R

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")

U = 2.0 ** -24
SHAPES = [(1, 1), (3, 7), (1, 4096), (2, 128), (5, 513), (9, 2049), (4, 4099), (700, 300),
          (3, 8200), (2, 16400), (3, 33000), (1, 100003), (1500, 64)]
DTYPES = [torch.bfloat16, torch.float32]


def terms(n):
    return 8 * -(-n // 512) + 24 if n <= 512 else n / 64 + 32


def half_ulp(dtype):
    return 2.0 ** -9 if dtype == torch.bfloat16 else U


def inputs(shape, dtype, seed, gain_dtype=None):
    gen = torch.Generator().manual_seed(seed)
    x, r, dy = (torch.randn(shape, generator=gen).to(dtype) for _ in range(3))
    g = (1 + 0.2 * torch.randn(shape[1], generator=gen)).to(gain_dtype or dtype)
    return x, r, dy, g


def forward64(h, g, eps):
    h, g = h.double(), g.double()
    rstd = (h.square().mean(1) + eps).rsqrt()
    return rstd, h * rstd[:, None] * g


def check_forward(out, x, res, g, eps, dtype):
    h = x if res is None else (x.float() + res.float()).to(dtype)
    assert torch.equal(out.h.cpu(), h)
    rstd, y = forward64(h, g, eps)
    tol = (terms(h.shape[1]) / 2 + 6) * U
    err = (out.rstd.cpu().double() / rstd - 1).abs()
    assert (err <= tol).all(), err.max()
    if out.y is not None:
        # the types' smallest subnormal, for values that round to one
        lim = (tol + 3 * U + 2 * half_ulp(dtype)) * y.abs() + 2.0 ** -130
        assert ((out.y.cpu().double() - y).abs() <= lim).all()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("pad", [0, 3, 8])
def test_forward(shape, dtype, residual, pad):
    x, r, _, g = inputs(shape, dtype, 1, torch.float32 if pad == 3 else None)
    xd, rd = R.strided(x, pad, pad % 2), R.strided(r, pad) if residual else None
    res = r if residual else None
    q, data, scale = R.fp8_buffers(zf, *shape, 1)
    out = zf.rmsnorm(xd, g.cuda(), rd, eps=1e-5, q=q)
    check_forward(out, x, res, g, 1e-5, dtype)
    # the 8-bit output is y, quantised
    want, code = R.quantize(out.y.cpu().double(), 1)
    assert torch.equal(q.scale.view(torch.uint8).cpu(), code)
    assert torch.equal(q.data.float().cpu().double(), want)
    d, s = data.cpu(), scale.cpu()
    d[:shape[0], :shape[1]], s[:code.shape[0], :code.shape[1]] = 0x7F, 0xFF
    assert (d == 0x7F).all() and (s == 0xFF).all(), "written outside"
    # each output alone gives the same
    assert torch.equal(zf.rmsnorm(xd, g.cuda(), rd, eps=1e-5).y, out.y)
    alone = zf.rmsnorm(xd, g.cuda(), rd, eps=1e-5, want_y=False, want_q=True)
    assert alone.y is None
    assert torch.equal(alone.q.data.view(torch.uint8), q.data.view(torch.uint8))


@pytest.mark.parametrize("shape", [(5, 513), (2, 33000)], ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
def test_forward_in_place(shape, dtype):
    x, r, _, g = inputs(shape, dtype, 2)
    want = zf.rmsnorm(x.cuda(), g.cuda(), r.cuda())
    stream = r.cuda()  # the residual stream, updated where it is
    out = zf.rmsnorm(x.cuda(), g.cuda(), stream, h=stream)
    assert out.h is stream and torch.equal(stream, want.h) and torch.equal(out.y, want.y)
    xd = x.cuda()
    out = zf.rmsnorm(xd, g.cuda(), r.cuda(), h=xd)
    assert torch.equal(xd, want.h) and torch.equal(out.y, want.y)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
def test_forward_values(dtype):
    """Rows of zeros, of tiny elements (eps decides), and with an infinity or a
    NaN (that row alone)."""
    x, _, _, g = inputs((6, 300), dtype, 3)
    x[0], x[2, 5], x[4, 299] = 0, float("inf"), float("nan")
    x[1] *= 2.0 ** -40
    out = zf.rmsnorm(x.cuda(), g.cuda(), eps=1e-6, want_q=True)
    y, rstd = out.y.cpu(), out.rstd.cpu()
    assert (y[0] == 0).all() and rstd[0] == pytest.approx(1e3)
    assert y[4].isnan().all()
    assert y[2, 5].isnan() and (y[2, :5] == 0).all()  # inf / inf, x / inf
    fine = [0, 1, 3, 5]
    r64, y64 = forward64(x[fine], g, 1e-6)
    assert ((y[fine].double() - y64).abs() <= (2 * half_ulp(dtype) + 1e-5) * y64.abs()).all()
    code = out.q.scale.view(torch.uint8).cpu()
    assert (code[4] == 255).all() and code[2].tolist()[0] == 255
    assert (code[fine] != 255).all()


def backward64(dy, h, g, rstd, dres):
    dy, h, g, rstd = (t.double() for t in (dy, h, g, rstd))
    hh, t = h * rstd[:, None], dy * g
    c = (t * hh).mean(1, keepdim=True)
    dx = rstd[:, None] * (t - hh * c)
    if dres is not None:
        dx = dx + dres.double()
    return dx, (dy * hh).sum(0), (dy * hh).abs().sum(0), hh, t


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("dres", [False, True])
@pytest.mark.parametrize("pad", [0, 3, 8])
def test_backward(shape, dtype, dres, pad):
    h, r, dy, g = inputs(shape, dtype, 4, torch.float32 if pad == 3 else None)
    rstd = (h.double().square().mean(1) + 1e-5).rsqrt().float()
    res = r if dres else None
    args = (R.strided(dy, pad), R.strided(h, pad, pad % 2), g.cuda(), rstd.cuda())
    rd = R.strided(r, pad) if dres else None
    dx, dgain = zf.rmsnorm_backward(*args, dresidual=rd)
    dx64, dg64, size, hh, t = backward64(dy, h, g, rstd, res)
    n = shape[1]
    lim = rstd.double()[:, None] * U * (6 * t.abs() + hh.abs() * (terms(n) + 8)
                                        * (t * hh).abs().mean(1, keepdim=True))
    lim = lim + (2 * half_ulp(dtype) + 2 * U) * dx64.abs() + 2.0 ** -130
    if dres:
        lim = lim + 2 * U * (dx64 - r.double()).abs()
    assert ((dx.cpu().double() - dx64).abs() <= lim).all()
    assert ((dgain.cpu().double() - dg64).abs() <= (shape[0] + 4) * U * size).all()
    # without the gain's gradient, and in place of dy or of dresidual
    only, none = zf.rmsnorm_backward(*args, dresidual=rd, want_dgain=False)
    assert none is None and torch.equal(only, dx)
    again, dgain2 = zf.rmsnorm_backward(*args, dresidual=rd, dx=args[0])
    assert torch.equal(again, dx) and torch.equal(dgain2, dgain), "equal calls, equal bits"
    if dres:
        own, _ = zf.rmsnorm_backward(R.strided(dy, pad), *args[1:], dresidual=rd, dx=rd)
        assert torch.equal(own, dx)


def test_backward_formula_against_differences():
    """The formula the tests compare with, against central differences of the
    forward pass in 64 bits."""
    gen = torch.Generator().manual_seed(6)
    x, dy = (torch.randn(3, 9, generator=gen, dtype=torch.float64) for _ in range(2))
    g = 1 + 0.2 * torch.randn(9, generator=gen, dtype=torch.float64)
    rstd, _ = forward64(x, g, 1e-5)
    dx, dg, *_ = backward64(dy, x, g, rstd, None)
    step = 1e-5

    def loss(x, g):
        return (forward64(x, g, 1e-5)[1] * dy).sum()

    for i in range(3):
        for j in range(9):
            d = torch.zeros_like(x)
            d[i, j] = step
            diff = (loss(x + d, g) - loss(x - d, g)) / (2 * step)
            assert abs(diff - dx[i, j]) < 1e-8
    for j in range(9):
        d = torch.zeros_like(g)
        d[j] = step
        assert abs((loss(x, g + d) - loss(x, g - d)) / (2 * step) - dg[j]) < 1e-8


def test_no_rows():
    g = torch.ones(5, device="cuda", dtype=torch.bfloat16)
    x = torch.empty(0, 5, device="cuda", dtype=torch.bfloat16)
    out = zf.rmsnorm(x, g, want_q=True)
    assert out.y.shape == (0, 5)
    dx, dgain = zf.rmsnorm_backward(x, x, g, out.rstd, dgain=torch.full((5,), 3.0, device="cuda"))
    assert dx.shape == (0, 5) and (dgain == 0).all()


@pytest.mark.parametrize("cols", [*range(65, 73), 512, 1025, 2047, 2049, 3080, 4102, 5123, 6145,
                                  8193, 11007, 12289, 16383])
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
def test_every_tail_and_block(cols, dtype):
    """Rows that end at each element of a thread's eight, and rows either side of
    each number of threads."""
    test_forward((3, cols), dtype, True, 1)
    test_backward((3, cols), dtype, True, 1)


@pytest.mark.parametrize("shape", [(16500, 40), (4111, 4100)], ids=str)
def test_backward_many_rows(shape):
    test_backward(shape, torch.bfloat16, True, 0)


def test_more_rows_than_blocks():
    """A dispatch has at most 2^21 blocks; its rows are walked in strides."""
    test_forward((2 ** 21 + 5, 8), torch.bfloat16, True, 0)
    test_backward((2 ** 21 + 5, 8), torch.bfloat16, True, 0)
