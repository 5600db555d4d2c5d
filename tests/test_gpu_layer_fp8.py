"""zf_quantize_fp8 and zf_matmul_fp8 against 64 bits.

The quantiser is exact: its only rounding is the one to e4m3.  An fp32
product's error is bounded by that of an fp32 sum: the accumulator takes 16
products at a time, so at most k / 16 + 8 roundings of at most the sum of
magnitudes each (8 for those inside an instruction and for sums split over
waves).  A bf16 product may besides lose 2^-10 of the largest of every 64
products (zf_layer.h), and half an ulp of its own rounding."""
import pytest
import torch

from tests import _layer as R

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")

SHAPES = [(1, 1), (1, 128), (3, 17), (128, 128), (127, 129), (130, 257), (257, 15), (5, 1000),
          (300, 1), (1, 5003)]


def values(shape, dtype, seed):
    """Activations with a spread of scales, some zero rows and tiny elements."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=gen) * torch.exp(3 * torch.randn(shape[1], generator=gen))
    x[shape[0] // 2] *= 2.0 ** -60
    if shape[0] > 2:
        x[shape[0] - 1] = 0
    return x.to(dtype)


def check(got, data, scale, x64, group):
    q, code = R.quantize(x64, group)
    r, c = x64.shape
    sr, sc = code.shape
    assert torch.equal(got.scale.view(torch.uint8).cpu(), code)
    assert torch.equal(got.data.float().cpu().double(), q)
    d, s = data.cpu(), scale.cpu()
    d[:r, :c], s[:sr, :sc] = 0x7F, 0xFF
    assert (d == 0x7F).all() and (s == 0xFF).all(), "written outside"


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 128])
@pytest.mark.parametrize("pad,off", [(0, 0), (3, 1), (8, 0)])
def test_quantize(shape, dtype, group, pad, off):
    x = values(shape, dtype, 3)
    xd = R.strided(x, pad, off)
    r, c = shape
    for want in ("rows", "transposed", "both"):
        a, da, sa = R.fp8_buffers(zf, r, c, group)
        b, db, sb = R.fp8_buffers(zf, c, r, group)
        zf.quantize_fp8(xd, group, rows=False, out=a if want != "transposed" else None,
                        out_t=b if want != "rows" else None)
        torch.cuda.synchronize()
        if want != "transposed":
            check(a, da, sa, x.double(), group)
        if want != "rows":
            check(b, db, sb, x.double().t().contiguous(), group)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_quantize_every_scale(dtype):
    """Magnitudes over the whole exponent range: at 448 and 1.75 times powers of
    two, the next value above, ties between codes, subnormals."""
    tops = []
    for e in range(-149 if dtype == torch.float32 else -133, 128):
        for f in (1.0, 1.75, 1.7578125, 1.9921875):
            tops.append(f * 2.0 ** e)
    top = torch.tensor(tops, dtype=torch.float64).to(dtype)
    gen = torch.Generator().manual_seed(1)
    x = torch.zeros(len(tops), 128, dtype=torch.float64)
    x[:, 0] = top.double()
    x[:, 1:] = top.double()[:, None] * (torch.randint(-448, 449, (len(tops), 127), generator=gen) / 448)
    x[:, 5] = -top.double() * (17 / 16) * 2.0 ** -5
    x = x.to(dtype)
    x[-1, 0] = torch.finfo(dtype).max
    x[~torch.isfinite(x)] = 0
    a, da, sa = R.fp8_buffers(zf, len(tops), 128, 1)
    zf.quantize_fp8(x.cuda(), 1, out=a)
    check(a, da, sa, x.double(), 1)


@pytest.mark.parametrize("group", [1, 128])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_quantize_nonfinite(group, bad):
    """A group that holds one: code 255, zero elements; the others as ever."""
    x = values((200, 300), torch.bfloat16, 5)
    x[130, 140] = bad
    a, da, sa = R.fp8_buffers(zf, 200, 300, group)
    b, db, sb = R.fp8_buffers(zf, 300, 200, group)
    zf.quantize_fp8(x.cuda(), group, out=a, out_t=b)
    check(a, da, sa, x.double(), group)
    check(b, db, sb, x.double().t().contiguous(), group)
    assert int((a.scale.view(torch.uint8) == 255).sum()) == 1
    assert int((b.scale.view(torch.uint8) == 255).sum()) == 1


MATMULS = [(1, 1, 1), (1, 16, 128), (2, 5, 64), (7, 100, 127), (16, 256, 1000), (17, 33, 129),
           (33, 300, 640), (64, 64, 511), (100, 130, 2048), (128, 128, 128), (129, 257, 389),
           (300, 200, 1025), (511, 513, 3001), (1, 4099, 5003), (40, 1000, 11008), (700, 90, 4096),
           (256, 512, 65), (1000, 1000, 16), (3, 2, 100000), (257, 300, 20000)]


def largest(a, b):
    """The sum over every 64 elements of the reduction of the largest product's
    magnitude."""
    a, b = a.abs(), b.abs()
    out = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device=a.device)
    for k in range(0, a.shape[1], 64):
        x, y = a[:, k:k + 64], b[:, k:k + 64]
        for r in range(0, a.shape[0], 32):
            out[r:r + 32] += (x[r:r + 32, None, :] * y[None]).amax(2)
    return out


def product_check(a, b, a64, b64, dtype, out=None):
    k = a64.shape[1]
    a64, b64 = a64.cuda(), b64.cuda()
    got = zf.matmul_fp8(a, b, out=out, dtype=dtype)
    torch.cuda.synchronize()
    want = a64 @ b64.t()
    size = a64.abs() @ b64.abs().t()
    tol = (k / 16 + 8) * 2.0 ** -23 * size
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * want.abs() + 2.0 ** -10 * largest(a64, b64)
    err = (got.double() - want).abs()
    assert (err <= tol).all(), (err - tol).max()
    return got


@pytest.mark.parametrize("m,n,k", MATMULS)
@pytest.mark.parametrize("groups", [(1, 1), (1, 128), (128, 1)], ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_matmul(m, n, k, groups, dtype):
    gen = torch.Generator().manual_seed(m * 31 + n * 7 + k)
    a, a64 = R.random_fp8(zf, m, k, groups[0], gen)
    b, b64 = R.random_fp8(zf, n, k, groups[1], gen)
    buf = torch.full((m + 1, n + 3), 7.0, dtype=dtype, device="cuda")
    got = product_check(a, b, a64, b64, dtype, out=buf[:m, :n])
    assert (buf[m:] == 7.0).all() and (buf[:, n:] == 7.0).all(), "written outside"
    again = zf.matmul_fp8(a, b, dtype=dtype)
    assert torch.equal(again, got), "equal calls give equal bits"


# Enough tiles for the larger tile shapes (256 x 256 and, below, 128 x 256), with
# reductions of one step, of odd ends, of whole steps.
LARGE = [(4100, 2700, k) for k in (1, 65, 128, 129, 500, 640)] + \
        [(2100, 2600, k) for k in (16, 127, 256, 1100)] + [(5000, 2100, 384), (1300, 4000, 777)]


@pytest.mark.parametrize("m,n,k", LARGE)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_matmul_large(m, n, k, dtype):
    gen = torch.Generator().manual_seed(m + n + k)
    a, a64 = R.random_fp8(zf, m, k, 1, gen)
    b, b64 = R.random_fp8(zf, n, k, 128 if k % 2 else 1, gen)
    buf = torch.full((m + 1, n + 5), 7.0, dtype=dtype, device="cuda")
    got = product_check(a, b, a64, b64, dtype, out=buf[:m, :n])
    assert (buf[m:] == 7.0).all() and (buf[:, n:] == 7.0).all(), "written outside"
    assert torch.equal(zf.matmul_fp8(a, b, dtype=dtype), got), "equal calls give equal bits"


def test_matmul_empty():
    a, b = zf.alloc_fp8(5, 0), zf.alloc_fp8(7, 0)
    assert (zf.matmul_fp8(a, b, out=torch.full((5, 7), 3.0, device="cuda")) == 0).all()
    assert zf.matmul_fp8(zf.alloc_fp8(0, 64), zf.alloc_fp8(7, 64)).shape == (0, 7)
    assert zf.matmul_fp8(zf.alloc_fp8(5, 64), zf.alloc_fp8(0, 64)).shape == (5, 0)


@pytest.mark.parametrize("m", [1, 20, 300])
def test_matmul_nan_scale(m):
    """A NaN scale reaches exactly the outputs whose groups hold it."""
    gen = torch.Generator().manual_seed(11)
    a, a64 = R.random_fp8(zf, m, 700, 1, gen)
    b, b64 = R.random_fp8(zf, 260, 700, 1, gen)
    a.scale.view(torch.uint8)[m // 2, 5] = 255
    b.scale.view(torch.uint8)[129, 0] = 255
    got = zf.matmul_fp8(a, b, dtype=torch.float32).isnan().cpu()
    want = torch.zeros_like(got)
    want[m // 2], want[:, 129] = True, True
    assert torch.equal(got, want)


@pytest.mark.parametrize("m", [1, 300])
def test_matmul_extreme_scales(m):
    """Scales at both ends of the range: products of 2^-127 with 2^120."""
    gen = torch.Generator().manual_seed(12)
    a, a64 = R.random_fp8(zf, m, 256, 1, gen, spread=0)
    b, b64 = R.random_fp8(zf, 64, 256, 1, gen, spread=0)
    a.scale.view(torch.uint8).fill_(0)
    b.scale.view(torch.uint8).fill_(247)
    product_check(a, b, a64 * 2.0 ** -127, b64 * 2.0 ** 120, torch.bfloat16)


@pytest.mark.parametrize("m", [1, 300])
@pytest.mark.parametrize("codes", [(20, 200), (110, 0), (240, 20)])
def test_matmul_far_scales(m, codes):
    """fp32 results with scales far from 1, the values within bf16's range: bound
    as ever, plus what counts as zero (below 2^-126)."""
    gen = torch.Generator().manual_seed(14)
    a, a64 = R.random_fp8(zf, m, 256, 1, gen, spread=0)
    b, b64 = R.random_fp8(zf, 64, 256, 1, gen, spread=0)
    a.scale.view(torch.uint8).fill_(codes[0])
    b.scale.view(torch.uint8).fill_(codes[1])
    sa, sb = 2.0 ** (codes[0] - 127), 2.0 ** (codes[1] - 127)
    got = zf.matmul_fp8(a, b, dtype=torch.float32).double().cpu()
    want = (a64 @ b64.t()) * sa * sb
    lost = 2.0 ** -126 * (a64.abs().sum(1)[:, None] * sa + b64.abs().sum(1)[None] * sb)
    tol = 24 * 2.0 ** -23 * (a64.abs() @ b64.abs().t()) * sa * sb + lost
    assert ((got - want).abs() <= tol).all()


def test_graph_replays():
    """Norm and product of a token captured once, replayed on new inputs between
    eager work, every replay against the eager result."""
    gen = torch.Generator().manual_seed(8)
    x = torch.empty(3, 512, dtype=torch.bfloat16, device="cuda")
    res = torch.empty_like(x)
    g = torch.ones(512, dtype=torch.bfloat16, device="cuda")
    w, _ = zf.quantize_fp8((torch.randn(700, 512, generator=gen) / 20).to(torch.bfloat16).cuda(), 128)
    w300, _ = zf.quantize_fp8(torch.randn(256, 6000, generator=gen).to(torch.bfloat16).cuda(), 128)
    wide = torch.randn(40, 6000, generator=gen).to(torch.bfloat16).cuda()  # a split reduction

    def run():
        n = zf.rmsnorm(x, g, res, want_y=False, want_q=True)
        return n.h, zf.matmul_fp8(n.q, w), zf.matmul_fp8(zf.quantize_fp8(wide)[0], w300)

    def fill():
        for t in (x, res, wide):
            t.copy_(torch.randn(t.shape, generator=gen).to(t.dtype))

    fill()
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for _ in range(4):
        fill()
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_other_stream():
    """Work on a stream of its own, ordered by it."""
    gen = torch.Generator().manual_seed(4)
    x = torch.randn(300, 500, generator=gen).to(torch.bfloat16).cuda()
    w = torch.randn(200, 500, generator=gen).to(torch.bfloat16).cuda()
    want = zf.matmul_fp8(zf.quantize_fp8(x)[0], zf.quantize_fp8(w, 128)[0])
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        y = zf.matmul_fp8(zf.quantize_fp8(x)[0], zf.quantize_fp8(w, 128)[0])
    st.synchronize()
    assert torch.equal(y, want)


def test_linear_layer_gradients():
    """Forward, input gradient and weight gradient of a linear layer in both
    layouts against 64 bits of the quantised operands."""
    gen = torch.Generator().manual_seed(9)
    t, i, o = 333, 200, 300
    x = torch.randn(t, i, generator=gen).to(torch.bfloat16)
    dy = torch.randn(t, o, generator=gen).to(torch.bfloat16)
    w = (0.05 * torch.randn(o, i, generator=gen)).to(torch.bfloat16)
    (xq, xt), (dq, dt) = (zf.quantize_fp8(v.cuda(), transposed=True) for v in (x, dy))
    wq, wt = zf.quantize_fp8(w.cuda(), 128, transposed=True)

    def v64(v, group):
        return R.value(*R.quantize(v.double().contiguous(), group), group)

    product_check(xq, wq, v64(x, 1), v64(w, 128), torch.bfloat16)
    product_check(dq, wt, v64(dy, 1), v64(w.t(), 128), torch.bfloat16)
    product_check(dt, xt, v64(dy.t(), 1), v64(x.t(), 1), torch.bfloat16)
    product_check(xt, dt, v64(x.t(), 1), v64(dy.t(), 1), torch.float32)


@pytest.mark.parametrize("n", range(257, 265))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_every_tail(n, dtype):
    """Rows that end at each element of a 16-byte unit: of the product's result, and
    of what is quantised."""
    test_matmul(40, n, 130, (1, 1), dtype)
    test_quantize((40, n), dtype, 1, 1, 0)
    test_quantize((40, n), dtype, 128, 0, 1)
