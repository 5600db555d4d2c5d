"""The sums of zf_matmul_fp8 where an addition of fewer bits than fp32 shows.

The bound of an fp32 result is that of test_gpu_layer_fp8.py: at most k / 16 + 8
roundings of at most the sum of magnitudes each.  A bf16 result is that sum,
rounded once: half an ulp of the result more, whatever the data."""
import pytest
import torch

from tests import _layer as R

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")

# few rows; a split reduction; tiles, ragged and whole; many tiles
FORMS = [(1, 40, 2048), (5, 33, 1000), (16, 200, 4096), (40, 130, 4096), (129, 300, 1000),
         (1003, 700, 512), (2100, 2600, 256), (4100, 2700, 384)]
DTYPES = [torch.bfloat16, torch.float32]


def operand(row, rows):
    """Every row the same elements, scales 1, everything around them NaN."""
    k = row.numel()
    f, data, scale = R.fp8_buffers(zf, rows, k, 1)
    data[:rows, :k] = row.to(torch.float8_e4m3fn).view(torch.uint8).cuda()
    scale[:rows, :f.scale.shape[1]] = 127
    return f


def limit(want, size, k, dtype):
    tol = (k / 16 + 8) * 2.0 ** -23 * size
    if dtype == torch.bfloat16:
        tol += 2.0 ** (torch.tensor(abs(want) + tol).log2().floor().item() - 8)
    return tol


@pytest.mark.parametrize("m,n,k", FORMS)
@pytest.mark.parametrize("every", [64, 128])
@pytest.mark.parametrize("cancel", [False, True], ids=["add", "cancel"])
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
def test_one_large_product_among_small_ones(m, n, k, every, cancel, dtype):
    """In every 64 or 128 elements one product of 448 * 448, the others positive
    and 2^-11 to 2^-19 of it: none of them may be cut off.  With `cancel` the
    large ones have alternating signs, and the small ones are the result."""
    for p in range(-1, 7):
        x = torch.full((k,), 2.0 ** (p // 2), dtype=torch.float64)
        y = torch.full((k,), 2.0 ** (p - p // 2), dtype=torch.float64)
        at = torch.arange(5, k, every)
        at = at[:len(at) // 2 * 2] if cancel else at
        x[at], y[at] = 448.0, 448.0
        if cancel:
            y[at[1::2]] = -448.0
        want, size = float((x * y).sum()), float((x * y).abs().sum())
        got = zf.matmul_fp8(operand(x, m), operand(y, n), dtype=dtype).double()
        err = (got - want).abs().max().item()
        assert err <= limit(want, size, k, dtype), (p, want, err)


@pytest.mark.parametrize("m,n,k", FORMS + [(1, 1, 1), (1, 4099, 5003), (257, 300, 20000)])
@pytest.mark.parametrize("group", [1, 128])
def test_bf16_result_is_the_rounded_fp32_result(m, n, k, group):
    gen = torch.Generator().manual_seed(m + n + k)
    a, _ = R.random_fp8(zf, m, k, 1, gen)
    b, _ = R.random_fp8(zf, n, k, group, gen)
    want = zf.matmul_fp8(a, b, dtype=torch.float32).to(torch.bfloat16)
    assert torch.equal(zf.matmul_fp8(a, b), want)


@pytest.mark.parametrize("m,n,k", [(1, 260, 700), (16, 260, 700), (20, 260, 700), (300, 260, 700),
                                   (40, 260, 8000), (2100, 2600, 384), (4100, 2700, 384)])
@pytest.mark.parametrize("group", [1, 128])
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
def test_nan_scales(m, n, k, group, dtype):
    """A group that holds an infinity or a NaN (zero elements, code 255) reaches
    exactly the results that it enters, in either type and every form."""
    gen = torch.Generator().manual_seed(11)
    a, _ = R.random_fp8(zf, m, k, 1, gen)
    b, _ = R.random_fp8(zf, n, k, group, gen)
    a.data.view(torch.uint8)[m // 2, 256:384] = 0
    a.scale.view(torch.uint8)[m // 2, 2] = 255
    b.scale.view(torch.uint8)[129 // group, 0] = 255
    b.data.view(torch.uint8)[129 // group * group:129 // group * group + group, :128] = 0
    got = zf.matmul_fp8(a, b, dtype=dtype).isnan()
    want = torch.zeros_like(got)
    want[m // 2] = True
    want[:, 129 // group * group:129 // group * group + group] = True
    assert torch.equal(got, want)


@pytest.mark.parametrize("m,n,k", [(1, 260, 5003), (16, 65, 700), (20, 260, 9000), (300, 260, 700),
                                   (2100, 1300, 1000)])
@pytest.mark.parametrize("codes", [((0, 140), (0, 140)), ((100, 247), (0, 60)),
                                   ((0, 30), (200, 247)), ((0, 0), (0, 247))], ids=str)
@pytest.mark.parametrize("group", [1, 128])
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
def test_scales_far_apart(m, n, k, codes, group, dtype):
    """Scales anywhere in their range and far apart within a row: an element is held
    to within 2^-118 of the largest scale of its row, and sums as ever."""
    gen = torch.Generator().manual_seed(m + n)
    ops, vals, tops = [], [], []
    for rows, grp, (lo, hi) in ((m, 1, codes[0]), (n, group, codes[1])):
        f, v = R.random_fp8(zf, rows, k, grp, gen, spread=0)
        code = torch.randint(lo, hi + 1, f.scale.shape, generator=gen)
        f.scale.view(torch.uint8).copy_(code.to(torch.uint8))
        s = 2.0 ** (code.double() - 127)
        s = s.repeat_interleave(128, 1)[:, :k].repeat_interleave(grp, 0)[:rows]
        ops.append(f)
        vals.append((v * s).cuda())
        tops.append(s.amax(1).cuda())
    (a, b), (sa, sb) = vals, tops
    want, size = a @ b.t(), a.abs() @ b.abs().t()
    tol = (k / 16 + 8) * 2.0 ** -23 * size + (k / 128 + 2) * 2.0 ** -149
    tol += 2.0 ** -118 * (sa[:, None] * b.abs().sum(1) + a.abs().sum(1)[:, None] * sb)
    if dtype == torch.bfloat16:
        tol += torch.ldexp(torch.ones_like(tol), (want.abs() + tol).log2().floor().clamp(min=-126).int() - 8)
    got = zf.matmul_fp8(*ops, dtype=dtype).double()
    assert ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max()
