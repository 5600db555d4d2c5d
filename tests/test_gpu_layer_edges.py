"""Edges of the operators of include/zf_layer.h: matrices without elements."""
import pytest
import torch

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")

DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
def test_norm_of_rows_without_elements(dtype, residual):
    """They count as rows of zeros: every output that has elements is written."""
    x = torch.empty(5, 0, dtype=dtype, device="cuda")
    gain = torch.empty(0, dtype=dtype, device="cuda")
    rstd = torch.full((6,), 7.0, device="cuda")
    out = zf.rmsnorm(x, gain, x.clone() if residual else None, eps=1e-6, want_q=True, rstd=rstd[:5])
    assert out.y.shape == out.h.shape == out.q.shape == (5, 0)
    assert rstd.tolist() == pytest.approx([1e3] * 5 + [7.0])
    dx, dgain = zf.rmsnorm_backward(x, x, gain, out.rstd)
    assert dx.shape == (5, 0) and dgain.shape == (0,)


def test_workspaces_that_no_kernel_may_write():
    """In host memory, strided, or too small; one of any type serves."""
    x = torch.randn(40, 6000, generator=torch.Generator().manual_seed(1)).cuda()
    a, b = zf.quantize_fp8(x)[0], zf.quantize_fp8(x[:30], 128)[0]
    need = zf.matmul_fp8_workspace_bytes(40, 30, 6000)
    h, gain = x[:, :64].contiguous(), torch.ones(64, device="cuda")
    rstd = torch.ones(40, device="cuda")
    need_norm = zf.rmsnorm_backward_workspace_bytes(40, 64)
    grad = torch.zeros(40, 64, dtype=torch.bfloat16, device="cuda")
    need_col = zf.colnorm_workspace_bytes(40, 64)
    assert need and need_norm and need_col
    for call, size in ((lambda w: zf.matmul_fp8(a, b, workspace=w), need),
                       (lambda w: zf.rmsnorm_backward(h, h, gain, rstd, workspace=w)[0], need_norm),
                       (lambda w: zf.colnorm(grad, workspace=w), need_col)):
        with pytest.raises(ValueError, match="workspace"):
            call(torch.empty(size, dtype=torch.uint8))
        with pytest.raises(ValueError, match="workspace"):
            call(torch.empty(size, 2, dtype=torch.uint8, device="cuda")[:, 0])
        with pytest.raises(zf.ZfError):
            call(torch.empty(size - 1, dtype=torch.uint8, device="cuda"))
        want = call(None)
        assert torch.equal(call(torch.empty(-(-size // 8), dtype=torch.float64, device="cuda")), want)
