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
