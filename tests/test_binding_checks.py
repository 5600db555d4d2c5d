"""What the binding's checks of tensors refuse (no GPU needed)."""
import pytest
import torch

zf = pytest.importorskip("paper_2505_12242_amd")
from paper_2505_12242_amd import _lib  # noqa: E402


@pytest.mark.parametrize("t", [torch.zeros(6, 8).t()[:1], torch.zeros(1, 8)[:, ::2],
                               torch.zeros(8, 3)[:, 1:2].t()], ids=["t", "step", "column"])
def test_a_single_rows_elements_are_contiguous(t):
    """One row (a single token) whose elements are not next to each other is refused,
    as more rows are: the kernels would read its neighbours."""
    with pytest.raises(ValueError, match="contiguous"):
        _lib._mat(t, torch.float32, "x", host=True)


@pytest.mark.parametrize("t", [torch.zeros(1, 8)[:, 2:7], torch.zeros(6, 8)[:1], torch.zeros(8, 1).t(),
                               torch.zeros(8, 3)[2:3, 1:2], torch.zeros(1, 8)[:, :0],
                               torch.zeros(8, 0).t()[:0], torch.zeros(0, 4)], ids=str)
def test_a_single_row_needs_no_row_stride(t):
    assert _lib._mat(t, torch.float32, "x", host=True) == t.shape[1]


def test_workspace_is_on_the_gpu():
    """A workspace in host memory is refused before the kernels would write to it."""
    assert _lib._workspace(None) == 0
    with pytest.raises(ValueError, match="workspace"):
        _lib._workspace(torch.empty(64, dtype=torch.uint8))
