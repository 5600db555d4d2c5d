"""The embedding's gradient of examples/train_decoder.py."""
import pytest
import torch

from test_gpu_layer_decoder import example

zf = pytest.importorskip("paper_2505_12242_amd")


@pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def test_rows_are_summed_in_one_order(device):
    """Rows of sizes far apart, whose sums' last bits follow the order of addition: the
    same bits every time, those of adding row after row, and zeros for tokens that do
    not occur."""
    ex = example()
    gen = torch.Generator().manual_seed(7)
    tokens = torch.randint(0, 24, (524,), generator=gen)
    tokens[tokens == 5] = 6
    dx = (torch.randn(524, 256, generator=gen)
          * torch.exp2(torch.randint(-12, 12, (524, 1), generator=gen).float())).bfloat16()
    want = torch.zeros(32, 256)
    for t, row in zip(tokens.tolist(), dx):
        want[t] += row.float()
    for _ in range(20):
        got = ex.embedding_gradient(tokens.to(device), dx.to(device), 32)
        assert torch.equal(got.cpu(), want)
    assert (want[5] == 0).all() and (want[24:] == 0).all()
