"""The operators together, as a training program runs them."""
import importlib.util
import os

import pytest
import torch

from tests.conftest import ROOT

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")


def example():
    spec = importlib.util.spec_from_file_location(
        "train_block", os.path.join(ROOT, "examples", "train_block.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_training_learns_the_map():
    """From about ln(512) = 6.2 plus what the head's start adds, to well below a
    fifth of it; the same losses from the same seed."""
    ex = example()
    losses = ex.train(steps=120)
    assert 5.5 < losses[0] < 8.0, losses[0]
    assert sum(losses[-10:]) / 10 < 0.2 * losses[0], losses[-10:]


def test_gradients_against_autograd():
    """One step's gradients against fp32 autograd of the same network: the 8-bit
    operands' rounding (up to 2^-4 an element, independent errors) leaves the
    directions: cosines above 0.98."""
    ex = example()
    block = ex.Block(seed=3)
    gen = torch.Generator().manual_seed(5)
    tokens = torch.randint(0, 512, (777,), generator=gen).cuda()
    targets = torch.randint(0, 512, (777,), generator=gen).cuda()
    w = [t.float().clone().requires_grad_() for t in block.w]
    p = [t.float().clone().requires_grad_() for t in block.params]

    def norm(x, g):
        return x * (x.square().mean(1, keepdim=True) + 1e-6).rsqrt() * g

    x = p[2][tokens]
    a = (norm(x, p[0]) @ w[0]).relu()
    logits = norm(a @ w[1] + x, p[1]) @ w[2]
    want = torch.nn.functional.cross_entropy(logits, targets)
    want.backward()
    loss = block.step(tokens, targets)
    torch.cuda.synchronize()
    assert abs(loss.item() - want.item()) < 0.05 * want.item()
    pairs = list(zip(block.slots[0], w)) + list(zip(block.grads, p))
    for got, ref in pairs:
        c = torch.nn.functional.cosine_similarity(got.float().flatten(), ref.grad.flatten(), 0)
        assert c > 0.98, c
    block.close()
