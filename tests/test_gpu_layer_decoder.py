"""Layer norm, linear layers, attention and their gradients together, as a
training program runs them."""
import importlib.util
import os

import pytest
import torch

from tests.conftest import ROOT

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")


def example():
    spec = importlib.util.spec_from_file_location(
        "train_decoder", os.path.join(ROOT, "examples", "train_decoder.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_training_runs():
    """Finite losses, the first about ln(64) plus what the head's start adds (its
    logits are of order one: half their variance); the same from the same seed."""
    ex = example()
    a, b = ex.train(steps=6), ex.train(steps=6)
    assert a == b and all(x == x and x < 12 for x in a)
    assert 4.0 < a[0] < 6.0, a[0]


def test_gradients_against_autograd():
    """One step's gradients against fp32 autograd of the same network.  A product of
    two 8-bit operands has a relative error (2-norm) of sqrt(2) times an element's
    root mean square rounding, at most 2^-4 / sqrt(3): 5%.  At most 14 products
    lie on a gradient's way (7 forward, 7 back) and their errors are independent:
    below 19%, a cosine above 0.98."""
    ex = example()
    model = ex.Decoder(seed=3)
    tokens, targets, starts = ex.batch(torch.Generator().manual_seed(5))
    w = [t.float().clone().requires_grad_() for t in model.w]
    p = [t.float().clone().requires_grad_() for t in model.params]

    def norm(x, i):
        c = x - x.mean(1, keepdim=True)
        return c * (c.square().mean(1, keepdim=True) + 1e-5).rsqrt() * p[i] + p[i + 1]

    def attention(qkv):
        out, s = [], starts.tolist()
        for a, b in zip(s, s[1:]):
            q, k, v = model.split(qkv[a:b])
            k, v = (t.repeat_interleave(2, 1) for t in (k, v))
            n = b - a
            scores = (q[:, None] * k[None]).sum(3) / 8.0  # [queries, keys, heads]
            hidden = torch.ones(n, n, device="cuda").triu(1).bool()[:, :, None]
            weights = scores.masked_fill(hidden, float("-inf")).softmax(1)
            out.append((weights[..., None] * v[None]).sum(1))
        return torch.cat(out).flatten(1)

    x = p[10][tokens]
    h1 = attention(norm(x, 0) @ w[0] + p[6]) @ w[1] + p[7] + x
    u = torch.nn.functional.gelu(norm(h1, 2) @ w[2] + p[8])
    h2 = u @ w[3] + p[9] + h1
    logits = norm(h2, 4) @ w[4]
    want = torch.nn.functional.cross_entropy(logits, targets, ignore_index=-1)
    want.backward()
    loss = model.step(tokens, targets, starts)
    torch.cuda.synchronize()
    assert abs(loss.item() - want.item()) < 0.05 * want.item()
    pairs = list(zip(model.slots[0], [t.grad for t in w])) + \
        list(zip(model.grads, [t.grad for t in p]))
    for i, (got, ref) in enumerate(pairs):
        got, ref = got.float().flatten(), ref.flatten()
        if i == 5 + 6:  # a key's bias shifts all of a query's scores: its gradient is none
            keep = torch.ones(512, device="cuda", dtype=torch.bool)
            keep[256:384] = False
            got, ref = got[keep], ref[keep]
        c = torch.nn.functional.cosine_similarity(got, ref, 0)
        assert c > 0.98, (i, c)
    model.close()
