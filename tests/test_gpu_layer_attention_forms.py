"""zf_attention_forward and zf_attention_backward against 64 bits, in the forms
that sizes select: many pieces of few rows' keys; blocks of the gradients of k
and v; a prompt among single tokens; keys that are not finite."""
import math

import pytest
import torch

from _attention import F64, forward, seen
from test_gpu_layer_attention import Case, check_backward, check_forward

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")


@pytest.mark.parametrize("lq,heads,kv,keys", [
    (1, 16, 1, 16640), (1, 16, 1, 32768), (1, 16, 1, 131072),
    (2, 8, 1, 16640), (2, 8, 1, 32768),
    (5, 28, 4, 16640), (5, 28, 4, 32768),
    (64, 8, 1, 16640), (64, 8, 1, 131072),
])
def test_few_rows_over_many_keys(lq, heads, kv, keys):
    c = Case([(lq, keys)], heads, kv, 64 if keys > 100000 else 128)
    check_forward(c, *c.run())


@pytest.mark.parametrize("lens", [[(5, 900), (1, 20000)], [(9, 32768), (3, 17)]], ids=str)
@pytest.mark.parametrize("dim", [80, 128])
def test_few_rows_over_a_large_cache(lens, dim):
    """The pieces follow what the cache has room for."""
    c = Case(lens, 16, 1, dim, room=32768)
    check_forward(c, *c.run())


def test_gradients_of_few_rows_over_many_keys():
    c = Case([(3, 16640)], 8, 1, 64)
    got = c.run()
    check_forward(c, *got)
    check_backward(c, *got, zf.attention_backward(c.gdo, c.gq, c.gk, c.gv, *got, c.seq_q, c.seq_k,
                                                  c.causal, c.scale))


RAGGED = [(40, 60), (33, 20), (130, 140), (1, 129), (17, 17)] * 9
# (128 keys a block: (keys / 128 + sequences) * kv blocks, 448 and more)
GRADIENTS = [
    # 1120 blocks: one group of waves
    dict(lens=RAGGED, heads=48, kv=16, dim=128),
    dict(lens=RAGGED, heads=48, kv=16, dim=80),
    dict(lens=RAGGED, heads=32, kv=16, dim=40, layout="heads"),
    dict(lens=RAGGED, heads=32, kv=16, dim=96, causal=False),
    # 576: two groups where causal
    dict(lens=[(150, 200), (260, 260), (70, 190)] * 3, heads=48, kv=24, dim=128),
    dict(lens=[(150, 200), (260, 260), (70, 190)] * 3, heads=48, kv=24, dim=88, layout="wide"),
    # fewer: 32 keys a block, eight waves where walks are long
    dict(lens=[(420, 300), (17, 40)], heads=8, kv=1, dim=128),
    dict(lens=[(420, 300), (17, 40)], heads=8, kv=1, dim=128, causal=False),
    dict(lens=[(420, 300), (17, 40)], heads=8, kv=1, dim=64),
]


@pytest.mark.parametrize("kw", GRADIENTS, ids=lambda kw: f"{len(kw['lens'])}x{kw['heads']}x{kw['dim']}")
def test_gradients_by_form(kw):
    c = Case(**kw)
    got = c.run()
    check_forward(c, *got)
    check_backward(c, *got, zf.attention_backward(c.gdo, c.gq, c.gk, c.gv, *got, c.seq_q, c.seq_k,
                                                  c.causal, c.scale))


@pytest.mark.parametrize("heads,kv,dim,causal", [(2, 2, 128, True), (1, 1, 64, False), (2, 1, 80, True)])
def test_a_prompt_among_single_tokens(heads, kv, dim, causal):
    """Up to 8 rows a sequence on average: a block walks the prompt's rows, 32 at a time."""
    c = Case([(1, 50)] * 31 + [(310 * kv // heads, 600)] + [(1, 7)] * 40, heads, kv, dim, causal)
    check_forward(c, *c.run())


@pytest.mark.parametrize("lens,heads,kv", [([(130, 200), (7, 90)], 4, 2), ([(1, 300), (2, 77)], 2, 1),
                                           ([(40, 1000)], 4, 1)])
@pytest.mark.parametrize("dim", [8, 40, 72, 80, 104, 120, 128])
@pytest.mark.parametrize("value", [-math.inf, math.inf, math.nan])
def test_an_infinite_element_of_a_key(lens, heads, kv, dim, value):
    """In the last unit of 16 bytes, behind which a width's padding begins: a score of
    minus infinity hides the key, others are NaN in the end."""
    for e in (dim - 1, dim - 8):
        c = Case(lens, heads, kv, dim)
        at = lens[0][1] // 2
        c.gk[c.ks[0] + at, 0, e] = value
        out, lse = c.run()
        k = c.k[c.ks[0]:c.ks[1], 0].clone()
        rows = slice(c.qs[0], c.qs[1])
        for h in range(heads // kv):
            mask = seen(*lens[0], True)
            s = c.q[rows, h, e].float() * value
            bad = mask[:, at] & (s != -math.inf)
            mask[:, at] = False
            o, l, tol, ltol = forward(c.q[rows, h], k, c.v[c.ks[0]:c.ks[1], 0], mask, c.scale)
            got, gl = out[rows, h].cpu().to(F64), lse[h, rows].cpu().to(F64)
            assert not torch.isfinite(got[bad]).any() and not torch.isfinite(gl[bad]).any()
            assert ((got - o).abs() <= tol)[~bad].all(), (h, e)
            assert ((gl - l).abs() <= ltol)[~bad].all()


@pytest.mark.parametrize("lens,heads,kv", [([(130, 200)], 4, 2), ([(1, 300)], 2, 1)])
@pytest.mark.parametrize("dim", [72, 128])
def test_scores_of_minus_infinity_alone(lens, heads, kv, dim):
    """A query whose scores all are has zeros, as if it saw no key."""
    c = Case(lens, heads, kv, dim)
    c.gq[..., dim - 1] = 1.0
    c.gk[c.ks[0]:c.ks[1], :, dim - 1] = -math.inf
    out, lse = c.run()
    rows = slice(c.qs[0], c.qs[1])
    assert (out[rows] == 0).all() and (lse[:, rows] == -math.inf).all()
