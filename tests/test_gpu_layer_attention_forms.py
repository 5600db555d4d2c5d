"""zf_attention_forward and zf_attention_backward against 64 bits, in the forms
that sizes select: many pieces of few rows' keys."""
import pytest

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
