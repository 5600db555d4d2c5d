"""How the attention of include/zf_layer.h divides its calls, read from the
workspace that it asks for (on the host, before any HIP call)."""
import ctypes

import pytest

zf = pytest.importorskip("paper_2505_12242_amd")
from paper_2505_12242_amd import _lib  # noqa: E402

# pieces that the joining kernel can hold: one a lane
MOST = 64


def pieces(tokens, keys, sequences, heads, kv, dim):
    """Pieces of the keys: each keeps `dim` sums and an lse of every row, in fp32."""
    a = _lib.ZfAttention(tokens, keys, sequences, heads, kv, dim, 1, 0.1, 16, 16, None)
    need = _lib.LIB.zf_attention_forward_workspace_bytes(ctypes.byref(a))
    each = tokens * heads * (dim + 1) * 4
    assert need % each == 0
    return need // each


def sizes():
    for tokens in (1, 2, 3, 5, 8, 9, 17, 64, 69, 128, 129, 500, 1024, 8192):
        for keys in (1, 127, 128, 129, 512, 4096, 16639, 16640, 32768, 131072, 1 << 20, (1 << 27) - 64):
            for sequences in (1, 2, 3, 7, 8, 48, 129, 1024):
                for heads, kv in ((1, 1), (8, 1), (16, 1), (64, 1), (28, 4), (8, 8), (32, 8), (32, 32)):
                    yield tokens, keys, sequences, heads, kv


def test_pieces_fit_the_join():
    """No sizes give more pieces than are joined."""
    many = 0
    for case in sizes():
        for dim in (8, 128):
            n = pieces(*case, dim)
            assert n <= MOST, (case, dim, n)
            many = max(many, n)
    assert many == MOST
