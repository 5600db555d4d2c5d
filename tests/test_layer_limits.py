"""Limits that include/zf_layer.h states, at their edges (host-side checks on
addresses that are never dereferenced)."""
import pytest

zf = pytest.importorskip("paper_2505_12242_amd")
from paper_2505_12242_amd import _lib  # noqa: E402
from tests.test_layer_refusals import EINVAL, OK, query, tensor  # noqa: E402

BLOCKS = 1 << 24


def test_adamw_blocks():
    """The sum over the tensors of ceil(n / 1024) is below 2^24."""
    most = (BLOCKS - 1) * 1024
    assert query(tensor(1, n=most))[0] == OK
    assert query(tensor(1, n=most + 1))[0] == EINVAL
    assert query(tensor(1, n=most - 1024), tensor(11, n=1))[0] == OK
    assert query(tensor(1, n=most - 1024), tensor(11, n=1025))[0] == EINVAL
    # 1000 tensors of one element take a block each
    small = [_lib.ZfAdamwTensor(n=1, grad=0x1000 + 64 * i, grad_dtype=0, master=0x1010 + 64 * i,
                                exp_avg=0x1018 + 64 * i, exp_avg_sq=0x1020 + 64 * i)
             for i in range(1000)]
    assert query(tensor(1, n=most - 1000 * 1024), *small)[0] == OK
    assert query(tensor(1, n=most - 999 * 1024), *small)[0] == EINVAL
