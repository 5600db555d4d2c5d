"""Calls of attention, layer norm and the linear layer on a stream of their own,
with workspaces given, and captured: two graphs that share one workspace."""
import pytest
import torch

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")

BF16, F32 = torch.bfloat16, torch.float32


def randn(*shape, dtype=BF16, seed=0):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=gen).to(dtype).cuda()


def raw(q):
    return [t.view(torch.uint8) for t in (q.data, q.scale)]


def attention():
    """One token over 3000 keys: pieces joined through a workspace."""
    q, k, v = randn(1, 8, 64), randn(3000, 2, 64, seed=1), randn(3000, 2, 64, seed=2)
    need = zf.attention_workspace_bytes(q, k)
    assert need > 0
    return need, lambda **kw: list(zf.attention(q, k, v, want_lse=True, **kw))


def attention_backward():
    q, k, v = randn(300, 4, 64), randn(300, 2, 64, seed=1), randn(300, 2, 64, seed=2)
    out, lse = zf.attention(q, k, v, want_lse=True)
    do = randn(300, 4, 64, seed=3)
    return (zf.attention_backward_workspace_bytes(q, k),
            lambda **kw: list(zf.attention_backward(do, q, k, v, out, lse, **kw)))


def layernorm_backward():
    dy, h, g = randn(3000, 700), randn(3000, 700, seed=1), randn(700, seed=2)
    y = zf.layernorm(h, g)
    return (zf.layernorm_backward_workspace_bytes(3000, 700),
            lambda **kw: list(zf.layernorm_backward(dy, h, g, y.mean, y.rstd, **kw)))


def linear():
    """40 x 256 x 6000: a reduction split over blocks."""
    a = zf.quantize_fp8(randn(40, 6000))[0]
    b = zf.quantize_fp8(randn(256, 6000, seed=1), 128)[0]
    bias, res = randn(256, seed=2), randn(40, 256, seed=3)

    def call(**kw):
        out = zf.linear_fp8(a, b, bias, "gelu", res, want_z=True, want_q=True, **kw)
        return [out.y, out.z, *raw(out.q)]
    return zf.linear_fp8_workspace_bytes(40, 256, 6000, True), call


def linear_rows():
    """8 rows and an 8-bit output: the products' sums pass through a workspace."""
    a = zf.quantize_fp8(randn(8, 512))[0]
    b = zf.quantize_fp8(randn(1000, 512, seed=1), 128)[0]

    def call(**kw):
        out = zf.linear_fp8(a, b, activation="silu", want_q=True, **kw)
        return [out.y, *raw(out.q)]
    return zf.linear_fp8_workspace_bytes(8, 1000, 512, True), call


def linear_backward():
    dy, z = randn(1000, 520), randn(1000, 520, seed=1)

    def call(**kw):
        out = zf.linear_fp8_backward(dy, z, "gelu_tanh", want_dz=True, **kw)
        return [out.dz, out.dbias, *raw(out.q), *raw(out.qt)]
    return zf.linear_fp8_backward_workspace_bytes(1000, 520), call


CALLS = [attention, attention_backward, layernorm_backward, linear, linear_rows, linear_backward]


def layernorm():
    x, r, g, b = randn(500, 700), randn(500, 700, seed=1), randn(700, seed=2), randn(700, seed=3)

    def call(**kw):
        out = zf.layernorm(x, g, b, r, want_q=True, **kw)
        return [out.y, out.h, out.mean, out.rstd, *raw(out.q)]
    return 0, call


def same(a, b):
    return len(a) == len(b) and all(torch.equal(x, y) for x, y in zip(a, b))


def owner(address):
    """The stream whose block of torch's allocator holds this address."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= address < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not torch's memory")


@pytest.mark.parametrize("make", CALLS + [layernorm], ids=lambda f: f.__name__)
def test_allocations_belong_to_the_calls_stream(make, monkeypatch):
    (_, call), st = make(), torch.cuda.Stream()
    want = call()
    torch.cuda.synchronize()
    real, seen = torch.empty, []

    def empty(*a, **kw):
        t = real(*a, **kw)
        if t.is_cuda and t.numel():
            seen.append(t)
        return t

    monkeypatch.setattr(torch, "empty", empty)
    got = call(stream=st)
    st.synchronize()
    assert seen and all(owner(t.data_ptr()) == st.cuda_stream for t in seen)
    assert same(got, want)


@pytest.mark.parametrize("make", CALLS, ids=lambda f: f.__name__)
def test_workspace_of_the_callers(make):
    """Of exactly the bytes asked for, whatever it holds, nothing behind it written;
    one byte less is refused."""
    need, call = make()
    want = call()
    assert need > 0
    buf = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        assert same(call(workspace=buf[:need]), want)
    assert (buf[need:] == 255).all()
    with pytest.raises(RuntimeError):
        call(workspace=buf[:need - 1])


@pytest.mark.parametrize("make", CALLS, ids=lambda f: f.__name__)
def test_two_graphs_share_a_workspace(make):
    """Replayed in turn on one stream: each call leaves nothing in the workspace that
    another one needs."""
    need, call = make()
    _, other = make()
    want = call()
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graphs, got = [], []
    with torch.cuda.stream(st):
        for f in (call, other):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=st):
                got.append(f(workspace=ws))
            graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for out in got:
            for t in out:
                t.zero_()
        ws.fill_(255)
        torch.cuda.synchronize()
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert same(got[0], want) and same(got[1], want)
        assert same(call(), want)
