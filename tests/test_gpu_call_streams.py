"""Calls launched on a stream of their own through `stream=`: what they allocate,
outputs and workspaces, belongs to that stream, so that torch's allocator gives
none of it to another stream while the call's kernels run."""
import pytest
import torch

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")

BF16, F32 = torch.bfloat16, torch.float32


def randn(*shape, dtype=BF16, seed=0):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=gen).to(dtype).cuda()


def split_product():
    """40 x 256 x 6000: a reduction split over blocks, joined through a workspace."""
    a, b = randn(40, 6000), randn(256, 6000, seed=1)
    assert zf.matmul_fp8_workspace_bytes(40, 256, 6000) > 0
    qa, qb = zf.quantize_fp8(a)[0], zf.quantize_fp8(b, 128)[0]
    return lambda st: [zf.matmul_fp8(qa, qb, stream=st), zf.matmul_fp8(qa, qb, dtype=F32, stream=st)]


def norm_backward():
    dy, h, g = randn(3000, 700), randn(3000, 700, seed=1), randn(700, seed=2)
    rstd = h.float().square().mean(1).add(1e-6).rsqrt()
    return lambda st: list(zf.rmsnorm_backward(dy, h, g, rstd, stream=st))


def norm():
    x, r, g = randn(500, 700), randn(500, 700, seed=1), randn(700, seed=2)

    def call(st):
        out = zf.rmsnorm(x, g, r, want_q=True, stream=st)
        return [out.y, out.h, out.rstd, out.q.data.view(torch.uint8), out.q.scale.view(torch.uint8)]
    return call


def quantize():
    x = randn(500, 640)

    def call(st):
        both = zf.quantize_fp8(x, transposed=True, stream=st)
        return [t.view(torch.uint8) for q in both for t in (q.data, q.scale)]
    return call


def adamw():
    g = randn(5000, dtype=F32, seed=1)
    hp = zf.AdamHparams(lr=1e-3)

    def call(st):
        with torch.cuda.stream(st):
            b = zf.AdamWBuffers.fresh(g, randn(5000, dtype=F32), bits=8)
        plan = zf.AdamWPlan([b], stream=st)
        plan.step(hp, 1, stream=st)
        plan.close()
        return [b.master, b.exp_avg_scale]
    return call


def selective():
    """Scores, selection and hand-over of the selective update."""
    n, m = 600, 500
    g = randn(n, m)

    def call(st):
        norms = zf.colnorm(g, stream=st)
        sel = zf.topk_select(norms, 0.1, stream=st)
        acc = torch.zeros(n, m - sel.k, device="cuda")
        torch.cuda.synchronize()
        zf.pack_accumulate(g, sel, acc, 1, 2, stream=st)
        return [norms, sel.sel_idx, sel.mask, zf.unpack(acc, sel, stream=st)]
    return call


CALLS = [split_product, norm_backward, norm, quantize, adamw, selective]


def owner(address):
    """The stream whose block of torch's allocator holds this address."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= address < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not torch's memory")


@pytest.mark.parametrize("make", CALLS, ids=lambda f: f.__name__)
def test_allocations_belong_to_the_calls_stream(make, monkeypatch):
    call, st = make(), torch.cuda.Stream()
    want = call(torch.cuda.current_stream())
    torch.cuda.synchronize()
    real, seen = torch.empty, []

    def empty(*a, **kw):
        t = real(*a, **kw)
        if t.is_cuda and t.numel():
            seen.append(t)
        return t

    monkeypatch.setattr(torch, "empty", empty)
    got = call(st)
    st.synchronize()
    assert seen and all(owner(t.data_ptr()) == st.cuda_stream for t in seen)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("make", [split_product, norm_backward], ids=lambda f: f.__name__)
def test_current_stream_keeps_its_own_memory(make):
    """The current stream allocates and fills memory while a busy stream still has
    the call in front of it: neither the workspace nor the outputs are among it."""
    call, st = make(), torch.cuda.Stream()
    want = call(torch.cuda.current_stream())
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(st):
            torch.cuda._sleep(20_000_000)
        got = call(st)
        for size in (1 << 12, 1 << 16, 1 << 18, 1 << 20, 1 << 22):
            for _ in range(4):
                torch.full((size,), float("nan"), device="cuda")
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
