"""AdamW over many tensors, bit for bit against the element sequence in numpy
(one fp32 operation at a time; the 8-bit states' codes too), and against 64
bits."""
import numpy as np
import pytest
import torch

from tests import _layer as R

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")

SIZES = [0, 1, 5, 127, 128, 129, 4095, 4096, 4097, 10007]


class Tensor:
    """One parameter on the GPU (at `off` elements into larger buffers filled
    with a guard value) and in numpy."""

    def __init__(self, n, bits, gdt, off, seed, weight=True, values="normal"):
        gen = torch.Generator().manual_seed(seed)
        g = (torch.randn(n, generator=gen) * 1e-2).to(gdt)
        p = torch.randn(n, generator=gen) * 0.02
        m = torch.randn(n, generator=gen) * 1e-3
        v = (torch.randn(n, generator=gen) * 1e-2).square()
        if values == "wide":  # magnitudes over the whole range, zeros among them
            e = torch.randint(-44, 18, (n,), generator=gen)
            g = torch.ldexp(g.float(), e).to(gdt)
            m, v = torch.ldexp(m, e), torch.ldexp(v, 2 * e)
            for t in (g, m, v):
                t[::7] = 0
            if n > 600:
                for t in (g, m, v):
                    t[128:256] = 0
                g[256:384] = 2.0 ** -120
                m[256:384], v[256:384] = 2.0 ** -110, 0
        elif values == "bad":
            g[n // 2] = float("nan")
            g[n // 3] = float("inf")
        self.n, self.bits, self.off = n, bits, off
        self.bufs = []
        if bits == 8:
            (mq, ms), (vq, vs) = R.np_encode(m.numpy(), False), R.np_encode(v.numpy(), True)
            self.m, self.v, self.ms, self.vs = mq, vq, ms, vs
            f8 = torch.float8_e4m3fn
            dm, dv = self.dev(torch.from_numpy(mq), f8), self.dev(torch.from_numpy(vq), f8)
            scales = self.dev(torch.from_numpy(ms)), self.dev(torch.from_numpy(vs))
        else:
            self.m, self.v = m.numpy(), v.numpy()
            dm, dv, scales = self.dev(m), self.dev(v), (None, None)
        self.g, self.p = g.float().numpy(), p.numpy()
        w = self.dev(p.to(torch.bfloat16)) if weight else None
        self.b = zf.AdamWBuffers(self.dev(g), self.dev(p), dm, dv, w, *scales)

    def dev(self, t, view=None):
        size = t.element_size()
        buf = torch.full(((t.numel() + self.off + 16) * size,), 0xA5, dtype=torch.uint8,
                         device="cuda")
        at = self.off * size
        self.bufs.append((buf, at, t.numel() * size))
        out = buf[at:at + t.numel() * size]
        # (a view of an unaligned byte slice is not a tensor of its type: slice after it)
        out = buf.view(t.dtype)[self.off:self.off + t.numel()]
        out.copy_(t)
        return out.view(view) if view is not None else out

    def step(self, hp, step, gs):
        a = (hp.lr, hp.beta1, hp.beta2, hp.eps, hp.weight_decay, step, gs)
        if self.bits == 8:
            m, r = R.np_decode(self.m, self.ms), R.np_decode(self.v, self.vs)
            with np.errstate(all="ignore"):
                self.p, m, v = R.np_adamw(self.g, self.p, m, r * r, *a)
                self.m, self.ms = R.np_encode(m, False)
                self.v, self.vs = R.np_encode(v, True)
        else:
            self.p, self.m, self.v = R.np_adamw(self.g, self.p, self.m, self.v, *a)

    def check(self):
        def same(t, want):
            got = t.detach()
            got = got.view(torch.uint8).cpu().numpy() if want.dtype == np.uint8 else got.cpu().numpy()
            if want.dtype == np.uint8:  # (the sign of a NaN's code is left open)
                got, want = (np.where((x & 0x7F) == 0x7F, 0x7F, x) for x in (got, want))
            assert np.array_equal(got, want, equal_nan=want.dtype != np.uint8), self.n
            if want.dtype != np.uint8:
                zero = want == 0
                assert np.array_equal(np.signbit(got[zero]), np.signbit(want[zero]))

        same(self.b.master, self.p)
        same(self.b.exp_avg, self.m)
        same(self.b.exp_avg_sq, self.v)
        if self.bits == 8:
            same(self.b.exp_avg_scale, self.ms)
            same(self.b.exp_avg_sq_scale, self.vs)
        if self.b.weight is not None:
            want = torch.from_numpy(self.p).to(torch.bfloat16).float().numpy()
            same(self.b.weight.float(), want)
        for buf, at, size in self.bufs:
            rest = torch.cat([buf[:at], buf[at + size:]])
            assert (rest == 0xA5).all(), "written outside"


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gdt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("off", [0, 1, 8])
@pytest.mark.parametrize("wd,gs", [(0.0, None), (0.01, 0.37)])
@pytest.mark.parametrize("values", ["normal", "wide"])
def test_step(bits, gdt, off, wd, gs, values):
    ts = [Tensor(n, bits, gdt, off, 7 * n + bits, weight=n % 2 == 0, values=values) for n in SIZES]
    hp = zf.AdamHparams(lr=1e-3, weight_decay=wd)
    plan = zf.AdamWPlan([t.b for t in ts])
    scale = torch.tensor([gs], device="cuda") if gs is not None else None
    for step in (1, 2, 3, 1000):
        plan.step(hp, step, grad_scale=scale)
        torch.cuda.synchronize()
        for t in ts:
            t.step(hp, step, gs)
            t.check()
    plan.close()


def test_mixed_tensors_and_stream():
    ts = [Tensor(n, b, d, o, n, values="normal") for n, b, d, o in
          [(5000, 8, torch.bfloat16, 0), (3, 32, torch.float32, 1), (0, 8, torch.float32, 0),
           (9000, 32, torch.bfloat16, 8), (129, 8, torch.float32, 3), (1, 8, torch.bfloat16, 0)]]
    hp = zf.AdamHparams(lr=1e-3)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    plan = zf.AdamWPlan([t.b for t in ts], stream=st)
    plan.step(hp, 1, stream=st)
    st.synchronize()
    for t in ts:
        t.step(hp, 1, None)
        t.check()


@pytest.mark.parametrize("bits", [32, 8])
def test_nonfinite_gradients(bits):
    """An infinity or a NaN spoils its element (32 bits) or its 128-element block's
    states (8 bits) and nothing else."""
    t = Tensor(1000, bits, torch.float32, 0, 3, values="bad")
    hp = zf.AdamHparams(lr=1e-3)
    plan = zf.AdamWPlan([t.b])
    plan.step(hp, 1)
    t.step(hp, 1, None)
    t.check()
    plan.step(hp, 2)
    t.step(hp, 2, None)
    t.check()
    bad = torch.isnan(t.b.master).cpu()
    assert bad[500] and int(bad.sum()) == (2 if bits == 32 else 256)


def test_fresh_states_against_64_bits():
    """20 steps from zero states: 32-bit states within rounding of 64 bits, 8-bit
    states within what their codes hold (a code is off by at most 1/16 of a
    value or 2^-10 of the block's largest 448th; the update's direction keeps its
    sign where the first moment is not lost)."""
    gen = torch.Generator().manual_seed(2)
    n, lr = 2000, 1e-3
    p0 = torch.randn(n, generator=gen) * 0.02
    grads = [torch.randn(n, generator=gen) * 1e-2 for _ in range(20)]
    hp = zf.AdamHparams(lr=lr)
    got = {}
    for bits in (32, 8):
        g, p = torch.zeros(n, device="cuda"), p0.cuda()
        plan = zf.AdamWPlan([zf.AdamWBuffers.fresh(g, p, bits=bits)])
        for i, x in enumerate(grads):
            g.copy_(x)
            plan.step(hp, i + 1)
        got[bits] = p.cpu().double()
    p, m, v = p0.double(), 0.0, 0.0
    moved = torch.zeros(n, dtype=torch.float64)
    for i, x in enumerate(grads):
        x = x.double()
        m, v = 0.9 * m + 0.1 * x, 0.999 * v + 0.001 * x * x
        u = (m / (1 - 0.9 ** (i + 1))) / ((v / (1 - 0.999 ** (i + 1))).sqrt() + 1e-8)
        p, moved = p - lr * u, moved + lr * u.abs()
    assert ((got[32] - p).abs() <= 20 * 2.0 ** -23 * (p.abs() + moved)).all()
    # each step's relative error: 1/16 per stored moment and step, most of it forgotten
    rms = ((got[8] - p).square().mean() / moved.square().mean()).sqrt()
    assert rms < 0.1, rms


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("low,high", [(-62, -38), (38, 62)])
def test_second_moments_at_the_ends_of_the_range(bits, low, high):
    """Second moments on both sides of 2^-96 and of 2^100, in the same lanes and
    in lanes of their own, up to where a square leaves fp32's range."""
    t = Tensor(2053, bits, torch.float32, 0, 3, values="normal")
    gen = torch.Generator().manual_seed(low)
    e = torch.randint(low, high, (t.n,), generator=gen)
    e[512:1536] = torch.arange(low, high).repeat_interleave(128)[:1024]
    g = torch.ldexp(1 + torch.rand(t.n, generator=gen), e)
    t.b.grad.copy_(g)
    t.g = g.numpy()
    plan = zf.AdamWPlan([t.b])
    hp = zf.AdamHparams(lr=1e-3)
    for step in (1, 2):
        plan.step(hp, step)
        torch.cuda.synchronize()
        t.step(hp, step, None)
        t.check()
    plan.close()
