"""zf_attention_forward and zf_attention_backward against 64 bits."""
import math

import pytest
import torch

from _attention import F64, H, backward, forward, seen, starts

pytestmark = pytest.mark.gpu

zf = pytest.importorskip("paper_2505_12242_amd")

BF16, F32 = torch.bfloat16, torch.float32


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def stored(x, layout):
    """x [tokens, heads, dim] on the GPU: dense, head by head, or inside rows that
    hold more, whatever is not x's own a NaN."""
    n, h, d = x.shape
    if layout == "heads":
        buf = torch.full((h, n + 3, d), float("nan"), dtype=BF16, device="cuda")
        out = buf[:, 1:n + 1].transpose(0, 1)
    elif layout == "wide":
        buf = torch.full((n + 2, h + 2, d + 8), float("nan"), dtype=BF16, device="cuda")
        out = buf[1:n + 1, 1:h + 1, :d]
    else:
        return x.cuda()
    out.copy_(x)
    return out


class Case:
    """Packed sequences of (queries, keys) lengths, some tokens before and after."""

    def __init__(self, lens, heads=2, kv=1, dim=64, causal=True, scale=None, layout="dense", seed=0,
                 std=1.0, ahead=2, behind=3, room=None):
        gen = torch.Generator().manual_seed(seed)
        self.lens, self.heads, self.kv, self.dim, self.causal = lens, heads, kv, dim, causal
        self.scale = dim ** -0.5 if scale is None else scale
        self.qs = starts([a for a, _ in lens], ahead)
        self.ks = starts([room if room else b for _, b in lens], ahead)
        self.room = room

        def rand(n, h):
            return (torch.randn(n, h, dim, generator=gen) * std).to(BF16)

        tq, tk = self.qs[-1] + behind, self.ks[-1] + behind
        self.q, self.k, self.v, self.do = rand(tq, heads), rand(tk, kv), rand(tk, kv), rand(tq, heads)
        if room:  # what lies behind a sequence's keys is anything
            for (_, lk), at in zip(lens, self.ks):
                self.k[at + lk:at + room] = float("nan")
                self.v[at + lk:at + room] = float("inf")
        for t in (self.q, self.do):
            t[:ahead] = float("nan")
            t[tq - behind:] = float("nan")
        for t in (self.k, self.v):
            t[:ahead] = float("nan")
            t[tk - behind:] = float("inf")
        self.gq, self.gk, self.gv, self.gdo = (stored(t, layout)
                                               for t in (self.q, self.k, self.v, self.do))
        self.seq_q, self.seq_k = ints(self.qs), ints(self.ks)
        self.len_k = ints([b for _, b in lens]) if room else None

    def run(self, **kw):
        return zf.attention(self.gq, self.gk, self.gv, seq_q=self.seq_q, seq_k=self.seq_k,
                            len_k=self.len_k, causal=self.causal, scale=self.scale, want_lse=True,
                            **kw)

    def pieces(self):
        """(head, key head, rows, keys, mask) of every sequence and head."""
        for i, (lq, lk) in enumerate(self.lens):
            rows = slice(self.qs[i], self.qs[i] + lq)
            keys = slice(self.ks[i], self.ks[i] + lk)
            for h in range(self.heads):
                yield h, h // (self.heads // self.kv), rows, keys, seen(lq, lk, self.causal)


def check_forward(c, out, lse):
    out, lse = out.cpu().to(F64), lse.cpu().to(F64)
    for h, g, rows, keys, mask in c.pieces():
        o, l, tol, ltol = forward(c.q[rows, h], c.k[keys, g], c.v[keys, g], mask, c.scale)
        got = out[rows, h]
        assert torch.isfinite(got).all(), (h, rows)
        bad = (got - o).abs() > tol
        assert not bad.any(), (h, rows, ((got - o).abs() / tol).max().item())
        empty = l.isinf()
        assert (lse[h, rows][empty] == -math.inf).all() and (got[empty] == 0).all()
        assert ((lse[h, rows] - l)[~empty].abs() <= ltol[~empty]).all(), (h, rows)


def check_backward(c, out, lse, grads):
    out, lse = out.cpu(), lse.cpu()
    want = [torch.zeros(t.shape, dtype=F64) for t in (c.q, c.k, c.v)]
    tol = [torch.zeros(t.shape, dtype=F64) for t in (c.q, c.k, c.v)]
    inside = [torch.zeros(t.shape[0], dtype=torch.bool) for t in (c.q, c.k, c.v)]
    for h, g, rows, keys, mask in c.pieces():
        d, e = backward(c.q[rows, h], c.k[keys, g], c.v[keys, g], out[rows, h], lse[h, rows],
                        c.do[rows, h], mask, c.scale)
        for i, (at, head) in enumerate(((rows, h), (keys, g), (keys, g))):
            want[i][at, head] += d[i]
            tol[i][at, head] += e[i]
            inside[i][at] = True
    for name, got, w, t, m in zip(("dq", "dk", "dv"), grads, want, tol, inside):
        got = got.cpu().to(F64)[m]
        assert torch.isfinite(got).all(), name
        limit = 1.01 * (t[m] * (1 + H) + H * w[m].abs()) + 1e-37
        assert ((got - w[m]).abs() <= limit).all(), (name, ((got - w[m]).abs() / limit).max().item())


RAGGED = [(33, 33), (64, 64), (1, 1), (0, 0), (65, 129), (7, 7), (130, 130)]
CASES = [
    dict(lens=[(1, 1)], heads=1, dim=8),
    dict(lens=[(5, 3)], heads=2, dim=64),                    # two queries see nothing
    dict(lens=[(0, 7), (7, 0), (3, 3)], heads=4, kv=2, dim=40),
    dict(lens=RAGGED, heads=4, kv=4, dim=128),
    dict(lens=RAGGED, heads=6, kv=2, dim=72, layout="wide"),
    dict(lens=RAGGED, heads=8, kv=1, dim=96, layout="heads"),
    dict(lens=RAGGED, heads=5, kv=1, dim=104, causal=False),
    dict(lens=[(257, 400), (40, 1000)], heads=7, kv=1, dim=128),
    dict(lens=[(127, 128), (128, 127), (129, 129)], heads=1, dim=64),
    dict(lens=[(300, 300)], heads=2, kv=2, dim=64, causal=False, layout="heads"),
    dict(lens=[(1 + i % 5, 1 + i % 7) for i in range(150)], heads=3, kv=3, dim=16),
    dict(lens=[(i % 3, i % 4) for i in range(4200)], heads=1, dim=8, causal=False),
    dict(lens=[(90, 150)], heads=2, dim=128, std=6.0),       # scores of some hundreds
    dict(lens=[(200, 200)], heads=2, dim=64, scale=1e-3),
    dict(lens=[(31, 2000)], heads=4, kv=2, dim=128),
    # gradients by blocks of 32 keys, eight waves each
    dict(lens=[(420, 300)], heads=4, dim=96),
    dict(lens=[(800, 800), (17, 40)], heads=4, kv=1, dim=40),
    # by blocks of 128 keys, one group of waves or two
    dict(lens=[(150, 200), (260, 260), (33, 190)] * 3, heads=32, kv=32, dim=72),
    dict(lens=[(150, 200), (260, 260), (33, 190)] * 3, heads=32, kv=32, dim=128, causal=False),
    dict(lens=[(150, 200), (260, 260), (70, 190)] * 3, heads=40, kv=20, dim=64),
]


@pytest.mark.parametrize("kw", CASES, ids=lambda kw: f"{len(kw['lens'])}x{kw['heads']}x{kw['dim']}")
def test_forward_and_backward(kw):
    c = Case(**kw)
    out = torch.full(c.q.shape, 7.0, dtype=BF16, device="cuda")
    lse = torch.full((c.heads, c.q.shape[0]), 9.0, device="cuda")
    c.run(out=out, lse=lse)
    check_forward(c, out, lse)
    assert (out[:c.qs[0]] == 7).all() and (out[c.qs[-1]:] == 7).all()
    assert (lse[:, :c.qs[0]] == 9).all() and (lse[:, c.qs[-1]:] == 9).all()
    grads = [torch.full(t.shape, 5.0, dtype=BF16, device="cuda") for t in (c.q, c.k, c.v)]
    zf.attention_backward(c.gdo, c.gq, c.gk, c.gv, out, lse, c.seq_q, c.seq_k, c.causal, c.scale,
                          *grads)
    check_backward(c, out, lse, grads)
    for g, at in zip(grads, (c.qs, c.ks, c.ks)):
        assert (g[:at[0]] == 5).all() and (g[at[-1]:] == 5).all()


@pytest.mark.parametrize("heads,kv,dim", [(8, 8, 128), (8, 1, 128), (12, 4, 64), (5, 1, 80), (64, 2, 96)])
@pytest.mark.parametrize("lq", [1, 2, 5])
def test_tokens_over_a_cache(heads, kv, dim, lq):
    lens = [(lq, n) for n in (1, 5, 31, 32, 33, 64, 100, 0, 511, 1024)]
    c = Case(lens, heads, kv, dim, room=1024, layout="wide" if lq == 2 else "dense")
    check_forward(c, *c.run())


@pytest.mark.parametrize("lens", [[(1, 5000)], [(1, 4097), (1, 63), (3, 9000)]], ids=len)
@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 1), (32, 32)])
def test_one_token_over_long_keys(lens, heads, kv):
    c = Case(lens, heads, kv, 128)
    check_forward(c, *c.run())


def test_one_sequence_without_starts():
    c = Case([(77, 77)], 4, 2, 64, ahead=0, behind=0)
    got = zf.attention(c.gq, c.gk, c.gv, want_lse=True)
    check_forward(c, *got)
    check_backward(c, *got, zf.attention_backward(c.gdo, c.gq, c.gk, c.gv, *got))
    assert zf.attention(c.gq, c.gk, c.gv).lse is None


def test_fused_projection_and_gradient_buffer():
    """q, k, v are columns of one buffer, and so are their gradients."""
    c = Case([(70, 70), (50, 50)], 4, 2, 64, ahead=0, behind=0)
    buf = torch.cat([c.q, c.k, c.v], 1).cuda()
    q, k, v = buf.split([4, 2, 2], 1)
    got = zf.attention(q, k, v, c.seq_q, want_lse=True)
    check_forward(c, *got)
    grad = torch.full_like(buf, float("nan"))
    check_backward(c, *got, zf.attention_backward(c.gdo, q, k, v, *got, c.seq_q, None, True, None,
                                                  *grad.split([4, 2, 2], 1)))
    assert torch.isfinite(grad).all()


@pytest.mark.parametrize("starts_q,starts_k", [([-5, 40, 1000], [0, 50, 70]),
                                               ([0, 100, 100], [-9, 2000, 60])])
def test_starts_outside_the_tensors_are_cut_off(starts_q, starts_k):
    c = Case([(100, 70)], 2, 1, 64, ahead=0, behind=0)
    got = zf.attention(c.gq, c.gk, c.gv, ints(starts_q), ints(starts_k), want_lse=True)
    cut_q = [min(max(x, 0), 100) for x in starts_q]
    cut_k = [min(max(x, 0), 70) for x in starts_k]
    want = zf.attention(c.gq, c.gk, c.gv, ints(cut_q), ints(cut_k), want_lse=True)
    assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)


@pytest.mark.parametrize("far", ["tokens", "heads"])
def test_offsets_beyond_32_bits(far):
    """Vectors more than 2^32 bytes apart, of tokens or of heads."""
    c = Case([(130, 260), (1, 30)], heads=2, kv=2 if far == "heads" else 1, ahead=0, behind=0)
    token, head = ((1 << 23) - 64, 64) if far == "tokens" else (64, (1 << 31) + 64)

    def spread(buf, shape, column=0):
        return buf.as_strided((*shape[:2], 64), (token, head, 1), column)

    column = 1024 if far == "tokens" else 64 * 512
    size = (c.k.shape[0] - 1) * token + (c.heads - 1) * head + 4 * column
    bufs = [torch.empty(size, dtype=BF16, device="cuda") for _ in range(5)]
    q, k, v, do = (spread(bufs[0], t.shape, i * column).copy_(t)
                   for i, t in enumerate((c.q, c.k, c.v, c.do)))
    got = zf.attention(q, k, v, c.seq_q, c.seq_k, scale=c.scale, out=spread(bufs[1], q.shape),
                       want_lse=True)
    check_forward(c, got.out, got.lse)
    # (single tokens, by pieces of keys)
    near = [t.contiguous() for t in (q[:1], k, v)]
    assert torch.equal(zf.attention(q[:1], k, v).out, zf.attention(*near).out)
    dq, dk, dv = (spread(b, t.shape) for b, t in zip(bufs[2:], (q, k, v)))
    grads = zf.attention_backward(do, q, k, v, *got, c.seq_q, c.seq_k, scale=c.scale, dq=dq, dk=dk,
                                  dv=dv)
    check_backward(c, *got, grads)


def test_no_tokens():
    q, k = torch.zeros(0, 4, 64, dtype=BF16, device="cuda"), torch.zeros(5, 2, 64, dtype=BF16, device="cuda")
    assert zf.attention(q, k, k, ints([0, 0]), ints([0, 5])).out.shape == (0, 4, 64)
    lse = torch.zeros(4, 0, device="cuda")
    _, dk, dv = zf.attention_backward(q, q, k, k, q, lse, ints([0, 0]), ints([0, 5]))
    assert (dk == 0).all() and (dv == 0).all()
    got = zf.attention(torch.ones(5, 4, 64, dtype=BF16, device="cuda"), k[:0], k[:0], ints([0, 5]),
                       ints([0, 0]), want_lse=True)
    assert (got.out == 0).all() and (got.lse == -math.inf).all()


def test_equal_calls_give_equal_bits():
    c = Case([(500, 500), (300, 700)], 8, 2, 128)
    first = c.run()
    grads = zf.attention_backward(c.gdo, c.gq, c.gk, c.gv, *first, c.seq_q, c.seq_k)
    for _ in range(3):
        again = c.run()
        m = slice(c.qs[0], c.qs[-1])
        assert torch.equal(again.out[m], first.out[m]) and torch.equal(again.lse[:, m], first.lse[:, m])
        g2 = zf.attention_backward(c.gdo, c.gq, c.gk, c.gv, *first, c.seq_q, c.seq_k)
        for a, b, at in zip(grads, g2, (c.qs, c.ks, c.ks)):
            assert torch.equal(a[at[0]:at[-1]], b[at[0]:at[-1]])


def test_differences():
    """The gradients against differences of the 64-bit function."""
    c = Case([(9, 9)], 2, 1, 16, ahead=0, behind=0, std=0.7)
    got = c.run()
    grads = zf.attention_backward(c.gdo, c.gq, c.gk, c.gv, *got, c.seq_q, c.seq_k)

    def loss(q, k, v):
        total = 0.0
        for h, g, rows, keys, mask in c.pieces():
            total += (forward(q[rows, h], k[keys, g], v[keys, g], mask, c.scale)[0]
                      * c.do[rows, h].to(F64)).sum()
        return total

    base = [t.to(F64) for t in (c.q, c.k, c.v)]
    gen = torch.Generator().manual_seed(5)
    for i in range(3):
        for _ in range(4):
            d = torch.randn(base[i].shape, generator=gen, dtype=F64)
            step = 1e-5
            ends = [loss(*[b + sign * step * d if j == i else b for j, b in enumerate(base)])
                    for sign in (1, -1)]
            slope = (ends[0] - ends[1]) / (2 * step)
            g = grads[i].cpu().to(F64)
            # out enters with its rounding to bf16 (D), p and dS with theirs, the
            # gradient with its own: four roundings of what is summed, at most
            assert abs(slope - (g * d).sum()) <= 4 * H * (g * d).abs().sum() * 3


@pytest.mark.parametrize("lens,heads,kv,dim", [([(70, 70), (40, 40)], 2, 2, 64),
                                               ([(200, 260)], 4, 1, 128), ([(5, 9)], 8, 2, 80),
                                               ([(4, 300), (1, 7)], 4, 2, 96)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("which", ["k", "v"])
def test_hidden_keys_reach_nothing(lens, heads, kv, dim, value, which):
    """A key that is not finite changes the queries that see it, and no other."""
    c = Case(lens, heads, kv, dim)
    want = c.run()
    for at in {lens[0][1] - 1, lens[0][1] // 2}:
        d = Case(lens, heads, kv, dim)
        (d.gk if which == "k" else d.gv)[d.ks[0] + at, 0, 3] = value
        got = d.run()
        lq, lk = lens[0]
        mask = seen(lq, lk, True)[:, at].cuda()
        group = heads // kv
        for h in range(heads):
            a, b = got.out[d.qs[0]:d.qs[1], h], want.out[d.qs[0]:d.qs[1], h]
            if h >= group:  # another key head's
                assert torch.equal(a, b)
                continue
            assert torch.equal(a[~mask], b[~mask])
            if which == "k":
                # a score of minus infinity hides the key, others are NaN in the end
                bad = ~torch.isfinite(a[mask]).all(1)
                s = c.q[d.qs[0]:d.qs[1], h, 3].cuda()[mask].float() * value
                assert (bad == (s != -math.inf)).all()
            else:
                assert torch.equal(a[mask][:, :3], b[mask][:, :3])
                x = a[mask][:, 3].float()
                assert x.isnan().all() if value != value else (x == value).all()
        assert torch.equal(got.out[d.qs[1]:d.qs[-1]], want.out[d.qs[1]:d.qs[-1]])


@pytest.mark.parametrize("lens,heads,kv", [([(128, 300)], 2, 2), ([(40, 40)], 4, 1), ([(4, 300)], 2, 1)])
def test_hidden_scores_round_nothing(lens, heads, kv):
    """Keys of large scores, seen by the last queries alone: the others' results keep
    their bits."""
    c, d = Case(lens, heads, kv, 64, behind=0), Case(lens, heads, kv, 64, behind=0)
    lq, lk = lens[0]
    half = lq // 2
    d.gk[d.ks[0] + lk - half:] *= 64.0
    want, got = c.run(), d.run()
    rows = slice(c.qs[0], c.qs[0] + lq - half)
    assert torch.equal(got.out[rows], want.out[rows])
    assert torch.equal(got.lse[:, rows], want.lse[:, rows])
    assert not torch.equal(got.out, want.out)


@pytest.mark.parametrize("lens,heads,kv,dim,causal", [([(90, 70), (5, 131)], 2, 1, 64, False),
                                                      ([(1, 45), (1, 300)], 8, 2, 128, True),
                                                      ([(3, 50)], 4, 1, 96, False)])
@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
def test_an_infinity_that_every_query_sees(lens, heads, kv, dim, causal, value):
    """In the last key's v, whose copies fill its tile: the sum is that infinity, as the
    weight of the key is positive (no score is farther than exp(-60) from another)."""
    c = Case(lens, heads, kv, dim, causal)
    want = c.run()
    for i, (_, lk) in enumerate(lens):
        d = Case(lens, heads, kv, dim, causal)
        d.gv[d.ks[i] + lk - 1, 0, 5] = value
        got = d.run()
        rows = slice(d.qs[i], d.qs[i + 1])
        assert (got.out[rows, :heads // kv, 5] == value).all()
        got.out[rows, :heads // kv, 5] = want.out[rows, :heads // kv, 5]
        m = slice(d.qs[0], d.qs[-1])
        assert torch.equal(got.out[m], want.out[m])


def test_captured_call_follows_the_lengths():
    c = Case([(1, 700), (1, 20), (1, 0)], 8, 2, 128, room=1024)
    stream = torch.cuda.Stream()
    out, lse = torch.zeros_like(c.gq), torch.zeros(8, c.q.shape[0], device="cuda")
    with torch.cuda.stream(stream):
        c.run(out=out, lse=lse)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            c.run(out=out, lse=lse)
    for lens in ([700, 20, 0], [701, 21, 1], [3, 1000, 64], [1024, 1, 512]):
        d = Case([(1, n) for n in lens], 8, 2, 128, room=1024)
        for a, b in ((c.gq, d.gq), (c.gk, d.gk), (c.gv, d.gv), (c.len_k, d.len_k)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        check_forward(d, out, lse)


def test_training_step_captured():
    c = Case([(100, 100), (60, 60)], 4, 2, 64, ahead=0, behind=0)
    want = c.run()
    grads = zf.attention_backward(c.gdo, c.gq, c.gk, c.gv, *want, c.seq_q, c.seq_k)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = c.run()
            g2 = zf.attention_backward(c.gdo, c.gq, c.gk, c.gv, *got, c.seq_q, c.seq_k)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)
        assert all(torch.equal(a, b) for a, b in zip(grads, g2))
        c.run()


def test_calls_on_a_stream_of_their_own():
    c = Case([(1, 4000)], 8, 1, 128)
    want = c.run()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = c.run(stream=st)
    st.synchronize()
    m = slice(c.qs[0], c.qs[-1])
    assert torch.equal(got.out[m], want.out[m])
