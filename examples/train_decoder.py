"""A decoder block trained on packed sequences of different lengths.

    python examples/train_decoder.py [--steps 120]

Layer norm, the projection to queries, keys and values, causal attention (two
query heads to a key head), the output projection with the residual's addition,
a second norm, a feed-forward pair with GELU, and an output projection behind a
third norm; the task is to name the token three places back, which only
attention can do.

  * the norms write the 8-bit operands of the products behind them; the
    products add bias, activation and residual and write the next operand
    (linear_fp8); what their gradients read is one pass (linear_fp8_backward);
  * attention reads the projection's columns where they are, and its gradients
    are written into columns of one buffer;
  * each weight gradient is written straight to a gradient slot of
    SelectiveUpdateRunner, in its channel-major layout;
  * norms, biases and the embedding are stepped by one AdamWPlan.

PyTorch computes what lies between (the embedding's lookup and gradient, the
loss).
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2505_12242_amd as zf  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
QKV, OUT, UP, DOWN, HEAD = range(5)


def embedding_gradient(tokens, dx, vocab):
    """[vocab, dim] in fp32: the rows of dx summed by token, in their order (index_add_'s
    atomics would add them in another order on every run)."""
    order = tokens.argsort(stable=True)
    starts = torch.searchsorted(tokens[order], torch.arange(vocab + 1, device=tokens.device))
    return torch.segment_reduce(dx[order].float(), "sum", offsets=starts, initial=0)


class Decoder:
    def __init__(self, vocab=64, dim=256, heads=4, kv=2, width=64, ffn=512, lr=2e-3, seed=0,
                 device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)

        def rand(*shape, std):
            return torch.randn(*shape, generator=gen, device=device) * std

        self.heads, self.kv, self.width = heads, kv, width
        # linear weights, stored channel-major ([in, out])
        self.shapes = [((heads + 2 * kv) * width, dim), (dim, heads * width), (ffn, dim), (dim, ffn),
                       (vocab, dim)]  # (outputs, inputs)
        self.w = [rand(m, n, std=m ** -0.5).to(BF16) for n, m in self.shapes]
        self.slots = [[torch.zeros(m, n, dtype=BF16, device=device) for n, m in self.shapes]
                      for _ in range(2)]
        hp = zf.AdamHparams(lr=lr)
        self.runner = zf.SelectiveUpdateRunner(self.shapes, 0.25, hp, refresh=4, accum=4,
                                               grad_slots=self.slots, weights=self.w,
                                               device=device, layout=zf.CHANNEL_MAJOR,
                                               offload=True)
        # what is not split by channel: three norms (gain, bias), four biases, the embedding
        masters = [torch.ones(dim, device=device) if i % 2 == 0 else torch.zeros(dim, device=device)
                   for i in range(6)]
        masters += [torch.zeros(n, device=device) for n, _ in self.shapes[:HEAD]]
        masters += [rand(vocab, dim, std=1.0)]
        self.params = [p.to(BF16) for p in masters]
        self.grads = [torch.zeros_like(p) for p in masters]
        self.hp = hp
        self.plan = zf.AdamWPlan([
            zf.AdamWBuffers.fresh(g, p, weight=w, bits=8 if p.dim() == 2 else 32)
            for g, p, w in zip(self.grads, masters, self.params)])
        self.clip = torch.ones(1, device=device)
        self.steps = 0
        self.quantize_weights()

    def quantize_weights(self):
        # of the stored [in, out] matrix: its transposed copy is the forward
        # product's operand [out, in], itself the backward product's
        both = [zf.quantize_fp8(w, group=128, transposed=True) for w in self.w]
        self.w_bwd, self.w_fwd = zip(*both)

    def split(self, qkv):
        return qkv.view(len(qkv), -1, self.width).split([self.heads, self.kv, self.kv], 1)

    def step(self, tokens, targets, starts):
        """One training step over packed sequences (starts: int32, each one's first
        token and the end); targets below 0 do not count.  The loss (a GPU
        scalar)."""
        norms, biases, table = self.params[:6], self.params[6:10], self.params[10]
        dnorms, dbiases = self.grads[:6], self.grads[6:10]
        slot = self.slots[self.steps % 2]
        w, wt = self.w_fwd, self.w_bwd
        # forward
        x = table[tokens]
        n1 = zf.layernorm(x, norms[0], norms[1], want_q=True)
        qkv = zf.linear_fp8(n1.q, w[QKV], biases[QKV]).y
        q, k, v = self.split(qkv)
        att = zf.attention(q, k, v, starts, want_lse=True)
        aq, at = zf.quantize_fp8(att.out.flatten(1), transposed=True)
        h1 = zf.linear_fp8(aq, w[OUT], biases[OUT], residual=x).y
        n2 = zf.layernorm(h1, norms[2], norms[3], want_q=True)
        u = zf.linear_fp8(n2.q, w[UP], biases[UP], "gelu", want_z=True, want_q=True)
        h2 = zf.linear_fp8(u.q, w[DOWN], biases[DOWN], residual=h1).y
        n3 = zf.layernorm(h2, norms[4], norms[5], want_q=True)
        logits = zf.matmul_fp8(n3.q, w[HEAD], dtype=F32)
        count = (targets >= 0).sum()
        logp = torch.log_softmax(logits, 1)
        at_target = targets.clamp(min=0)[:, None]
        loss = -(logp.gather(1, at_target)[:, 0] * (targets >= 0)).sum() / count
        # backward
        d = logp.exp_()
        d.scatter_add_(1, at_target, torch.full_like(at_target, -1.0, dtype=F32))
        d.mul_((targets >= 0)[:, None]).div_(count)

        def weight(i, xt, dt):  # a linear weight's gradient, [in, out]
            zf.matmul_fp8(xt, dt, out=slot[i])

        def columns(y):
            return zf.quantize_fp8(y, rows=False, transposed=True)[1]

        g = zf.linear_fp8_backward(d, want_dbias=False)
        weight(HEAD, columns(n3.y), g.qt)
        dh2, _, _ = zf.layernorm_backward(zf.matmul_fp8(g.q, wt[HEAD]), h2, norms[4], n3.mean, n3.rstd,
                                          dgain=dnorms[4], dbias=dnorms[5])
        g = zf.linear_fp8_backward(dh2, dbias=dbiases[DOWN])
        weight(DOWN, columns(u.y), g.qt)
        g = zf.linear_fp8_backward(zf.matmul_fp8(g.q, wt[DOWN]), u.z, "gelu", dbias=dbiases[UP])
        weight(UP, columns(n2.y), g.qt)
        dh1, _, _ = zf.layernorm_backward(zf.matmul_fp8(g.q, wt[UP]), h1, norms[2], n2.mean, n2.rstd,
                                          dresidual=dh2, dgain=dnorms[2], dbias=dnorms[3])
        g = zf.linear_fp8_backward(dh1, dbias=dbiases[OUT])
        weight(OUT, at, g.qt)
        dout = zf.matmul_fp8(g.q, wt[OUT]).view_as(att.out)
        dqkv = torch.empty_like(qkv)
        dq, dk, dv = self.split(dqkv)
        zf.attention_backward(dout, q, k, v, att.out, att.lse, starts, dq=dq, dk=dk, dv=dv)
        g = zf.linear_fp8_backward(dqkv, dbias=dbiases[QKV])
        weight(QKV, columns(n1.y), g.qt)
        dx, _, _ = zf.layernorm_backward(zf.matmul_fp8(g.q, wt[QKV]), x, norms[0], n1.mean, n1.rstd,
                                         dresidual=dh1, dgain=dnorms[0], dbias=dnorms[1])
        self.grads[10].copy_(embedding_gradient(tokens, dx, len(table)))
        # update: the linear weights by channel, the rest in one launch, clipped
        self.steps += 1
        self.runner.step()
        norm = torch.stack([t.norm() for t in self.grads]).norm()
        torch.clamp(1.0 / (norm + 1e-6), max=1.0, out=self.clip[0])
        self.plan.step(self.hp, self.steps, grad_scale=self.clip)
        self.quantize_weights()
        return loss

    def close(self):
        self.runner.sync()
        self.runner.close()
        self.plan.close()


def batch(gen, vocab=64, lengths=(200, 37, 130, 1, 96, 60)):
    """Packed sequences; the target of a token is the one three places back in its
    own sequence, or -1 where there is none."""
    tokens, targets, starts = [], [], [0]
    for n in lengths:
        t = torch.randint(0, vocab, (n,), generator=gen)
        tokens.append(t)
        targets.append(torch.cat([torch.full((min(n, 3),), -1), t[:max(n - 3, 0)]]))
        starts.append(starts[-1] + n)
    return (torch.cat(tokens).cuda(), torch.cat(targets).cuda(),
            torch.tensor(starts, dtype=torch.int32, device="cuda"))


def train(steps=120, seed=0, report=0):
    """The losses of `steps` steps."""
    gen = torch.Generator().manual_seed(seed)
    model = Decoder(seed=seed)
    losses = []
    for i in range(steps):
        losses.append(model.step(*batch(gen)))
        if report and (i + 1) % report == 0:
            print(f"step {i + 1}: loss {losses[-1].item():.3f}", flush=True)
    model.close()
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=120)
    args = ap.parse_args()
    train(args.steps, report=20)
