"""One feed-forward block trained with every operator of the library.

    python examples/train_block.py [--steps 120]

A token's embedding goes through an RMS norm, two linear layers with a ReLU
between them, the residual's addition with a second norm, and an output
projection; the task is a fixed random map from tokens to tokens.

  * the norms write the 8-bit operands of the products behind them, and the
    products run forward and backward in 8 bits (matmul_fp8);
  * each product's weight gradient is written straight to a gradient slot of
    SelectiveUpdateRunner, in its channel-major layout; the runner updates the
    linear weights selectively, with the offloaded optimizer;
  * norm gains and the embedding are stepped by one AdamWPlan, the embedding
    with states in 8 bits;
  * the weights are quantised again after every update, both ways at once.

PyTorch computes what lies between (the embedding's lookup and gradient, the
ReLU, the loss).
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2505_12242_amd as zf  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


class Block:
    def __init__(self, vocab=512, dim=256, ffn=1024, lr=2e-3, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)

        def rand(*shape, std):
            return torch.randn(*shape, generator=gen, device=device) * std

        # linear weights, stored channel-major ([in, out]): up, down, head
        self.shapes = [(ffn, dim), (dim, ffn), (vocab, dim)]  # (outputs, inputs)
        self.w = [rand(m, n, std=m ** -0.5).to(BF16) for n, m in self.shapes]
        self.slots = [[torch.zeros(m, n, dtype=BF16, device=device) for n, m in self.shapes]
                      for _ in range(2)]
        hp = zf.AdamHparams(lr=lr)
        self.runner = zf.SelectiveUpdateRunner(self.shapes, 0.25, hp, refresh=4, accum=4,
                                               grad_slots=self.slots, weights=self.w,
                                               device=device, layout=zf.CHANNEL_MAJOR,
                                               offload=True)
        # what is not split by channel: two gains, the embedding
        masters = [torch.ones(dim, device=device), torch.ones(dim, device=device),
                   rand(vocab, dim, std=1.0)]
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

    def step(self, tokens, targets):
        """One training step; the loss (a GPU scalar)."""
        g1, g2, table = self.params
        up, down, head = self.slots[self.steps % 2]
        # forward
        x = table[tokens]
        n1 = zf.rmsnorm(x, g1, want_q=True)
        a = zf.matmul_fp8(n1.q, self.w_fwd[0]).relu_()
        aq, at = zf.quantize_fp8(a, transposed=True)
        n2 = zf.rmsnorm(zf.matmul_fp8(aq, self.w_fwd[1]), g2, residual=x, want_q=True)
        logits = zf.matmul_fp8(n2.q, self.w_fwd[2], dtype=F32)
        logp = torch.log_softmax(logits, 1)
        loss = -logp.gather(1, targets[:, None]).mean()
        # backward
        d = logp.exp_()
        d.scatter_add_(1, targets[:, None], torch.full_like(targets[:, None], -1.0, dtype=F32))
        dq, dt = zf.quantize_fp8(d.div_(len(tokens)), transposed=True)
        _, n2t = zf.quantize_fp8(n2.y, rows=False, transposed=True)
        zf.matmul_fp8(n2t, dt, out=head)
        dh, _ = zf.rmsnorm_backward(zf.matmul_fp8(dq, self.w_bwd[2]), n2.h, g2, n2.rstd,
                                    dgain=self.grads[1])
        dq, dt = zf.quantize_fp8(dh, transposed=True)
        zf.matmul_fp8(at, dt, out=down)
        da = zf.matmul_fp8(dq, self.w_bwd[1]).mul_(a > 0)
        dq, dt = zf.quantize_fp8(da, transposed=True)
        _, n1t = zf.quantize_fp8(n1.y, rows=False, transposed=True)
        zf.matmul_fp8(n1t, dt, out=up)
        dx, _ = zf.rmsnorm_backward(zf.matmul_fp8(dq, self.w_bwd[0]), x, g1, n1.rstd,
                                    dresidual=dh, dgain=self.grads[0])
        self.grads[2].zero_().index_add_(0, tokens, dx.float())
        # update: the linear weights by channel, the rest in one launch, clipped
        self.steps += 1
        self.runner.step()
        norm = torch.stack([g.norm() for g in self.grads]).norm()
        torch.clamp(1.0 / (norm + 1e-6), max=1.0, out=self.clip[0])
        self.plan.step(self.hp, self.steps, grad_scale=self.clip)
        self.quantize_weights()
        return loss

    def close(self):
        self.runner.sync()
        self.runner.close()
        self.plan.close()


def train(steps=120, batch=1000, vocab=512, seed=0, report=0):
    """The losses of `steps` steps."""
    gen = torch.Generator().manual_seed(seed)
    target = torch.randperm(vocab, generator=gen).cuda()
    block = Block(vocab=vocab, seed=seed)
    losses = []
    for i in range(steps):
        tokens = torch.randint(0, vocab, (batch,), generator=gen).cuda()
        losses.append(block.step(tokens, target[tokens]))
        if report and (i + 1) % report == 0:
            print(f"step {i + 1}: loss {losses[-1].item():.3f}", flush=True)
    block.close()
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=120)
    args = ap.parse_args()
    train(args.steps, report=20)
