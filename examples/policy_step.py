"""Fine-tuning steps from token ids to clipped gradients with this package's
entry points: embedding lookup, a chain of LoRA linears, the frozen head's
logits, a policy loss (or a preference loss), the way back, and one global norm
over the adapters' and the embedding's gradients.

    python examples/policy_step.py                       # a small chain, 20 steps
    python examples/policy_step.py --loss preference
    python examples/policy_step.py --tokens 4096 --vocab 128256 --width 3072 --hidden 8192 --rank 32 --steps 5

The ids are random and the weights untrained; what a step does with them is
what it does in a fine-tuning run.  The update is plain gradient descent.
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_19528_amd as lm  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


class Chain:
    """Embedding [V, D], LoRA linears D -> hidden -> D, ..., a frozen head [V, D], and
    every buffer that a step over T tokens uses."""

    def __init__(self, T, V, D, hidden, pairs, r, seed=0, alpha=16.0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def randn(*shape, std):
            return (torch.randn(*shape, generator=g, device="cuda") * std).to(BF16)

        def new(*shape, dtype=BF16):
            return torch.empty(*shape, dtype=dtype, device="cuda")

        self.T, self.V, self.D, self.scale = T, V, D, alpha / r
        self.table, self.head = randn(V, D, std=1.0), randn(V, D, std=1.0 / math.sqrt(D))
        dims = [D, hidden] * pairs + [D]
        self.W = [randn(o, i, std=1.0 / math.sqrt(i)) for i, o in zip(dims, dims[1:])]
        # fp32 masters of the trained A and B, and the bf16 copies that the kernels read
        self.masters = [(torch.randn(r, w.shape[1], generator=g, device="cuda") / math.sqrt(w.shape[1]),
                         torch.randn(w.shape[0], r, generator=g, device="cuda") * 0.02) for w in self.W]
        self.AB = [(a.to(BF16), b.to(BF16)) for a, b in self.masters]
        self.x = [new(T, d) for d in dims]
        self.dx = [new(T, d) for d in dims]
        self.u = [new(T, r, dtype=F32) for _ in self.W]
        self.dAB = [(torch.empty_like(a), torch.empty_like(b)) for a, b in self.masters]
        self.logits = new(T, V)
        n = min(T, V)
        self.tokens, self.rows = new(n, dtype=torch.int32), new(n, D, dtype=F32)
        # all gradients of a step, clipped in place
        self.grads = lm.grad_list([t for ab in self.dAB for t in ab] + [self.rows])
        self.norm, self.logp, self.loss = new(2, dtype=F32), new(T, dtype=F32), new(1, dtype=F32)

    def forward(self, ids):
        lm.embed_fwd(self.table, ids, self.x[0])
        for i, (w, (a, b)) in enumerate(zip(self.W, self.AB)):
            lm.lora_linear_fwd(self.x[i], w, a, b, self.x[i + 1], self.u[i], self.scale)
        lm.lora_linear_fwd(self.x[-1], self.head, None, None, self.logits, None, 0.0)
        return self.logits

    def backward(self, ids):
        """From the gradient that the loss left in the logits' place."""
        lm.frozen_linear_bwd_dx(self.logits, self.head, self.dx[-1])
        for i in reversed(range(len(self.W))):
            (a, b), (da, db) = self.AB[i], self.dAB[i]
            lm.lora_linear_bwd(self.x[i], self.W[i], a, b, self.u[i], self.dx[i + 1], self.dx[i], da, db, self.scale)
        lm.embed_bwd_rows(ids, self.dx[0], self.V, self.tokens, self.rows)

    def update(self, max_norm, lr):
        lm.grad_clip(self.grads, max_norm, self.norm)
        for (a, b), (ha, hb), (da, db) in zip(self.masters, self.AB, self.dAB):
            a.sub_(da, alpha=lr)
            b.sub_(db, alpha=lr)
            ha.copy_(a)
            hb.copy_(b)
        # the rows past the distinct tokens are zeros: any row may take them
        self.table.index_add_(0, self.tokens.clamp(min=0), (-lr * self.rows).to(BF16))

    def reference(self, ids, targets, weights):
        """Log-probabilities of the targets under the present weights."""
        out = torch.empty_like(self.logp)
        return lm.token_logp(self.forward(ids), targets, out, weights=weights)

    def policy_step(self, ids, targets, weights, advantages, old, ref, kl_coef=0.05):
        z = self.forward(ids)
        lm.policy_loss(z, targets, weights, advantages, old, ref, self.loss, self.logp, z, kl_coef=kl_coef)
        self.backward(ids)

    def preference_step(self, ids, targets, weights, ref, seq, margins, beta=0.1):
        z = self.forward(ids)
        lm.preference_loss(z, targets, weights, ref, seq, self.loss, margins, self.logp, z, beta=beta)
        self.backward(ids)


def batch(T, V, sequences, prompt=0.25, seed=1):
    """Ids, next-token targets, weights that leave each sequence's prompt out, and the
    sequences' offsets."""
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    targets = torch.roll(ids, -1)
    ends = [round(T * i / sequences) for i in range(sequences + 1)]
    w = torch.zeros(T)
    for lo, hi in zip(ends, ends[1:]):
        w[lo + int((hi - lo) * prompt):hi - 1] = 1.0
    return ids.cuda(), targets.cuda(), w.cuda(), torch.tensor(ends, dtype=torch.int32, device="cuda")


def run(loss="policy", T=512, V=2048, D=256, hidden=512, pairs=2, r=8, steps=20, lr=0.5, max_norm=0.5, sequences=8, quiet=False):
    """The losses of `steps` steps on one batch."""
    net = Chain(T, V, D, hidden, pairs, r)
    ids, targets, w, seq = batch(T, V, sequences)
    ref = net.reference(ids, targets, w)
    margins = torch.empty(sequences // 2, device="cuda")
    adv = torch.ones(T, device="cuda")
    for i in range(1, sequences, 2):  # every other sequence scored badly
        adv[int(seq[i]):int(seq[i + 1])] = -1.0
    share = w / w.sum()
    losses = []
    for step in range(steps):
        torch.cuda.synchronize()
        start = time.perf_counter()
        if loss == "policy":
            net.policy_step(ids, targets, share, adv, ref, ref)
        else:
            net.preference_step(ids, targets, w, ref, seq, margins)
        net.update(max_norm, lr)
        losses.append(float(net.loss))
        if not quiet:
            norm, factor = net.norm.tolist()
            print(f"step {step}: loss {losses[-1]:+.5f}  norm {norm:.4f}  factor {factor:.3f}  "
                  f"{(time.perf_counter() - start) * 1e3:.2f} ms", flush=True)
    return losses


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--loss", choices=["policy", "preference"], default="policy")
    for name, default in (("tokens", 512), ("vocab", 2048), ("width", 256), ("hidden", 512), ("pairs", 2), ("rank", 8), ("steps", 20)):
        p.add_argument("--" + name, type=int, default=default)
    a = p.parse_args()
    run(a.loss, a.tokens, a.vocab, a.width, a.hidden, a.pairs, a.rank, a.steps)
