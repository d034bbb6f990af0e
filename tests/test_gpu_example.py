"""The fine-tuning step of examples/policy_step.py: its gradients against automatic
differentiation of the same chain in 64 bits on the CPU, and that steps lower the loss."""
import math
import os
import sys

import pytest
import torch

import step_reference as R
from gpu_helpers import relerr

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import policy_step  # noqa: E402

# The chain's activations and gradients are rounded to bf16 about ten times on the
# way, 2^-9 each.
TOL = 10 * 2.0 ** -9


def _double(net, ids):
    """(logits, leaves) of the chain in 64 bits."""
    E = net.table.cpu().double().requires_grad_()
    leaves, x = [E], E[ids.cpu().long()]
    for w, (a, b) in zip(net.W, net.AB):
        a, b = a.cpu().double().requires_grad_(), b.cpu().double().requires_grad_()
        leaves += [a, b]
        x = x @ w.cpu().double().T + net.scale * (x @ a.T) @ b.T
    return x @ net.head.cpu().double().T, leaves


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_step_gradients(loss):
    print(f"[case] example step {loss}", file=sys.stderr, flush=True)
    T, V, sequences = 96, 512, 4
    net = policy_step.Chain(T, V, 128, 256, 1, 8)
    ids, targets, w, seq = policy_step.batch(T, V, sequences)
    ref = net.reference(ids, targets, w)
    g = torch.Generator().manual_seed(5)
    old = ref + 0.1 * torch.randn(T, generator=g).cuda()
    adv = torch.randn(T, generator=g).cuda()
    z, leaves = _double(net, ids)
    lp = torch.log_softmax(z, 1)[torch.arange(T), targets.cpu().long()]
    wd, rd = w.cpu().double(), ref.cpu().double()
    if loss == "policy":
        net.policy_step(ids, targets, w, adv, old, ref, kl_coef=0.1)
        ratio, A, d = (lp - old.cpu().double()).exp(), adv.cpu().double(), rd - lp
        # The gradient jumps where the clip sets in, and logp differs by the chain's roundings:
        # a position is clipped here where the chain's own logp says so.
        own = (net.logp.cpu().double() - old.cpu().double()).exp()
        clipped = own.clamp(0.8, 1.2) * A < own * A
        want = (wd * (torch.where(clipped, 0.0, -ratio * A) + 0.1 * (d.exp() - d - 1.0))).sum()
    else:
        margins = torch.empty(sequences // 2, device="cuda")
        net.preference_step(ids, targets, w, ref, seq, margins, beta=0.5)
        x, e = wd * (lp - rd), seq.tolist()
        s = torch.stack([x[a:b].sum() for a, b in zip(e, e[1:])])
        want = -torch.nn.functional.logsigmoid(0.5 * (s[0::2] - s[1::2])).mean()
    want.backward()
    dE = torch.zeros(V, 128, dtype=torch.float64)
    n = int((net.tokens >= 0).sum())
    dE[net.tokens[:n].cpu().long()] = net.rows[:n].cpu().double()
    got = [dE] + [t.cpu().double() for ab in net.dAB for t in ab]
    errs = [relerr(a, b.grad) for a, b in zip(got, leaves)]
    assert max(errs) <= TOL, errs
    norm = math.sqrt(sum(float(t.square().sum()) for t in got))
    net.update(0.5 * norm, 0.0)
    assert abs(float(net.norm[0]) - norm) <= 2.0 ** -20 * norm and abs(float(net.norm[1]) - 0.5) <= 2.0 ** -20


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_steps_lower_the_loss(loss):
    print(f"[case] example run {loss}", file=sys.stderr, flush=True)
    losses = policy_step.run(loss, steps=6, quiet=True)
    assert all(math.isfinite(x) for x in losses) and losses[-1] < losses[0]
