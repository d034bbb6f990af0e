"""Token losses where an error of one rounding decides or adds up: margins over many
rows."""
import sys

import pytest
import torch

import step_reference as R

pytestmark = pytest.mark.gpu

import paper_2606_19528_amd as lm  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def _announce(msg):
    print(f"[case] {msg}", file=sys.stderr, flush=True)


def _logp64(z, y, V):
    """log p(y_t) in 64 bits, on the GPU."""
    out = torch.empty(z.shape[0], dtype=R.F64, device="cuda")
    for a in range(0, z.shape[0], 256):
        b = min(z.shape[0], a + 256)
        ls = torch.log_softmax(z[a:b, :V].double(), 1)
        out[a:b] = ls.gather(1, y[a:b, None].long())[:, 0]
    return out


@pytest.mark.parametrize("V,dt", [(32001, F32), (128256, BF16)])
def test_margin_has_no_common_offset(V, dt):
    """A margin over 2400 chosen and 200 rejected positions of a decoder's logits.  What the rows'
    log-probabilities are off by independently averages out: about 1.5 u a row
    (the rounding of some twenty-four joins and of the sums before them, and the exponential's
    own 0.44 u where log s is corrected), six standard deviations allowed.  What they are off
    by alike adds up, and may be 0.2 u a row beside that: the hardware's exponential is 0.06 u
    low in the mean, in the terms and in the factors that bring partial sums to one maximum;
    no other rounding has a direction.  (log2 e rounded to 32 bits alone makes 1.1 u of it.)"""
    _announce(f"margin offset V={V} {dt}")
    n, chosen, beta = 2600, 2400, 0.1
    ld = -(-V // 8) * 8
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (torch.randn(n, ld, generator=g, device="cuda") * 2.5).to(dt)
    y = torch.randint(0, V, (n,), generator=g, dtype=torch.int32, device="cuda")
    lp = _logp64(z, y, V)
    ref = (lp + 0.3 * torch.randn(n, generator=g, device="cuda", dtype=R.F64)).float()
    seq = torch.tensor([0, chosen, n], dtype=torch.int32, device="cuda")
    L, M, got = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty(n, device="cuda")
    lm.preference_loss(z, y, None, ref, seq, L, M, got, beta=beta, vocab=V)
    d = lp - ref.double()
    want = beta * float(d[:chosen].sum() - d[chosen:].sum())
    tol = beta * R.U * (0.2 * (2 * chosen - n) + 6 * 1.5 * n ** 0.5) + 2 * R.U * abs(want)
    assert abs(float(M[0]) - want) <= tol, (float(M[0]) - want, tol)
