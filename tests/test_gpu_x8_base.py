"""The LoRA backward from 8 bits at the edges of its values: dx over a quantized base against W = s q + b as it is defined,
and gradients that are not finite."""
import pytest
import torch

import block_reference as ref
from test_gpu_x8 import case, check, run
from workloads import quant_weight

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,group", [(4, 128), (8, 128), (4, 16), (8, 64)])
@pytest.mark.parametrize("T,K,N,r", [(1, 128, 264, 8), (5, 256, 1032, 16), (203, 512, 1032, 16), (1030, 1024, 264, 33)])
def test_dx_over_a_quantized_base(T, K, N, r, bits, group):
    """The product takes W rounded to bf16, by at most 2^-8 of it (and two fp32 roundings of s q and s q + b before), so
    dx is off by |dy| times these in each element, and by the spectral norm of dy times the Frobenius norm of 2^-8 W in all,
    beside what a 32-bit evaluation is off by."""
    s = -0.5
    inp, d, x8, xq, W, _ = case(T, K, N, r, bits, group)
    Wq = quant_weight(N, K, bits, group, seed=1)  # (what `case` made)
    q = Wq["codes"]
    if bits == 4:
        q = torch.stack([q & 15, q >> 4], 2).view(N, K)
    sq, b = q.double() * Wq["scale"].double().T.repeat_interleave(group, 1), Wq["offset"].double().T.repeat_interleave(group, 1)
    u = (xq @ inp["A"].double().T).float()
    dx = run(d, x8, W, u.cuda(), s)[0].cpu().double()
    want = ref.linear_bwd(xq, sq + b, inp["A"], inp["B"], u, inp["dy"], s)[0]
    err = ref.linear_bwd_bounds(xq, sq + b, inp["A"], inp["B"], u, inp["dy"], s)[0]
    dy = inp["dy"].double()
    off = 2.0 ** -8 * (1 + 2.0 ** -22) * (sq + b).abs() + 2.0 ** -23 * (sq.abs() + b.abs())
    own = err + 2.0 ** -8 * (want.abs() + err + dy.abs() @ off)  # a 32-bit evaluation, and the output's rounding
    assert bool(((dx - want).abs() <= dy.abs() @ off + own).all())
    whole = torch.linalg.matrix_norm(dy, 2) * off.norm() + (err + 2.0 ** -8 * (dx.abs() + err)).norm()
    assert float((dx - want).norm()) <= float(whole)


@pytest.mark.parametrize("T,K,N,r", [(24, 264, 256, 8), (300, 520, 264, 32), (600, 264, 520, 33)])
def test_a_gradient_that_is_not_finite(T, K, N, r):
    """One infinite value of dy, in a token and a column of the output: dx of that token, all of dA and that column's row of
    dB are not finite; the rest is what it is without the value."""
    inp, d, x8, xq, W, wide = case(T, K, N, r)
    u = (xq @ inp["A"].double().T).float()
    d["dy"][3, 5] = torch.inf
    dx, dA, dB = run(d, x8, W, u.cuda(), 1.0)
    assert not bool(dx[3].isfinite().any()) and not bool(dA.isfinite().any()) and not bool(dB[5].isfinite().any())
    inp["dy"][3, 5] = 0.0
    want = ref.linear_bwd(xq, wide, inp["A"], inp["B"], u, inp["dy"], 1.0)
    err = ref.linear_bwd_bounds(xq, wide, inp["A"], inp["B"], u, inp["dy"], 1.0)
    rows, cols = torch.arange(T) != 3, torch.arange(N) != 5
    ref.check(dx.cpu()[rows], want[0][rows], err[0][rows], "dx")
    ref.check(dB.cpu()[cols], want[2][cols], err[2][cols], "dB")
    d["dy"][3, 5] = 0.0
    check(run(d, x8, W, u.cuda(), 1.0), inp, xq, wide, u, 1.0)
