"""Token losses where an error of one rounding decides or adds up: margins over many
rows, positions at the edge of the clip."""
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


def _at_the_edge(T, V, dt, sign, seed):
    """A policy loss with clip_lo = clip_hi = 0 right after the rollout: old_logp is the current
    logp rounded to fp32, so every ratio is 1 within a few roundings and the branch of every
    position hangs on them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = (torch.randn(T, V, generator=g, device="cuda") * 2.0).to(dt)
    y = torch.randint(0, V, (T,), generator=g, dtype=torch.int32, device="cuda")
    adv, old = torch.full((T,), sign, device="cuda"), torch.empty(T, device="cuda")
    L, dz = torch.empty(1, device="cuda"), torch.empty_like(z)
    lm.policy_loss(z, y, None, adv, torch.zeros(T, device="cuda"), None, L, old)  # (old: logp)
    lm.policy_loss(z, y, None, adv, old, None, L, torch.empty(T, device="cuda"), dz, clip_lo=0.0, clip_hi=0.0)
    return float(L[0]), dz


# rows in one wave's registers, in a workgroup's, and in parts
@pytest.mark.parametrize("T,V", [(1500, 512), (1500, 2048), (300, 9000), (150, 32768), (60, 128256)])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_gradient_rows_at_the_clips_edge_are_whole(T, V, dt):
    """A position is clipped or it is not: its row of dlogits is zero, or no element of it
    is (c softmax is above 1e-12 everywhere)."""
    _announce(f"clip edge T={T} V={V} {dt}")
    for sign in (1.0, -1.0):
        _, dz = _at_the_edge(T, V, dt, sign, T + V)
        n = (dz != 0).sum(1)
        some = (n != 0) & (n != V)
        assert not some.any(), f"{int(some.sum())} of {T} rows are partly zero"
        assert 0 < int((n == 0).sum()) < T  # both sides occur


def test_loss_and_gradient_take_one_side_of_the_clip():
    """One position, its row in parts: where the gradient is that of a clipped position, the
    loss is that of the bound, exactly -1 times the advantage."""
    _announce("clip edge, loss and gradient")
    clipped = 0
    for seed in range(60):
        for sign in (1.0, -1.0):
            loss, dz = _at_the_edge(1, 65536, F32, sign, seed)
            if not dz.any():
                clipped += 1
                assert loss == -sign, (seed, sign, loss)
    assert clipped


def _along(f, z, X, h):
    """(central difference of f along X, bound of its truncation): the third derivative from
    the five points of f in 64 bits, twice for what it changes in between."""
    v = [float(f(z + k * h * X)) for k in (-2, -1, 1, 2)]
    return (v[2] - v[1]) / (2 * h), 2 * h * h / 6 * abs(v[3] - 2 * v[2] + 2 * v[1] - v[0]) / (2 * h ** 3)


@pytest.mark.parametrize("which", ["policy", "preference"])
def test_kernel_gradients_along_themselves(which):
    """The kernels' gradients against central differences of the kernels' own losses, in
    the gradient's direction, where the derivative is its norm.  A loss in 32 bits is off
    by its positions' c times what their log-probabilities are off by, and its rounding;
    what is allowed in all has to be under 3 % of the derivative."""
    _announce(f"{which} gradient along itself")
    T, V, h, kl, beta, eps = 24, 64, 1.0 / 32, 0.2, 0.8, 0.1
    g = torch.Generator().manual_seed(8)
    z = torch.randn(T, V, generator=g) * 2.0
    y = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    w = (0.5 + torch.rand(T, generator=g)) / (T if which == "policy" else 1.0)
    lp = R.logp(z, y, V)[0]
    # ratios well inside the clip's edges or well beyond them, so that none is crossed
    lr = torch.tensor([0.05, -0.05, 0.7, -0.7], dtype=R.F64)[torch.arange(T) % 4]
    old, ref = (lp - lr).float(), (lp + 0.3 * torch.randn(T, generator=g, dtype=R.F64)).float()
    adv = torch.randn(T, generator=g)
    seq = [0, 7, 12, 20, 24]
    cu = [t.cuda() for t in (y, w, adv, old, ref, torch.tensor(seq, dtype=torch.int32))]

    def kernel(zz):
        zz = zz.float().cuda()
        L, M, o, dz = (torch.empty(1, device="cuda"), torch.empty(2, device="cuda"), torch.empty(T, device="cuda"),
                       torch.empty(T, V, device="cuda"))
        if which == "policy":
            lm.policy_loss(zz, cu[0], cu[1], cu[2], cu[3], cu[4], L, o, dz, clip_lo=0.2, clip_hi=0.3, kl_coef=kl)
        else:
            lm.preference_loss(zz, cu[0], cu[1], cu[4], cu[5], L, M, o, dz, beta=beta, label_smoothing=eps)
        return float(L[0]), dz.cpu().double()

    def exact(zz):
        if which == "policy":
            out = R.policy(zz, y, V, w, adv, old, ref, 0.2, 0.3, kl)
            return out[0], out[2]
        out = R.preference(zz, y, V, w, ref, seq, beta, eps)
        return out[0], out[3]

    loss, dz = kernel(z)
    norm = float(dz.norm())
    # the points are fp32 values, so that both see the same ones
    X = (dz / norm).float().double()
    step = torch.stack([(z.double() + k * h * X).float().double() for k in (-1, 1)])
    want = float((dz * (step[1] - step[0])).sum()) / (2 * h)
    diff = (kernel(step[1])[0] - kernel(step[0])[0]) / (2 * h)
    _, cut = _along(lambda p: exact(p)[0], z.double(), X, h)
    off = float(exact(z.double())[1].abs().sum()) * (float(R.logp_bound(z, y, V).max()) + 16 * R.U) + 4 * R.U * (1 + abs(loss))
    tol = off / h + cut + 16 * R.U * norm
    assert abs(want - norm) <= 1e-4 * norm
    assert tol <= 0.03 * norm, (tol, norm)
    assert abs(diff - want) <= tol, (diff, want, tol)


@pytest.mark.parametrize("seq,falls", [([0, 10, 20, 12, 30], [1]), ([5, 3, 9], [0]), ([0, 3, 10, 4, 6, 8, 12], [1]),
                                       ([0, 10, 8, 20, 31], [0])])
@pytest.mark.parametrize("T,V", [(40, 64), (40, 128256)])
def test_offsets_that_are_not_ascending(T, V, seq, falls):
    """Two pairs may then hold the same rows: NaN in the loss and every row of the gradient,
    instead of what the one that comes last leaves.  The next call is not touched by it."""
    _announce(f"falling offsets {seq} V={V}")
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.randn(T, V, generator=g, device="cuda")
    y = torch.randint(0, V, (T,), generator=g, dtype=torch.int32, device="cuda")
    P = len(seq) // 2
    ws = torch.empty(lm.token_loss_workspace_bytes(lm.TOKEN_LOSS_OP_PREFERENCE, T, V, V, P, lm.LORA_F32), dtype=torch.uint8,
                     device="cuda")
    L, M, lp, dz = (torch.empty(1, device="cuda"), torch.empty(P, device="cuda"), torch.empty(T, device="cuda"),
                    torch.empty(T, V, device="cuda"))

    def call(offsets):
        lm.preference_loss(z, y, None, None, torch.tensor(offsets, dtype=torch.int32, device="cuda"), L, M, lp, dz, ws=ws)
        return [t.clone() for t in (L, M, lp, dz)]

    good = call(sorted(seq))
    bad = call(seq)
    assert torch.isnan(bad[0]).all() and torch.isnan(bad[3]).all()
    assert torch.isnan(bad[1]).nonzero()[:, 0].tolist() == falls
    assert torch.equal(bad[2], good[2])
    assert all(torch.equal(a, b) for a, b in zip(call(sorted(seq)), good)) and torch.isfinite(good[3]).all()
