"""Log-probabilities, policy loss and preference loss with their gradients against
the definitions in 64 bits (step_reference), within bounds of a 32-bit evaluation:
over one position and many, vocabularies of one to more than a workgroup holds,
odd ones in padded rows, masked rows, forbidden tokens, infinities and NaN in
places that are not read."""
import sys

import pytest
import torch

import step_reference as R

pytestmark = pytest.mark.gpu

import paper_2606_19528_amd as lm  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
INF = float("inf")


def _announce(msg):
    print(f"[case] {msg}", file=sys.stderr, flush=True)


# (T, V, ld): few and many rows, short and long rows, both sides of a vector, of a
# workgroup's width and of what a workgroup holds of a row.
SHAPES = [(1, 1, 8), (1, 8, 8), (3, 9, 16), (5, 100, 104), (2, 2047, 2048), (7, 4096, 4104), (33, 1000, 1000),
          (300, 520, 520), (700, 77, 80), (4, 32001, 32008), (260, 8200, 8200), (2, 128256, 128256), (5, 151936, 151936),
          (270, 33000, 33008), (1, 262147, 262152), (520, 65537, 65544), (600, 128256, 128264)]


def _inputs(T, V, ld, dt, seed, live=0.7):
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn(T, ld, generator=g) * 2.5).to(dt)
    z[:, V:] = float("nan")  # columns past the vocabulary are never used
    y = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    w = torch.where(torch.rand(T, generator=g) < live, 0.5 + torch.rand(T, generator=g), 0.0)
    w[T // 2] = 1.0
    dead = w == 0
    y[dead] = -100
    z[dead, 0] = float("nan")
    z[dead, V - 1] = INF
    return g, z, y, w


def _close(got, ref, bound, what):
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: error {float(err[bad].max()):.3e} above its bound, reference up to {float(ref.abs().max()):.3e}"


def _check_dz(dz, c, dc, p, y, ld, dt, V):
    """dz = c (onehot - p): c is off by dc, p relatively by the exponent's rounding
    (its argument is up to 100 units off by u each way) and 2 ulp of exp."""
    ref = R.dlogits(c, p, y, ld)
    logs = p.clamp(min=1e-45).log().abs().clamp(max=104.0)
    rel = (3 * logs + 8) * R.U + (V / 256 + 20) * R.U
    hot = torch.zeros_like(p)
    ok = (y >= 0) & (y < V)
    hot[torch.nonzero(ok)[:, 0], y[ok].long()] = 1.0
    bound = torch.zeros_like(ref)
    bound[:, :V] = dc[:, None] * (p + hot) + c.abs()[:, None] * (p * rel + (p + hot) * 2 * R.U) + 2e-38
    if dt == BF16:
        bound = bound + ref.abs() * 2.0 ** -8
    _close(dz.cpu(), ref, bound, "dlogits")
    assert not dz[:, V:].any()


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_logp(shape, dt):
    T, V, ld = shape
    _announce(f"token_logp T={T} V={V} ld={ld} {dt}")
    _, z, y, w = _inputs(T, V, ld, dt, T + V)
    got = torch.full((T,), 9.0, device="cuda")
    lm.token_logp(z.cuda(), y.cuda(), got, weights=w.cuda(), vocab=V)
    live = w != 0
    ref = R.logp(z[live], y[live], V)[0]
    _close(got.cpu()[live], ref, R.logp_bound(z[live], y[live], V), "logp")
    assert not got.cpu()[~live].any()
    zl, yl = z[live].cuda(), y[live].cuda()
    every = torch.empty(int(live.sum()), device="cuda")
    lm.token_logp(zl, yl, every, vocab=V)  # no weights: every position
    _close(every.cpu(), ref, R.logp_bound(z[live], y[live], V), "logp without weights")


def _policy_inputs(g, z, y, w, V):
    T = z.shape[0]
    live = w != 0
    lp = torch.zeros(T, dtype=R.F64)
    lp[live] = R.logp(z[live], y[live], V)[0]
    lr = 0.3 * torch.randn(T, generator=g, dtype=R.F64)
    for edge in (0.8, 1.3):  # clear of the clip's edges, where the gradient jumps
        d = lr.exp() - edge
        lr = torch.where(d.abs() < 2e-3, (edge + torch.where(d < 0, -2e-3, 2e-3)).log(), lr)
    old, ref, adv = (lp - lr).float(), (lp + 0.3 * torch.randn(T, generator=g, dtype=R.F64)).float(), torch.randn(T, generator=g)
    for t in (old, ref, adv):
        t[~live] = float("nan")
    return adv, old, ref


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("kl", [0.0, 0.25])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_policy(shape, kl, dt):
    T, V, ld = shape
    _announce(f"policy_loss T={T} V={V} ld={ld} kl={kl} {dt}")
    g, z, y, w = _inputs(T, V, ld, dt, 3 * T + V)
    adv, old, ref = _policy_inputs(g, z, y, w, V)
    zc = torch.where((w != 0)[:, None], z.float(), 0.0).to(dt)
    clean = [torch.nan_to_num(t) for t in (adv, old, ref)]
    loss, lp, c, p = R.policy(zc, y, V, w, *clean, 0.2, 0.3, kl)
    dev = [t.cuda() for t in (z, y, w, adv, old, ref)]
    L, got, dz = torch.empty(1, device="cuda"), torch.empty(T, device="cuda"), torch.full_like(dev[0], 3.0)

    def call(zt, out):
        lm.policy_loss(zt, dev[1], dev[2], dev[3], dev[4], dev[5] if kl else None, L, got, out, clip_lo=0.2, clip_hi=0.3,
                       kl_coef=kl, vocab=V)

    call(dev[0], dz)
    dlp = torch.where(w != 0, R.logp_bound(zc, y, V), 0.0)
    _close(got.cpu(), lp, dlp, "logp")
    A, o, r = (t.double() for t in clean)
    ratio, e = (lp - o).exp(), (r - lp).exp()
    # ratio and exp(d) inherit logp's error and round in their argument and value
    drop = dlp + (8 + (lp - o).abs() + o.abs() * 0) * R.U
    dk = dlp + (8 + (r - lp).abs()) * R.U
    wd = w.double()
    dl = wd * (A.abs() * ratio * drop + kl * ((e + 1) * dk + 4 * R.U * (r - lp).abs()) + 4 * R.U * (A.abs() * ratio + kl * e))
    dl = torch.where(w != 0, dl, 0.0).sum() + 2 * R.U * abs(float(loss))
    assert abs(float(L[0]) - float(loss)) <= float(dl), (float(L[0]), float(loss), float(dl))
    dc = torch.where(w != 0, wd * (A.abs() * ratio * (drop + 4 * R.U) + kl * (e * dk + 4 * R.U * e)), 0.0)
    _check_dz(dz, c, dc, p, y, ld, dt, V)
    # the loss alone, and the gradient in the logits' place: the same bits
    first = (L.clone(), got.clone())
    call(dev[0], None)
    assert torch.equal(L, first[0]) and torch.equal(got, first[1])
    z2 = dev[0].clone()
    call(z2, z2)
    assert torch.equal(L, first[0]) and torch.equal(got, first[1]) and torch.equal(z2, dz)


def _seq(T, P):
    ends = [int(round(T * (i + 0.3 * (i % 2)) / (2 * P + 0.3))) for i in range(2 * P)] + [T]
    return ends


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("pairs,eps", [(1, 0.0), (3, 0.1)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_preference(shape, pairs, eps, dt):
    T, V, ld = shape
    _announce(f"preference_loss T={T} V={V} ld={ld} pairs={pairs} {dt}")
    g, z, y, w = _inputs(T, V, ld, dt, 5 * T + V)
    seq = _seq(T, pairs)  # short ones leave sequences empty
    live = w != 0
    zc = torch.where(live[:, None], z.float(), 0.0).to(dt)
    ref = (R.logp(zc, y.clamp(min=0), V)[0] + 0.3 * torch.randn(T, generator=g, dtype=R.F64)).float()
    refn = torch.where(live, ref, torch.nan)
    beta = 0.2
    loss, margins, lp, c, p = R.preference(zc, y, V, w, ref, seq, beta, eps)
    dev = [t.cuda() for t in (z, y, w, refn, torch.tensor(seq, dtype=torch.int32))]
    L, M, got, dz = (torch.empty(1, device="cuda"), torch.empty(pairs, device="cuda"), torch.empty(T, device="cuda"),
                     torch.full_like(dev[0], 3.0))

    def call(zt, out):
        lm.preference_loss(zt, *dev[1:], L, M, got, out, beta=beta, label_smoothing=eps, vocab=V)

    call(dev[0], dz)
    dlp = torch.where(live, R.logp_bound(zc, y, V), 0.0)
    _close(got.cpu(), lp, dlp, "logp")
    wd = w.double()
    dm = torch.stack([beta * (wd * dlp)[seq[2 * i]:seq[2 * i + 2]].sum() for i in range(pairs)]) + 4 * R.U * margins.abs() + 1e-30
    _close(M.cpu(), margins, dm, "margins")
    # loss and c are smooth in the margin with derivatives of at most 1 and 1/4
    assert abs(float(L[0]) - loss) <= float(dm.mean()) + 16 * R.U * (abs(loss) + 1.0)
    dc = torch.zeros(T, dtype=R.F64)
    for i in range(pairs):
        dc[seq[2 * i]:seq[2 * i + 2]] = beta / pairs * (float(dm[i]) + 16 * R.U)
    _check_dz(dz, c, torch.where(live, wd * dc, 0.0), p, y, ld, dt, V)
    first = [t.clone() for t in (L, M, got)]
    call(dev[0], None)
    assert all(torch.equal(a, b) for a, b in zip(first, (L, M, got)))
    z2 = dev[0].clone()
    call(z2, z2)
    assert all(torch.equal(a, b) for a, b in zip(first, (L, M, got))) and torch.equal(z2, dz)


def test_reference_gradients_against_differences():
    """The 64-bit gradients themselves against central differences of the 64-bit losses."""
    g, z, y, w = _inputs(12, 40, 40, F32, 5)
    z = torch.nan_to_num(z, posinf=0.0).double()
    y = y.clamp(min=0)
    adv, old, ref = (torch.nan_to_num(t) for t in _policy_inputs(g, z, y, w, 40))
    seq, h = [0, 5, 7, 9, 12], 1e-6
    X = torch.randn(z.shape, generator=g, dtype=R.F64)

    def both(zz):
        return R.policy(zz, y, 40, w, adv, old, ref, 0.2, 0.3, 0.25), R.preference(zz, y, 40, w, ref, seq, 0.3, 0.1)

    (_, _, c, p), (_, _, _, c2, p2) = both(z)
    up, down = both(z + h * X), both(z - h * X)
    for i, (cc, pp) in enumerate(((c, p), (c2, p2))):
        want = float((R.dlogits(cc, pp, y, 40) * X).sum())
        diff = (float(up[i][0]) - float(down[i][0])) / (2 * h)
        assert abs(diff - want) <= 1e-6 * (1.0 + abs(want))


def test_kernel_gradients_against_differences():
    """Central differences of the kernels' own fp32 losses along a direction, h = 1/64: the
    third-order term is at most h^2 of terms of order one, the losses' rounding 2^-22 / h."""
    _announce("loss gradients against differences")
    T, V, h = 24, 64, 1.0 / 64
    g, z, y, w = _inputs(T, V, V, F32, 8, live=2.0)
    adv, old, ref = _policy_inputs(g, z, y, w, V)
    old = old + 0.02 * adv.sign()  # all ratios free of the clip along the way
    adv = adv.abs() * torch.where((R.logp(z, y, V)[0] - old.double()) > 0, -1.0, 1.0).float()
    X = torch.randn(z.shape, generator=g)
    X[:, :] /= X.norm()
    w = w / T
    seq = torch.tensor([0, 7, 12, 20, 24], dtype=torch.int32).cuda()
    cu = [t.cuda() for t in (y, w, adv, old, ref)]

    def both(zz):
        L, M, lp, dz = (torch.empty(1, device="cuda"), torch.empty(2, device="cuda"), torch.empty(T, device="cuda"),
                        torch.empty(T, V, device="cuda"))
        lm.policy_loss(zz.cuda(), *cu, L, lp, dz, kl_coef=0.2, clip_lo=INF, clip_hi=INF)
        a = float(L[0]), dz.cpu().double()
        lm.preference_loss(zz.cuda(), cu[0], cu[1], cu[4], seq, L, M, lp, dz, beta=0.5)
        return a, (float(L[0]), dz.cpu().double())

    mid, up, down = both(z), both(z + h * X), both(z - h * X)
    for i in range(2):
        want = float((mid[i][1] * X.double()).sum())
        diff = (up[i][0] - down[i][0]) / (2 * h)
        assert abs(diff - want) <= 2.0 ** -21 / h * (1 + abs(mid[i][0])) + h * h, (i, diff, want)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_forbidden_and_lowest_logits(dt):
    """-inf logits are tokens of probability 0; a row of the type's lowest value is uniform;
    a row of only -inf, a NaN, +inf or a target outside the vocabulary gives NaN there
    and nowhere else."""
    _announce(f"special logits {dt}")
    V, low = 1000, torch.finfo(dt).min
    T = 9
    g = torch.Generator().manual_seed(2)
    z = torch.randn(T, V, generator=g).to(dt)
    y = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    z[0, 1::2] = -INF
    y[0] = 4
    z[1] = low
    z[2, : V // 2] = low
    y[2] = V - 1
    z[3] = -INF
    z[4, 17] = float("nan")
    z[5, 3] = INF
    y[6] = V
    y[7] = -1
    w = torch.ones(T)
    adv, old = torch.ones(T), torch.full((T,), -7.0)
    L, lp, dz = torch.empty(1, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, V, dtype=dt, device="cuda")
    lm.policy_loss(z.cuda(), y.cuda(), w.cuda(), adv.cuda(), old.cuda(), None, L, lp, dz, clip_hi=INF)
    lp, dz = lp.cpu(), dz.cpu()
    good = [0, 1, 2, 8]
    _close(lp[good], R.logp(z[good], y[good], V)[0], R.logp_bound(z[good], y[good], V) + 1e-6, "logp")
    assert torch.isfinite(dz[good]).all() and not dz[0, 1::2].any() and not dz[2, : V // 2].any()
    assert torch.isnan(lp[3:8]).all() and torch.isnan(L[0])
    assert all(torch.isnan(dz[t]).any() for t in range(3, 8))
    # the same rows at weight 0 leave no trace
    w[3:8] = 0
    lm.policy_loss(z.cuda(), y.cuda(), w.cuda(), adv.cuda(), old.cuda(), None, L, lp2 := torch.empty(T, device="cuda"),
                   dz2 := torch.empty(T, V, dtype=dt, device="cuda"), clip_hi=INF)
    assert torch.isfinite(L[0]) and not lp2[3:8].any() and not dz2[3:8].any()
    assert torch.equal(lp2.cpu()[good], lp[good]) and torch.equal(dz2.cpu()[good], dz[good])


def test_all_positions_masked():
    _announce("all masked")
    T, V = 20, 304
    z = torch.full((T, V), float("nan"), dtype=BF16, device="cuda")
    y, w, o = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    L, M, lp, dz = torch.ones(1, device="cuda"), torch.ones(2, device="cuda"), torch.ones(T, device="cuda"), torch.ones_like(z)
    lm.policy_loss(z, y, w, o, o, o, L, lp, dz, kl_coef=1.0)
    assert not L.any() and not lp.any() and not dz.any()
    seq = torch.tensor([0, 5, 5, 5, 20], dtype=torch.int32, device="cuda")
    lm.preference_loss(z, y, w, None, seq, L, M, lp, dz)
    assert abs(float(L[0]) - 0.6931472) < 1e-6 and not M.any() and not lp.any() and not dz.any()


def test_positions_outside_the_sequences_and_bad_offsets():
    """Positions that no sequence holds have no gradient; offsets beyond the positions
    are cut to them."""
    _announce("seq offsets")
    T, V = 30, 64
    g, z, y, w = _inputs(T, V, V, F32, 9, live=2.0)
    c = [t.cuda() for t in (z, y, w)]
    L, M, lp, dz = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, V, device="cuda")
    lm.preference_loss(*c, None, torch.tensor([4, 9, 20], dtype=torch.int32, device="cuda"), L, M, lp, dz)
    rows = dz.abs().sum(1).cpu() > 0
    assert rows[4:20].all() and not rows[:4].any() and not rows[20:].any()
    lm.preference_loss(*c, None, torch.tensor([-5, 9, 2000000000], dtype=torch.int32, device="cuda"), L, M, lp, dz)
    a = dz.clone()
    lm.preference_loss(*c, None, torch.tensor([0, 9, T], dtype=torch.int32, device="cuda"), L, M, lp, dz)
    assert torch.equal(a, dz)


def test_large_margins_stay_finite():
    _announce("large margins")
    T, V = 16, 128
    g, z, y, w = _inputs(T, V, V, F32, 4, live=2.0)
    c = [t.cuda() for t in (z, y, w)]
    seq = torch.tensor([0, 8, 16], dtype=torch.int32, device="cuda")
    L, M, lp, dz = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, V, device="cuda")
    for sign in (1.0, -1.0):
        ref = torch.zeros(T)
        ref[:8] = sign * 1e4
        lm.preference_loss(*c, ref.cuda(), seq, L, M, lp, dz, beta=10.0)
        assert torch.isfinite(L[0]) and torch.isfinite(dz).all()
        assert abs(float(L[0]) - max(0.0, -float(M[0]))) <= 1e-3


def test_offsets_beyond_32_bits():
    """Logits of 2^31 elements and more: the last rows are found and written."""
    _announce("more than 2^31 logits")
    T, V = 8200, 262152
    assert T * V > 2 ** 31
    z = torch.zeros(T, V, dtype=BF16, device="cuda")
    g = torch.Generator().manual_seed(1)
    rows = [0, 1, T - 2, T - 1]
    part = torch.randn(4, V, generator=g).to(BF16)
    z[rows] = part.cuda()
    y = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    w = torch.zeros(T)
    w[rows] = 0.25
    adv, old = torch.ones(T), torch.full((T,), -13.0)
    L, lp = torch.empty(1, device="cuda"), torch.empty(T, device="cuda")
    lm.policy_loss(z, y.cuda(), w.cuda(), adv.cuda(), old.cuda(), None, L, lp, z, clip_hi=INF)
    lpr, p = R.logp(part, y[rows], V)
    _close(lp.cpu()[rows], lpr, R.logp_bound(part, y[rows], V), "logp")
    c = -0.25 * (lpr + 13.0).exp()
    ref = R.dlogits(c, p, y[rows], V)
    err = (z[rows].cpu().double() - ref).abs()
    assert (err <= 2.0 ** -7 * ref.abs() + 1e-9 * c.abs()[:, None]).all()
    assert not z[2:T - 2].any()


def test_graph_replays_and_other_stream():
    """A captured step replays on changed inputs; a call on another stream with a
    workspace of its own."""
    _announce("loss graph")
    T, V = 64, 2000
    g, z, y, w = _inputs(T, V, V, BF16, 12, live=2.0)
    c = [t.cuda() for t in (z, y, w, torch.randn(T, generator=g), torch.full((T,), -8.0))]
    L, lp, dz = torch.empty(1, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(c[0])
    ws = torch.empty(lm.token_loss_workspace_bytes(lm.TOKEN_LOSS_OP_POLICY, T, V, V), dtype=torch.uint8, device="cuda")

    def call(stream=None):
        lm.policy_loss(*c, None, L, lp, dz, ws=ws, stream=stream)

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    call(st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(4):
        c[0].copy_(torch.randn(T, V, generator=torch.Generator().manual_seed(seed)))
        call()
        want = [t.clone() for t in (L, lp, dz)]
        for t in (L, lp, dz):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (L, lp, dz)))


def test_logp_in_parts_replays():
    """Rows in parts that meet within the launch: a captured call replayed, with eager
    calls on the same workspace in between, and a workspace of arbitrary contents."""
    _announce("logp parts graph")
    T, V = 24, 128256
    g = torch.Generator().manual_seed(3)
    n = lm.token_loss_workspace_bytes(lm.TOKEN_LOSS_OP_LOGP, T, V, V)
    ws = torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda")
    y = torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda()
    z, lp, want = torch.empty(T, V, dtype=BF16, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    z.normal_()
    lm.token_logp(z, y, lp, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lm.token_logp(z, y, lp, ws=ws)
    for seed in range(6):
        z.normal_(std=1.0 + seed)
        lp.fill_(5.0)
        graph.replay()
        lm.token_logp(z, y, want, ws=ws if seed % 2 else None)
        torch.cuda.synchronize()
        assert torch.equal(lp, want)
        if seed == 3:
            ws.random_(0, 256)
    ref = R.logp(z.cpu(), y.cpu(), V)[0]
    _close(lp.cpu(), ref, R.logp_bound(z.cpu(), y.cpu(), V), "logp")


def test_python_refusals():
    T, V = 4, 16
    z = torch.zeros(T, V, device="cuda")
    y, f = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, device="cuda")
    with pytest.raises(TypeError):
        lm.token_logp(z, y.long(), f)
    with pytest.raises(TypeError):
        lm.token_logp(z.half(), y, f)
    with pytest.raises(ValueError):
        lm.token_logp(z, y, torch.zeros(T + 1, device="cuda"))
    with pytest.raises(ValueError):
        lm.token_logp(z.t().contiguous().t(), y, f)
    with pytest.raises(ValueError):
        lm.token_logp(z, y.cpu(), f)
    with pytest.raises(lm.LoraError):
        lm.token_logp(z, y, f, vocab=V + 1)
    with pytest.raises(lm.LoraError):
        lm.policy_loss(z, y, None, f, f, None, torch.zeros(1, device="cuda"), torch.zeros(T, device="cuda"), kl_coef=0.1)
