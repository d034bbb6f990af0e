"""Embedding lookup and gradient: the lookup bitwise, the gradient against the sums in
64 bits within the bound of their 32-bit evaluation, over lengths from one token
on, tokens that all differ or are all the same, and ids outside the table."""
import sys

import pytest
import torch

import step_reference as R

pytestmark = pytest.mark.gpu

import paper_2606_19528_amd as lm  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def _announce(msg):
    print(f"[case] {msg}", file=sys.stderr, flush=True)


def _ids(T, V, kind, g):
    if kind == "uniform":
        return torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    if kind == "text":  # few tokens often, most seldom
        return (V * torch.rand(T, generator=g, dtype=torch.float64) ** 6).to(torch.int32).clamp(max=V - 1)
    if kind == "same":
        return torch.full((T,), V // 2, dtype=torch.int32)
    if kind == "edges":
        ids = torch.randint(0, 3, (T,), generator=g, dtype=torch.int32)
        return torch.where(ids == 2, V - 1, ids * 0)
    ids = torch.randint(-2, V + 2, (T,), generator=g, dtype=torch.int32)  # "outside"
    ids[: T // 3] = -100
    return ids


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("shape", [(1, 1, 8), (1, 500, 3072), (5, 7, 24), (24, 1000, 2048), (333, 128, 520), (1000, 257, 8192)])
def test_lookup(shape, dt):
    T, V, D = shape
    _announce(f"embed_fwd T={T} V={V} D={D} {dt}")
    g = torch.Generator().manual_seed(T + V)
    table = torch.randn(V, D, generator=g).to(dt)
    for kind in ("uniform", "outside"):
        ids = _ids(T, V, kind, g)
        ok = (ids >= 0) & (ids < V)
        for scale in (1.0, 45.2548):
            out = torch.full((T, D), 7.0, dtype=dt, device="cuda")
            lm.embed_fwd(table.cuda(), ids.cuda(), out, scale)
            want = (table[torch.where(ok, ids, 0).long()].float() * torch.tensor(scale, dtype=F32)).to(dt)
            assert torch.equal(out.cpu(), torch.where(ok[:, None], want, torch.zeros_like(want)))


def _check_grad(got, ids, dout, V, scale, base=None):
    ref, bound = R.embed_grad(ids, dout, V, scale)
    if base is not None:
        ref, bound = ref + base.double(), bound + R.U * (base.double().abs() + ref.abs()) * 2 + bound * 2 ** -20
    err = (got.double() - ref).abs()
    assert (err <= bound).all(), f"largest error {float(err.max()):.3e}, over its bound by {float((err - bound).max()):.3e}"
    if base is None:
        absent = torch.ones(V, dtype=torch.bool)
        absent[ids[(ids >= 0) & (ids < V)].long()] = False
        assert not got[absent].any()


CASES = [(1, 1, 8), (1, 1000, 64), (2, 3, 24), (8, 50, 136), (9, 50, 136), (64, 40, 1032), (32, 1, 2048), (31, 3, 24), (33, 2, 1032), (65, 700, 2048), (257, 513, 72),
         (1023, 1000, 64), (2048, 511, 40), (2049, 512, 40), (4100, 30000, 72), (6144, 700, 16), (6145, 5000, 16), (8200, 1024, 16), (8193, 300000, 16), (8300, 262144, 8), (300, 262145, 24), (300, 262144, 24),
         (20011, 130001, 16), (32769, 600, 8), (70001, 900, 8)]


@pytest.mark.parametrize("kind", ["uniform", "text", "same", "edges", "outside"])
@pytest.mark.parametrize("shape", CASES, ids=lambda s: "x".join(map(str, s)))
def test_gradient(shape, kind):
    T, V, D = shape
    dt = F32 if T % 2 else BF16
    _announce(f"embed_bwd T={T} V={V} D={D} {kind} {dt}")
    g = torch.Generator().manual_seed(T * 7 + V)
    ids = _ids(T, V, kind, g)
    dout = torch.randn(T, D, generator=g).to(dt)
    scale = 0.75
    di, dd = ids.cuda(), dout.cuda()
    dense = torch.full((V, D), 3.0, device="cuda")
    lm.embed_bwd(di, dd, dense, scale)
    _check_grad(dense.cpu(), ids, dout, V, scale)
    # the compact form holds the same sums, bit for bit
    n = min(T, V)
    tokens = torch.full((n,), 77, dtype=torch.int32, device="cuda")
    rows = torch.full((n, D), 3.0, device="cuda")
    lm.embed_bwd_rows(di, dd, V, tokens, rows, scale)
    want = torch.unique(ids[(ids >= 0) & (ids < V)])
    m = want.numel()
    assert torch.equal(tokens[:m].cpu(), want) and (tokens[m:] == -1).all()
    assert torch.equal(rows[:m].cpu(), dense.cpu()[want.long()]) and not rows[m:].any()
    # added to what is there
    base = torch.randn(V, D, generator=g)
    acc = base.cuda()
    lm.embed_bwd(di, dd, acc, scale, accumulate=True)
    _check_grad(acc.cpu(), ids, dout, V, scale, base)
    absent = torch.ones(V, dtype=torch.bool)
    absent[want.long()] = False
    assert torch.equal(acc.cpu()[absent], base[absent])


def test_gradient_is_the_lookups_difference():
    """<dout, lookup(E + h X) - lookup(E - h X)> / 2h = <dE, X> for the linear lookup."""
    _announce("embed gradient against differences")
    g = torch.Generator().manual_seed(3)
    T, V, D, scale, h = 300, 90, 64, 1.5, 0.5
    E, X = torch.randn(V, D, generator=g), torch.randn(V, D, generator=g)
    ids, dout = _ids(T, V, "outside", g), torch.randn(T, D, generator=g)
    outs = []
    for s in (h, -h):
        out = torch.empty(T, D, device="cuda")
        lm.embed_fwd((E + s * X).cuda(), ids.cuda(), out, scale)
        outs.append(out.cpu().double())
    dE = torch.empty(V, D, device="cuda")
    lm.embed_bwd(ids.cuda(), dout.cuda(), dE, scale)
    diff = float(((outs[0] - outs[1]) * dout.double()).sum()) / (2 * h)
    # each of T D products carries a few roundings of values of a few units
    assert abs(diff - float((dE.cpu().double() * X.double()).sum())) <= 64 * R.U * T * D


def test_repeatable_and_ordered_on_its_stream():
    """Bitwise the same from call to call, with a workspace that holds another call's
    remains, and on another stream than the current one."""
    _announce("embed repeat and stream")
    g = torch.Generator().manual_seed(11)
    T, V, D = 5000, 900, 72
    ids, dout = _ids(T, V, "text", g).cuda(), torch.randn(T, D, generator=g).cuda()
    ws = torch.randint(0, 256, (lm.embed_bwd_workspace_bytes(T, V, D),), dtype=torch.uint8, device="cuda")
    a, b = torch.empty(V, D, device="cuda"), torch.empty(V, D, device="cuda")
    lm.embed_bwd(ids, dout, a, ws=ws)
    lm.embed_bwd(ids.flip(0).contiguous(), dout, b, ws=ws)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    lm.embed_bwd(ids, dout, b, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(a, b)


@pytest.mark.parametrize("T", [300, 9000])  # without and with a sort
def test_graph_replays(T):
    """A captured lookup and its gradients replay on changed tokens."""
    _announce(f"embed graph T={T}")
    g = torch.Generator().manual_seed(T)
    V, D = 800, 40
    table, dout = torch.randn(V, D, generator=g).cuda(), torch.randn(T, D, generator=g).cuda()
    ids, out = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.empty(T, D, device="cuda")
    n = min(T, V)
    dense, rows, tokens = torch.empty(V, D, device="cuda"), torch.empty(n, D, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    ws = torch.empty(lm.embed_bwd_workspace_bytes(T, V, D), dtype=torch.uint8, device="cuda")

    def call():
        lm.embed_fwd(table, ids, out)
        lm.embed_bwd(ids, dout, dense, ws=ws)
        lm.embed_bwd_rows(ids, dout, V, tokens, rows, ws=ws)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for kind in ("uniform", "text", "same", "outside", "uniform"):
        ids.copy_(_ids(T, V, kind, g))
        call()
        want = [t.clone() for t in (out, dense, rows, tokens)]
        for t in (out, dense, rows, tokens):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (out, dense, rows, tokens)))


def test_infinities_stay_in_their_row():
    _announce("embed inf")
    g = torch.Generator().manual_seed(5)
    T, V, D = 40, 9, 16
    ids = _ids(T, V, "uniform", g)
    ids[3] = 4
    dout = torch.randn(T, D, generator=g)
    dout[3, 2] = float("inf")
    dE = torch.empty(V, D, device="cuda")
    lm.embed_bwd(ids.cuda(), dout.cuda(), dE)
    dE = dE.cpu()
    assert torch.isinf(dE[4, 2])
    dE[4, 2] = 0
    assert torch.isfinite(dE).all()
