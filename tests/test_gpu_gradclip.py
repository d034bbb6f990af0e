"""Global norm and clipping of a list of gradients against 64-bit sums.

The norm's squares are summed in 64 bits, so the norm is within a few 2^-53 of the
exact one before it is rounded to fp32, and the factor likewise: 2^-23 relatively.
An output is g times the rounded factor, rounded: 2^-23 more in fp32, 2^-8 in bf16."""
import sys

import pytest
import torch

import step_reference as R

pytestmark = pytest.mark.gpu

import paper_2606_19528_amd as lm  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
LISTS = [
    [(1,)],
    [(3,), (1,), (8,), (4097,)],
    [(8, 256), (256, 8)],
    [(13, 2048), (256, 13), (0,), (5,)],
    [(16, 3000), (8191,), (100003,)],
    [(7,)] * 300,                       # more entries than one launch lays out
    [(32, 8192)] * 40 + [(1,)] * 70,    # many chunks
]


def _announce(msg):
    print(f"[case] {msg}", file=sys.stderr, flush=True)


def _grads(shapes, dts, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(*s, generator=g) * size).to(dts[i % len(dts)]) for i, s in enumerate(shapes)]


@pytest.mark.parametrize("i", range(len(LISTS)))
@pytest.mark.parametrize("dts,out", [([F32], F32), ([BF16], BF16), ([F32, BF16], F32), ([BF16, F32], BF16)])
def test_clip(i, dts, out):
    shapes = LISTS[i]
    _announce(f"clip list {i} {dts} -> {out}")
    grads = _grads(shapes, dts, 17 + i)
    norm, _, _ = R.clip(grads, 1.0)
    dev = [g.cuda() for g in grads]
    outs = [torch.full(g.shape, 5.0, dtype=out, device="cuda") for g in grads]
    gl = lm.grad_list(dev, outs)
    for max_norm in (0.37 * norm, 2.0 * norm):
        _, c, ref = R.clip(grads, max_norm)
        res = torch.empty(2, device="cuda")
        lm.grad_clip(gl, max_norm, res)
        assert abs(float(res[0]) - norm) <= 2.0 ** -23 * norm
        assert abs(float(res[1]) - c) <= 2.0 ** -22 * c
        for o, r, g, d in zip(outs, ref, grads, dev):
            tol = (2.0 ** -22 if out == F32 else 2.0 ** -8) * r.abs() + 1e-40
            assert ((o.cpu().double() - r).abs() <= tol).all()
            assert torch.equal(d.cpu(), g)  # the gradients themselves are only read
    one = torch.empty(1, device="cuda")
    lm.grad_norm(gl, one)
    assert float(one[0]) == float(res[0])


@pytest.mark.parametrize("dt", [F32, BF16])
def test_in_place(dt):
    _announce(f"clip in place {dt}")
    grads = _grads(LISTS[4], [dt], 3)
    norm, c, ref = R.clip(grads, 2.5)
    dev = [g.cuda() for g in grads]
    gl = lm.grad_list(dev)
    res = torch.empty(2, device="cuda")
    lm.grad_clip(gl, 1e9, res)  # not clipped: bitwise unchanged
    assert float(res[1]) == 1.0 and all(torch.equal(a.cpu(), b) for a, b in zip(dev, grads))
    lm.grad_clip(gl, 2.5, res)
    for o, r in zip(dev, ref):
        assert ((o.cpu().double() - r).abs() <= (2.0 ** -22 if dt == F32 else 2.0 ** -8) * r.abs()).all()


@pytest.mark.parametrize("size", [1e-30, 1e25])
def test_squares_beyond_32_bits(size):
    _announce(f"clip size {size}")
    grads = _grads([(16, 256), (9,)], [F32], 5, size)
    norm, c, ref = R.clip(grads, 0.5 * size)
    gl = lm.grad_list([g.cuda() for g in grads], outs := [torch.empty(g.shape, device="cuda") for g in grads])
    res = torch.empty(2, device="cuda")
    lm.grad_clip(gl, 0.5 * size, res)
    assert abs(float(res[0]) - norm) <= 2.0 ** -23 * norm
    for o, r in zip(outs, ref):
        assert ((o.cpu().double() - r).abs() <= 2.0 ** -21 * r.abs() + 1e-40).all()


def test_zero_and_not_finite():
    _announce("clip zero, inf, nan")
    res = torch.empty(2, device="cuda")
    z = torch.zeros(100, device="cuda")
    lm.grad_clip(lm.grad_list([z]), 0.0, res)
    assert res.tolist() == [0.0, 1.0] and not z.any()
    g = torch.ones(100, device="cuda")
    lm.grad_clip(lm.grad_list([g]), 0.0, res)  # nothing is allowed
    assert res.tolist() == [10.0, 0.0] and not g.any()
    g = torch.ones(100, device="cuda")
    g[7] = float("inf")
    lm.grad_clip(lm.grad_list([g]), 1.0, res)
    assert res.tolist() == [float("inf"), 0.0] and torch.isnan(g[7]) and not g[:7].any()
    g = torch.ones(100, device="cuda")
    g[7] = float("nan")
    lm.grad_clip(lm.grad_list([g]), 1.0, res)
    assert torch.isnan(res).all() and torch.isnan(g).all()


def test_list_follows_the_buffers_and_repeats():
    _announce("clip list reused")
    buf = torch.empty(70001, device="cuda")
    out = torch.empty_like(buf)
    gl = lm.grad_list([buf], [out])
    res = torch.empty(2, device="cuda")
    seen = []
    for seed in (1, 2, 1):
        buf.copy_(torch.randn(70001, generator=torch.Generator().manual_seed(seed)))
        lm.grad_clip(gl, 1.0, res)
        seen.append((out.clone(), res.clone()))
    assert torch.equal(seen[0][0], seen[2][0]) and torch.equal(seen[0][1], seen[2][1])
    assert not torch.equal(seen[0][0], seen[1][0])


@pytest.mark.parametrize("n", [5000, 500001])  # one launch and two
def test_graph_replays(n):
    _announce(f"clip graph {n}")
    buf, out, res = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(2, device="cuda")
    gl = lm.grad_list([buf], [out])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lm.grad_clip(gl, 1.0, res)
    for seed in range(4):
        buf.normal_(std=10.0 ** (seed - 4))
        lm.grad_clip(gl, 1.0, res)
        want = out.clone(), res.clone()
        out.zero_(), res.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(res, want[1])


def test_python_refusals():
    a = torch.ones(8, device="cuda")
    with pytest.raises(lm.LoraError):
        lm.grad_list([])
    with pytest.raises(ValueError):
        lm.grad_list([a], [torch.ones(7, device="cuda")])
    with pytest.raises(ValueError):
        lm.grad_list([a.cpu()])
    with pytest.raises(TypeError):
        lm.grad_list([a.half()])
    with pytest.raises(lm.LoraError):
        lm.grad_list([a, a])  # two outputs in one place
    with pytest.raises(ValueError):
        lm.grad_clip(lm.grad_list([a]), 1.0, torch.empty(1, device="cuda"))
    with pytest.raises(lm.LoraError):
        lm.grad_clip(lm.grad_list([a]), float("nan"), torch.empty(2, device="cuda"))
