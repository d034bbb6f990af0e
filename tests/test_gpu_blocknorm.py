"""Norms with gate, residual scale and residual sum on the GPU, forward and backward,
against their definitions in 64 bits."""
import itertools

import pytest
import torch

import block_reference as ref
import paper_2606_19528_amd as lm

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
TYPES = [(BF16, BF16), (BF16, F32), (F32, F32)]
EPS = 1e-6


def make(T, D, dt, rt, post=True, gate="channel", seed=0):
    g = torch.Generator().manual_seed(seed + 1000 * T + D)

    def randn(*shape, dtype=dt):
        return torch.randn(*shape, generator=g).to(dtype)

    shape = {"none": None, "channel": (D,), "token": (T, 1), "full": (T, D)}[gate]
    return {"h": randn(T, D, dtype=rt), "y": (3.0 * torch.randn(T, D, generator=g)).to(dt),
            "gate": None if shape is None else torch.rand(*shape, generator=g).to(dt),
            "w_pre": (1.0 + 0.3 * torch.randn(D, generator=g)).to(dt),
            "w_post": (1.0 + 0.3 * torch.randn(D, generator=g)).to(dt) if post else None,
            "dn": randn(T, D), "dh_out": randn(T, D, dtype=rt)}


def dev(d):
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in d.items()}


def forward(c, post, off=0.0, a=0.75, eps=EPS, keep=(), **kw):
    """Outputs of block_norm_fwd on the CPU tensors of `c`."""
    d = dev(c)
    T, D = c["h"].shape
    dt, rt = c["y"].dtype, c["h"].dtype
    o = {"h": torch.full((T, D), 9.0, dtype=rt, device="cuda"), "n": torch.full((T, D), 9.0, dtype=dt, device="cuda"),
         "rstd_pre": torch.empty(T, device="cuda"), "rstd_post": torch.empty(T, device="cuda") if post else None}
    k8 = {k + "8": lm.act8_empty(T, D) for k in keep}
    lm.block_norm_fwd(d["h"], d["y"], h_out=o["h"], n=o["n"], w_pre=d["w_pre"], w_post=d["w_post"], gate=d["gate"], post_norm=post,
                      rstd_pre=o["rstd_pre"], rstd_post=o["rstd_post"], eps=eps, gain_offset=off, res_scale=a, **k8, **kw)
    return {**o, **k8}


def check_forward(c, got, post, off=0.0, a=0.75, eps=EPS):
    want, err = ref.norm_fwd(c["h"], c["y"], post, c["w_post"], c["gate"], c["w_pre"], eps, off, a)
    for k in want:
        ref.check(got[k], want[k], err[k], k)


# widths of every form of the kernel, one vector and odd numbers of them, each with its last
# threads idle and all of them busy
WIDTHS = [8, 120, 512, 520, 1024, 1032, 2048, 2056, 4096, 4104, 8192, 8200, 16384]


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_forward_widths(D, dt, rt):
    for T in (1, 6):
        c = make(T, D, dt, rt)
        check_forward(c, forward(c, True), True)


@pytest.mark.parametrize("post,gate", itertools.product([False, True], ["none", "channel", "token", "full"]))
@pytest.mark.parametrize("dt,rt", TYPES)
def test_forward_parts(dt, rt, post, gate):
    c = make(37, 328, dt, rt, post, gate)
    if gate != "none":
        c["gate"].view(-1)[0] = 0.0
    check_forward(c, forward(c, post), post)
    # gains stored as their distance from 1
    for w in ("w_pre", "w_post"):
        if c[w] is not None:
            c[w] = (c[w].float() - 1.0).to(dt)
    check_forward(c, forward(c, post, off=1.0, a=-1.5, eps=0.1), post, off=1.0, a=-1.5, eps=0.1)


def test_forward_many_rows():
    c = make(4099, 1096, BF16, BF16)
    check_forward(c, forward(c, True), True)


@pytest.mark.parametrize("dt,rt", TYPES)
def test_norm_alone_and_without_gains(dt, rt):
    """No block: the first norm of a decoder; and a norm without gains."""
    T, D = 19, 264
    c = make(T, D, dt, rt)
    h = c["h"].cuda()
    n, r = torch.empty(T, D, dtype=dt, device="cuda"), torch.empty(T, device="cuda")
    lm.block_norm_fwd(h, n=n, w_pre=c["w_pre"].cuda(), rstd_pre=r)
    want, err = ref.norm_fwd(c["h"], None, False, None, None, c["w_pre"], EPS, 0.0, 1.0)
    ref.check(n, want["n"], err["n"], "n")
    ref.check(r, want["rstd_pre"], err["rstd_pre"], "rstd")
    lm.block_norm_fwd(h, n=n, gain_offset=5.0)  # (an offset has no gains to go with)
    want, err = ref.norm_fwd(c["h"], None, False, None, None, None, EPS, 0.0, 1.0)
    ref.check(n, want["n"], err["n"], "n")
    c["w_pre"] = c["w_post"] = None
    check_forward(c, forward(c, True, off=5.0), True)


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("T,D", [(1, 8), (33, 1000), (5, 4104)])
def test_copies_in_8_bits(T, D, dt, rt):
    """Bitwise what act8_quantize makes of the stored tensors; the other outputs unchanged by them."""
    c = make(T, D, dt, rt)
    got, plain = forward(c, True, keep="yhn"), forward(c, True)
    for k in ("h", "n", "rstd_pre", "rstd_post"):
        assert torch.equal(got[k], plain[k]), k
    for k, t in (("y8", c["y"].cuda()), ("h8", got["h"]), ("n8", got["n"])):
        want = lm.act8_quantize(t, lm.act8_empty(T, D))
        assert torch.equal(got[k][0], want[0]) and torch.equal(got[k][1], want[1]), k
    # n and h only as copies
    d = dev(c)
    n8, h8 = lm.act8_empty(T, D), lm.act8_empty(T, D)
    lm.block_norm_fwd(d["h"], d["y"], w_pre=d["w_pre"], w_post=d["w_post"], gate=d["gate"], n8=n8, h8=h8, res_scale=0.75)
    assert torch.equal(n8[0], got["n8"][0]) and torch.equal(n8[1], got["n8"][1]) and torch.equal(h8[0], got["h8"][0])


@pytest.mark.parametrize("dt,rt", TYPES)
def test_stream_in_place(dt, rt):
    c = make(21, 2056, dt, rt)
    want = forward(c, True)
    d = dev(c)
    n = torch.empty_like(d["y"])
    lm.block_norm_fwd(d["h"], d["y"], h_out=d["h"], n=n, w_pre=d["w_pre"], w_post=d["w_post"], gate=d["gate"], res_scale=0.75)
    assert torch.equal(d["h"], want["h"]) and torch.equal(n, want["n"])


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("D", [264, 4104])
def test_large_small_and_not_finite_rows(D, dt, rt):
    """Rows of zeros, of squares outside fp32, and with infinities or NaN: each row by itself."""
    c = make(8, D, dt, rt, gate="none")
    c["y"][0], c["h"][0] = 0.0, 0.0
    c["y"][1] = (c["y"][1].float() * 1e25).to(dt)
    c["h"][2] = (c["h"][2].float() * 1e30).to(rt)
    c["y"][3] = (c["y"][3].float() * 1e-30).to(dt)
    c["y"][4, 7] = torch.nan
    c["h"][5, D - 1] = torch.inf
    c["y"][6, 3] = -torch.inf
    got = forward(c, True)
    finite = [0, 1, 2, 3, 7]
    part = {k: (v[finite] if v is not None and v.ndim == 2 else v) for k, v in c.items()}
    check_forward(part, {k: (v[finite] if v is not None else None) for k, v in got.items()}, True)
    assert bool(got["h"][4].isnan().all()) and bool(got["n"][4].isnan().all())
    # an infinity: the mean is infinite, so the others are 0 and it is inf * 0
    assert bool(got["n"][5, D - 1].isnan()) and bool((got["n"][5, : D - 1] == 0).all())
    assert bool(got["h"][6, 3].isnan()) and bool(got["n"][6].isnan().all())
    assert torch.equal(got["h"][6, 4:].cpu(), c["h"][6, 4:])  # (y's norm there is 0)


# ---- backward ---------------------------------------------------------------------------
def backward(c, r1, r2, post, want_grads, off=0.0, a=0.75, h=None, y=None, **kw):
    d = dev(c)
    T, D = c["h"].shape
    dt, rt = c["y"].dtype, c["h"].dtype
    o = {"dh": torch.full((T, D), 9.0, dtype=rt, device="cuda"), "dy": torch.full((T, D), 9.0, dtype=dt, device="cuda"),
         "dw_pre": None, "dw_post": None, "dgate": None}
    if want_grads:
        o["dw_pre"] = torch.full((D,), 9.0, device="cuda")
        o["dw_post"] = torch.full((D,), 9.0, device="cuda") if post else None
        if c["gate"] is not None:
            o["dgate"] = torch.full(c["gate"].shape, 9.0, dtype=dt if c["gate"].shape == (T, D) else F32, device="cuda")
    lm.block_norm_bwd(d["dn"], d["dh_out"], d["h"] if h is None else h, d["y"] if y is None else y, w_pre=d["w_pre"],
                      w_post=d["w_post"], gate=d["gate"], post_norm=post, rstd_pre=r1.cuda(), rstd_post=r2.cuda() if post else None,
                      gain_offset=off, res_scale=a, **o, **kw)
    return o


def roots(c):
    return tuple((c[k].double().square().mean(1) + EPS).rsqrt().float() for k in ("h", "y"))


def check_backward(c, got, r1, r2, post, off=0.0, a=0.75, h=None, y=None):
    want, err = ref.norm_bwd(c["dn"], c["dh_out"], c["h"] if h is None else h, c["y"] if y is None else y, post, c["w_post"],
                             c["gate"], c["w_pre"], r2, r1, off, a)
    for k, v in got.items():
        if v is not None:
            ref.check(v, want[k], err[k], k)


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_backward_widths(D, dt, rt):
    for T, grads in ((1, False), (6, True)):
        c = make(T, D, dt, rt)
        r1, r2 = roots(c)
        check_backward(c, backward(c, r1, r2, True, grads), r1, r2, True)


@pytest.mark.parametrize("post,gate", itertools.product([False, True], ["none", "channel", "token", "full"]))
@pytest.mark.parametrize("dt,rt", TYPES)
def test_backward_parts(dt, rt, post, gate):
    c = make(37, 328, dt, rt, post, gate)
    r1, r2 = roots(c)
    for grads in (False, True):
        check_backward(c, backward(c, r1, r2, post, grads), r1, r2, post)
    for w in ("w_pre", "w_post"):
        if c[w] is not None:
            c[w] = (c[w].float() - 1.0).to(dt)
    check_backward(c, backward(c, r1, r2, post, True, off=1.0, a=-1.5), r1, r2, post, off=1.0, a=-1.5)
    c["w_pre"] = c["w_post"] = None
    check_backward(c, backward(c, r1, r2, post, True, off=1.0), r1, r2, post)


@pytest.mark.parametrize("T", [511, 513, 2051])
def test_backward_many_rows(T):
    """More rows than workgroups, at a width with several rows a workgroup and one with one."""
    for D in (264, 2056):
        c = make(T, D, BF16, F32)
        r1, r2 = roots(c)
        got = backward(c, r1, r2, True, True)
        check_backward(c, got, r1, r2, True)
        again = backward(c, r1, r2, True, True)
        assert all(torch.equal(got[k], again[k]) for k in got)  # (a fixed order)


# rows of one to 25 vectors of a wave, as many as leave the forms for few rows
MANY = [512, 1024, 1536, 2040, 2056, 3592, 4104, 6152, 8192, 12288, 12296]


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("D", MANY)
def test_many_rows_of_every_width(D, dt, rt):
    T = 1024 // ((D + 511) // 512) + 3
    c = make(T, D, dt, rt, gate="token")
    check_forward(c, forward(c, True), True)
    r1, r2 = roots(c)
    check_backward(c, backward(c, r1, r2, True, False), r1, r2, True)


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("D", MANY[1:])
def test_large_calls_are_their_rows(D, dt, rt):
    """Calls large enough to be read past the caches: the bits of calls over parts of their rows."""
    T = (1 << 24) // D + 5
    g = torch.Generator(device="cuda").manual_seed(D)
    d = {k: torch.randn(T, D, generator=g, device="cuda").to(rt if k in ("h", "dh_out") else dt) for k in ("h", "y", "dn", "dh_out")}
    w = {k: (1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(dt) for k in ("w_pre", "w_post", "gate")}
    r = {k: 0.5 + torch.rand(T, generator=g, device="cuda") for k in ("rstd_pre", "rstd_post")}

    def run(a, b):
        p = {k: v[a:b] for k, v in d.items()}
        n8, dh, dy = lm.act8_empty(b - a, D), torch.empty_like(p["h"]), torch.empty_like(p["y"])
        ho, n = torch.empty_like(p["h"]), torch.empty_like(p["y"])
        lm.block_norm_fwd(p["h"], p["y"], h_out=ho, n=n, n8=n8, **w)
        lm.block_norm_bwd(p["dn"], p["dh_out"], p["h"], p["y"], dh=dh, dy=dy, **w, **{k: v[a:b].clone() for k, v in r.items()})
        return ho, n, *n8, dh, dy

    whole, cuts = run(0, T), [T * k // 5 for k in range(6)]
    parts = [run(a, b) for a, b in zip(cuts, cuts[1:])]
    for k, x in enumerate(whole):
        assert torch.equal(x, torch.cat([p[k] for p in parts])), k


@pytest.mark.parametrize("dt,rt,gate", [(BF16, BF16, "channel"), (BF16, F32, "full"), (F32, F32, "token")])
def test_backward_of_long_rows(dt, rt, gate):
    """Rows that are passed over twice, two of them a workgroup, from whole values and from copies, the stream's
    gradient in place."""
    T, D = 258, 8264
    c = make(T, D, dt, rt, gate=gate)
    r1, r2 = roots(c)
    got = backward(c, r1, r2, True, True)
    check_backward(c, got, r1, r2, True)
    d = dev(c)
    dh = d["dh_out"].clone()
    lm.block_norm_bwd(d["dn"], dh, d["h"], d["y"], dh=dh, w_pre=d["w_pre"], w_post=d["w_post"], gate=d["gate"], rstd_pre=r1.cuda(),
                      rstd_post=r2.cuda(), res_scale=0.75, dw_pre=torch.empty(D, device="cuda"))
    assert torch.equal(dh, got["dh"])
    h8, y8 = (lm.act8_quantize(d[k], lm.act8_empty(T, D)) for k in ("h", "y"))
    again = backward(c, r1, r2, True, True, h=h8, y=y8)
    check_backward(c, again, r1, r2, True, h=ref.act8_values(*(t.cpu() for t in h8)), y=ref.act8_values(*(t.cpu() for t in y8)))


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("D", [256, 768, 1536, 3072])
def test_an_infinite_gradient_in_the_last_row(D, dt, rt):
    """Its column's sums are infinite, not NaN: rows of a workgroup behind the last add nothing to them."""
    T = 5
    c = make(T, D, dt, rt)
    c["dh_out"][T - 1, 9] = float("inf")
    r1, r2 = roots(c)
    got = backward(c, r1, r2, True, True)
    assert got["dw_post"][9].isinf() and got["dgate"][9].isinf()
    for k in ("dw_pre", "dw_post", "dgate"):
        assert got[k][torch.arange(D, device="cuda") != 9].isfinite().all(), k


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("kept", ["h", "y", "hy"])
def test_backward_from_copies(dt, rt, kept):
    T, D = 45, 1000
    c = make(T, D, dt, rt)
    r1, r2 = roots(c)
    k8, val = {}, {}
    for k in kept:
        k8[k] = lm.act8_quantize(c[k].cuda(), lm.act8_empty(T, D))
        val[k] = ref.act8_values(k8[k][0].cpu(), k8[k][1].cpu())
    for grads in (False, True):
        check_backward(c, backward(c, r1, r2, True, grads, **k8), r1, r2, True, **val)


def test_backward_of_one_side():
    """A gradient through the stream alone, through the norm alone, and in place."""
    T, D = 23, 264
    c = make(T, D, BF16, F32)
    r1, r2 = roots(c)
    for missing in ("dn", "dh_out"):
        d = {**c, missing: None}
        got = backward(d, r1, r2, True, False)
        check_backward(d, got, r1, r2, True)
    d = dev(c)
    want = backward(c, r1, r2, True, False)
    lm.block_norm_bwd(d["dn"], d["dh_out"], d["h"], dh=d["dh_out"], w_pre=d["w_pre"], rstd_pre=r1.cuda())
    assert torch.equal(d["dh_out"], want["dh"])


@pytest.mark.parametrize("gate", ["channel", "token", "full"])
def test_gradients_by_differences(gate):
    """The backward's gradients against differences of the definition in 64 bits along random directions."""
    T, D = 3, 24
    c = make(T, D, F32, F32, gate=gate)
    names = ["h0", "y", "w_pre", "w_post", "gate"]
    h0 = torch.randn(T, D, generator=torch.Generator().manual_seed(5), dtype=torch.float64).float()

    def outs(v):
        o, _ = ref.norm_fwd(v["h0"], v["y"], True, v["w_post"], v["gate"], v["w_pre"], EPS, 0.0, 0.75)
        return (o["n"] * c["dn"].double()).sum() + (o["h"] * c["dh_out"].double()).sum()

    at = {"h0": h0, "y": c["y"], "w_pre": c["w_pre"], "w_post": c["w_post"], "gate": c["gate"]}
    fwd, _ = ref.norm_fwd(h0, c["y"], True, c["w_post"], c["gate"], c["w_pre"], EPS, 0.0, 0.75)
    d = {**c, "h": fwd["h"].float()}
    got = backward(d, fwd["rstd_pre"].float(), fwd["rstd_post"].float(), True, True)
    grads = {"h0": got["dh"], "y": got["dy"], "w_pre": got["dw_pre"], "w_post": got["dw_post"], "gate": got["dgate"]}
    g = torch.Generator().manual_seed(6)
    for k in names:
        way = torch.randn(at[k].shape, generator=g, dtype=torch.float64)
        # the fourth-order difference: its own error is below 1e-9 of these sums
        t, f = 1e-3, lambda s: float(outs({**at, k: at[k].double() + s * way}))
        slope = (8 * (f(t) - f(-t)) - (f(2 * t) - f(-2 * t))) / (12 * t)
        mine = float((grads[k].cpu().double().reshape(way.shape) * way).sum())
        size = float((grads[k].cpu().double().reshape(way.shape) * way).abs().sum())
        # fp32 gradients of rows of 24: 2 SUM + 20 roundings of what they are sums of, at most 4 times the gradient
        assert abs(mine - slope) <= (2 * ref.SUM + 20) * 4 * ref.U * size + 1e-8 * abs(slope) + 1e-9, k


def test_stream_and_graph():
    """Both directions captured together, replayed on new values with eager work in between."""
    T, D = 65, 1000
    c = make(T, D, BF16, F32)
    d = dev(c)
    o = {k: torch.empty_like(d["h"]) for k in ("h", "dh")}
    o |= {k: torch.empty_like(d["y"]) for k in ("n", "dy")}
    r1, r2 = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    col = {k: torch.empty(D, device="cuda") for k in ("dw_pre", "dw_post", "dgate")}
    ws = torch.empty(lm.block_norm_workspace_bytes(T, D), dtype=torch.uint8, device="cuda")
    par = {k: d[k] for k in ("w_pre", "w_post", "gate")}

    def both(stream=None):
        lm.block_norm_fwd(d["h"], d["y"], h_out=o["h"], n=o["n"], rstd_pre=r1, rstd_post=r2, stream=stream, **par)
        lm.block_norm_bwd(d["dn"], d["dh_out"], o["h"], d["y"], dh=o["dh"], dy=o["dy"], rstd_pre=r1, rstd_post=r2, ws=ws,
                          stream=stream, **col, **par)

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    both(st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    everything = {**o, **col}
    for seed in range(4):
        n = make(T, D, BF16, F32, seed=seed)
        for k in ("h", "y", "dn", "dh_out"):
            d[k].copy_(n[k])
        graph.replay()
        got = {k: v.clone() for k, v in everything.items()}
        for v in everything.values():
            v.zero_()
        both()
        torch.cuda.synchronize()
        for k, v in everything.items():
            assert torch.equal(v, got[k]), k


@pytest.mark.parametrize("D,kept", [(1032, False), (2048, True), (16384, False)])
def test_offsets_past_32_bits(D, kept):
    """More than 2^31 values: the last rows, which repeat the first ones, have their bits."""
    n = 520  # rows that are repeated
    k = (1 << 31) // (n * D) + 1
    T = n * k
    assert T * D > 1 << 31
    c = {a: (b if b is None or b.shape[0] != n else b.repeat(k, 1)) for a, b in dev(make(n, D, BF16, BF16)).items()}
    r = {a: (0.5 + torch.rand(n, device="cuda")).repeat(k) for a in ("rstd_pre", "rstd_post")}
    w = {a: c[a] for a in ("w_pre", "w_post", "gate")}
    n8, h8, y8 = (lm.act8_empty(T, D) if kept else None for _ in range(3))
    ho, nn = torch.empty_like(c["h"]), torch.empty_like(c["y"])
    lm.block_norm_fwd(c["h"], c["y"], h_out=ho, n=nn, n8=n8, h8=h8, y8=y8, **w)
    out = [ho, nn]
    dh, dy = torch.empty_like(c["h"]), torch.empty_like(c["y"])
    lm.block_norm_bwd(c["dn"], c["dh_out"], h8 if kept else ho, y8 if kept else c["y"], dh=dh, dy=dy, **w, **r)
    out += [dh, dy]
    if kept:
        out += [*n8, *h8, *y8]
        x8, back = lm.act8_quantize(c["y"], lm.act8_empty(T, D)), torch.empty_like(c["y"])
        lm.act8_dequantize(x8, back)
        out += [*x8, back]
    for i, t in enumerate(out):
        assert torch.equal(t[-n:], t[:n]), i
        assert torch.equal(t[(k // 2) * n:(k // 2 + 1) * n], t[:n]), i
