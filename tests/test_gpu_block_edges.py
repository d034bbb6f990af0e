"""Norms with gate and residual sum at the edges of their values, against their definitions in 64 bits."""
import pytest
import torch

import block_reference as ref
import paper_2606_19528_amd as lm

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
TYPES = [(BF16, BF16), (BF16, F32), (F32, F32)]
EPS = 1e-6


def inputs(T, D, dt, rt, post, gate, seed, off=0.0):
    """Rows of different size with a few large channels, on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def activation():
        x = randn(T, D) * torch.where(torch.rand(D, generator=g, device="cuda") < 0.01, 12.0, 1.0)
        return x * (0.5 * randn(T, 1)).exp()

    shape = {"none": None, "channel": (D,), "token": (T, 1), "full": (T, D)}[gate]
    return {"h": activation().to(rt), "y": activation().to(dt), "gate": None if shape is None else randn(*shape).sigmoid().to(dt),
            "w_pre": (1.0 - off + 0.2 * randn(D)).to(dt), "w_post": (1.0 - off + 0.2 * randn(D)).to(dt) if post else None}


def act8(x):
    """(codes, scale) of fp32 rows by the definition, quotients in 64 bits, on the GPU."""
    T, D = x.shape
    n = -(-D // 128)
    wide = torch.nn.functional.pad(x, (0, n * 128 - D)).view(T, n, 128).double()
    m = wide.abs().amax(2, keepdim=True)
    q = torch.floor(wide.abs() * 127.0 / torch.where(m > 0, m, 1.0) + 0.5) * wide.sign()
    return q.to(torch.int8).view(T, n * 128)[:, :D], (m[..., 0] / 127.0).float()


def definition(c, post, off, a, eps):
    y = c["y"].double()
    if post:
        y = y * (1.0 / torch.sqrt(y.square().mean(1, keepdim=True) + eps)) * (c["w_post"].double() + off)
    h = c["h"].double() + a * y * (1.0 if c["gate"] is None else c["gate"].double())
    return h, h * (1.0 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)) * (c["w_pre"].double() + off)


# rows of every number of waves, short last groups; 13 million values
COPIES = [(4099, 328, True, "token"), (2053, 1096, True, "channel"), (1021, 2056, False, "full"), (517, 4104, True, "none"),
          (301, 8200, True, "full"), (131, 12304, True, "channel"), (3, 1000, True, "token")]


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("T,D,post,gate", COPIES)
def test_copies_of_computed_fp32_values(T, D, post, gate, dt, rt):
    """fp32 values are computed in 64 bits and rounded once, so that their copies have the codes of the
    definition's.  Both sides evaluate it in 64 bits: at most 10 roundings of 2^-53, of the parts of h' (|h| + |a y g
    w r2|) or of n, and D of them in a mean, of which the root takes half.  A stored value is the nearest of the
    definition's, so off by half a step, and by those roundings: at most
    2^-24 |v| + 2^-53 ((10 + D) |v| + 10 parts).  (Which of two neighbours is stored where the value is within the
    latter of their middle is open: with a = 0.7 and products of two bf16 values such middles are met, 7 / 10
    times a multiple of 10.)  Of the values where the nearest is stored every code is the definition's."""
    for off, a, eps in ((0.0, 0.7, EPS), (1.0, -1.3, 0.1)):
        c = inputs(T, D, dt, rt, post, gate, seed=T + D, off=off)
        h_out, n = torch.empty_like(c["h"]), torch.empty_like(c["y"])
        y8, h8, n8 = (lm.act8_empty(T, D) for _ in range(3))
        lm.block_norm_fwd(c["h"], c["y"], h_out=h_out, n=n, w_pre=c["w_pre"], w_post=c["w_post"], gate=c["gate"], y8=y8, h8=h8,
                          n8=n8, eps=eps, gain_offset=off, res_scale=a)
        h64, n64 = definition(c, post, off, a, eps)
        parts = c["h"].double().abs() + (h64 - c["h"].double()).abs()
        for name, k8, got, want in (("y", y8, c["y"], c["y"]), ("h", h8, h_out, h64), ("n", n8, n, n64)):
            if name != "y":
                if got.dtype != F32:
                    continue  # (a computed bf16 value's copy is that of the value as it is stored)
                ratio = 1.0 if name == "h" else want.abs() / h64.abs().clamp(min=1e-30)
                bound = 2.0 ** -24 * want.abs() + 2.0 ** -53 * ((10 + D) * want.abs() + 10 * parts * ratio)
                wrong = int(((got.double() - want).abs() > bound).sum())
                assert wrong == 0, f"{name}: {wrong} values are not the nearest"
            nearest = want.float()
            codes, scale = act8(nearest)
            wrong = int(((k8[0] != codes) & (got == nearest)).sum())
            assert wrong == 0, f"{name}: {wrong} codes of {codes.numel()} are not the definition's"
            wide = torch.nn.functional.pad(got == nearest, (0, -D % 128), value=True).view(T, -1, 128).all(2)
            assert bool(((k8[1] == scale) | ~wide).all()), name
            # (of h' by such products; of n, which has a root in it, one in 10^7 where D is 10^4)
            assert float((got != nearest).double().mean()) <= (0.01 if name == "h" else 1e-6), name


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("D", [264, 1000, 8264])
def test_infinite_gate_and_gain(D, dt, rt):
    """Lanes behind a row's end take no part in its sums: a token's gate, or the gain of the last channel, may be
    infinite, then h' is (there), and 1 / sqrt of its mean square is 0."""
    T = 5
    c = inputs(T, D, dt, rt, True, "token", seed=D)
    c["y"][1].fill_(2.0)

    def run(**kw):
        o = {"h_out": torch.empty_like(c["h"]), "n": torch.empty_like(c["y"]), "rstd_pre": torch.empty(T, device="cuda")}
        lm.block_norm_fwd(c["h"], c["y"], **{**{k: c[k] for k in ("w_pre", "w_post", "gate")}, **kw}, **o)
        return o

    plain = run()
    gate = c["gate"].clone()
    gate[1] = torch.inf
    got = run(gate=gate)
    assert bool(got["h_out"][1].isinf().all()) and float(got["rstd_pre"][1]) == 0.0 and bool(got["n"][1].isnan().all())
    rows = [0, 2, 3, 4]
    assert all(torch.equal(got[k][rows], plain[k][rows]) for k in got)
    w = c["w_post"].clone()
    w[D - 1] = torch.inf
    got = run(w_post=w)
    assert bool(got["h_out"][:, D - 1].isinf().all()) and torch.equal(got["h_out"][:, :D - 1], plain["h_out"][:, :D - 1])
    assert bool((got["rstd_pre"] == 0).all())
    assert bool((got["n"][:, :D - 1] == 0).all()) and bool(got["n"][:, D - 1].isnan().all())


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("D", [264, 1000, 3080, 8264, 12296])
@pytest.mark.parametrize("sums", [False, True])
def test_an_infinite_stream_gradient_in_the_last_channel(D, dt, rt, sums):
    """Lanes behind a row's end hold its last values and add nothing to its sums: where dh' is infinite
    there, dy and a token's dgate are as by the definition, infinite and not NaN; other rows are what they are without it."""
    T = 6
    c = inputs(T, D, dt, rt, True, "token", seed=D)
    g = torch.Generator(device="cuda").manual_seed(1)
    dn, dho = (torch.randn(T, D, generator=g, device="cuda").to(t) for t in (dt, rt))
    r1, r2 = (0.5 + torch.rand(T, generator=g, device="cuda") for _ in range(2))

    def run():
        o = {"dh": torch.empty_like(c["h"]), "dy": torch.empty_like(c["y"]), "dgate": torch.empty(T, 1, device="cuda")}
        w = torch.empty(D, device="cuda") if sums else None
        lm.block_norm_bwd(dn, dho, c["h"], c["y"], **{k: c[k] for k in ("w_pre", "w_post", "gate")}, rstd_pre=r1, rstd_post=r2, dw_pre=w,
                          res_scale=0.75, **o)
        return o

    plain = run()
    dho[2, D - 1] = torch.inf
    got = run()
    cpu = {k: v.cpu() for k, v in c.items()}
    want, _ = ref.norm_bwd(dn.cpu(), dho.cpu(), cpu["h"], cpu["y"], True, cpu["w_post"], cpu["gate"], cpu["w_pre"], r2.cpu(), r1.cpu(),
                           0.0, 0.75)
    for k, v in got.items():
        rows = [0, 1, 3, 4, 5]
        assert torch.equal(v[rows], plain[k][rows]), k
        x, w = v[2].cpu().double(), want[k].reshape(v.shape)[2]
        assert torch.equal(x.isnan(), w.isnan()) and torch.equal(x.isinf(), w.isinf()), k
        inf = w.isinf()
        assert torch.equal(x[inf], w[inf]), k


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("D", [264, 8264, 12296])
@pytest.mark.parametrize("gate,sums", [("token", False), ("token", True), ("full", False), ("full", True), ("channel", True)])
def test_an_infinite_block_output_without_a_post_norm(D, dt, rt, gate, sums):
    """dy = a g dh does not read y, which dgate does: its infinity comes into dgate alone, in the forms of
    one pass over a row and of two."""
    T = 4
    c = inputs(T, D, dt, rt, False, gate, seed=D)
    g = torch.Generator(device="cuda").manual_seed(2)
    dn, dho = (torch.randn(T, D, generator=g, device="cuda").to(t) for t in (dt, rt))
    r1 = 0.5 + torch.rand(T, generator=g, device="cuda")

    def run():
        o = {"dh": torch.empty_like(c["h"]), "dy": torch.empty_like(c["y"])}
        o["dgate"] = torch.empty(c["gate"].shape, dtype=dt if gate == "full" else F32, device="cuda")
        w = torch.empty(D, device="cuda") if sums else None
        lm.block_norm_bwd(dn, dho, c["h"], c["y"], w_pre=c["w_pre"], gate=c["gate"], rstd_pre=r1, dw_pre=w, res_scale=0.75, **o)
        return o

    plain = run()
    c["y"][1, 9] = torch.inf
    got = run()
    assert torch.equal(got["dh"], plain["dh"]) and torch.equal(got["dy"], plain["dy"])
    at = {"token": (1, 0), "full": (1, 9), "channel": (9,)}[gate]
    assert bool(got["dgate"][at].isinf())
    got["dgate"][at] = plain["dgate"][at]
    assert torch.equal(got["dgate"], plain["dgate"])


@pytest.mark.parametrize("back", [False, True])
def test_the_most_rows(back):
    """2^22 rows in 16 waves each, forward and backward: 2^32 threads, which no dimension of a grid holds.  The rows
    repeat 512 of them, whose results they have."""
    n, T = 512, 1 << 22
    D = 6152 if back else 12296
    g = torch.Generator(device="cuda").manual_seed(3)
    few = torch.randn(n, D, generator=g, device="cuda").to(BF16)
    many = torch.empty(T, D, dtype=BF16, device="cuda")
    many.view(T // n, n, D).copy_(few.expand(T // n, n, D))

    def run(x):
        if back:
            dy = torch.empty_like(x)
            lm.block_norm_bwd(None, x, None, dh=x, dy=dy, res_scale=0.75)
            return dy
        r = torch.empty(x.shape[0], device="cuda")
        lm.block_norm_fwd(x, rstd_pre=r)
        return r

    want = run(few)
    got = run(many).view(T // n, *want.shape)
    for a in range(0, T // n, 512):
        assert bool((got[a:a + 512] == want).all()), a
    del many, got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kept", [False, True])
def test_the_gradient_of_a_post_gain_alone(kept):
    """bf16 y and gain behind an fp32 stream, through which alone a gradient comes."""
    T, D = 70, 264
    c = inputs(T, D, BF16, F32, True, "none", seed=4)
    dho = torch.randn(T, D, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    r2 = 0.5 + torch.rand(T, device="cuda")
    y8 = lm.act8_quantize(c["y"], lm.act8_empty(T, D))
    y = ref.act8_values(*(t.cpu() for t in y8)) if kept else c["y"].cpu()
    dh, w = torch.empty_like(dho), torch.empty(D, device="cuda")
    lm.block_norm_bwd(None, dho, None, y8 if kept else c["y"], dh=dh, w_post=c["w_post"], rstd_post=r2, dw_post=w, res_scale=0.75)
    want, err = ref.norm_bwd(None, dho.cpu(), None, y, True, c["w_post"].cpu(), None, None, r2.cpu(), None, 0.0, 0.75)
    assert torch.equal(dh, dho)
    ref.check(w, want["dw_post"], err["dw_post"], "dw_post")
