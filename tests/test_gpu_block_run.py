"""The operators between the linears and the backward from 8 bits as a step uses them:
embedding, norm, two LoRA linears, norm behind the block with its gate and residual sum, norm before the
head, the head's LoRA linear; and back, from the copies in 8 bits alone.  Against
automatic differentiation of the same function in 64 bits on the CPU."""
import pytest
import torch

import paper_2606_19528_amd as lm

pytestmark = pytest.mark.gpu
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
EPS, RES, S = 1e-6, 0.75, 0.5


def weights(T, D, F, V, r, gate, seed=0):
    g = torch.Generator().manual_seed(seed)

    def n(*shape, scale=1.0, dt=BF16):
        return (scale * torch.randn(*shape, generator=g, dtype=F32)).to(dt)

    w = {"table": n(V, D), "w0": 1 + n(D, scale=0.1), "w1": 1 + n(D, scale=0.1), "w2": 1 + n(D, scale=0.1)}
    w["gate"] = n(*{"channel": (D,), "token": (T, 1), "full": (T, D)}[gate])
    for k, (a, b) in {"up": (D, F), "down": (F, D), "head": (D, V)}.items():
        w["W_" + k], w["A_" + k], w["B_" + k] = n(b, a, scale=a ** -0.5), n(r, a, scale=a ** -0.5), n(b, r, scale=r ** -0.5)
    ids = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    return w, ids, n(T, V)


def exact(w, ids, dz):
    """Gradients of <dz, logits> in 64 bits."""
    p = {k: v.double().requires_grad_() for k, v in w.items()}

    def norm(x, gain):
        return x * (x.square().mean(1, keepdim=True) + EPS).rsqrt() * gain

    def linear(x, k):
        return x @ p["W_" + k].T + S * (x @ p["A_" + k].T) @ p["B_" + k].T

    h = p["table"][ids.long()]
    y = linear(linear(norm(h, p["w0"]), "up"), "down")
    h1 = h + RES * p["gate"] * norm(y, p["w2"])
    (linear(norm(h1, p["w1"]), "head") * dz.double()).sum().backward()
    return {k: v.grad for k, v in p.items()}


class Step:
    """The same on the GPU: every buffer made once, `run` only calls."""

    def __init__(self, w, ids, dz, rt):
        self.w, self.ids, self.dz = {k: v.cuda() for k, v in w.items()}, ids.cuda(), dz.cuda()
        (T,), (V, D), F, r = ids.shape, w["table"].shape, w["W_up"].shape[0], w["A_up"].shape[0]

        def e(*shape, dt=BF16):
            return torch.empty(*shape, dtype=dt, device="cuda")

        self.e, self.h0, self.h1 = e(T, D), e(T, D, dt=rt), e(T, D, dt=rt)
        self.n0, self.z, self.y, self.n1, self.logits = e(T, D), e(T, F), e(T, D), e(T, D), e(T, V)
        self.r0, self.r1, self.r2 = (e(T, dt=F32) for _ in range(3))
        self.k = {k: lm.act8_empty(T, d) for k, d in (("n0", D), ("z", F), ("y", D), ("h1", D), ("n1", D))}
        self.dn1, self.dy, self.dz1, self.dn0 = e(T, D), e(T, D), e(T, F), e(T, D)
        self.dh = e(T, D, dt=rt)
        self.dh0 = self.dh if rt == BF16 else e(T, D)
        self.g = {"w0": e(D, dt=F32), "w1": e(D, dt=F32), "w2": e(D, dt=F32), "table": e(V, D, dt=F32)}
        gate = self.w["gate"]
        self.g["gate"] = torch.empty_like(gate) if gate.shape == (T, D) and gate.shape != (T, 1) else e(*gate.shape, dt=F32)
        for k, a, b in (("up", D, F), ("down", F, D), ("head", D, V)):
            self.g["A_" + k], self.g["B_" + k] = e(r, a, dt=F32), e(b, r, dt=F32)
        n = max(lm.lora_linear_workspace_bytes(lm.LORA_OP_FWD, T, a, b, r, lm.LORA_BF16) for a, b in ((D, F), (F, D), (D, V)))
        n = max([n] + [lm.lora_linear_x8_workspace_bytes(T, a, b, r) for a, b in ((D, F), (F, D), (D, V))])
        n = max(n, lm.block_norm_workspace_bytes(T, D), lm.embed_bwd_workspace_bytes(T, V, D))
        self.ws = e(n, dt=torch.uint8)

    def forward(self):
        w, k, ws = self.w, self.k, self.ws
        lm.embed_fwd(w["table"], self.ids, self.e)
        self.h0.copy_(self.e)
        lm.block_norm_fwd(self.h0, n=self.n0, w_pre=w["w0"], rstd_pre=self.r0, n8=k["n0"], eps=EPS)
        lm.lora_linear_fwd(self.n0, w["W_up"], w["A_up"], w["B_up"], self.z, scale=S, ws=ws)
        lm.act8_quantize(self.z, k["z"])
        lm.lora_linear_fwd(self.z, w["W_down"], w["A_down"], w["B_down"], self.y, scale=S, ws=ws)
        lm.block_norm_fwd(self.h0, self.y, h_out=self.h1, n=self.n1, w_post=w["w2"], w_pre=w["w1"], gate=w["gate"], rstd_pre=self.r1,
                          rstd_post=self.r2, y8=k["y"], h8=k["h1"], n8=k["n1"], eps=EPS, res_scale=RES)
        lm.lora_linear_fwd(self.n1, w["W_head"], w["A_head"], w["B_head"], self.logits, scale=S, ws=ws)

    def backward(self):
        w, k, g, ws = self.w, self.k, self.g, self.ws
        lm.lora_linear_bwd_x8(k["n1"], w["W_head"], w["A_head"], w["B_head"], None, self.dz, self.dn1, g["A_head"], g["B_head"], S, ws=ws)
        lm.block_norm_bwd(self.dn1, None, k["h1"], k["y"], dh=self.dh, dy=self.dy, w_pre=w["w1"], w_post=w["w2"], gate=w["gate"],
                          rstd_pre=self.r1, rstd_post=self.r2, dw_pre=g["w1"], dw_post=g["w2"], dgate=g["gate"], res_scale=RES, ws=ws)
        lm.lora_linear_bwd_x8(k["z"], w["W_down"], w["A_down"], w["B_down"], None, self.dy, self.dz1, g["A_down"], g["B_down"], S, ws=ws)
        lm.lora_linear_bwd_x8(k["n0"], w["W_up"], w["A_up"], w["B_up"], None, self.dz1, self.dn0, g["A_up"], g["B_up"], S, ws=ws)
        lm.block_norm_bwd(self.dn0, self.dh, self.h0, dh=self.dh, w_pre=w["w0"], rstd_pre=self.r0, dw_pre=g["w0"], ws=ws)
        if self.dh0 is not self.dh:
            self.dh0.copy_(self.dh)
        lm.embed_bwd(self.ids, self.dh0, g["table"], ws=ws)


# Norm-wise: a value stored in bf16 is off by 2^-8 of it at most, and 14 stand between the table and its
# gradient; a value in 8 bits by half a scale, at most 4 / 254 of a group's root mean square where none is beyond
# four of them, and three copies enter a gradient (x, h, y).  Linears and norms of
# independent errors do not enlarge them.  14 / 256 + 12 / 254 = 0.102.
TOL = 14 / 256 + 12 / 254


def close(step, want):
    for k, got in step.g.items():
        err = (got.double().cpu() - want[k]).norm() / want[k].norm()
        assert err <= TOL, (k, float(err))


@pytest.mark.parametrize("T,D,F,V,r,rt,gate", [
    (1, 128, 264, 72, 4, BF16, "channel"), (61, 264, 520, 96, 8, BF16, "channel"), (203, 512, 1000, 520, 16, F32, "token"),
    (700, 256, 1032, 264, 13, F32, "full"), (1030, 520, 264, 128, 40, BF16, "full")])
def test_a_step_from_kept_bits(T, D, F, V, r, rt, gate):
    w, ids, dz = weights(T, D, F, V, r, gate)
    step = Step(w, ids, dz, rt)
    step.forward()
    step.backward()
    close(step, exact(w, ids, dz))


@pytest.mark.parametrize("T,D,F,V", [(61, 264, 520, 96), (700, 256, 520, 264)])
def test_the_step_as_two_graphs_on_one_workspace(T, D, F, V):
    """Forward and backward captured each for itself, with the workspace in common; replayed on new tokens and
    gradients, with eager steps in between."""
    w, ids, dz = weights(T, D, F, V, 8, "channel")
    step, eager = Step(w, ids, dz, F32), Step(w, ids, dz, F32)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        step.forward()
        step.backward()
    torch.cuda.synchronize()
    fwd, bwd = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(fwd):
        step.forward()
    with torch.cuda.graph(bwd):
        step.backward()
    for seed in range(4):
        _, ids, dz = weights(T, D, F, V, 8, "channel", seed=seed)
        for s in (step, eager):
            s.ids.copy_(ids)
            s.dz.copy_(dz)
        eager.forward()
        fwd.replay()
        eager.backward()
        bwd.replay()
        torch.cuda.synchronize()
        for k in eager.g:
            assert torch.equal(step.g[k], eager.g[k]), (seed, k)
        if seed == 3:
            close(step, exact(w, ids, dz))
