"""CPU tests of the host logic around activations in 8 bits and the norms between blocks: sizes
rejected, workspaces, and refusals before any device work (fake, never-dereferenced pointers)."""
import ctypes
import math

import pytest
import torch

import paper_2606_19528_amd as lm
from paper_2606_19528_amd import lora as L

EINVAL, EUNSUP, EWS = L.LORA_EINVAL, L.LORA_EUNSUPPORTED, L.LORA_EWORKSPACE
BAD = ctypes.c_size_t(-1).value
NAN, INF = float("nan"), math.inf


def P(i, off=0):
    return 0x7F0000000000 + i * 0x1000000000 + off


def _run(fn, spec, kw):
    assert not set(kw) - set(spec), kw
    return fn(*{**spec, **kw}.values())


def quantize(**kw):
    return _run(lm.lib().act8_quantize, dict(x=P(1), codes=P(2), scale=P(3), T=64, D=200, dt=0, st=None), kw)


def dequantize(**kw):
    return _run(lm.lib().act8_dequantize, dict(codes=P(2), scale=P(3), x=P(1), T=64, D=200, dt=0, st=None), kw)


def block(**kw):
    b = dict(T=64, D=256, dt=0, res_dt=1, post_norm=1, gate_mode=1, gain_offset=0.0, res_scale=1.0, w_post=P(20), w_pre=P(21),
             gate=P(22))
    return {k: kw.pop(k, v) for k, v in b.items()}, kw


def k8(at):
    return None if at is None else ctypes.byref(L._Act8(*at))


def fwd(**kw):
    b, kw = block(**kw)
    spec = dict(h=P(1), y=P(2), h_out=P(3), n=P(4), r2=P(5), r1=P(6), y8=(P(7), P(8)), h8=(P(9), P(10)), n8=(P(11), P(12)), eps=1e-6,
                st=None)
    assert not set(kw) - set(spec), kw
    a = {**spec, **kw}
    for k in ("y8", "h8", "n8"):
        a[k] = k8(a[k])
    return lm.lib().block_norm_fwd(ctypes.byref(L._BlockNorm(**b)), *a.values())


def bwd(**kw):
    b, kw = block(**kw)
    spec = dict(dn=P(1), dho=P(2), h=P(3), h8=None, y=P(4), y8=None, r2=P(5), r1=P(6), dh=P(7), dy=P(8), dw1=P(9), dw2=P(10),
                dg=P(11), ws=P(12), wsb=1 << 24, st=None)
    assert not set(kw) - set(spec), kw
    a = {**spec, **kw}
    for k in ("y8", "h8"):
        a[k] = k8(a[k])
    return lm.lib().block_norm_bwd(ctypes.byref(L._BlockNorm(**b)), *a.values())


def x8(**kw):
    return _run(lm.lib().lora_linear_bwd_x8, dict(xc=P(1), xs=P(2), W=P(3), A=P(4), B=P(5), u=P(6), dy=P(7), dx=P(8), dA=P(9),
                                                  dB=P(10), T=64, K=256, N=512, r=8, s=1.0, ws=P(11), wsb=1 << 26, st=None), kw)


def x8q(**kw):
    return _run(lm.lib().lora_linear_bwd_q_x8, dict(xc=P(1), xs=P(2), W=P(3), ws_=P(12), wo=P(13), bits=4, group=64, A=P(4),
                                                    B=P(5), u=P(6), dy=P(7), dx=P(8), dA=P(9), dB=P(10), T=64, K=256, N=512, r=8,
                                                    s=1.0, ws=P(11), wsb=1 << 26, st=None), kw)


@pytest.mark.parametrize("fn,kw,code", [
    *[(f, kw, code) for f in (quantize, dequantize) for kw, code in (
        (dict(x=None), EINVAL), (dict(codes=None), EINVAL), (dict(scale=None), EINVAL), (dict(T=0), EINVAL), (dict(D=0), EINVAL),
        (dict(D=12), EUNSUP), (dict(D=1 << 21), EUNSUP), (dict(T=(1 << 28) + 1), EUNSUP), (dict(T=1 << 62), EUNSUP),
        (dict(dt=2), EINVAL), (dict(x=P(1, 8)), EINVAL), (dict(codes=P(2, 8)), EINVAL), (dict(scale=P(3, 4)), EINVAL),
        (dict(codes=P(1, 16)), EINVAL), (dict(x=P(3, -16)), EINVAL))],
    (quantize, dict(codes=P(3, -64 * 200 + 16)), EINVAL),
    (fwd, dict(h=None), EINVAL), (fwd, dict(y=None), EINVAL), (fwd, dict(eps=0.0), EINVAL), (fwd, dict(eps=NAN), EINVAL),
    (fwd, dict(eps=INF), EINVAL), (fwd, dict(eps=-1.0), EINVAL), (fwd, dict(T=0), EINVAL), (fwd, dict(D=0), EINVAL),
    (fwd, dict(D=20), EUNSUP), (fwd, dict(D=16392), EUNSUP), (fwd, dict(T=(1 << 22) + 1), EUNSUP), (fwd, dict(dt=3), EINVAL),
    (fwd, dict(res_dt=3), EINVAL), (fwd, dict(dt=1, res_dt=0), EUNSUP), (fwd, dict(gate_mode=4), EINVAL),
    (fwd, dict(gate_mode=-1), EINVAL), (fwd, dict(gate=None), EINVAL), (fwd, dict(gate_mode=0), EINVAL),
    (fwd, dict(post_norm=2), EINVAL), (fwd, dict(post_norm=0), EINVAL), (fwd, dict(post_norm=0, w_post=None), EINVAL),
    (fwd, dict(res_scale=NAN), EINVAL), (fwd, dict(gain_offset=INF), EINVAL), (fwd, dict(h=P(1, 8)), EINVAL),
    (fwd, dict(gate=P(22, 2)), EINVAL), (fwd, dict(w_pre=P(21, 8)), EINVAL), (fwd, dict(h_out=P(2)), EINVAL),
    (fwd, dict(n=P(1, 64)), EINVAL), (fwd, dict(h_out=P(1, 16)), EINVAL), (fwd, dict(n=P(3)), EINVAL), (fwd, dict(r1=P(5)), EINVAL),
    (fwd, dict(n8=(P(11), None)), EINVAL), (fwd, dict(y8=(None, P(8))), EINVAL), (fwd, dict(h8=(P(9), P(9, 16))), EINVAL),
    (fwd, dict(n8=(P(20), P(12))), EINVAL), (fwd, dict(n8=(P(11, 8), P(12))), EINVAL),
    (fwd, dict(h_out=None, n=None, r1=None, r2=None, y8=None, h8=None, n8=None), EINVAL),
    (fwd, dict(y=None, post_norm=0, w_post=None, r2=None, y8=None), EINVAL),  # a gate without a block
    (bwd, dict(dh=None), EINVAL), (bwd, dict(dn=None, dho=None), EINVAL), (bwd, dict(h=None), EINVAL), (bwd, dict(r1=None), EINVAL),
    (bwd, dict(r2=None), EINVAL), (bwd, dict(y=None), EINVAL), (bwd, dict(h8=(P(13), P(14))), EINVAL),
    (bwd, dict(y8=(P(13), P(14))), EINVAL), (bwd, dict(h=None, h8=(P(13), None)), EINVAL), (bwd, dict(dn=None), EINVAL),
    (bwd, dict(gate=None, gate_mode=0), EINVAL), (bwd, dict(post_norm=0, w_post=None), EINVAL), (bwd, dict(ws=None), EWS),
    (bwd, dict(wsb=64), EWS), (bwd, dict(ws=P(12, 4)), EINVAL), (bwd, dict(ws=P(7)), EINVAL), (bwd, dict(dh=P(1)), EINVAL),
    (bwd, dict(dh=P(2, 16)), EINVAL), (bwd, dict(dy=P(4)), EINVAL), (bwd, dict(dw1=P(10)), EINVAL), (bwd, dict(dg=P(22)), EINVAL),
    (bwd, dict(dw2=P(10, 4)), EINVAL), (bwd, dict(D=16400), EUNSUP), (bwd, dict(T=-3), EINVAL),
    *[(f, kw, code) for f in (x8, x8q) for kw, code in (
        (dict(xc=None), EINVAL), (dict(xs=None), EINVAL), (dict(W=None), EINVAL), (dict(A=None), EINVAL), (dict(B=None), EINVAL),
        (dict(dy=None), EINVAL), (dict(dA=None), EINVAL), (dict(dB=None), EINVAL), (dict(s=NAN), EINVAL), (dict(T=0), EINVAL),
        (dict(r=-1), EINVAL), (dict(r=129), EINVAL), (dict(K=12), EUNSUP), (dict(N=1 << 21), EUNSUP), (dict(T=1 << 30), EUNSUP),
        (dict(xc=P(1, 8)), EINVAL), (dict(xs=P(2, 4)), EINVAL), (dict(dx=P(7)), EINVAL), (dict(dA=P(1)), EINVAL),
        (dict(dB=P(2)), EINVAL), (dict(dA=P(10, 64)), EINVAL), (dict(ws=None), EWS), (dict(wsb=1024), EWS), (dict(ws=P(11, 8)), EINVAL),
        (dict(ws=P(8, 16)), EINVAL))],
    (x8q, dict(bits=5), EINVAL), (x8q, dict(group=24), EUNSUP), (x8q, dict(r=72), EUNSUP), (x8q, dict(wo=None), EINVAL),
    (x8, dict(r=0, dx=None), EINVAL),
])
def test_refusals(fn, kw, code):
    assert fn(**kw) == code
    assert lm.lib().lora_last_error()


def test_workspace_queries():
    lib = lm.lib()
    assert lib.block_norm_workspace_bytes(0, 64) == BAD and lib.block_norm_workspace_bytes(4, 12) == BAD
    assert lib.block_norm_workspace_bytes(4, 16392) == BAD
    for T, D in ((1, 8), (97, 1000), (4096, 2048), (16384, 16384)):
        n = lib.block_norm_workspace_bytes(T, D)  # a few hundred sums of a row, however many rows
        assert 2 * 4 * D <= n <= 2 * 4 * D * min(T + 3, 1024) + 256
    assert lib.lora_linear_x8_workspace_bytes(0, 64, 64, 8) == BAD and lib.lora_linear_x8_workspace_bytes(4, 64, 60, 8) == BAD
    assert lib.lora_linear_x8_workspace_bytes(4096, 64, 64, 0) == 0
    for T, K, N, r in ((128, 256, 256, 8), (4096, 8192, 3072, 32), (1891, 2048, 11008, 16)):
        n = lib.lora_linear_x8_workspace_bytes(T, K, N, r)
        assert n <= 2 * T * K + (1 << 20)  # less than a bf16 copy of x
    with pytest.raises(lm.LoraError):
        lm.block_norm_workspace_bytes(1, 4)
    with pytest.raises(lm.LoraError):
        lm.lora_linear_x8_workspace_bytes(1, 4, 8, 8)


def _nodes(*dims, r=8, **kw):
    arr = (L._Node * (len(dims) - 1))()
    for i in range(len(dims) - 1):
        arr[i] = L._Node(P(20 + 5 * i), P(21 + 5 * i), P(22 + 5 * i), P(23 + 5 * i), P(24 + 5 * i), dims[i], dims[i + 1], r, 1.0)
    return arr


def test_chain_refusals_and_sizes():
    lib = lm.lib()
    T, dims = 128, (256, 512, 264, 256)
    nodes = _nodes(*dims)
    host, ws = lib.lora_ckpt_host_bytes_x8(nodes, 3, T), lib.lora_ckpt_workspace_bytes_x8(nodes, 3, T)
    kept = sum(T * d + 4 * T * -(-d // 128) for d in dims[:-1])
    assert kept <= host <= kept + 6 * 256
    assert ws < lib.lora_ckpt_workspace_bytes(nodes, 3, T) and host < 0.54 * lib.lora_ckpt_host_bytes(nodes, 3, T)
    assert lib.lora_ckpt_host_bytes_x8(_nodes(*dims, r=0), 3, T) == 0
    broken = _nodes(*dims)
    broken[1].d_in = 520
    assert lib.lora_ckpt_workspace_bytes_x8(broken, 3, T) == BAD and lib.lora_ckpt_host_bytes_x8(nodes, 0, T) == BAD
    for fn in (lib.lora_ckpt_forward_x8, lib.lora_ckpt_backward_x8):
        def call(arr=nodes, n=3, a=P(1), b=P(2), stash=P(3), hb=host, w=P(4), wb=ws):
            return fn(arr, n, T, a, b, stash, hb, w, wb, None, None)
        assert call(n=0) == EINVAL and call(arr=broken) == EINVAL and call(a=None) == EINVAL
        assert call(stash=None) == EWS and call(hb=host - 1) == EWS and call(w=None) == EWS and call(wb=ws - 1) == EWS
        assert call(w=P(4, 16)) == EINVAL
        bare = _nodes(*dims)
        bare[2].dB = None
        assert call(arr=bare) == EINVAL
    assert lib.lora_ckpt_forward_x8(nodes, 3, T, P(1), None, P(3), host, P(4), ws, None, None) == EINVAL


# ---- the binding: what it refuses itself ---------------------------------------------
class _T:
    """What the binding reads of a tensor on GPU 0."""

    def __init__(self, *shape, dtype=torch.bfloat16, contiguous=True, device=0):
        self.shape, self.dtype, self._c, self._d = torch.Size(shape), dtype, contiguous, device

    def is_contiguous(self):
        return self._c

    def get_device(self):
        return self._d

    def data_ptr(self):
        return 0x1000

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize


F32, BF16, I8 = torch.float32, torch.bfloat16, torch.int8


@pytest.fixture
def gpu0(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)


def _pair(T, D, dtype=I8, groups=None, **kw):
    return _T(T, D, dtype=dtype, **kw), _T(T, -(-D // 128) if groups is None else groups, dtype=F32, **kw)


@pytest.mark.parametrize("x,x8,error", [
    (_T(4, 136, dtype=torch.float16), _pair(4, 136), TypeError), (_T(4, 136), _pair(4, 136, dtype=torch.uint8), TypeError),
    (_T(4, 136), _pair(4, 136, groups=1), ValueError), (_T(4, 136), _pair(5, 136), ValueError),
    (_T(4, 136, contiguous=False), _pair(4, 136), ValueError), (_T(4, 136, device=-1), _pair(4, 136), ValueError),
    (_T(4, 136, device=1), _pair(4, 136), ValueError), (_T(4, 136), _pair(4, 136, device=1), ValueError),
])
def test_binding_refuses_activations(gpu0, x, x8, error):
    for call in (lambda: lm.act8_quantize(x, x8), lambda: lm.act8_dequantize(x8, x)):
        with pytest.raises(error):
            call()


@pytest.mark.parametrize("kw,error", [
    (dict(gate=_T(4)), ValueError), (dict(gate=_T(1, 136)), ValueError), (dict(gate=_T(136, dtype=F32)), TypeError),
    (dict(w_pre=_T(128)), ValueError), (dict(w_post=_T(136, dtype=F32)), TypeError), (dict(n=_T(4, 136, dtype=F32)), TypeError),
    (dict(n=_T(4, 136, contiguous=False)), ValueError), (dict(h_out=_T(4, 136, dtype=F32)), TypeError),
    (dict(rstd_pre=_T(4)), TypeError), (dict(rstd_pre=_T(4, 1, dtype=F32)), ValueError), (dict(n8=_pair(4, 128)), ValueError),
    (dict(y=_T(4, 136, device=1)), ValueError),
])
def test_binding_refuses_norm_arguments(gpu0, kw, error):
    with pytest.raises(error):
        lm.block_norm_fwd(_T(4, 136), **{"y": _T(4, 136), "n": _T(4, 136), **kw})


@pytest.mark.parametrize("kw,error", [
    (dict(dgate=_T(136, dtype=F32)), ValueError), (dict(gate=_T(136), dgate=_T(136)), TypeError),
    (dict(gate=_T(4, 1), dgate=_T(4, dtype=F32)), ValueError), (dict(gate=_T(4, 136), dgate=_T(4, 136, dtype=F32)), TypeError),
    (dict(dw_pre=_T(136)), TypeError), (dict(dy=_T(4, 128)), ValueError), (dict(dh_out=_T(4, 136, dtype=F32)), TypeError),
])
def test_binding_refuses_norm_gradients(gpu0, kw, error):
    with pytest.raises(error):
        lm.block_norm_bwd(_T(4, 136), kw.pop("dh_out", None), _T(4, 136), _T(4, 136), dh=_T(4, 136),
                          ws=_T(1 << 20, dtype=torch.uint8), rstd_pre=_T(4, dtype=F32), **kw)


@pytest.mark.parametrize("kw,error", [
    (dict(W=_T(64, 128)), ValueError), (dict(A=_T(8, 128)), ValueError), (dict(B=_T(64, 4)), ValueError),
    (dict(dx=_T(4, 136, dtype=F32)), TypeError), (dict(dA=_T(8, 136)), TypeError), (dict(u=_T(4, 4, dtype=F32)), ValueError),
    (dict(x8=_pair(3, 136)), ValueError), (dict(dy=_T(4, 64, contiguous=False)), ValueError),
])
def test_binding_refuses_linear_arguments(gpu0, kw, error):
    a = dict(x8=_pair(4, 136), W=_T(64, 136), A=_T(8, 136), B=_T(64, 8), u=None, dy=_T(4, 64), dx=None, dA=_T(8, 136, dtype=F32),
             dB=_T(64, 8, dtype=F32))
    with pytest.raises(error):
        lm.lora_linear_bwd_x8(*{**a, **kw}.values())
