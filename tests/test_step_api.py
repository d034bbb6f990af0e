"""CPU tests of the host logic around the embedding, loss and clipping entry points:
sizes rejected, workspaces, and refusals before any device work (fake,
never-dereferenced pointers)."""
import ctypes
import math

import pytest

import paper_2606_19528_amd as lm
from paper_2606_19528_amd import lora as L

EINVAL, EUNSUP, EWS = L.LORA_EINVAL, L.LORA_EUNSUPPORTED, L.LORA_EWORKSPACE
BAD = ctypes.c_size_t(-1).value


def P(i, off=0):
    return ctypes.c_void_p(0x7F0000000000 + i * 0x1000000000 + off)


def _run(fn, spec, kw):
    a = dict(spec)
    a.update(kw)
    return fn(*a.values())


def embed_fwd(**kw):
    return _run(lm.lib().embed_fwd, dict(table=P(1), ids=P(2), out=P(3), T=64, V=100, D=64, scale=1.0, dt=0, st=None), kw)


def embed_bwd(**kw):
    return _run(lm.lib().embed_bwd, dict(ids=P(2), dout=P(3), dtable=P(4), T=64, V=100, D=64, scale=1.0, acc=0, dt=0, ws=P(5),
                                         wsb=1 << 24, st=None), kw)


def embed_rows(**kw):
    return _run(lm.lib().embed_bwd_rows, dict(ids=P(2), dout=P(3), tokens=P(6), rows=P(4), T=64, V=100, D=64, scale=1.0, dt=0,
                                              ws=P(5), wsb=1 << 24, st=None), kw)


def logp(**kw):
    return _run(lm.lib().token_logp, dict(z=P(1), ld=104, y=P(2), w=P(3), logp=P(4), T=64, V=100, dt=0, ws=P(5), wsb=1 << 24,
                                          st=None), kw)


def policy(**kw):
    return _run(lm.lib().policy_loss, dict(z=P(1), ld=104, y=P(2), w=P(3), adv=P(6), old=P(7), ref=P(8), loss=P(9), logp=P(4),
                                           dz=P(10), T=64, V=100, lo=0.2, hi=0.2, kl=0.1, dt=0, ws=P(5), wsb=1 << 24, st=None), kw)


def pref(**kw):
    return _run(lm.lib().preference_loss, dict(z=P(1), ld=104, y=P(2), w=P(3), ref=P(8), seq=P(11), pairs=3, loss=P(9),
                                               margins=P(12), logp=P(4), dz=P(10), T=64, V=100, beta=0.1, eps=0.0, dt=0,
                                               ws=P(5), wsb=1 << 24, st=None), kw)


NAN, INF = float("nan"), math.inf


@pytest.mark.parametrize("fn,kw,code", [
    (embed_fwd, dict(table=None), EINVAL), (embed_fwd, dict(ids=None), EINVAL), (embed_fwd, dict(out=None), EINVAL),
    (embed_fwd, dict(T=0), EINVAL), (embed_fwd, dict(V=0), EINVAL), (embed_fwd, dict(D=0), EINVAL),
    (embed_fwd, dict(D=12), EUNSUP), (embed_fwd, dict(D=1 << 21), EUNSUP), (embed_fwd, dict(dt=5), EINVAL),
    (embed_fwd, dict(scale=NAN), EINVAL), (embed_fwd, dict(out=P(3, 8)), EINVAL), (embed_fwd, dict(out=P(1, 64)), EINVAL),
    (embed_fwd, dict(T=(1 << 25) + 1, D=8), EUNSUP), (embed_fwd, dict(T=1 << 25, D=1 << 11), EUNSUP), (embed_fwd, dict(V=1 << 40), EUNSUP),
    (embed_bwd, dict(ids=None), EINVAL), (embed_bwd, dict(dout=None), EINVAL), (embed_bwd, dict(dtable=None), EINVAL),
    (embed_bwd, dict(ws=None), EWS), (embed_bwd, dict(wsb=64), EWS), (embed_bwd, dict(ws=P(5, 4)), EINVAL),
    (embed_bwd, dict(scale=INF), EINVAL), (embed_bwd, dict(dtable=P(3, 16)), EINVAL), (embed_bwd, dict(ws=P(4, 16)), EINVAL),
    (embed_bwd, dict(D=20), EUNSUP), (embed_bwd, dict(T=1 << 30, D=1 << 11, V=8), EUNSUP),
    (embed_rows, dict(tokens=None), EINVAL), (embed_rows, dict(tokens=P(4)), EINVAL), (embed_rows, dict(rows=P(5)), EINVAL),
    (logp, dict(z=None), EINVAL), (logp, dict(y=None), EINVAL), (logp, dict(logp=None), EINVAL), (logp, dict(V=0), EINVAL),
    (logp, dict(T=-1), EINVAL), (logp, dict(V=105), EINVAL), (logp, dict(ld=100), EUNSUP), (logp, dict(ld=102, dt=1), EUNSUP),
    (logp, dict(dt=2), EINVAL), (logp, dict(z=P(1, 2)), EINVAL), (logp, dict(logp=P(3)), EINVAL), (logp, dict(T=(1 << 23) + 1), EUNSUP),
    (policy, dict(adv=None), EINVAL), (policy, dict(old=None), EINVAL), (policy, dict(loss=None), EINVAL),
    (policy, dict(ref=None), EINVAL), (policy, dict(lo=-0.1), EINVAL), (policy, dict(hi=NAN), EINVAL),
    (policy, dict(kl=INF), EINVAL), (policy, dict(ws=None), EWS), (policy, dict(wsb=8), EWS), (policy, dict(dz=P(1, 16)), EINVAL),
    (policy, dict(loss=P(4)), EINVAL), (policy, dict(adv=P(6, 4)), EINVAL), (policy, dict(T=0), EINVAL),
    (policy, dict(T=1 << 62), EUNSUP),
    (pref, dict(seq=None), EINVAL), (pref, dict(margins=None), EINVAL), (pref, dict(pairs=0), EINVAL), (pref, dict(beta=NAN), EINVAL),
    (pref, dict(eps=-0.1), EINVAL), (pref, dict(eps=1.1), EINVAL), (pref, dict(ws=None), EWS), (pref, dict(margins=P(9)), EINVAL),
    (pref, dict(dz=P(2)), EINVAL), (pref, dict(pairs=(1 << 22) + 1), EUNSUP), (pref, dict(ld=100), EUNSUP),
])
def test_refusals(fn, kw, code):
    assert fn(**kw) == code
    assert lm.lib().lora_last_error()


def test_workspace_queries():
    lib = lm.lib()
    assert lib.embed_bwd_workspace_bytes(0, 10, 8) == BAD and lib.embed_bwd_workspace_bytes(4, 10, 12) == BAD
    # sorted keys and positions, chunk sums: a few words a position and an eighth of the fp32 gradient rows
    T, D = 4096, 2048
    assert 4 * T <= lib.embed_bwd_workspace_bytes(T, 128256, D) <= 64 * T + T * D + (1 << 20)
    for op in range(3):
        assert lib.token_loss_workspace_bytes(op, 4096, 128256, 128256, 4, 0) <= 1 << 20  # no copy of the logits
    assert lib.token_loss_workspace_bytes(3, 4, 8, 8, 1, 0) == BAD
    assert lib.token_loss_workspace_bytes(2, 4, 8, 8, 0, 0) == BAD
    assert lib.token_loss_workspace_bytes(1, 4, 8, 9, 0, 0) == BAD


def _grads(*entries):
    arr = (L._Grad * len(entries))()
    for i, e in enumerate(entries):
        arr[i] = L._Grad(*e)
    return arr


def _init(arr, mem=P(15), nbytes=1 << 30, n=None):
    gl = L._GradList()
    return lm.lib().grad_list_init(ctypes.byref(gl), arr, len(arr) if n is None else n, mem, nbytes, None)


A, B = P(1).value, P(2).value


@pytest.mark.parametrize("entries,code", [
    ([(None, A, 8, 1, 1)], EINVAL), ([(A, B, -1, 1, 1)], EINVAL), ([(A, B, 8, 3, 1)], EINVAL), ([(A, B, 8, 1, 3)], EINVAL),
    ([(A + 4, B, 8, 1, 1)], EINVAL), ([(A, B + 8, 8, 1, 1)], EINVAL), ([(A, A, 8, 1, 0)], EINVAL),
    ([(A, A, 8, 1, 1), (A + 16, B, 8, 1, 1)], EINVAL),      # an in-place output overlaps another gradient
    ([(A, B, 8, 1, 1), (A + 64, B + 16, 8, 1, 1)], EINVAL),  # two outputs overlap
    ([(A, A + 16, 8, 1, 1)], EINVAL),                        # an output over its own gradient, shifted
    ([(A, B, 1 << 41, 1, 1)], EUNSUP),
    ([(P(15).value + 64, B, 8, 1, 1)], EINVAL),              # a gradient in the list's memory
])
def test_list_refusals(entries, code):
    assert _init(_grads(*entries)) == code


def test_list_memory():
    one = _grads((A, B, 8, 1, 1))
    need = lm.lib().grad_list_bytes(one, 1)
    assert need != BAD and _init(one, nbytes=need - 1) == EWS and _init(one, mem=None) == EWS
    assert _init(one, n=0) == EINVAL and lm.lib().grad_list_bytes(None, 1) == BAD
    many = _grads(*[(A + 4096 * i, B + 4096 * i, 1000, 1, 1) for i in range(392)])
    assert lm.lib().grad_list_bytes(many, 392) <= 1 << 20


def test_calls_on_a_list_that_was_not_laid_out():
    gl = L._GradList()
    assert lm.lib().grad_norm(ctypes.byref(gl), P(1), None) == EINVAL
    assert lm.lib().grad_clip(ctypes.byref(gl), 1.0, P(1), None) == EINVAL
    gl = L._GradList(P(3).value, 8, 1, 4096, 0)
    assert lm.lib().grad_clip(ctypes.byref(gl), 1.0, P(1), None) == EINVAL  # no outputs
    gl.has_out = 1
    assert lm.lib().grad_clip(ctypes.byref(gl), -1.0, P(1), None) == EINVAL
    assert lm.lib().grad_clip(ctypes.byref(gl), 1.0, P(3), None) == EINVAL  # norm inside the list's memory
    assert lm.lib().grad_clip(ctypes.byref(gl), 1.0, None, None) == EINVAL
