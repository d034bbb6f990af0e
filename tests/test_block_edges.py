"""CPU tests of the host logic around the norms between blocks at the edges of its arguments (fake,
never-dereferenced pointers; refusals before any device work)."""
import os
from types import SimpleNamespace

import pytest
import torch

import paper_2606_19528_amd as lm
from paper_2606_19528_amd import lora as L
from test_block_api import EINVAL, _pair, _T, bwd, fwd, gpu0  # noqa: F401 (gpu0: a fixture)


@pytest.mark.parametrize("fn,kw", [(fwd, dict(res_scale=1e39)), (fwd, dict(gain_offset=-1e39)), (bwd, dict(res_scale=1e39)),
                                   (bwd, dict(gain_offset=1e300)), (fwd, dict(eps=1e39)), (fwd, dict(eps=0.99e-30))])
def test_scalars_outside_32_bits(fn, kw):
    """They are given in 64 bits; rows of bf16 values and gradients take them in 32."""
    assert fn(**kw) == EINVAL
    assert lm.lib().lora_last_error()



def test_launches_leave_no_error_behind():
    """A launch that fails says so by what hipGetLastError returns, which also clears it: peeked at, it would be the
    next call's failure too.  (Without a GPU the runtime answers every question with an error, and with one no launch
    of an accepted call fails, so this reads the sources.)"""
    csrc = os.path.join(os.path.dirname(lm.__file__), "csrc")
    for name in sorted(os.listdir(csrc)):
        with open(os.path.join(csrc, name)) as f:
            assert "hipPeekAtLastError" not in f.read(), name


F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("kw,dt", [
    (dict(y=_T(4, 136), w_post=_T(136), rstd_post=_T(4, dtype=F32), dw_post=_T(136, dtype=F32)), BF16),
    (dict(y=_pair(4, 136), w_post=_T(136), rstd_post=_T(4, dtype=F32), dw_post=_T(136, dtype=F32)), BF16),
    (dict(y=_T(4, 136), post_norm=True, rstd_post=_T(4, dtype=F32), dw_post=_T(136, dtype=F32)), BF16),
    (dict(y=_T(4, 136, dtype=F32), post_norm=True, rstd_post=_T(4, dtype=F32), dw_post=_T(136, dtype=F32)), F32),
    (dict(), F32),
])
def test_any_tensor_names_the_type(gpu0, monkeypatch, kw, dt):  # noqa: F811
    """The gradient of a post norm's gain alone, through an fp32 stream: the block's type is that of y or of the
    gain where neither dn, dy, w_pre nor a gate is given."""
    seen = []

    class Lib:
        @staticmethod
        def block_norm_bwd(b, *args):
            seen.append(b._obj)
            return 0

    monkeypatch.setattr(L, "lib", lambda: Lib)
    lm.block_norm_bwd(None, _T(4, 136, dtype=F32), None, dh=_T(4, 136, dtype=F32), ws=_T(1 << 20, dtype=torch.uint8), stream=SimpleNamespace(cuda_stream=0), **kw)
    assert seen[0].dt == {BF16: lm.LORA_BF16, F32: lm.LORA_F32}[dt] and seen[0].res_dt == lm.LORA_F32
