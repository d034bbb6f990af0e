"""CPU tests of the host logic around the norms between blocks at the edges of its arguments (fake,
never-dereferenced pointers; refusals before any device work)."""
import os

import pytest

import paper_2606_19528_amd as lm
from test_block_api import EINVAL, bwd, fwd


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
