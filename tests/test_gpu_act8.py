"""Activations in 8 bits on the GPU against their definition: codes, scales and restored
values to the bit."""
import pytest
import torch

import block_reference as ref
import paper_2606_19528_amd as lm

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _activation(T, D, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, D, generator=g) * (torch.randn(T, 1, generator=g)).exp()
    return x.to(dtype)


def _round_trip(x):
    T, D = x.shape
    codes, scale = ref.act8(x)
    x8 = lm.act8_empty(T, D)
    x8[0].fill_(99)
    x8[1].fill_(-1.0)
    assert lm.act8_quantize(x.cuda(), x8) is x8
    assert torch.equal(x8[0].cpu(), codes)
    assert torch.equal(x8[1].cpu().nan_to_num(-1.0), scale.nan_to_num(-1.0))  # (no scale is -1)
    for dtype in (BF16, F32):
        out = torch.full((T, D), 7.0, dtype=dtype, device="cuda")
        lm.act8_dequantize(x8, out)
        wide = scale.repeat_interleave(128, 1)[:, :D] * codes.float()  # one fp32 product, as there
        assert torch.equal(out.cpu().nan_to_num(5.0), wide.to(dtype).nan_to_num(5.0))
    return x8


# (T, D): one group, short last groups, several rows of groups, more groups than the launch for few takes
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,D", [(1, 8), (1, 128), (3, 136), (7, 120), (64, 1000), (203, 4096), (1, 11008), (5, 16384),
                                 (1027, 2048), (517, 8200), (20001, 104)])
def test_codes_scales_and_values(T, D, dtype):
    x = _activation(T, D, dtype)
    x8 = _round_trip(x)
    err = (ref.act8_values(x8[0].cpu(), x8[1].cpu()) - x.double()).abs()
    half = x8[1].cpu().double().repeat_interleave(128, 1)[:, :D] / 2
    assert bool((err <= half * (1 + 2.0 ** -15)).all())  # (the scale's rounding, 2^-24 of 127 steps)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_halves(dtype):
    """Quotients on a half go away from zero; all of them occur where the largest is 127."""
    k = torch.arange(0, 127, dtype=F32)
    x = torch.zeros(4, 256)
    x[0, :127], x[0, 127] = k + 0.5, 127.0
    x[1, :127], x[1, 127] = -(k + 0.5), 127.0
    x[2, ::2], x[2, 1] = 0.5, -1.0  # half the largest: 63.5
    x[3] = torch.linspace(-1.0, 1.0, 256)
    _round_trip(x.to(dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_extremes(dtype):
    """Zeros, the largest and the smallest numbers, and values that are not finite, each in groups of
    their own and beside others."""
    big, small = torch.finfo(dtype).max, torch.finfo(dtype).tiny
    x = torch.zeros(12, 264)
    x[1] = -0.0
    x[2, 5] = big
    x[3] = -big
    x[4, :130] = small * torch.linspace(-1.0, 1.0, 130)  # below the normal numbers
    x[5, 3], x[5, 200] = torch.inf, 1.0
    x[6, 140], x[6, 2] = torch.nan, 3.0
    x[7, 263], x[7, 0] = -torch.inf, 2.0
    x[8, ::2] = 1e-38
    x[9] = 2.0 ** -60
    x[10] = 2.0 ** -61 * torch.linspace(0.0, 1.0, 264)
    x[11, 7], x[11, 8] = torch.nan, torch.inf
    x8 = _round_trip(x.to(dtype))
    bad = x8[1].isnan().cpu()
    assert bad.nonzero().tolist() == [[5, 0], [6, 1], [7, 2], [11, 0]]


def test_rows_behind_the_activation_stay():
    """What follows codes, scales and values in larger buffers is left as it was."""
    T, D = 37, 136
    x = _activation(T, D, BF16)
    codes = torch.full((T + 4, D), 77, dtype=torch.int8, device="cuda")
    scale = torch.full((T + 4, 2), 5.0, device="cuda")
    out = torch.full((T + 4, D), 3.0, dtype=BF16, device="cuda")
    x8 = (codes[:T], scale[:T])
    lm.act8_quantize(x.cuda(), x8)
    lm.act8_dequantize(x8, out[:T])
    assert bool((codes[T:] == 77).all()) and bool((scale[T:] == 5.0).all()) and bool((out[T:] == 3.0).all())


def test_stream_and_graph():
    """On a stream of the caller's, and captured: each replay takes the input as it is then."""
    T, D = 301, 1000
    x = _activation(T, D, BF16).cuda()
    x8, out = lm.act8_empty(T, D), torch.empty(T, D, dtype=BF16, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    lm.act8_quantize(x, x8, stream=st)
    lm.act8_dequantize(x8, out, stream=st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lm.act8_quantize(x, x8)
        lm.act8_dequantize(x8, out)
    for seed in range(4):
        x.copy_(_activation(T, D, BF16, seed))
        graph.replay()
        got = out.clone()
        codes, scale = ref.act8(x.cpu())
        torch.cuda.synchronize()
        assert torch.equal(x8[0].cpu(), codes) and torch.equal(x8[1].cpu(), scale)
        assert torch.equal(got.cpu(), (scale.repeat_interleave(128, 1)[:, :D] * codes.float()).to(BF16))
