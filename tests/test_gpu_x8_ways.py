"""The LoRA backward from 8 bits on two streams at a time, and as two graphs that share a workspace, at sizes that
reach every way to dx, and every sum and meeting, that its plan knows."""
import pytest
import torch

import paper_2606_19528_amd as lm
from test_gpu_x8 import case, run

# few tokens in one part and in several (flags of the parts in the workspace), producers, rows with one sum of du
# and with several, u in one sum and in several, tokens in one range and in several
REPLAYED = [(1, 264, 256, 8, 16), (24, 1024, 4096, 16, 16), (128, 2048, 2056, 12, 16), (30, 2056, 2048, 64, 16), (300, 520, 264, 32, 16),
            (1040, 1032, 1032, 16, 16), (600, 264, 520, 33, 16), (24, 2048, 4096, 16, 4), (1891, 2048, 520, 16, 8)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,K,N,r,bits", REPLAYED)
def test_two_calls_at_once_and_replays(T, K, N, r, bits):
    """u saved in one call and recomputed in another; each call's values are its own, so that sums taken from
    the other call, or from an earlier replay, show."""
    calls = []
    for seed in range(2):
        inp, d, x8, xq, W, _ = case(T, K, N, r, bits=bits, seed=10 * seed)
        calls.append((d, x8, W, (xq @ inp["A"].double().T).float().cuda() if seed == 0 else None))
    n = lm.lora_linear_x8_workspace_bytes(T, K, N, r)
    wss = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in calls]
    want = [run(*c[:4], 1.0) for c in calls]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(4):
        both = []
        for c, ws, st in zip(calls, wss, streams):
            with torch.cuda.stream(st):  # (the outputs are made there too)
                both.append(run(*c, 1.0, ws=ws))
        got.append(both)
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for x, y in zip(g, want) for a, b in zip(x, y))
    graphs, outs = [], []
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(*c, 1.0, ws=wss[0]))
        graphs.append(g)
    for k in range(5):
        for o in outs:
            for t in o:
                t.zero_()
        if k == 3:
            wss[0].fill_(255)  # (what it holds does not matter)
        graphs[k % 2].replay()
        run(*calls[0], 1.0, ws=wss[1])
        graphs[1 - k % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(outs, want) for a, b in zip(x, y)), k
