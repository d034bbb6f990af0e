"""Workspaces of the embedding gradient, with and without a sort (host logic)."""
import pytest

import paper_2606_19528_amd as lm


@pytest.mark.parametrize("D", [64, 2048])
@pytest.mark.parametrize("V", [900, 128256])
def test_embedding_gradient(V, D):
    # searched: slots for an eighth of the positions' fp32 rows, and three words a position
    for T in (1, 4096, 8192):
        n = lm.embed_bwd_workspace_bytes(T, V, D)
        assert T * D // 2 <= n <= T * D // 2 + 4 * D + 16 * T + (1 << 12)
    # sorted: two keys, two positions and a number a position, a chunk's sum for 32 of them,
    # and the tiles' counts (512 for 1024 positions)
    for T in (8193, 100000):
        n = lm.embed_bwd_workspace_bytes(T, V, D)
        assert 20 * T + T * D // 8 <= n <= 24 * T + T * D // 8 + 4 * D + (1 << 13)
    # a vocabulary whose bitmap does not fit is sorted with few positions too
    assert lm.embed_bwd_workspace_bytes(4096, 300000, D) >= 20 * 4096
