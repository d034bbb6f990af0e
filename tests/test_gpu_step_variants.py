"""Each variant of the kernels around the linears at sizes that only it takes, and where
its workgroups go on to further rows: the checks of test_gpu_tokenloss and
test_gpu_embed at more shapes."""
import pytest
import torch

import test_gpu_embed as embed
import test_gpu_tokenloss as loss

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


# Rows kept by 64 threads (4096 workgroups at most), by 256 with 8 and with 16 vectors each
# (1024), by 1024 with 8 and with 16 (256): more rows than workgroups, a third of them masked.
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("T,V,ld", [(4200, 77, 80), (1100, 5000, 5000), (1100, 8200, 8200), (1100, 20000, 20000),
                                    (300, 32001, 32008), (600, 40001, 40008)])
def test_policy_rows(T, V, ld, dt):
    loss.test_policy((T, V, ld), 0.25, dt)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_preference_rows(dt):
    loss.test_preference((1100, 8200, 8200), 3, 0.1, dt)


# Both sides of where the search takes 8 positions a workgroup instead of 4, its largest
# size, the dense form cleared ahead of the sums (256 MB), sorts of one pass and of three.
@pytest.mark.parametrize("T,V,D,kind", [(4096, 700, 16, "text"), (4097, 700, 16, "text"), (8192, 700, 16, "text"),
                                        (8192, 9, 24, "edges"), (40, 131072, 512, "uniform"), (3001, 131072, 512, "text"),
                                        (9000, 511, 16, "outside"), (8193, 100, 24, "text"), (8200, 511, 8, "same"),
                                        (8193, 270000, 16, "edges")])
def test_embedding_gradients(T, V, D, kind):
    embed.test_gradient((T, V, D), kind)
