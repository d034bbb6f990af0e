"""The plan of the LoRA backward from 8 bits: its query, and that the sizes which the GPU tests run reach every way that
the plan knows (host logic, no GPU)."""
import ctypes

import pytest

import paper_2606_19528_amd as lm
from paper_2606_19528_amd import lora as L
from test_gpu_x8 import SIZES
from test_gpu_x8_ways import REPLAYED


def test_query():
    none = dict(few_tokens=0, few_parts=0, fused=0, du_parts=0, u_parts=0, token_ranges=0)
    assert lm.lora_linear_x8_plan(24, 264, 136, 0) == none
    p = lm.lora_linear_x8_plan(24, 1024, 4096, 16)
    assert p["few_tokens"] == 1 and p["few_parts"] > 1 and p["fused"] == p["du_parts"] == 0 and p["token_ranges"] == 1
    p = lm.lora_linear_x8_plan(24, 1024, 4096, 16, quantized=True)  # (no few-token kernel over a quantized base)
    assert p["few_tokens"] == p["few_parts"] == p["fused"] == 0 and p["du_parts"] >= 1
    p = lm.lora_linear_x8_plan(24, 1024, 4096, 16, want_dx=False)
    assert p["few_tokens"] == p["fused"] == 0 and p["du_parts"] >= 1
    plan, fn = L._X8Plan(), lm.lib().lora_linear_x8_plan
    for args, code in (((0, 128, 128, 8, 0, 1), L.LORA_EINVAL), ((64, 100, 128, 8, 0, 1), L.LORA_EUNSUPPORTED),
                       ((64, 128, 128, 8, 2, 1), L.LORA_EINVAL), ((64, 128, 128, 8, 0, -1), L.LORA_EINVAL),
                       ((64, 128, 128, 72, 1, 1), L.LORA_EUNSUPPORTED), ((64, 128, 128, 129, 0, 1), L.LORA_EINVAL)):
        assert fn(*args, ctypes.byref(plan)) == code, args
    assert fn(64, 128, 128, 8, 0, 1, None) == L.LORA_EINVAL


def ways(sizes):
    """What the calls of these sizes run: dx's kernel, and its sums and meetings."""
    seen = set()
    for T, K, N, r, bits in sizes:
        p = lm.lora_linear_x8_plan(T, K, N, r, quantized=bits != 16)
        if p["few_tokens"]:
            seen.add(("few tokens", "parts" if p["few_parts"] > 1 else "one part"))
            seen.add(("few tokens", "65 and more" if T > 64 else "up to 64", "33 ranks and more" if r > 32 else "up to 32 ranks"))
        elif p["fused"]:
            seen.add(("producers",))
        else:
            seen.add(("rows", "sums" if p["du_parts"] > 1 else "one sum"))
        seen.add(("u", "sums" if p["u_parts"] > 1 else "one sum"))
        seen.add(("tokens", "ranges" if p["token_ranges"] > 1 else "one range"))
    return seen


EVERY = {("few tokens", "parts"), ("few tokens", "one part"), ("few tokens", "65 and more", "up to 32 ranks"),
         ("few tokens", "up to 64", "up to 32 ranks"), ("producers",), ("rows", "sums"), ("rows", "one sum"), ("u", "sums"),
         ("u", "one sum"), ("tokens", "ranges"), ("tokens", "one range")}


@pytest.mark.parametrize("name,sizes", [("against the definition", [(*s, 16) for s in SIZES]), ("at once and replayed", REPLAYED)])
def test_the_sizes_reach_every_way(name, sizes):
    missing = EVERY - ways(sizes)
    assert not missing, missing


def test_two_blocks_of_ranks_in_the_few_token_kernel():
    assert ("few tokens", "up to 64", "33 ranks and more") in ways([(*s, 16) for s in SIZES])


def test_few_tokens_or_producers():
    """65 to 128 tokens over a W of fewer than 2^22 weights: the few-token kernel, but producers where they are and measured
    faster, at more than 16 ranks and reductions of middle length."""
    for K, N, r, few in ((256, 256, 8, 1), (1024, 1024, 16, 1), (1024, 1024, 20, 1), (1024, 1024, 32, 0), (2048, 768, 24, 0),
                         (256, 640, 32, 0), (1024, 512, 32, 1), (1024, 1536, 32, 1), (512, 4096, 32, 1)):
        for T in (72, 128):
            p = lm.lora_linear_x8_plan(T, K, N, r)
            assert p["few_tokens"] == few and p["fused"] == 1 - few, (T, K, N, r, p)
