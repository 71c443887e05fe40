"""Causal attention of requests of more than 64 tokens, every value of every row against the formula in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu

SHAPES = [(8, 8, 64), (8, 1, 128), (4, 2, 128), (8, 2, 64), (4, 4, 128)]
ALL = 1 << 30


@pytest.fixture(scope="module")
def mods():
    import test_gpu_causal
    from paper_2410_11744_b200 import build
    build.build()
    from paper_2410_11744_b200 import binding
    return binding, test_gpu_causal


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("contexts,ns", [([700, 0, 129], [65, 300, 1]), ([0, 1000], [513, 200]), ([5000], [129])])
def test_chunks(mods, hq, hkv, d, contexts, ns):
    B, causal = mods
    causal.Chunk(B, hq + d, hq, hkv, d, contexts, ns, 128).check_after_call(sample=ALL)


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("fused", [False, True])
def test_prompts(mods, hq, hkv, d, fused):
    B, causal = mods
    causal.Prompt(B, hq + d, hq, hkv, d, [130, 2, 700, 256, 1501], fused).check_after_call(sample=ALL)


@pytest.mark.parametrize("combine,ctas", [(0, 0), (2, 7), (2, 400)])
def test_split_groups_and_short_queues(mods, combine, ctas):
    B, causal = mods
    B.dyspec_set_tuning(-1, ctas, combine)
    try:
        c = causal.Chunk(B, 3, 8, 2, 128, [6000, 0], [100, 300], 256)
        p = causal.Prompt(B, 3, 4, 2, 64, [900, 1100])
    finally:
        B.dyspec_set_tuning(-1, 0, 2)
    c.check_after_call(sample=ALL)
    p.check_after_call(sample=ALL)
