"""Random shapes of the append and causal-attention calls, against the formula in 64 bits (seeded; each seed is one batch)."""
import random

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

SHAPES = [(8, 8, 64), (8, 1, 64), (12, 3, 128), (4, 2, 64), (16, 2, 128), (6, 6, 128), (2, 1, 128)]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


@pytest.fixture(scope="module")
def mods():
    import test_gpu_append
    import test_gpu_causal
    from paper_2410_11744_b200 import build
    build.build()
    from paper_2410_11744_b200 import binding
    return binding, test_gpu_append, test_gpu_causal


@pytest.mark.parametrize("seed", range(30))
def test_random_chunks(mods, seed):
    B, _, causal = mods
    rng = random.Random(1000 + seed)
    hq, hkv, d = rng.choice(SHAPES)
    n_req = _log(rng, 1, 12)
    n_hi = rng.choice([1, 1, 4, 40, 300, 900])
    contexts = [rng.choice([0, _log(rng, 1, 3000)]) for _ in range(n_req)]
    ns = [rng.choice([0, 1, _log(rng, 1, n_hi), n_hi]) for _ in range(n_req)]
    B.dyspec_set_tuning(rng.choice([-1, -1, 0, 1]), rng.choice([0, 0, 0, 1, 7, 200]), rng.choice([2, 2, 0]))
    try:
        c = causal.Chunk(B, seed, hq, hkv, d, contexts, ns, rng.choice([128, 256, 1024]), q_scale=rng.choice([0.1, 1.0, 3.0]))
    finally:
        B.dyspec_set_tuning(-1, 0, 2)
    c.check_after_call(sample=40)
    want = c.out.clone()
    c.out[:c.n] = 0
    c.call()
    import torch
    torch.cuda.synchronize()
    assert torch.equal(c.out, want)


@pytest.mark.parametrize("seed", range(20))
def test_random_prompts(mods, seed):
    B, _, causal = mods
    rng = random.Random(2000 + seed)
    hq, hkv, d = rng.choice(SHAPES)
    ns = [rng.choice([0, 1, _log(rng, 1, 1500)]) for _ in range(_log(rng, 1, 10))]
    causal.Prompt(B, seed, hq, hkv, d, ns, fused=rng.random() < 0.5).check_after_call(sample=40)


@pytest.mark.parametrize("seed", range(30))
def test_random_appends(mods, seed):
    B, append, _ = mods
    rng = random.Random(3000 + seed)
    hq, hkv, d = rng.choice(SHAPES + [(5, 7, 64), (71, 9, 128)])
    n_req = _log(rng, 1, 60)
    contexts = [rng.choice([0, _log(rng, 1, 500)]) for _ in range(n_req)]
    ns = [rng.choice([0, 1, _log(rng, 1, 200)]) for _ in range(n_req)]
    if sum(ns) == 0:
        ns[0] = 3
    tree = rng.choice(["", "", "apart", "in_pages"])
    s = append._case(seed, hq, hkv, d, contexts, ns, rng.choice([1, 8, 128, 512]), rng.choice([0, 16, d // 2, d]), rng.random() < 0.5,
                     tree=tree, fused=rng.random() < 0.5, pad=rng.choice([0, 17]))
    append._check(B, s)
    assert int(s["status"].item()) == 0
