"""The 64-bit references that the append and causal-attention calls are tested with, against definitions written out by hand (CPU)."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from attention64 import causal, check, rope_table, rotate  # noqa: E402


def _bf16(gen, *shape):
    return torch.randn(shape, generator=gen).to(torch.bfloat16)


@pytest.mark.parametrize("hq,hkv,context", [(2, 2, 0), (4, 1, 3), (6, 3, 7)])
def test_causal_is_the_sum_over_keys_up_to_the_row(hq, hkv, context):
    gen = torch.Generator().manual_seed(hq + context)
    n, d = 5, 64
    q, k, v = _bf16(gen, n, hq, d), _bf16(gen, context + n, hkv, d), _bf16(gen, context + n, hkv, d)
    out, bound = causal(q, k, v, context)
    for i in range(n):
        for h in range(hq):
            keys = [k[t, h * hkv // hq].tolist() for t in range(context + i + 1)]
            w = [math.exp(sum(a * b for a, b in zip(q[i, h].tolist(), key)) / math.sqrt(d)) for key in keys]
            want = sum(x * v[t, h * hkv // hq].double() for t, x in enumerate(w)) / sum(w)
            assert torch.allclose(out[i, h], want, rtol=1e-12, atol=1e-14)
    rows, _ = causal(q, k, v, context, rows=[0, n - 1])
    assert torch.equal(rows, out[[0, n - 1]])
    assert (bound > 0).all() and (bound < 0.05).all()
    check(out.to(torch.bfloat16), out, bound)
    with pytest.raises(AssertionError):
        check(out + 2 * bound, out, bound)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 32)])
def test_rotation_turns_pairs_by_position_and_keeps_their_length(interleaved, d, rot):
    gen = torch.Generator().manual_seed(rot)
    table = rope_table(50, rot, device="cpu")
    x = _bf16(gen, 50, 3, d)
    y, _ = rotate(x, table, interleaved)
    assert torch.equal(y[..., rot:], x[..., rot:].double()) and torch.equal(y[0], x[0].double())
    for i in (0, rot // 2 - 1):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        angle = 17 * 10000.0 ** (-2.0 * i / rot)
        p, q = x[17, 1, a].double(), x[17, 1, b].double()
        assert abs(y[17, 1, a] - (p * math.cos(angle) - q * math.sin(angle))) < 1e-6
        assert abs(y[17, 1, b] - (q * math.cos(angle) + p * math.sin(angle))) < 1e-6
        assert abs(p * p + q * q - y[17, 1, a] ** 2 - y[17, 1, b] ** 2) < 1e-5
    # scores depend on the distance of two positions only
    u, w = x[:1].expand(50, 3, d), x[1:2].expand(50, 3, d)
    s = (rotate(u, table, interleaved)[0][5:45] * rotate(w, table, interleaved)[0][:40]).sum(-1)
    assert (s - s[0]).abs().max() < 1e-4
