"""Causal attention with all weights alike, where the softmax is exact: scores of 0 give exponentials of exactly 1, their sum counts the
keys, and V of multiples of 2^-7 sums without rounding.  The output is then the mean of the values that a row sees, rounded once: every
value of every row is compared with it bit for bit, so that an exponential off by 2^-14 shows through the output's 2^-8."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    import test_gpu_causal
    from paper_2410_11744_b200 import build
    build.build()
    from paper_2410_11744_b200 import binding
    return binding, test_gpu_causal


def _check_means(out, v, context):
    """out [n][Hq][D] (bf16) against the running means of v [context + n][Hkv][D]."""
    import torch
    n, hq, d = out.shape
    sums = v.double().cumsum(dim=0)[context:]
    assert sums.abs().max() * 128 < 2 ** 24                       # exact in fp32, in whatever order
    mean = sums / torch.arange(context + 1, context + n + 1, device=v.device, dtype=torch.float64)[:, None, None]
    mean = mean.repeat_interleave(hq // v.shape[1], dim=1)
    # The kernels multiply the sum with 1 / count, each within 2^-22: a mean that close to the middle of two bf16 values may go either way.
    lo, hi = (mean * (1 - 2.0 ** -21)).to(torch.bfloat16), (mean * (1 + 2.0 ** -21)).to(torch.bfloat16)
    assert ((out == lo) | (out == hi)).all()
    return int((lo == hi).sum())


def _values(gen, *shape):
    import torch
    return (torch.randint(-255, 256, shape, generator=gen, device="cuda").float() / 128.0).to(torch.bfloat16)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (8, 1, 64), (4, 4, 128)])
@pytest.mark.parametrize("contexts,ns", [([1500, 0, 77], [300, 700, 1]), ([700, 3000], [1, 3]), ([9000], [130])])
def test_uniform_weights_give_the_rounded_mean(mods, hq, hkv, d, contexts, ns):
    import torch
    B, causal = mods
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d + hq)
    c = causal.Chunk(B, d, hq, hkv, d, contexts, ns, 128)
    p = causal.Prompt(B, d, hq, hkv, d, [x + 200 for x in ns])
    c.q[:], p.q[:] = 0.0, 0.0
    for rows in c.seq_rows:
        c.v[rows] = _values(gen, len(rows), hkv, d)
    p.v.copy_(_values(gen, *p.v.shape))
    c.call()
    p.call()
    torch.cuda.synchronize()
    at = decided = 0
    for r, (context, n) in enumerate(zip(contexts, ns)):
        decided += _check_means(c.out[at:at + n], c.v[c.seq_rows[r]], context)
        at += n
    assert decided > 0.9 * c.n * hq * d
    at = 0
    for n in p.ns:
        _check_means(p.out[at:at + n], p.v[at:at + n], 0)
        at += n
    assert int(c.status.item()) == 0 and int(p.status.item()) == 0
