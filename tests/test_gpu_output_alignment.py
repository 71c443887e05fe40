"""Attention outputs that are 16-byte but not 32-byte aligned: every kernel and every way of merging split groups writes the same bits
as into an aligned buffer, and nothing in front of or behind its rows."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

SHIFT = 8                          # values: 16 bytes behind a boundary of 32


@pytest.fixture(scope="module")
def mods():
    import test_gpu_causal
    from paper_2410_11744_b200 import build
    build.build()
    from paper_2410_11744_b200 import binding, runner
    return binding, runner, test_gpu_causal


def _shifted(like):
    """(buffer, view of like's shape that starts 16 bytes behind a boundary of 32)"""
    import torch
    buf = torch.full((like.numel() + SHIFT + 64,), 7.0, dtype=like.dtype, device=like.device)
    assert buf.data_ptr() % 32 == 0
    view = buf[SHIFT:SHIFT + like.numel()].view(like.shape)
    assert view.data_ptr() % 32 == 16
    return buf, view


def _same(buf, view, want, rows):
    import torch
    torch.cuda.synchronize()
    assert torch.equal(view[:rows], want[:rows])
    assert (buf[:SHIFT] == 7.0).all() and (buf[SHIFT + rows * want[0].numel():] == 7.0).all()


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (8, 1, 64), (4, 4, 128)])
@pytest.mark.parametrize("contexts,ns", [([300, 0], [1, 2]), ([300, 0, 65], [1, 150, 300]), ([20000], [1]), ([9000, 50], [40, 1])])
@pytest.mark.parametrize("combine", [2, 0])
def test_causal_outputs(mods, hq, hkv, d, contexts, ns, combine):
    B, _, causal = mods
    B.dyspec_set_tuning(-1, 0, combine)
    try:
        c = causal.Chunk(B, d + hq, hq, hkv, d, contexts, ns, 128)
    finally:
        B.dyspec_set_tuning(-1, 0, 2)
    c.call()
    buf, view = _shifted(c.out)
    c.call(out=view)
    _same(buf, view, c.out, c.n)
    p = causal.Prompt(B, d + hq, hq, hkv, d, [n + 1 for n in ns])
    p.call()
    buf, view = _shifted(p.out)
    p.call(out=view)
    _same(buf, view, p.out, p.n)


@pytest.mark.parametrize("g,hkv,d", [(1, 4, 64), (8, 1, 128), (2, 2, 128), (4, 2, 64)])
@pytest.mark.parametrize("prefix,nodes", [([100, 7], [3, 5]), ([70, 500, 0], [300, 129, 90]), ([6000], [64]), ([5000, 900], [256, 20])])
@pytest.mark.parametrize("ctas,combine", [(0, 2), (0, 1), (0, 0), (3, 2), (0, 2 + 16 * 2)])
def test_tree_outputs(mods, g, hkv, d, prefix, nodes, ctas, combine):
    B, R, _ = mods
    from paper_2410_11744_b200 import workloads as wl
    rng = np.random.default_rng(5)
    w = wl.make_custom(60, g * hkv, hkv, d, prefix, [wl.random_tree(rng, n) for n in nodes])
    B.dyspec_set_tuning(-1, ctas, combine)
    try:
        b = R.DeviceBatch(w)
    finally:
        B.dyspec_set_tuning(-1, 0, 2)
    b.step()
    want = b.out
    buf, b.out = _shifted(want)
    b.step()
    _same(buf, b.out, want, b.total_nodes)
    if len(nodes) == 1:
        B.dyspec_set_default_shape(g * hkv, hkv, d, b.W)
        buf, view = _shifted(want)
        B.dyspec_tree_attention(b.q, b.k, b.v, prefix[0], b.bits, nodes[0], view)
        single = want.clone()
        B.dyspec_tree_attention(b.q, b.k, b.v, prefix[0], b.bits, nodes[0], single)
        _same(buf, view, single, b.total_nodes)
