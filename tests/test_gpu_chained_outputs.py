"""Attention outputs as inputs of the next attention call, the ways that the stream-order rule allows: through a copy, and through the
append (which takes them as q and k and writes q and the cache).  The chains run without any host synchronisation and in a
replayed graph, and give the bits of the same calls with the device idle between any two."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    import test_gpu_causal
    from paper_2410_11744_b200 import build
    build.build()
    from paper_2410_11744_b200 import binding, runner
    return binding, runner, test_gpu_causal


def _chain(steps, reset, result):
    """The result of `steps` one by one with the device idle in between, and without: five times in a row, and replayed."""
    import torch
    reset()
    for step in steps:
        torch.cuda.synchronize()
        step()
    torch.cuda.synchronize()
    want = result().clone()
    for _ in range(5):
        reset()
        for step in steps:
            step()
        torch.cuda.synchronize()
        assert torch.equal(result(), want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for step in steps:
                step()
    for _ in range(5):
        reset()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(result(), want)


@pytest.mark.parametrize("hq,hkv,d", [(8, 8, 128), (4, 4, 64), (8, 2, 128)])
@pytest.mark.parametrize("ns", [[3, 1], [150, 70], [900, 2]])
def test_prompt_outputs_through_a_copy(mods, hq, hkv, d, ns):
    """Six layers; with as many kv heads as heads the output is the next layer's q, k and v."""
    B, _, causal = mods
    p = causal.Prompt(B, d, hq, hkv, d, ns)
    start = [t.clone() for t in (p.q, p.k, p.v)]

    def reset():
        for t, s in zip((p.q, p.k, p.v), start):
            t.copy_(s)

    def onwards():
        p.q.copy_(p.out[:p.n])
        if hq == hkv:
            p.k.copy_(p.out[:p.n])
            p.v.copy_(p.out[:p.n])

    _chain([p.call, onwards] * 6, reset, lambda: p.out)


@pytest.mark.parametrize("ns", [[1, 1, 1], [4, 100, 33]])
def test_chunk_outputs_through_the_append(mods, ns):
    """The output is appended as the next step's keys and rotated as its queries, in place of a projection."""
    import torch
    from attention64 import rope_table
    B, _, causal = mods
    hq = hkv = 8
    c = causal.Chunk(B, 3, hq, hkv, 128, [300, 64, 5], ns, 128)
    rope = rope_table(1024, 128)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(ns)]), dtype=torch.int32, device="cuda")
    contexts = torch.tensor(c.contexts, dtype=torch.int32, device="cuda")
    first, k0 = c.q.clone(), c.k.clone()

    def reset():
        c.q.copy_(first)
        c.k.copy_(k0)
        c.out.fill_(0.0)

    def append():
        B.dyspec_append_kv_paged(c.out, c.v[:c.n], c.out, c.q, c.k, c.v2, c.rows, offsets, contexts, None, None, c.table, c.table.shape[1],
                                 128, rope, 1024, 128, False, c.n, len(ns), hq, hkv, 128, status=c.status)

    c.v2 = c.v.clone()                                   # (the values that the call writes are not looked at)
    _chain([c.call, append] * 5 + [c.call], reset, lambda: c.out)
    assert int(c.status.item()) == 0 and torch.isfinite(c.out[:c.n]).all()


def test_tree_outputs_through_a_copy(mods):
    B, R, _ = mods
    from paper_2410_11744_b200 import workloads as wl
    rng = np.random.default_rng(1)
    for prefix, nodes in (([100, 7], [20, 33]), ([900, 300], [200, 64]), ([4000], [64])):
        w = wl.make_custom(61, 8, 2, 128, prefix, [wl.random_tree(rng, n) for n in nodes])
        b = R.DeviceBatch(w)
        first = b.q.clone()
        _chain([b.step, lambda: b.q.copy_(b.out)] * 5, lambda: b.q.copy_(first), lambda: b.out)
        assert int(b.status.item()) == 0


def test_buffers_that_swap_roles(mods):
    """A buffer that one call reads and the next one writes needs nothing in between: writes wait for the calls in front."""
    import torch
    B, _, causal = mods
    p = causal.Prompt(B, 7, 8, 2, 128, [700, 3])
    q0, other = p.q.clone(), torch.zeros_like(p.q)

    def first():
        B.dyspec_prompt_attention(p.plan, p.q, p.k, p.v, other, p.ws, p.status, None)

    def second():                                        # overwrites the first call's q
        B.dyspec_prompt_attention(p.plan, q0, p.k, p.v, p.q, p.ws, p.status, None)

    _chain([first, second], lambda: p.q.copy_(q0), lambda: other)
    assert torch.equal(p.q, other)
