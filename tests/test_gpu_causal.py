"""Causal attention of chunks over a paged cache and of packed prompts, against the formula in 64 bits; every value within the
bound that the kernels' arithmetic has (attention64.causal)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available()
    from paper_2410_11744_b200 import build
    build.build()
    from paper_2410_11744_b200 import binding
    return binding


@pytest.fixture
def tuning(B):
    yield B.dyspec_set_tuning
    B.dyspec_set_tuning(-1, 0, 2)


def _bf16(gen, *shape, scale=1.0):
    import torch
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(torch.bfloat16)


def _zeros(*shape, dtype=None):
    import torch
    return torch.zeros(shape, dtype=dtype or torch.bfloat16, device="cuda")


def _workspace(plan):
    import torch
    return _zeros(max(256, plan.workspace_bytes()), dtype=torch.uint8)


class Chunk:
    """A batch of chunks over a pool whose rows that belong to nobody hold NaN, and whose pages are shuffled."""

    def __init__(self, B, seed, hq, hkv, d, contexts, ns, page, q_scale=1.0, extra=3, scale=0.0):
        import torch
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.B, self.shape, self.contexts, self.ns = B, (hq, hkv, d), contexts, ns
        need = [-(-(c + k) // page) for c, k in zip(contexts, ns)]
        ids = np.random.default_rng(seed).permutation(sum(need) + 2)
        table = np.full((len(ns), max(1, max(need))), -1, np.int32)
        self.seq_rows = []
        for r, k in enumerate(need):
            table[r, :k] = ids[sum(need[:r]):sum(need[:r + 1])]
            t = np.arange(contexts[r] + ns[r])
            self.seq_rows.append(torch.tensor(table[r][t // page].astype(np.int64) * page + t % page, device="cuda"))
        self.rows, self.n = (sum(need) + 2) * page, sum(ns)
        self.k, self.v = (torch.full((self.rows, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for rows in self.seq_rows:
            self.k[rows], self.v[rows] = _bf16(gen, len(rows), hkv, d), _bf16(gen, len(rows), hkv, d)
        self.q = _bf16(gen, self.n, hq, d, scale=q_scale)
        self.out = torch.full((self.n + extra, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
        self.table = torch.tensor(table, device="cuda")
        self.plan = B.dyspec_plan_create_chunk(hq, hkv, d, contexts, ns, self.rows, page, scale)
        self.scale = scale if scale > 0 else None
        self.ws, self.status = _workspace(self.plan), _zeros(1, dtype=torch.int32)

    def call(self, **over):
        a = dict(q=self.q, out=self.out, ws=self.ws, table=self.table, stream=None, q_stride=0)
        a.update(over)
        self.B.dyspec_chunk_attention_paged(self.plan, a["q"], self.k, self.v, a["table"], a["table"].shape[1], a["out"], a["ws"],
                                            self.status, a["stream"], a["q_stride"])

    def check(self, out=None, sample=64):
        """All rows of short chunks, `sample` rows (the first, the last, some between) of long ones."""
        import torch
        from attention64 import causal, check
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0
        out = self.out if out is None else out
        at = 0
        for r, (c, n) in enumerate(zip(self.contexts, self.ns)):
            if n:
                rows = None
                if n > sample:
                    rng = np.random.default_rng(r)
                    rows = sorted(set([0, 1, n - 2, n - 1] + [int(x) for x in rng.integers(0, n, sample)]))
                want, bound = causal(self.q[at:at + n], self.k[self.seq_rows[r]], self.v[self.seq_rows[r]], c, scale=self.scale, rows=rows)
                got = out[at:at + n]
                check(got if rows is None else got[rows], want, bound)
            at += n
        if len(out) > self.n:
            assert (out[self.n:] == 7.0).all()              # rows behind the last request are left as they were
        return self


SHAPES = [(8, 8, 64), (8, 1, 128), (4, 2, 128), (8, 2, 64), (32, 32, 128)]


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("page", [128, 512])
def test_single_tokens(B, hq, hkv, d, page):
    contexts = [0, 1, 62, 63, 64, 65, 127, 128, 129, 511, 512, 1000, 2047]
    Chunk(B, hq + d + page, hq, hkv, d, contexts, [1] * len(contexts), page).check_after_call()


Chunk.check_after_call = lambda self, **kw: (self.call(), self.check(**kw))[1]


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
def test_one_single_token(B, hq, hkv, d):
    for c in (0, 5, 300, 3000):
        Chunk(B, c + d, hq, hkv, d, [c], [1], 256).check_after_call()


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
def test_small_chunks_of_odd_sizes(B, hq, hkv, d):
    g = hq // hkv
    most = 64 // g
    Chunk(B, 3 * d + g, hq, hkv, d, [0, 63, 64, 500, 0, 129, 7], [most, 1, min(2, most), most - most // 3, 0, most, 1], 128).check_after_call()


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("page", [128, 1024])
def test_chunks_of_all_sizes(B, hq, hkv, d, page):
    ns = [1, 64, 65, 0, 127, 128, 129, 255, 257, 300]
    contexts = [700, 0, 1, 40, 128, 127, 129, 1000, 0, 384]
    Chunk(B, hq * 3 + d + page, hq, hkv, d, contexts, ns, page).check_after_call()


@pytest.mark.parametrize("ctas", [1, 3, 40])
def test_a_short_queue_of_few_ctas(B, tuning, ctas):
    tuning(-1, ctas, 2)
    Chunk(B, ctas, 8, 2, 128, [700, 0, 90, 1], [130, 300, 1, 77], 128).check_after_call()
    Chunk(B, ctas, 8, 8, 64, [700, 0, 90, 1], [130, 300, 1, 77], 128).check_after_call()


@pytest.mark.parametrize("regime", [0, 1])
def test_both_kernels_serve_any_size(B, tuning, regime):
    """The choice between them is one of speed: either answers chunks of every size."""
    tuning(regime, 0, 2)
    Chunk(B, 5 + regime, 16, 4, 128, [260, 0, 33], [1, 70, 200], 128).check_after_call()
    Chunk(B, 6 + regime, 4, 4, 64, [1300], [3], 128).check_after_call()


@pytest.mark.parametrize("regime,combine", [(0, 0), (0, 2), (1, 2)])
@pytest.mark.parametrize("hq,hkv,d,n", [(8, 1, 128, 1), (8, 2, 64, 9), (8, 1, 128, 40)])
def test_long_contexts_are_split_and_joined(B, tuning, regime, combine, hq, hkv, d, n):
    tuning(regime, 0, combine)
    c = Chunk(B, n + combine, hq, hkv, d, [9000, 20011], [n, 1], 256)
    assert c.plan.describe()["max_splits"] > 1
    c.check_after_call()


def test_large_scores_and_growing_maxima(B):
    """Rows whose maximum grows tile after tile (the output is rescaled), and scores of many units."""
    import torch
    for n, seed in ((1, 1), (200, 2)):
        c = Chunk(B, seed, 8, 2, 128, [1000], [n], 128, q_scale=4.0)
        ramp = torch.linspace(0.05, 2.0, 1000 + n, device="cuda")
        c.k[c.seq_rows[0]] = (c.k[c.seq_rows[0]].float() * ramp[:, None, None]).to(torch.bfloat16)
        c.check_after_call()


@pytest.mark.parametrize("scale", [0.01, 0.4, -1.0])
def test_a_scale_of_the_callers(B, scale):
    """Not 1 / sqrt(d); one that is not positive stands for that."""
    Chunk(B, 9, 8, 2, 128, [700, 3], [1, 2], 128, scale=scale).check_after_call()
    Chunk(B, 10, 8, 8, 64, [700, 0], [130, 70], 128, scale=scale).check_after_call()


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("n", [1, 200])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_beyond_2_to_the_30(B, hq, hkv, d, n, sign):
    """Scores of one product, sign * 2^40 * step(key): the softmax is 1 / ties on the keys of the largest one that a row sees.  Their weights
    are exactly 1, so the output is the mean of their values but for P's rounding, the fp32 sum's and the output's."""
    import torch
    context = 500
    c = Chunk(B, n, hq, hkv, d, [context], [n], 128)
    step = (torch.arange(context + n, device="cuda") // 90 % 5 + 1).float()           # 1 .. 5, in runs of 90 keys
    c.q[:], c.k[c.seq_rows[0]] = 0.0, 0.0
    c.q[:, :, 3] = sign * 2.0 ** 40
    c.k[c.seq_rows[0], :, 3] = step[:, None].to(torch.bfloat16)
    c.call()
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    v = c.v[c.seq_rows[0]].double()
    for i in {0, n // 2, n - 1}:
        seen = sign * step[:context + i + 1]
        ties = seen == seen.max()
        for h in range(hq):
            w = v[:context + i + 1][ties][:, h // (hq // hkv)]
            want, size = w.mean(dim=0), w.abs().mean(dim=0)
            bound = 2.0 ** -8 * (want.abs() + size) + 2.0 ** -15 * size + 2.0 ** -126
            assert ((c.out[i, h].double() - want).abs() <= bound).all()


def test_many_requests(B):
    rng = np.random.default_rng(4)
    ns = [int(x) for x in rng.integers(0, 3, 900)]
    Chunk(B, 11, 4, 2, 64, [int(x) for x in rng.integers(0, 200, 900)], ns, 128).check_after_call()
    ns[450] = 150                                                    # all of them on the tensor-core kernel
    Chunk(B, 12, 4, 2, 64, [int(x) for x in rng.integers(0, 200, 900)], ns, 128).check_after_call()


def test_strided_queries(B):
    import torch
    for ns in ([1, 1], [90, 200]):
        c = Chunk(B, 41, 8, 2, 128, [300, 64], ns, 128)
        wide = torch.full((c.n, 8 * 128 + 40), 3.0, dtype=torch.bfloat16, device="cuda")
        wide[:, :1024] = c.q.view(c.n, 1024)
        c.call(q=wide, q_stride=wide.stride(0))
        c.check()


def test_bad_pages_harm_no_other_request(B):
    """Page numbers outside the pool read as zeros."""
    import torch
    for ns in ([1, 1, 1], [1, 150, 70]):
        c = Chunk(B, 43, 8, 2, 128, [300, 200, 257], ns, 128)
        table = c.table.clone()
        for i, bad in enumerate((-1, c.rows // 128, 0x7fffffff)):
            table[1, 1] = bad
            c.call(table=table)
            torch.cuda.synchronize()
            assert torch.isfinite(c.out).all()
        c.out[ns[0]:ns[0] + ns[1]] = 0
        c.call()
        c.check()
        whole = c.out.clone()
        c.call(table=table)
        torch.cuda.synchronize()
        keep = [i for i in range(c.n) if not ns[0] <= i < ns[0] + ns[1]]
        assert torch.equal(c.out[keep], whole[keep])


def test_not_finite_neighbours_do_not_show(B):
    """Another request's NaN and infinities stay with that request, in the pool and in packed prompts."""
    import torch
    for ns in ([1, 1, 1], [64, 130, 50]):
        c = Chunk(B, 47, 8, 2, 128, [300, 200, 257], ns, 128)
        c.call()
        torch.cuda.synchronize()
        whole = c.out.clone()
        c.k[c.seq_rows[1]] = float("nan")
        c.v[c.seq_rows[1]] = float("inf")
        c.call()
        torch.cuda.synchronize()
        keep = [i for i in range(c.n) if not ns[0] <= i < ns[0] + ns[1]]
        assert torch.equal(c.out[keep], whole[keep])
        assert not torch.isfinite(c.out[ns[0]:ns[0] + ns[1]]).any()


def test_keys_in_a_pool_beyond_32_bit_offsets(B):
    import torch
    for n in (1, 90):
        c = Chunk(B, 53, 8, 8, 128, [300], [n], 256)
        pages = 2200000 // 256
        big = [torch.zeros((pages * 256, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        table = c.table.clone()
        for i in range(c.table.shape[1]):
            old, new = int(c.table[0, i]), pages - 1 - i
            table[0, i] = new
            big[0][new * 256:(new + 1) * 256] = c.k[old * 256:(old + 1) * 256]
            big[1][new * 256:(new + 1) * 256] = c.v[old * 256:(old + 1) * 256]
        c.call()
        torch.cuda.synchronize()
        want = c.out.clone()
        c.check()
        plan = B.dyspec_plan_create_chunk(8, 8, 128, [300], [n], pages * 256, 256)
        c.out.zero_()
        B.dyspec_chunk_attention_paged(plan, c.q, big[0], big[1], table, table.shape[1], c.out, _workspace(plan), c.status)
        torch.cuda.synchronize()
        assert torch.equal(c.out[:n], want[:n])


# ---- packed prompts ------------------------------------------------------------------------------------------------
class Prompt:
    def __init__(self, B, seed, hq, hkv, d, ns, fused=False):
        import torch
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.B, self.ns, self.n = B, ns, sum(ns)
        if fused:
            x = _bf16(gen, self.n, (hq + 2 * hkv) * d + 8)
            self.q, self.k, self.v = (x[:, a * d:b * d].view(self.n, b - a, d) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
        else:
            self.q, self.k, self.v = _bf16(gen, self.n, hq, d), _bf16(gen, self.n, hkv, d), _bf16(gen, self.n, hkv, d)
        self.out = torch.full((self.n + 2, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
        self.plan = B.dyspec_plan_create_prompt(hq, hkv, d, ns)
        self.ws, self.status = _workspace(self.plan), _zeros(1, dtype=torch.int32)

    def call(self, stream=None, ws=None, out=None):
        self.B.dyspec_prompt_attention(self.plan, self.q, self.k, self.v, self.out if out is None else out, self.ws if ws is None else ws,
                                       self.status, stream, self.q.stride(0), self.k.stride(0), self.v.stride(0))

    def check(self, sample=64):
        import torch
        from attention64 import causal, check
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0
        at = 0
        for r, n in enumerate(self.ns):
            if n:
                rows = None
                if n > sample:
                    rng = np.random.default_rng(r)
                    rows = sorted(set([0, 1, n - 2, n - 1] + [int(x) for x in rng.integers(0, n, sample)]))
                s = slice(at, at + n)
                want, bound = causal(self.q[s], self.k[s], self.v[s], 0, rows=rows)
                check(self.out[s] if rows is None else self.out[s][rows], want, bound)
            at += n
        assert (self.out[self.n:] == 7.0).all()
        return self


Prompt.check_after_call = lambda self, **kw: (self.call(), self.check(**kw))[1]


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("fused", [False, True])
def test_packed_prompts(B, hq, hkv, d, fused):
    Prompt(B, hq + d, hq, hkv, d, [1, 130, 0, 64, 257, 500, 2, 128], fused).check_after_call()
    Prompt(B, hq + d, hq, hkv, d, [1, 3, 0, 64 // (hq // hkv), 2], fused).check_after_call()
    Prompt(B, hq + d, hq, hkv, d, [1], fused).check_after_call()


def test_long_prompts(B):
    Prompt(B, 1, 8, 1, 128, [5000], True).check_after_call()
    Prompt(B, 2, 4, 4, 64, [3111, 17, 4096]).check_after_call()


def test_prompt_neighbours_that_are_not_finite(B):
    import torch
    for ns in ([5, 8, 7], [200, 70, 130]):
        p = Prompt(B, 5, 8, 2, 128, ns)
        p.call()
        torch.cuda.synchronize()
        want = p.out.clone()
        s = slice(ns[0], ns[0] + ns[1])
        p.q[s], p.k[s], p.v[s] = float("nan"), float("inf"), float("nan")
        p.call()
        torch.cuda.synchronize()
        keep = [i for i in range(p.n) if not ns[0] <= i < ns[0] + ns[1]]
        assert torch.equal(p.out[keep], want[keep])


def test_a_nan_key_shows_in_the_rows_behind_it_only(B):
    import torch
    for n in (7, 400):
        for at in range(0, n, max(1, n // 16)):
            p = Prompt(B, 9, 8, 1, 128, [n])
            p.k[at, 0, 5] = float("nan")
            p.call()
            torch.cuda.synchronize()
            assert torch.isfinite(p.out[:at]).all() and torch.isnan(p.out[at:n]).all()


def test_prompt_and_chunk_agree_over_one_sequence(B):
    """The same tokens as one prompt, and chunk by chunk over a cache."""
    import torch
    from attention64 import causal, check
    p = Prompt(B, 11, 8, 2, 128, [700])
    c = Chunk(B, 12, 8, 2, 128, [0], [700], 128)
    c.q.copy_(p.q)
    c.k[c.seq_rows[0]], c.v[c.seq_rows[0]] = p.k, p.v
    p.check_after_call()
    for lo, hi in ((0, 333), (333, 334), (334, 700)):
        plan = B.dyspec_plan_create_chunk(8, 2, 128, [lo], [hi - lo], c.rows, 128)
        out = _zeros(hi - lo, 8, 128)
        B.dyspec_chunk_attention_paged(plan, p.q[lo:hi], c.k, c.v, c.table, c.table.shape[1], out, _workspace(plan), c.status)
        torch.cuda.synchronize()
        want, bound = causal(p.q[lo:hi], p.k[:hi], p.v[:hi], lo)
        check(out, want, bound)


# ---- streams, graphs, plans ----------------------------------------------------------------------------------------
def test_repeated_calls_share_a_workspace_and_give_the_same_bits(B):
    import torch
    for make in (lambda: Chunk(B, 3, 8, 2, 128, [9000, 50, 0], [40, 1, 300], 128), lambda: Prompt(B, 3, 8, 8, 64, [900, 300, 2000]),
                 lambda: Chunk(B, 3, 8, 1, 128, [9000, 50, 0], [1, 2, 3], 128)):
        c = make().check_after_call()
        want = c.out.clone()
        for _ in range(20):
            c.out[:c.n] = 0
            c.call()
            torch.cuda.synchronize()
            assert torch.equal(c.out, want)


def test_one_workspace_serves_the_plans_of_a_loop(B):
    """Plans of different batches, which split, queue and merge differently, in turn over one buffer that was zeroed once."""
    import torch
    runs = [Chunk(B, 1, 8, 2, 128, [9000, 50, 0], [40, 1, 300], 128), Chunk(B, 2, 8, 1, 128, [12000, 50], [1, 1], 128),
            Chunk(B, 3, 8, 2, 128, [700] * 30, [1] * 30, 128), Prompt(B, 4, 8, 8, 64, [900, 300, 2000]),
            Chunk(B, 5, 8, 1, 128, [9001, 51], [1, 2], 128), Chunk(B, 6, 8, 2, 64, [20000], [9], 256), Prompt(B, 7, 4, 2, 128, [1, 3])]
    ws = _zeros(max([256] + [c.plan.workspace_bytes() for c in runs]), dtype=torch.uint8)
    torch.cuda.synchronize()
    for _ in range(3):
        for c in runs:
            c.out[:c.n] = 0
            c.call(ws=ws)
    for c in runs:
        c.check()


def test_neighbouring_rows_change_no_bit(B):
    """Rows of another request in the same tile of packed rows: whatever they hold, the request's own bits stay."""
    import torch
    for ns in ([3, 9, 5], [67, 70, 131], [131, 1, 90]):
        p = Prompt(B, 8, 8, 2, 128, ns)
        p.call()
        torch.cuda.synchronize()
        want = p.out[:ns[0]].clone()
        for fill in (float("nan"), 300.0, 0.0):
            p.q[ns[0]:] = fill
            p.call()
            torch.cuda.synchronize()
            assert torch.equal(p.out[:ns[0]], want)


def test_two_streams_with_workspaces_of_their_own(B):
    import torch
    a = Chunk(B, 3, 8, 2, 128, [5000, 50, 0], [200, 1, 300], 128)
    b = Chunk(B, 4, 8, 1, 128, [12000, 50], [1, 1], 128)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [_zeros(a.n, 8, 128), _zeros(a.n, 8, 128), _zeros(b.n, 8, 128)]
    works = [_workspace(a.plan), _workspace(a.plan), _workspace(b.plan)]
    torch.cuda.synchronize()
    for _ in range(10):
        for c, st, out, ws in zip((a, a, b), streams, outs, works):
            c.call(stream=st, out=out, ws=ws)
    torch.cuda.synchronize()
    a.check(outs[0]), a.check(outs[1]), b.check(outs[2])


def test_captured_and_replayed(B):
    import torch
    for ns in ([1, 1], [300, 1], [1, 40]):
        c = Chunk(B, 5, 8, 2, 128, [9000, 300], ns, 128)
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            c.call()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                c.call()
        for seed in (6, 7):
            gen = torch.Generator(device="cuda")
            gen.manual_seed(seed)
            c.q.copy_(_bf16(gen, *c.q.shape))
            for rows in c.seq_rows:
                c.k[rows] = _bf16(gen, len(rows), 2, 128)
            c.out[:c.n] = 0
            torch.cuda.synchronize()
            graph.replay()
            c.check()


def test_plans_serve_their_own_calls_only(B):
    import torch
    c = Chunk(B, 3, 8, 2, 128, [300], [4], 128)
    p = Prompt(B, 3, 8, 2, 128, [40])
    tree = B.Plan(8, 2, 128, [300], [4], None, c.rows, 4, 0.0, page_size=128)
    flat = B.Plan(8, 2, 128, [0], [40], [0], 40, 4, 0.0)
    bits, ints = _zeros(64, 4, dtype=torch.int32), _zeros(64, dtype=torch.int32)
    ws = _zeros(1 << 22, dtype=torch.uint8)
    before = c.out.clone()
    refused = [
        lambda: B.dyspec_chunk_attention_paged(tree, c.q, c.k, c.v, c.table, c.table.shape[1], c.out, ws),
        lambda: B.dyspec_chunk_attention_paged(p.plan, c.q, c.k, c.v, c.table, c.table.shape[1], c.out, ws),
        lambda: B.dyspec_prompt_attention(c.plan, p.q, p.k, p.v, c.out, ws),
        lambda: B.dyspec_prompt_attention(flat, p.q, p.k, p.v, c.out, ws),
        lambda: B.dyspec_tree_attention_paged(c.plan, c.q, c.k, c.v, c.table, c.table.shape[1], bits, None, c.out, ws),
        lambda: B.dyspec_tree_attention_ragged(p.plan, p.q, p.k, p.v, bits, c.out, ws),
        lambda: B.dyspec_tree_attention_ragged(c.plan, p.q, p.k, p.v, bits, c.out, ws),
        lambda: B.dyspec_plan_build_tree_mask(c.plan, ints, bits),
        lambda: B.dyspec_plan_build_tree_mask_tiles(p.plan, ints, bits, None, ints),
        lambda: B.dyspec_plan_dfs_reorder(p.plan, ints, ints),
        lambda: B.dyspec_chunk_attention_paged(c.plan, c.q, c.k, c.v, c.table, 2, c.out, ws),              # 304 tokens in 256
        lambda: B.dyspec_chunk_attention_paged(c.plan, c.q, c.k, c.v, None, 3, c.out, ws),
        lambda: B.dyspec_chunk_attention_paged(c.plan, c.q, c.k, c.v, c.table, 3, c.out, ws, q_stride=1020),
        lambda: B.dyspec_prompt_attention(p.plan, p.q, None, p.v, p.out, ws),
        lambda: B.dyspec_prompt_attention(p.plan, p.q, p.k, p.v, p.out, ws, k_stride=252),
    ]
    for call in refused:
        with pytest.raises(B.DyspecError) as e:
            call()
        assert e.value.code == -1
    long = B.dyspec_plan_create_chunk(8, 1, 128, [30000], [64], 30208, 128)
    assert long.workspace_bytes() > 256
    with pytest.raises(B.DyspecError) as e:
        B.dyspec_chunk_attention_paged(long, c.q, c.k, c.v, c.table, 300, c.out, ws[:256])
    assert e.value.code == -3
    torch.cuda.synchronize()
    assert torch.equal(c.out, before)


def test_empty_plans(B):
    import torch
    for contexts, ns in (([], []), ([5, 0], [0, 0])):
        plan = B.dyspec_plan_create_chunk(8, 2, 128, contexts, ns, 256, 128)
        B.dyspec_chunk_attention_paged(plan, None, None, None, None, 0, None)
        plan = B.dyspec_plan_create_prompt(8, 2, 128, ns)
        B.dyspec_prompt_attention(plan, None, None, None, None)
    torch.cuda.synchronize()
