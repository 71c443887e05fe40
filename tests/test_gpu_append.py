"""Appending rotated keys and values to the paged cache, against the formula in 64 bits: K, Q within one rounding, V and all rows
that are not the new tokens' bit for bit."""
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


def _bf16(gen, *shape):
    import torch
    return torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)


def _i32(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _case(seed, hq, hkv, d, contexts, ns, page, rot, inter, tree="", fused=False, pad=0, spare=2):
    """Inputs, page table and the rows and positions of the new tokens, as a dict."""
    import torch
    from attention64 import rope_table
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    n = sum(ns)
    need = [-(-(c + (0 if tree == "apart" else k)) // page) for c, k in zip(contexts, ns)]
    ids = rng.permutation(sum(need) + spare)
    table = np.full((len(ns), max(1, max(need, default=1))), -1, np.int32)
    for r, k in enumerate(need):
        table[r, :k] = ids[sum(need[:r]):sum(need[:r + 1])]
    rows = (sum(need) + spare) * page
    tree0 = None
    if tree == "apart":
        tree0 = rows + 3 + np.concatenate([[0], np.cumsum(ns)[:-1]]).astype(np.int64)
        rows += n + 5
    depths = np.concatenate([np.minimum(rng.integers(0, 9, k), np.arange(k)) for k in ns] or [[]]) if tree else None
    dst, pos = [], []
    for r, (c, k) in enumerate(zip(contexts, ns)):
        j = np.arange(k)
        dst.append(tree0[r] + j if tree0 is not None else table[r][(c + j) // page].astype(np.int64) * page + (c + j) % page)
        pos.append(c + (depths[sum(ns[:r]):sum(ns[:r + 1])] if tree else j))
    s = dict(hq=hq, hkv=hkv, d=d, n=n, page=page, rot=rot, inter=inter, rows=rows, n_req=len(ns),
             dst=torch.tensor(np.concatenate(dst), dtype=torch.int64, device="cuda"),
             pos=torch.tensor(np.concatenate(pos), dtype=torch.int64, device="cuda"),
             table=_i32(table), offsets=_i32(np.concatenate([[0], np.cumsum(ns)])), contexts=_i32(contexts),
             depths=None if depths is None else _i32(np.concatenate([depths, np.zeros(pad)])),
             tree0=None if tree0 is None else torch.tensor(tree0, dtype=torch.int64, device="cuda"),
             n_positions=max([c + k for c, k in zip(contexts, ns)] + [1]))
    s["rope"] = rope_table(s["n_positions"], rot) if rot else None
    if fused:
        x = _bf16(gen, n + pad, (hq + 2 * hkv) * d + 24)               # (columns behind them: a stride that is no row's size)
        s["q"], s["k"], s["v"] = (x[:, a * d:b * d].view(n + pad, b - a, d) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    else:
        s["q"], s["k"], s["v"] = _bf16(gen, n + pad, hq, d), _bf16(gen, n + pad, hkv, d), _bf16(gen, n + pad, hkv, d)
    s["k_cache"], s["v_cache"] = _bf16(gen, rows, hkv, d), _bf16(gen, rows, hkv, d)
    s["q_out"] = _bf16(gen, n + pad, hq, d)
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return s


def _call(B, s, **over):
    a = dict(s, **over)
    B.dyspec_append_kv_paged(a["k"], a["v"], a["q"], a["q_out"], a["k_cache"], a["v_cache"], a["rows"], a["offsets"], a["contexts"],
                             a["depths"], a["tree0"], a["table"], a["table"].shape[1], a["page"], a["rope"], a["n_positions"],
                             a["rot"], a["inter"], a["k"].shape[0], a["n_req"], a["hq"], a["hkv"], a["d"], k_stride=a["k"].stride(0),
                             v_stride=a["v"].stride(0), q_stride=0 if a["q"] is None else a["q"].stride(0),
                             q_out_stride=0 if a["q_out"] is None else a["q_out"].stride(0), status=a["status"])


def _check(B, s, live=None, **over):
    """Runs the call and compares everything; live: which tokens are expected to be written (all)."""
    import torch
    from attention64 import check, rotate
    before = {k: s[k].clone() for k in ("k_cache", "v_cache", "q_out")}
    _call(B, s, **over)
    torch.cuda.synchronize()
    n, dst = s["n"], s["dst"]
    live = torch.ones(n, dtype=torch.bool, device="cuda") if live is None else live
    old = torch.ones(s["rows"], dtype=torch.bool, device="cuda")
    old[dst[live]] = False
    assert torch.equal(s["k_cache"][old], before["k_cache"][old]) and torch.equal(s["v_cache"][old], before["v_cache"][old])
    assert torch.equal(s["v_cache"][dst[live]], s["v"][:n][live])
    assert torch.equal(s["q_out"][n:], before["q_out"][n:]) and torch.equal(s["q_out"][:n][~live], before["q_out"][:n][~live])
    for x, got in ((s["k"][:n][live], s["k_cache"][dst[live]]), (s["q"][:n][live], s["q_out"][:n][live])):
        if s["rot"]:
            want, bound = rotate(x, s["rope"][s["pos"][live]], s["inter"])
            check(got, want, bound + 1e-300)
        else:
            assert torch.equal(got, x)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("hq,hkv,d,rot", [(64, 8, 128, 128), (32, 32, 128, 64), (8, 8, 64, 64), (5, 3, 64, 16), (1, 1, 128, 112), (4, 2, 128, 0)])
def test_append_matches_the_formula(B, hq, hkv, d, rot, inter):
    contexts, ns = [0, 127, 128, 300, 5, 0], [3, 1, 130, 0, 64, 1]
    s = _case(hq + d + rot, hq, hkv, d, contexts, ns, 128, rot, inter, fused=bool(rot % 32), pad=5)
    _check(B, s)
    assert int(s["status"].item()) == 0


@pytest.mark.parametrize("page", [1, 16, 64, 4096])
def test_append_page_sizes(B, page):
    s = _case(page, 8, 2, 64, [0, 15, 16, 100], [33, 1, 2, 47], page, 32, False)
    _check(B, s)
    assert int(s["status"].item()) == 0


@pytest.mark.parametrize("tree", ["apart", "in_pages"])
def test_append_tree_nodes_take_their_depth_as_position(B, tree):
    s = _case(7, 32, 4, 128, [200, 0, 1023], [64, 7, 33], 256, 128, False, tree=tree, pad=3)
    _check(B, s)
    assert int(s["status"].item()) == 0


@pytest.mark.parametrize("n_req", [1, 31, 32, 33, 1000, 1025, 2500])
def test_append_finds_the_request_of_every_token(B, n_req):
    rng = np.random.default_rng(n_req)
    ns = [int(x) for x in rng.integers(0, 3, n_req)]
    ns[-1] = 1
    s = _case(n_req, 2, 1, 64, [int(x) for x in rng.integers(0, 40, n_req)], ns, 32, 64, True)
    _check(B, s)
    assert int(s["status"].item()) == 0


def test_append_many_tokens(B):
    s = _case(3, 16, 8, 128, [10, 0], [3001, 1200], 128, 128, False, fused=True)
    _check(B, s)
    assert int(s["status"].item()) == 0


def test_append_without_queries_and_in_place(B):
    import torch
    s = _case(11, 8, 4, 128, [9, 70], [40, 5], 64, 128, False)
    twin = _case(11, 8, 4, 128, [9, 70], [40, 5], 64, 128, False)
    _call(B, s)
    _call(B, twin, q=None, q_out=None, hq=0)
    torch.cuda.synchronize()
    assert torch.equal(s["k_cache"], twin["k_cache"]) and torch.equal(s["v_cache"], twin["v_cache"])
    q = s["q"].clone()
    _call(B, s, q=q, q_out=q)
    torch.cuda.synchronize()
    assert torch.equal(q, s["q_out"])


def test_append_reports_what_has_no_place_and_writes_the_rest(B):
    import torch
    s = _case(13, 4, 2, 64, [10, 30, 5, 40], [20, 20, 20, 20], 16, 64, False)
    live = torch.ones(s["n"], dtype=torch.bool, device="cuda")
    table = s["table"].clone()
    table[0, 1] = -1                                   # tokens 16 .. 29 of request 0: no page
    live[6:20] = False
    table[1, 2] = s["rows"] // 16                      # tokens 32 .. 47 of request 1: a page behind the pool
    live[22:38] = False
    table[2, 0] = 0x7fffffff                           # tokens 5 .. 15 of request 2
    live[40:51] = False
    s["rope"] = s["rope"][:55].contiguous()            # positions 55 .. 59 of request 3: behind the table
    live[75:80] = False
    _check(B, s, live=live, table=table, n_positions=55)
    assert int(s["status"].item()) == -1


def test_append_bad_tree_rows_contexts_and_narrow_tables(B):
    import torch
    s = _case(17, 4, 2, 64, [10, 30, 5], [8, 8, 8], 16, 64, False, tree="apart")
    live = torch.ones(s["n"], dtype=torch.bool, device="cuda")
    tree0 = s["tree0"].clone()
    tree0[0] = -3
    tree0[1] = s["rows"] - 2                           # (behind the rows of request 2)
    live[:8] = False
    s["dst"][8:16] = s["rows"] - 2 + torch.arange(8, device="cuda")
    live[10:16] = False
    _check(B, s, live=live, tree0=tree0)
    assert int(s["status"].item()) == -1
    s = _case(19, 4, 2, 64, [10, 30], [8, 8], 16, 64, False)
    live = torch.ones(s["n"], dtype=torch.bool, device="cuda")
    live[8:] = False                                   # two pages per request: tokens 32 .. have none; 30, 31 have
    live[8:10] = True
    table = s["table"][:, :2].contiguous()
    _check(B, s, live=live, table=table)
    assert int(s["status"].item()) == -1
    live[:8] = False                                   # a context below zero: nowhere
    contexts = s["contexts"].clone()
    contexts[0] = -5
    _check(B, s, live=live, table=table, contexts=contexts)


def test_append_keeps_not_finite_values(B):
    import torch
    s = _case(23, 2, 2, 64, [4], [6], 16, 32, False)
    s["v"][0, 0, 3], s["v"][1, 1, 5], s["k"][2, 0, 40] = float("nan"), float("-inf"), float("inf")
    _call(B, s)
    torch.cuda.synchronize()
    got = s["v_cache"][s["dst"]]
    assert torch.equal(torch.nan_to_num(got, 7.0), torch.nan_to_num(s["v"], 7.0)) and torch.isnan(got[0, 0, 3])
    assert torch.isinf(s["k_cache"][s["dst"]][2, 0, 40])


def test_append_into_a_pool_beyond_32_bit_offsets(B):
    """2.2 M rows of 1024 values: offsets of the last page are beyond 2^31 values and 2^32 bytes."""
    import torch
    s = _case(29, 8, 8, 128, [100], [40], 256, 128, False)
    rows = (2200000 // 256) * 256
    pool_k = torch.zeros((rows, 8, 128), dtype=torch.bfloat16, device="cuda")
    pool_v = torch.zeros((rows, 8, 128), dtype=torch.bfloat16, device="cuda")
    s["k_cache"], s["v_cache"], s["rows"] = pool_k, pool_v, rows
    s["table"][0, 0] = rows // 256 - 1
    s["dst"] = rows - 256 + 100 + torch.arange(40, device="cuda")
    _check(B, s)
    assert int(s["status"].item()) == 0


def test_append_in_a_replayed_graph_follows_its_device_inputs(B):
    """Lengths, contexts and the page table are device data: a captured call serves the next step's values."""
    import torch
    s = _case(31, 8, 2, 64, [20, 40, 7], [4, 1, 6], 16, 64, False, pad=9)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _call(B, s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            _call(B, s)
    torch.cuda.synchronize()
    t = _case(37, 8, 2, 64, [33, 0, 15], [1, 9, 5], 16, 64, False, pad=5, spare=2)
    assert t["table"].shape[1] <= s["table"].shape[1] and t["rows"] <= s["rows"] and t["n_positions"] <= s["n_positions"]
    for name in ("k", "v", "q"):
        s[name].copy_(t[name])
    s["offsets"].copy_(t["offsets"])
    s["contexts"].copy_(t["contexts"])
    s["table"][:, :t["table"].shape[1]].copy_(t["table"])
    graph.replay()
    torch.cuda.synchronize()
    _call(B, t)
    torch.cuda.synchronize()
    assert int(s["status"].item()) == 0
    assert torch.equal(s["k_cache"][t["dst"]], t["k_cache"][t["dst"]]) and torch.equal(s["v_cache"][t["dst"]], t["v"][:t["n"]])
    assert torch.equal(s["q_out"][:t["n"]], t["q_out"][:t["n"]])
