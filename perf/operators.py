"""The operators around the paged KV cache, what their speed is measured on, and their plain forms.

A serving stack that verifies draft trees with this library also has to get tokens into the cache and to run the
attention of everything that is not a tree.  `op` says which operator a case is:

  append   K and V of new tokens go into a paged cache, rotated by their positions on the way, and Q is rotated with
           them (`dyspec_append_kv_paged`).  New tokens are prompt chunks, single tokens of decoding requests, or the
           nodes of draft trees, whose position is context + depth and whose rows lie inside the pages or apart.
  chunk    causal attention of a chunk of new tokens over a paged cache that already holds them
           (`dyspec_chunk_attention_paged`): single tokens, chunks of a long prompt, both in one batch.
  prompt   causal attention over whole prompts, packed one behind the other, with grouped heads
           (`dyspec_prompt_attention`); Q, K and V may be columns of one fused projection.

Sizes of ragged batches come from the case (`shape_seed`), so that its work is known; values come from the seed that
`prepare` is given.  With `own` false, `run` computes the same in elementary torch operations in 32 bits.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"


def listed():
    return [
        # one decoding step of a serving batch: a token each, GQA 8; nothing but launch and a chain of small loads
        dict(name="append_decode_32", op="append", hq=64, hkv=8, d=128, n_req=32, c_lo=100, c_hi=2048, n_lo=1, n_hi=1,
             page=256, rot=128, inter=False, tree="", fused=False, shape_seed=3),
        # draft trees of a batch of 8, MHA: positions by depth, tree rows behind the pages
        dict(name="append_tree_8", op="append", hq=32, hkv=32, d=128, n_req=8, c_lo=64, c_hi=512, n_lo=48, n_hi=128,
             page=128, rot=128, inter=False, tree="apart", fused=False, shape_seed=5),
        # small heads, a quarter of them rotated as neighbouring pairs, appended behind odd contexts
        dict(name="append_partial_d64", op="append", hq=16, hkv=8, d=64, n_req=5, c_lo=0, c_hi=700, n_lo=33, n_hi=1500,
             page=128, rot=16, inter=True, tree="", fused=False, shape_seed=29),
        # a prefill step: ragged prompts straight from one fused projection, GQA 8
        dict(name="append_prompt_16k", op="append", hq=64, hkv=8, d=128, n_req=6, c_lo=0, c_hi=0, n_lo=1000, n_hi=4500,
             page=256, rot=128, inter=False, tree="", fused=True, shape_seed=11),
        # one decoding request, MHA, the chat length of the benchmark: latency
        dict(name="decode_one_mha", op="chunk", hq=32, hkv=32, d=128, n_req=1, c_lo=1024, c_hi=1024, n_lo=1, n_hi=1,
             long_req=0, long_n=0, page=256, shape_seed=0),
        # a decoding batch, GQA 8, ragged contexts: streams K and V
        dict(name="decode_batch_64", op="chunk", hq=64, hkv=8, d=128, n_req=64, c_lo=512, c_hi=8192, n_lo=1, n_hi=1,
             long_req=0, long_n=0, page=256, shape_seed=13),
        # two requests in very long contexts, a token each: few rows, a long axis to split
        dict(name="decode_long_131072", op="chunk", hq=64, hkv=8, d=128, n_req=2, c_lo=131072, c_hi=131072, n_lo=1,
             n_hi=1, long_req=0, long_n=0, page=512, shape_seed=0),
        # one chunk of a long prompt
        dict(name="chunk_512_over_8192", op="chunk", hq=64, hkv=8, d=128, n_req=1, c_lo=8192, c_hi=8192, n_lo=512,
             n_hi=512, long_req=0, long_n=0, page=256, shape_seed=0),
        # what a scheduler with chunked prefill submits: decoding requests and one chunk in a batch, odd sizes
        dict(name="mixed_batch_32", op="chunk", hq=32, hkv=8, d=128, n_req=32, c_lo=300, c_hi=6000, n_lo=1, n_hi=1,
             long_req=1, long_n=997, page=128, shape_seed=17),
        # a few short prompts of odd lengths, MHA
        dict(name="prompt_short_6", op="prompt", hq=32, hkv=32, d=128, n_req=6, n_lo=1, n_hi=512, fused=False,
             shape_seed=19),
        # ragged prompts with small heads, from one fused projection
        dict(name="prompt_ragged_d64", op="prompt", hq=16, hkv=8, d=64, n_req=8, n_lo=300, n_hi=4096, fused=True,
             shape_seed=23),
        # one long prompt, GQA 8: dense contraction
        dict(name="prompt_16384_gqa", op="prompt", hq=64, hkv=8, d=128, n_req=1, n_lo=16384, n_hi=16384, fused=False,
             shape_seed=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(32, 32, 128), (64, 8, 128), (32, 8, 128), (16, 8, 64), (8, 8, 64), (64, 64, 128), (8, 2, 128), (16, 4, 64)]


def draw(rng):
    op = rng.choice(["append", "chunk", "chunk", "prompt"])
    seed = rng.randrange(1 << 20)
    hq, hkv, d = rng.choice(HEADS)
    wide = hq * d // 2048                          # 1/4 .. 4 of 16 heads of 128: bounds the work
    if op == "append":
        tree = rng.choice(["", "", "apart", "in_pages"])
        n_hi = _log_int(rng, 1, 300 if tree else 4096)
        n_req = _log_int(rng, 1, max(1, min(48, 16000 // (n_hi * max(1, wide)))))
        return dict(op=op, hq=hq, hkv=hkv, d=d, n_req=n_req, c_lo=0, c_hi=_log_int(rng, 1, 1024),
                    n_lo=max(1, n_hi // rng.choice([1, 3, 20])), n_hi=n_hi, page=rng.choice([16, 128, 256, 1024]),
                    rot=rng.choice([d, d, d // 2, 16, 0]), inter=rng.random() < 0.4, tree=tree,
                    fused=rng.random() < 0.5, shape_seed=seed)
    if op == "chunk":
        kind = rng.choice(["decode", "decode", "chunk", "mixed"])
        if kind == "decode":
            n_req, n_hi = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 5])
            c_hi = _log_int(rng, 1, max(64, min(131072, 600000 * 1024 // (n_req * hkv * d))))
        else:
            n_req = _log_int(rng, 1, 12) if kind == "chunk" else rng.randint(2, 32)
            n_hi = _log_int(rng, 8, max(16, 4096 // n_req)) if kind == "chunk" else 1
            c_hi = _log_int(rng, 1, 16384 // max(1, n_req // 4))
        mixed = kind == "mixed"
        return dict(op=op, hq=hq, hkv=hkv, d=d, n_req=n_req, c_lo=c_hi // rng.choice([1, 4, 30]), c_hi=c_hi,
                    n_lo=max(1, n_hi // rng.choice([1, 4])), n_hi=n_hi, long_req=rng.randint(1, 2) if mixed else 0,
                    long_n=_log_int(rng, 65, 1500) if mixed else 0, page=rng.choice([128, 256, 512]), shape_seed=seed)
    n_hi = _log_int(rng, 2, 16384 // max(1, wide))
    n_req = _log_int(rng, 1, max(1, min(32, 16384 // n_hi)))
    return dict(op=op, hq=hq, hkv=hkv, d=d, n_req=n_req, n_lo=max(1, n_hi // rng.choice([1, 3, 20])), n_hi=n_hi,
                fused=rng.random() < 0.5, shape_seed=seed)


# ---- sizes of a case ---------------------------------------------------------------------------------------------
def _between(rng, lo, hi):
    return lo if hi <= lo else int(round(math.exp(rng.uniform(math.log(max(1, lo)), math.log(hi)))))


def _sizes(case):
    """(contexts, new tokens) of the batch: lengths log-uniform between the case's bounds; `long_req` of the requests
    bring a long chunk."""
    rng = random.Random(case["shape_seed"])
    cs = [_between(rng, case["c_lo"], case["c_hi"]) if "c_lo" in case else 0 for _ in range(case["n_req"])]
    ns = [_between(rng, case["n_lo"], case["n_hi"]) for _ in range(case["n_req"])]
    for r in range(min(case.get("long_req", 0), case["n_req"])):
        ns[r * 7 % case["n_req"]] = case["long_n"]
    return cs, ns


def work(case):
    cs, ns = _sizes(case)
    hq, hkv, d, n = case["hq"], case["hkv"], case["d"], sum(ns)
    if case["op"] == "append":      # Q, K and V in and out, a table row and a position a token; 3 operations a value
        rotated = n * (hq + hkv) * case["rot"]
        return {"bytes": 2 * n * (hq + 2 * hkv) * d * 2 + n * (case["rot"] + 1) * 4, "flops": 3 * rotated}
    pairs = sum(k * c + k * (k + 1) // 2 for c, k in zip(cs, ns))
    rows = sum(cs) + n
    return {"bytes": 2 * rows * hkv * d * 2 + 2 * n * hq * d * 2, "flops": 4 * hq * d * pairs}


# ---- inputs ------------------------------------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _ints(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).to(DEV)


def _pages(rng, lens, page):
    """Shuffled page table for sequences of these lengths, -1 behind a sequence's last page, and rows of the pool."""
    need = [-(-x // page) for x in lens]
    ids = rng.permutation(sum(need) + 2)
    table = np.full((len(lens), max(1, max(need))), -1, dtype=np.int32)
    at = 0
    for r, k in enumerate(need):
        table[r, :k] = ids[at:at + k]
        at += k
    return table, (sum(need) + 2) * page


def _qkv(g, n, hq, hkv, d, fused):
    """Projections of n tokens: three tensors, or columns of one."""
    if not fused:
        return _normal(g, n, hq, d), _normal(g, n, hkv, d), _normal(g, n, hkv, d)
    x = _normal(g, n, (hq + 2 * hkv) * d)
    return (x[:, :hq * d].view(n, hq, d), x[:, hq * d:(hq + hkv) * d].view(n, hkv, d),
            x[:, (hq + hkv) * d:].view(n, hkv, d))


def _rope_table(n_positions, rot):
    """[positions][rot]: cosines of the rot / 2 angles, then their sines (base 10000), in 64 bits before rounding."""
    freq = 10000.0 ** (-np.arange(rot // 2, dtype=np.float64) / max(1, rot // 2))
    angle = np.arange(n_positions, dtype=np.float64)[:, None] * freq[None, :]
    return torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], axis=1).astype(np.float32)).to(DEV)


def _depths(rng, ns, tree):
    """Depth of every node of random recursive trees (parents come before children); None without trees."""
    if not tree:
        return None
    out = []
    for n in ns:
        dep = np.zeros(n, dtype=np.int32)
        for i in range(1, n):
            dep[i] = dep[rng.integers(max(0, i - 8), i)] + 1
        out.append(dep)
    return np.concatenate(out)


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1009 + 7)
    rng = np.random.default_rng(seed)
    cs, ns = _sizes(case)
    hq, hkv, d, n = case["hq"], case["hkv"], case["d"], sum(ns)
    s = dict(case=case, cs=cs, ns=ns, n=n, scale=1.0 / math.sqrt(d))
    if case["op"] == "prompt":
        s["q"], s["k"], s["v"] = _qkv(g, n, hq, hkv, d, case["fused"])
        return s
    apart = case.get("tree") == "apart"
    table, rows = _pages(rng, [c + (0 if apart else k) for c, k in zip(cs, ns)], case["page"])
    s["tree0"] = None
    if apart:
        s["tree0"] = rows + np.concatenate([[0], np.cumsum(ns)[:-1]])
        rows += n
    s["table"], s["rows"] = table, rows
    s["k_cache"], s["v_cache"] = _normal(g, rows, hkv, d), _normal(g, rows, hkv, d)
    if case["op"] == "chunk":
        s["q"] = _normal(g, n, hq, d)
        return s
    s["q"], s["k"], s["v"] = _qkv(g, n, hq, hkv, d, case["fused"])
    s["depths"] = _depths(rng, ns, case["tree"])
    s["n_positions"] = max(c + k for c, k in zip(cs, ns))
    s["rope"] = _rope_table(s["n_positions"], case["rot"]) if case["rot"] else None
    return s


def _token_rows(table, page, c, n):
    """Pool rows of tokens c .. c + n - 1 of the sequence with this row of the page table."""
    t = np.arange(c, c + n)
    return table[t // page].astype(np.int64) * page + t % page


def _append_layout(s):
    """(pool row, position) of every new token."""
    case, rows, pos, at = s["case"], [], [], 0
    for r, (c, n) in enumerate(zip(s["cs"], s["ns"])):
        rows.append(s["tree0"][r] + np.arange(n) if s["tree0"] is not None else _token_rows(s["table"][r], case["page"], c, n))
        pos.append(c + (s["depths"][at:at + n] if s["depths"] is not None else np.arange(n)))
        at += n
    return np.concatenate(rows), np.concatenate(pos)


def prepare(case, seed):
    s = _inputs(case, seed)
    cs, ns, n = s["cs"], s["ns"], s["n"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "append":
        rows, pos = _append_layout(s)
        s["dst"], s["pos"] = _ints(rows, np.int64), _ints(pos, np.int64)
        s["offsets"], s["contexts"] = _ints(np.concatenate([[0], np.cumsum(ns)])), _ints(cs)
        s["depths"] = None if s["depths"] is None else _ints(s["depths"])
        s["tree0"] = None if s["tree0"] is None else _ints(s["tree0"], np.int64)
        s["q_out"] = torch.zeros((n, hq, d), dtype=torch.bfloat16, device=DEV)
    else:
        s["out"] = torch.zeros((n, hq, d), dtype=torch.bfloat16, device=DEV)
    if case["op"] == "chunk":
        s["kv_rows"] = [_ints(_token_rows(s["table"][r], case["page"], 0, c + k), np.int64) for r, (c, k) in enumerate(zip(cs, ns))]
    if case["op"] != "prompt":
        s["per_req"], s["table"] = s["table"].shape[1], _ints(s["table"])
    s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    if own and case["op"] != "append":
        from paper_2410_11744_b200 import binding as B
        if case["op"] == "chunk":
            s["plan"] = B.dyspec_plan_create_chunk(hq, hkv, d, cs, ns, s["rows"], case["page"])
        else:
            s["plan"] = B.dyspec_plan_create_prompt(hq, hkv, d, ns)
        s["workspace"] = torch.zeros(max(256, s["plan"].workspace_bytes()), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)[s["case"]["op"]](s)


def _own_append(s):
    from paper_2410_11744_b200 import binding as B
    case = s["case"]
    B.dyspec_append_kv_paged(s["k"], s["v"], s["q"], s["q_out"], s["k_cache"], s["v_cache"], s["rows"], s["offsets"],
                             s["contexts"], s["depths"], s["tree0"], s["table"], s["per_req"], case["page"], s["rope"],
                             s["n_positions"], case["rot"], case["inter"], s["n"], case["n_req"], case["hq"], case["hkv"],
                             case["d"], k_stride=s["k"].stride(0), v_stride=s["v"].stride(0), q_stride=s["q"].stride(0),
                             status=s["status"])
    return [s["q_out"], s["k_cache"], s["v_cache"], s["status"]]


def _own_chunk(s):
    from paper_2410_11744_b200 import binding as B
    B.dyspec_chunk_attention_paged(s["plan"], s["q"], s["k_cache"], s["v_cache"], s["table"], s["per_req"], s["out"],
                                   s["workspace"], s["status"])
    return [s["out"], s["status"]]


def _own_prompt(s):
    from paper_2410_11744_b200 import binding as B
    B.dyspec_prompt_attention(s["plan"], s["q"], s["k"], s["v"], s["out"], s["workspace"], s["status"],
                              q_stride=s["q"].stride(0), k_stride=s["k"].stride(0), v_stride=s["v"].stride(0))
    return [s["out"], s["status"]]


_run_own = dict(append=_own_append, chunk=_own_chunk, prompt=_own_prompt)


def _rotate(x, cos, sin, inter):
    """x [n][heads][d] in 32 bits; cos, sin [n][1][rot / 2]: pairs (i, i + rot / 2), or neighbours, turned."""
    half = cos.shape[-1]
    turned, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if inter else (turned[..., :half], turned[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], dim=-1).flatten(-2) if inter else torch.cat([a, b], dim=-1)
    return torch.cat([turned, rest], dim=-1)


def _plain_append(s):
    case = s["case"]
    q, k = s["q"].float(), s["k"].float()
    if case["rot"]:
        half = case["rot"] // 2
        row = s["rope"][s["pos"]][:, None, :]
        cos, sin = row[..., :half], row[..., half:]
        q, k = _rotate(q, cos, sin, case["inter"]), _rotate(k, cos, sin, case["inter"])
    s["q_out"].copy_(q.to(torch.bfloat16))
    s["k_cache"][s["dst"]] = k.to(torch.bfloat16)
    s["v_cache"][s["dst"]] = s["v"]
    return [s["q_out"], s["k_cache"], s["v_cache"], s["status"]]


def _plain_causal(q, k, v, first, scale, out):
    """Rows of q are tokens first .. of the sequence k, v; a block of rows at a time, over the keys that it sees."""
    n, hq, d = q.shape
    hkv = k.shape[1]
    g = hq // hkv
    kt, vt = k.float().permute(1, 2, 0), v.float().permute(1, 0, 2)                       # [hkv][d][S], [hkv][S][d]
    block = max(1, min(n, (1 << 28) // (hq * k.shape[0])))
    for i0 in range(0, n, block):
        i1 = min(n, i0 + block)
        seen = first + i1
        qb = q[i0:i1].float().view(i1 - i0, hkv, g, d).permute(1, 2, 0, 3).reshape(hkv, g * (i1 - i0), d)
        x = torch.matmul(qb, kt[:, :, :seen]).view(hkv, g, i1 - i0, seen).mul_(scale)
        if i1 - i0 > 1:
            late = torch.arange(seen, device=DEV)[None, :] > first + torch.arange(i0, i1, device=DEV)[:, None]
            x.masked_fill_(late, -math.inf)
        x = torch.exp(x.sub_(x.amax(dim=-1, keepdim=True)))
        o = torch.matmul(x.view(hkv, g * (i1 - i0), seen), vt[:, :seen]).view(hkv, g, i1 - i0, d)
        o = o / x.sum(dim=-1, keepdim=True)
        out[i0:i1] = o.permute(2, 0, 1, 3).reshape(i1 - i0, hq, d).to(torch.bfloat16)


def _plain_chunk(s):
    at = 0
    for r, (c, n) in enumerate(zip(s["cs"], s["ns"])):
        rows = s["kv_rows"][r]
        _plain_causal(s["q"][at:at + n], s["k_cache"][rows], s["v_cache"][rows], c, s["scale"], s["out"][at:at + n])
        at += n
    return [s["out"], s["status"]]


def _plain_prompt(s):
    at = 0
    for n in s["ns"]:
        _plain_causal(s["q"][at:at + n], s["k"][at:at + n], s["v"][at:at + n], 0, s["scale"], s["out"][at:at + n])
        at += n
    return [s["out"], s["status"]]


_run_plain = dict(append=_plain_append, chunk=_plain_chunk, prompt=_plain_prompt)


# ---- the same from the definitions in 64 bits ----------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "append":
        return _exact_append(s)
    outs, at = [], 0
    for r, (c, n) in enumerate(zip(s["cs"], s["ns"])):
        q = s["q"][at:at + n].double()
        if case["op"] == "chunk":
            rows = torch.from_numpy(_token_rows(s["table"][r], case["page"], 0, c + n)).to(DEV)
            k, v = s["k_cache"][rows], s["v_cache"][rows]
        else:
            k, v = s["k"][at:at + n], s["v"][at:at + n]
        out = torch.empty((n, case["hq"], case["d"]), dtype=torch.float64, device=DEV)
        key = torch.arange(c + n, device=DEV)
        for h in range(case["hq"]):
            kh, vh = (t[:, h * case["hkv"] // case["hq"]].double() for t in (k, v))
            for i in range(0, n, 2048):
                token = c + torch.arange(i, min(n, i + 2048), device=DEV)
                x = torch.einsum("id,td->it", q[i:i + 2048, h], kh) / math.sqrt(case["d"])
                w = torch.softmax(torch.where(key[None, :] <= token[:, None], x, -math.inf), dim=1)
                out[i:i + 2048, h] = torch.einsum("it,td->id", w, vh)
        outs.append(out)
        at += n
    return [torch.cat(outs), torch.zeros(1, dtype=torch.int32, device=DEV)]


def _exact_append(s):
    case, rot = s["case"], s["case"]["rot"]
    rows, pos = _append_layout(s)
    dst = torch.from_numpy(rows).to(DEV)
    got = []
    for x in (s["q"], s["k"]):
        x = x.double()
        y = x.clone()
        if rot:
            turn = torch.complex(*(t.double() for t in s["rope"][torch.from_numpy(pos.astype(np.int64)).to(DEV)].chunk(2, dim=1)))
            first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["inter"] else (slice(0, rot // 2), slice(rot // 2, rot))
            z = torch.complex(x[..., first], x[..., second]) * turn[:, None, :]
            y[..., first], y[..., second] = z.real, z.imag
        got.append(y)
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    k_cache[dst], v_cache[dst] = got[1], s["v"].double()
    return [got[0], k_cache, v_cache, torch.zeros(1, dtype=torch.int32, device=DEV)]
