"""Refusals of the append and causal-attention calls, on the host: nothing is launched, no GPU is needed."""
import ctypes

import pytest

P = 1 << 20        # stands for an aligned device pointer: the refusals come before anything reads it


@pytest.fixture(scope="module")
def lib():
    from paper_2410_11744_b200 import build
    build.build()
    from paper_2410_11744_b200 import binding
    return binding.lib


def _append(lib, **over):
    from paper_2410_11744_b200 import binding
    a = dict(k=P, ks=0, v=P, vs=0, q=P, qs=0, qo=2 * P, qos=0, hq=8, kc=P, vc=P, rows=1024, off=P, ctx=P, dep=None, tree=None, n_req=0,
             n=0, table=P, ppr=4, page=16, rope=P, npos=100, rot=64, inter=0, hkv=2, d=64, status=None)
    a.update(over)
    z = lambda *names: [a[name] or 0 for name in names]
    packed = binding._APPEND_ARGS.pack(*z("k", "v", "q", "qo", "kc", "vc", "ks", "vs", "qs", "qos", "rows", "off", "ctx", "dep", "tree", "table",
                                          "rope", "status", "n_req", "n", "hq", "hkv", "d", "ppr", "page", "npos", "rot", "inter"))
    return lib.dyspec_append_kv_paged(packed, None)


@pytest.mark.parametrize("code,over", [
    (0, {}), (0, dict(n_req=3)), (0, dict(n=3)),
    (-1, dict(hq=-1)), (-1, dict(hkv=0)), (-1, dict(n=-1)), (-1, dict(n_req=-1)), (-1, dict(rows=-1)), (-1, dict(rot=-16)),
    (-2, dict(d=96)), (-2, dict(rot=24)), (-1, dict(rot=128)), (-1, dict(page=0)), (-1, dict(page=48)), (-1, dict(ppr=0)),
    (-1, dict(ks=64)), (-1, dict(vs=132)), (-1, dict(qs=511)), (-1, dict(qos=-512)), (-1, dict(npos=-1)),
    (-2, dict(hq=1 << 17)), (0, dict(tree=P, page=0, ppr=0)),
] + [(-1, dict(n_req=1, n=1, **{name: None})) for name in ("k", "v", "q", "qo", "kc", "vc", "off", "ctx", "table", "rope")]
  + [(-1, dict(n_req=1, n=1, **{name: P + 8})) for name in ("k", "v", "q", "qo", "kc", "vc", "rope")]
  + [(-1, dict(n_req=1, n=1, **{name: P + 2})) for name in ("off", "ctx", "dep", "tree", "table", "status")]
  + [(-1, dict(n_req=1, n=1, qo=P, qs=1024))])
def test_append_refusals(lib, code, over):
    assert _append(lib, **over) == code


def _i32(values):
    return None if values is None else ctypes.cast((ctypes.c_int32 * max(1, len(values)))(*values), ctypes.c_void_p)


def _plan(lib, chunk, hq=8, hkv=2, d=64, ctx=(5,), n=(3,), rows=1024, page=128, n_req=None):
    h = ctypes.c_void_p()
    n_req = (0 if n is None else len(n)) if n_req is None else n_req
    if chunk:
        rc = lib.dyspec_plan_create_chunk(ctypes.byref(h), hq, hkv, d, n_req, _i32(ctx), _i32(n), rows, page, 0.0)
    else:
        rc = lib.dyspec_plan_create_prompt(ctypes.byref(h), hq, hkv, d, n_req, _i32(n), 0.0)
    return rc, h


@pytest.mark.parametrize("code,over", [
    (-1, dict(hq=0)), (-1, dict(hkv=-2)), (-2, dict(hq=7)), (-2, dict(hq=24)), (-2, dict(d=96)), (-1, dict(n=(-1,))),
    (-1, dict(n=None, n_req=1)), (-1, dict(n_req=-1)), (-2, dict(hq=2, n=(2 ** 31 - 100,))), (-2, dict(n=(2 ** 30,))),
    (-2, dict(n=(2 ** 28, 2 ** 28, 2 ** 28))), (-2, dict(hq=64, hkv=64, n=(2 ** 24,))),
])
@pytest.mark.parametrize("chunk", [True, False])
def test_plan_refusals(lib, chunk, code, over):
    if chunk and over.get("n"):
        over = dict(over, ctx=(5,) * len(over["n"]))
    rc, h = _plan(lib, chunk, **over)
    assert rc == code and not h.value


@pytest.mark.parametrize("code,over", [
    (-1, dict(ctx=(-1,))), (-1, dict(ctx=None)), (-1, dict(page=0)), (-1, dict(page=192)), (-2, dict(page=64)), (-2, dict(page=1 << 21)),
    (-1, dict(rows=-1)), (-1, dict(rows=0)), (-2, dict(rows=1 << 31)), (-2, dict(ctx=(2 ** 31 - 300,), n=(100,))),
])
def test_chunk_plan_refusals(lib, code, over):
    rc, h = _plan(lib, True, **over)
    assert rc == code and not h.value


def test_calls_without_a_plan(lib):
    assert lib.dyspec_append_kv_paged(None, None) == -1
    assert lib.dyspec_chunk_attention_paged(None, P, 0, P, P, P, 4, P, None, 0, None, None) == -1
    assert lib.dyspec_prompt_attention(None, P, 0, P, 0, P, 0, P, None, 0, None, None) == -1
    assert lib.dyspec_plan_create_chunk(None, 8, 2, 64, 0, None, None, 0, 128, 0.0) == -1
    assert lib.dyspec_plan_create_prompt(None, 8, 2, 64, 0, None, 0.0) == -1
