"""What the binding makes of tensors that are not packed: rows that lie apart give their own stride, any other layout is refused.
Host tensors: every refusal comes before the library is called."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2410_11744_b200 import build
    build.build()
    from paper_2410_11744_b200 import binding
    return binding


def test_row_strides(B):
    x = torch.zeros(6, 200, dtype=torch.bfloat16)
    rows = lambda t: B._row_stride(t, "call")
    assert rows(None) == 0 and rows(1 << 20) == 0
    assert rows(x) == 0 and rows(x.view(6, 25, 8)) == 0 and rows(x.view(-1)) == 0      # packed
    assert rows(x[:, 64:128]) == 200 and rows(x[:, 64:128].view(6, 4, 16)) == 200      # columns of a projection
    assert rows(x[::2]) == 400 and rows(x[2:4]) == 0                                  # every other row; some rows
    assert rows(x[:1, 64:128]) == 0                                                   # one row: nothing lies apart
    for bad in (x[:, ::2], x.view(6, 25, 8)[:, :, :4], x.view(6, 25, 8).transpose(1, 2), x.t(), x.view(-1)[::2], x[:1].expand(6, 200)):
        with pytest.raises(B.DyspecError) as e:
            rows(bad)
        assert e.value.code == -1


def test_layouts_without_a_stride_are_refused(B):
    """Caches side by side in one tensor, cut tables, an output in columns of another: nothing of them reaches the library."""
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    kv, table, rope = z(256, 2, 2, 64), z(2, 4, dtype=torch.int32), z(100, 128, dtype=torch.float32)
    q, out = z(3, 8, 64), z(3, 8, 128)
    plan = B.Plan._owning(None, 128, 3)                 # (no handle: a call that came through would be refused with -1 as well,
    called, own = [], B.lib                             #  so the library's entry points are replaced)

    class Lib:
        def __getattr__(self, name):
            return own.dyspec_error_string if name == "dyspec_error_string" else lambda *a: called.append(name) or 0

    def append(k_cache=kv[:, 0].contiguous(), v_cache=kv[:, 1].contiguous(), page_table=table, rope_table=rope, q_=q, q_out=q):
        B.dyspec_append_kv_paged(z(3, 2, 64), z(3, 2, 64), q_, q_out, k_cache, v_cache, 256, z(2, dtype=torch.int32), z(1, dtype=torch.int32), None,
                                 None, page_table, 4, 64, rope_table, 100, 64, False, 3, 1, 8, 2, 64, stream=1)

    def chunk(k=kv[:, 0].contiguous(), v=kv[:, 1].contiguous(), page_table=table, q_=q, o=q):
        B.dyspec_chunk_attention_paged(plan, q_, k, v, page_table, 4, o, stream=1)

    def prompt(k=q, v=q, q_=q, o=q):
        B.dyspec_prompt_attention(plan, q_, k, v, o, stream=1)

    B.lib = Lib()
    try:
        append(), chunk(), prompt(), append(q_=out[:, :, :64].reshape(3, 512)), append(q_=None, q_out=None)
        assert len(called) == 5
        called.clear()
        cols = out[:, :, :64]                           # heads 128 apart: no row of 8 packed heads
        for call in (lambda: append(k_cache=kv[:, 0]), lambda: append(v_cache=kv[:, 1]), lambda: append(page_table=table[:, :2]),
                     lambda: append(rope_table=rope[:, :64]), lambda: append(q_=cols), lambda: append(q_out=cols),
                     lambda: chunk(k=kv[:, 0]), lambda: chunk(v=kv[:, 1]), lambda: chunk(page_table=table[:, :2]), lambda: chunk(o=cols),
                     lambda: chunk(o=out.view(3, 1024)[:, :512]), lambda: chunk(q_=cols), lambda: prompt(o=cols), lambda: prompt(k=cols),
                     lambda: prompt(v=cols), lambda: prompt(q_=cols)):
            with pytest.raises(B.DyspecError) as e:
                call()
            assert e.value.code == -1 and not called
    finally:
        B.lib = own


@pytest.mark.gpu
def test_fused_projections_without_strides(B):
    """Columns of one projection, no stride named: the same bits as with the strides named."""
    import test_gpu_append
    import test_gpu_causal
    for ns in ([3, 1], [150, 70]):
        p = test_gpu_causal.Prompt(B, 3, 8, 2, 128, ns, fused=True)
        p.call()
        again = torch.zeros_like(p.out)
        B.dyspec_prompt_attention(p.plan, p.q, p.k, p.v, again, p.ws, p.status)
        wide = torch.zeros((p.n, 1064), dtype=torch.bfloat16, device="cuda")
        c = test_gpu_causal.Chunk(B, 4, 8, 2, 128, [300, 64], ns, 128)
        c.call()
        wide[:, :1024] = c.q.view(c.n, 1024)
        chunked = torch.zeros_like(c.out)
        B.dyspec_chunk_attention_paged(c.plan, wide[:, :1024], c.k, c.v, c.table, c.table.shape[1], chunked, c.ws, c.status)
        torch.cuda.synchronize()
        assert torch.equal(again[:p.n], p.out[:p.n]) and torch.equal(chunked[:c.n], c.out[:c.n])
    s, t = (test_gpu_append._case(5, 8, 2, 64, [9, 70], [40, 5], 64, 64, False, fused=True) for _ in range(2))
    test_gpu_append._call(B, s)
    wide = torch.zeros((t["n"], 8 * 64 + 8), dtype=torch.bfloat16, device="cuda")
    B.dyspec_append_kv_paged(t["k"], t["v"], t["q"], wide[:, :512], t["k_cache"], t["v_cache"], t["rows"], t["offsets"], t["contexts"], None,
                             None, t["table"], t["table"].shape[1], 64, t["rope"], t["n_positions"], 64, False, t["n"], 2, 8, 2, 64)
    torch.cuda.synchronize()
    assert torch.equal(s["k_cache"], t["k_cache"]) and torch.equal(s["v_cache"], t["v_cache"])
    assert torch.equal(s["q_out"].view(-1, 512), wide[:, :512]) and (wide[:, 512:] == 0).all()
