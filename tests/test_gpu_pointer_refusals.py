"""Pointers of the attention calls that are not aligned are refused on the host, before anything is launched: the outputs stay as they
were, and a good call behind the refusals is answered."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ns", [[1, 2], [150, 70]])
def test_misaligned_pointers(ns):
    import torch
    import test_gpu_causal as causal
    from paper_2410_11744_b200 import binding as B
    c, p = causal.Chunk(B, 3, 8, 2, 128, [300, 0], ns, 128), causal.Prompt(B, 4, 8, 2, 128, ns)
    before = c.out.clone(), p.out.clone()
    for name, off in (("q", 8), ("k", 8), ("v", 8), ("out", 8), ("table", 2), ("status", 2), ("status", 1)):
        a = dict(q=c.q.data_ptr(), k=c.k.data_ptr(), v=c.v.data_ptr(), table=c.table.data_ptr(), out=c.out.data_ptr(), status=c.status.data_ptr())
        a[name] += off
        with pytest.raises(B.DyspecError) as e:
            B.dyspec_chunk_attention_paged(c.plan, a["q"], a["k"], a["v"], a["table"], c.table.shape[1], a["out"], c.ws, a["status"])
        assert e.value.code == -1
        if name == "table":
            continue
        a = dict(q=p.q.data_ptr(), k=p.k.data_ptr(), v=p.v.data_ptr(), out=p.out.data_ptr(), status=p.status.data_ptr())
        a[name] += off
        with pytest.raises(B.DyspecError) as e:
            B.dyspec_prompt_attention(p.plan, a["q"], a["k"], a["v"], a["out"], p.ws, a["status"])
        assert e.value.code == -1
    torch.cuda.synchronize()
    assert torch.equal(c.out, before[0]) and torch.equal(p.out, before[1])
    c.check_after_call()
    p.check_after_call()
