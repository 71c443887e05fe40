"""The operators in the order of a serving loop, over one paged cache: prompt, chunk, speculative steps (draft tree appended with
its depths as positions, tree attention, verification, compaction), plain decoding.  At every step the attention's output is compared
with the formula over the sequence's own tokens, whose K is rotated in 64 bits from the unrotated projections."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("hq,hkv,d,page,rot", [(8, 2, 128, 128, 128), (8, 8, 64, 256, 32)])
def test_a_sequence_through_its_life(apart, hq, hkv, d, page, rot):
    import torch
    from attention64 import causal, check, rope_table, rotate
    from paper_2410_11744_b200 import build, workloads as wl
    build.build()
    from paper_2410_11744_b200 import binding as B
    dev, rng = "cuda", np.random.default_rng(hq + d)
    gen = torch.Generator(device=dev)
    gen.manual_seed(d)
    lens, n_req, per_req, vocab = [150, 1, 300], 3, 8, 256
    tree_rows, pool = 64, n_req * per_req * page
    rows = pool + n_req * tree_rows
    table = torch.tensor(rng.permutation(n_req * per_req).reshape(n_req, per_req).astype(np.int32), device=dev)
    k_cache, v_cache = (torch.zeros((rows, hkv, d), dtype=torch.bfloat16, device=dev) for _ in range(2))
    rope = rope_table(per_req * page, rot)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    # what every sequence consists of so far, before rotation: lists of [tokens][hkv][d]
    have = [[torch.zeros((0, hkv, d), dtype=torch.bfloat16, device=dev)] * 2 for _ in lens]
    contexts = [0] * n_req
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=dev)
    new = lambda n, h: torch.randn((n, h, d), generator=gen, device=dev).to(torch.bfloat16)

    def append(ns, depths=None, tree0=None):
        n = sum(ns)
        q, k, v, q_rot = new(n, hq), new(n, hkv), new(n, hkv), torch.empty((n, hq, d), dtype=torch.bfloat16, device=dev)
        B.dyspec_append_kv_paged(k, v, q, q_rot, k_cache, v_cache, rows, i32(np.concatenate([[0], np.cumsum(ns)])), i32(contexts), depths,
                                 tree0, table, per_req, page, rope, per_req * page, rot, False, n, n_req, hq, hkv, d, status=status)
        return q, k, v, q_rot

    def rounded(x, positions):
        """Rotated in fp64, then rounded to bf16 as the cache holds it."""
        return rotate(x, rope[positions], False)[0].to(torch.bfloat16)

    def causal_step(ns):
        q, k, v, q_rot = append(ns)
        out = torch.zeros_like(q_rot)
        plan = B.dyspec_plan_create_chunk(hq, hkv, d, contexts, ns, rows, page)
        ws = torch.zeros(max(256, plan.workspace_bytes()), dtype=torch.uint8, device=dev)
        B.dyspec_chunk_attention_paged(plan, q_rot, k_cache, v_cache, table, per_req, out, ws, status)
        if sum(contexts) == 0:                               # the prompt call, over the rotated rows as they are packed
            k_rot = torch.cat([rounded(k[sum(ns[:r]):sum(ns[:r + 1])], torch.arange(n, device=dev)) for r, n in enumerate(ns)])
            again = torch.zeros_like(out)
            prompt = B.dyspec_plan_create_prompt(hq, hkv, d, ns)
            pws = torch.zeros(max(256, prompt.workspace_bytes()), dtype=torch.uint8, device=dev)
            B.dyspec_prompt_attention(prompt, q_rot, k_rot, v, again, pws, status)
        torch.cuda.synchronize()
        at = 0
        for r, n in enumerate(ns):
            have[r] = [torch.cat([have[r][0], k[at:at + n]]), torch.cat([have[r][1], v[at:at + n]])]
            total = contexts[r] + n
            kr = rounded(have[r][0], torch.arange(total, device=dev))
            qr = rounded(q[at:at + n], torch.arange(contexts[r], total, device=dev))
            want, bound = causal(qr, kr, have[r][1], contexts[r])
            # a rotated value may fall on the other side of a rounding: K and Q each off by a step of 2^-8 in a few places at most,
            # which moves a score by 2^-7 of its parts; the outputs stay within a few of their bounds
            check(out[at:at + n], want, 8 * bound)
            if sum(contexts) == 0:
                check(again[at:at + n], want, 8 * bound)
            contexts[r] = total
            at += n

    causal_step(lens)
    causal_step([100, 37, 1])
    for step in range(2):
        trees = [wl.greedy_tree(rng, n, 4, 0.3) for n in (33, 20, 48)]
        ns = [len(t) for t in trees]
        n, W = sum(ns), B.dyspec_words_per_row(max(ns))
        off = np.concatenate([[0], np.cumsum(ns)])
        tree0 = None if not apart else torch.tensor(pool + tree_rows * np.arange(n_req), dtype=torch.int64, device=dev)
        plan = B.dyspec_plan_create_paged(hq, hkv, d, contexts, ns, None if tree0 is None else tree0.tolist(), rows, page, W)
        parents, bits = i32(np.concatenate(trees)), torch.zeros((n, W), dtype=torch.int32, device=dev)
        depths = torch.zeros(n, dtype=torch.int32, device=dev)
        B.dyspec_plan_build_tree_mask(plan, parents, bits, depths, status)
        q, k, v, q_rot = append(ns, depths, tree0)
        out = torch.zeros_like(q_rot)
        ws = torch.zeros(max(256, plan.workspace_bytes()), dtype=torch.uint8, device=dev)
        B.dyspec_tree_attention_paged(plan, q_rot, k_cache, v_cache, table, per_req, bits, None, out, ws, status)
        case = wl.make_verify_case(step, vocab, trees, sharpness=3.0, disagreement=0.3)
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)
        got_t, got_n, count = i32(np.zeros((n_req, 64))), i32(np.zeros((n_req, 64))), i32(np.zeros(n_req))
        B.dyspec_verify_tree(parents, t(np.concatenate(case.tokens)), t(case.draft_probs), t(case.target_probs), t(case.accept_u),
                             t(case.sample_u), t(case.node_offsets), n_req, max(ns), vocab, got_t, got_n, count, 64, status=status)
        new_len = i32(np.zeros(n_req))
        B.dyspec_compact_kv_paged(k_cache, v_cache, tree0, table, per_req, page, i32(contexts), got_n, count, n_req, 64, hkv, d, new_len,
                                  status, keep_root=True)
        torch.cuda.synchronize()
        for r in range(n_req):
            path = [0] + [int(a) for a in got_n[r, :int(count[r])].tolist() if a >= 0]
            # the path's nodes as the next tokens of the sequence: their rows of the tree attention are causal attention over it
            at = int(off[r])
            node = torch.tensor(path, device=dev) + at
            total = contexts[r] + len(path)
            assert depths[node].tolist() == list(range(len(path))) and int(new_len[r]) == total
            have[r] = [torch.cat([have[r][0], k[node]]), torch.cat([have[r][1], v[node]])]
            kr = rounded(have[r][0], torch.arange(total, device=dev))
            qr = rounded(q[node], torch.arange(contexts[r], total, device=dev))
            want, bound = causal(qr, kr, have[r][1], contexts[r])
            check(out[node], want, 8 * bound)
            contexts[r] = total
    causal_step([1, 1, 1])
    causal_step([5, 1, 60])
    assert int(status.item()) == 0
