"""One workspace, zeroed once, for plans of every kind in turn: trees whose split groups are merged inside the kernel, by clusters and by the
combine launch, trees from the shared queue, chunks and prompts.  Each call gives the bits that it gives with a workspace of its own."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _runs():
    """(call(workspace), output, status, plan) of every kind."""
    import torch
    import test_gpu_causal as causal
    from paper_2410_11744_b200 import build, workloads as wl
    build.build()
    from paper_2410_11744_b200 import binding as B, runner as R
    rng = np.random.default_rng(3)
    tree = lambda n: wl.random_tree(rng, n)
    runs = []

    def add_tree(tuning, hq, hkv, d, prefix, nodes, paged=None):
        w = wl.make_custom(70 + len(runs), hq, hkv, d, prefix, [tree(n) for n in nodes])
        B.dyspec_set_tuning(*tuning)
        try:
            b = R.DeviceBatch(w, paged=None if paged is None else wl.to_paged(w, 256, seed=1, tree_in_pages=paged))
        finally:
            B.dyspec_set_tuning(-1, 0, 2)

        def call(ws):
            b.workspace, b.workspace_bytes = ws, ws.numel()
            b.step()
        runs.append((call, b.out, b.status, b.plan))

    add_tree((-1, 0, 1), 4, 4, 128, [2500], [256])                     # merged inside the kernel
    add_tree((-1, 0, 1), 8, 1, 64, [9000, 300], [40, 129], paged=True)
    add_tree((-1, 0, 2), 32, 32, 128, [4096], [256])                   # clusters through the workspace
    add_tree((-1, 0, 0), 8, 8, 128, [3000, 700], [48, 17])             # small tiles, combine launch
    add_tree((-1, 0, 2), 32, 8, 128, [900] * 10, [200] * 10)           # whole groups from the queue
    add_tree((-1, 0, 2), 32, 32, 128, [1024], [64], paged=False)       # small tiles, clusters: no workspace
    for c in (causal.Chunk(B, 1, 8, 2, 128, [9000, 50, 0], [40, 1, 300], 128), causal.Chunk(B, 2, 8, 1, 128, [12000, 50], [1, 1], 128),
              causal.Chunk(B, 5, 8, 1, 128, [9001, 51], [1, 2], 128), causal.Chunk(B, 6, 8, 2, 64, [20000], [9], 256),
              causal.Prompt(B, 4, 32, 32, 64, [900, 300, 2000]), causal.Prompt(B, 7, 4, 2, 128, [1, 3])):
        runs.append((lambda ws, c=c: c.call(ws=ws), c.out, c.status, c.plan))
    kinds = {(p.describe()["regime"], p.describe()["cluster"] > 1, p.describe()["split_groups"] > 0, p.describe()["combine_launch"],
              p.describe()["dynamic"]) for _, _, _, p in runs}
    assert {(1, False, True, 0, 0), (1, True, False, 0, 0), (0, False, True, 1, 0), (1, False, False, 0, 1), (0, False, True, 0, 0)} <= kinds, kinds
    return torch, runs


def test_plans_of_every_kind_share_one_workspace():
    torch, runs = _runs()
    zeros = lambda n: torch.zeros(n, dtype=torch.uint8, device="cuda")
    wants = []
    for call, out, status, plan in runs:
        out.zero_()
        call(zeros(max(256, plan.workspace_bytes())))
        torch.cuda.synchronize()
        wants.append(out.clone())
    ws = zeros(max(plan.workspace_bytes() for _, _, _, plan in runs))
    rng = np.random.default_rng(9)
    n = len(runs)
    for order in [list(range(n)), list(range(n))[::-1]] + [rng.permutation(n).tolist() for _ in range(8)]:
        for i in order:
            runs[i][1].zero_()
            runs[i][0](ws)
        torch.cuda.synchronize()
        for (call, out, status, plan), want in zip(runs, wants):
            assert int(status.item()) == 0 and torch.equal(out, want)
    assert int(ws[:16384].to(torch.int32).sum().item()) == 0            # the control words are back at zero
