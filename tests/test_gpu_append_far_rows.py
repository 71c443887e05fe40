"""Tree rows at the far end of 64 bits are rows outside the pool like any other: reported, nothing of them written."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("row", [2 ** 63 - 1, 2 ** 63 - 4, 2 ** 62, 2 ** 33, -2 ** 63])
def test_tree_rows_at_the_end_of_64_bits(row):
    import torch
    import test_gpu_append as append
    from paper_2410_11744_b200 import binding as B
    s = append._case(41, 4, 2, 64, [10, 30, 5], [8, 8, 8], 16, 64, False, tree="apart")
    live = torch.ones(s["n"], dtype=torch.bool, device="cuda")
    live[8:16] = False
    tree0 = s["tree0"].clone()
    tree0[1] = row
    append._check(B, s, live=live, tree0=tree0)
    assert int(s["status"].item()) == -1
