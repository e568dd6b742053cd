"""lserve_tree_masks with positions in the place of the parents."""
import pytest
import torch

from tree_reference import ancestors, pack_bits, random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes", [(5, 64, 1), (200, 0, 70), (1024, 3)])
def test_positions_written_over_parents(sizes):
    import paper_2502_14866_amd as L

    L.load_library()
    g = torch.Generator().manual_seed(1)
    trees, dev = [random_tree(n, g) for n in sizes], "cuda:0"
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    words = -(-max(sizes) // 64)
    both = i32([x for t in trees for x in t])
    mask = torch.zeros((len(both), words), dtype=torch.int64, device=dev)
    cu = i32([0] + torch.tensor(sizes).cumsum(0).tolist())
    L.lserve_tree_masks(both, cu, i32([100] * len(sizes)), max(sizes), mask, both)
    want = [ancestors(t) for t in trees]
    assert both.tolist() == [100 + d for _, depth in want for d in depth]
    assert mask.tolist() == [row for see, _ in want for row in pack_bits(see, words)]
