"""lserve_sparse_decode_tree at the ends of its ranges: the widest trees under the largest groups, batches of thousands of which most draft nothing."""
import pytest
import torch

from tree_reference import Problem, random_tree

pytestmark = pytest.mark.gpu


def _both(p, **kw):
    import paper_2502_14866_amd as L

    L.load_library()
    out, lse = p.call(L, **kw)
    p.check(out, lse)


@pytest.mark.parametrize("bits,dtype", [(16, torch.bfloat16), (8, torch.bfloat16), (4, torch.float16)])
def test_the_widest_trees_under_eight_heads(bits, dtype):
    """64 tiles of rows of one sequence, over a list in pieces; another with a few tokens beside it."""
    g = torch.Generator().manual_seed(7)
    _both(Problem((500, 64), [random_tree(1024, g), random_tree(3, g)], hq=8, hkv=1, flags=[0], bits=bits, dtype=dtype), pad=2)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("batch", [300, 5000])
def test_batches_that_mostly_draft_nothing(batch, bits):
    g = torch.Generator().manual_seed(batch)
    lens = [int(x) for x in torch.randint(0, 70, (batch,), generator=g)]
    sizes = [int(x) if i % 37 == 0 else 0 for i, x in enumerate(torch.randint(1, 5, (batch,), generator=g))]
    lens[37], lens[-1] = 3000, 200
    _both(Problem(lens, [random_tree(n, g) for n in sizes], hq=2, hkv=1, flags=[0], bits=bits))
