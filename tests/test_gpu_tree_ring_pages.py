"""lserve_sparse_decode_tree over a ring table that names pages its pool does not have: the nearest there is, as with the page table."""
import pytest
import torch

from tree_reference import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("wrong", [-1, -2 ** 31, 2 ** 31 - 1, 1])
def test_pages_outside_the_pool(bits, wrong):
    import paper_2502_14866_amd as L

    L.load_library()
    p = Problem((700, 130), [[-1, 0, 0], [-1]], flags=[1, 0], two_way=True, bits=bits)
    last = p.pools["ks"].shape[0] - 1
    page, slot = (0 if wrong < 0 else last), (p.ring == (0 if wrong < 0 else last)).nonzero()
    if not len(slot):  # nobody has that page: sequence 0 gets it for its first one
        old = int(p.ring[0, 0])
        for pool in ("ks", "vs"):
            p.pools[pool][page] = p.pools[pool][old]
        p.ring[0, 0] = page
        slot = torch.tensor([[0, 0]])
    want = p.call(L)
    p.check(*want)
    b, i = slot[0].tolist()
    p.ring[b, i] = wrong if wrong != 1 else last + 1
    got = p.call(L)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
