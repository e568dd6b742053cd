"""lserve_sparse_decode_tree under selections of more entries than there are pages: every entry counts, as in a decode step."""
import pytest
import torch

from tree_reference import NP, Problem, random_tree

pytestmark = pytest.mark.gpu


def _lib():
    import paper_2502_14866_amd as L

    L.load_library()
    return L


def _problem(lens, sizes, budget, **kw):
    g = torch.Generator().manual_seed(100 + len(lens))
    return Problem(lens, [random_tree(n, g) for n in sizes], budget=budget, **kw)


def _both(p):
    out, lse = p.call(_lib())
    p.check(out, lse)


def _repeat(p, b, hk, count):
    pages = -(-p.lens[b] // NP)
    p.sel["pages"][b, hk, :count] = torch.arange(count, dtype=torch.int32) % pages
    p.sel["count"][b, hk] = count


@pytest.mark.parametrize("bits,dtype", [(16, torch.float16), (16, torch.bfloat16), (8, torch.float16), (4, torch.bfloat16)])
@pytest.mark.parametrize("nodes", [3, 20, 70])
def test_pages_named_again_and_again(bits, dtype, nodes):
    p = _problem((130, 60, 700), (nodes, 1, 5), 1024, bits=bits, dtype=dtype, flags=[0, 0])
    for b in range(3):
        for hk in range(2):
            _repeat(p, b, hk, 16 - 5 * hk - b)
    _both(p)


@pytest.mark.parametrize("bits", [16, 4])
def test_any_order_after_tokens_were_taken_back(bits):
    """A selection of a longer sequence, its pages in no order: those that are left are attended, wherever they stand."""
    p = _problem((200, 64), (7, 3), 512, bits=bits, flags=[0, 0])
    p.sel["lens"][:] = 640
    for b in range(2):
        p.sel["pages"][b, 0] = torch.tensor([9, 8, 7, 6, 3, 1, 0, 2], dtype=torch.int32)
        p.sel["pages"][b, 1] = torch.tensor([5, 4, 9, 8, 7, 6, 2, 0], dtype=torch.int32)
        p.sel["count"][b] = 8
    _both(p)


@pytest.mark.parametrize("stale", [0, 200])
@pytest.mark.parametrize("bits", [16, 8])
def test_in_pieces(bits, stale):
    """Lists twice as long as the history, cut into pieces by the lengths alone; heads of one sequence have lists of their own lengths."""
    p = _problem((5000, 300), (9, 40), 64 * 160, bits=bits, stale=stale, hq=8, hkv=4, flags=[0, 0, 1, 0])
    _repeat(p, 0, 0, 160)
    _repeat(p, 0, 1, 120)
    _repeat(p, 1, 3, 159)
    _both(p)


def test_lists_that_stay_whole():
    """So many lists that none is cut."""
    g = torch.Generator().manual_seed(3)
    lens = [int(x) for x in torch.randint(1, 130, (520,), generator=g)]
    p = _problem(lens, [1] * 520, 320, hq=8, hkv=8, flags=[0] * 8)
    assert _lib().lserve_tree_workspace_bytes(_lib().AttnDesc(8, 8, [0] * 8), 520, 520, 1, p.width, 5) == 0
    for b in range(0, 520, 7):
        _repeat(p, b, b % 8, 5)
    _both(p)


def test_counts_past_the_stride_are_not_read():
    p = _problem((130, 64), (3, 3), 256, flags=[0, 0])
    for b in range(2):
        for hk in range(2):
            _repeat(p, b, hk, 4)
    want = p.call(_lib())
    p.check(*want)
    p.sel["count"][:] = 2 ** 31 - 1
    got = p.call(_lib())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
