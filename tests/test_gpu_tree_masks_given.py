"""lserve_sparse_decode_tree with masks, positions and selections that no tree of tokens would give, but that its description allows."""
import numpy as np
import pytest
import torch

from tree_reference import Problem, random_tree

pytestmark = pytest.mark.gpu


def _lib():
    import paper_2502_14866_amd as L

    L.load_library()
    return L


def _trees(sizes, seed=0):
    g = torch.Generator().manual_seed(100 + seed)
    return [random_tree(n, g) for n in sizes]


def _both(p, **kw):
    out, lse = p.call(_lib(), **kw)
    p.check(out, lse)
    return out, lse


@pytest.mark.parametrize("bits", [16, 8])
def test_bits_of_tokens_that_are_not_there(bits):
    p = Problem((130, 700), _trees((9, 70)), bits=bits, words=3)
    want, lse = _both(p)
    p.see = [np.concatenate([s, np.ones((len(s), 192 - len(s)), dtype=bool)], 1) for s in p.see]
    out, lse_out = p.call(_lib())
    assert torch.equal(out, want) and torch.equal(lse_out, lse)


@pytest.mark.parametrize("two_way", [False, True])
@pytest.mark.parametrize("ahead", [1, 63, 64, 200, 100000, 2 ** 31 - 1 - 800])
def test_positions_far_ahead(two_way, ahead):
    """Windows of streaming heads follow the positions: history and siblings behind them go, sink pages stay."""
    p = Problem((700, 30), _trees((20, 6)), flags=[1, 0], two_way=two_way)
    p.pos = [x + ahead * (j % 2) for j, x in enumerate(p.pos)]
    _both(p)


def test_every_token_at_its_own_position_in_any_order():
    p = Problem((300,), [[-1] * 40], flags=[1, 1], sink=0, local=64)
    g = torch.Generator().manual_seed(4)
    p.pos = (300 + torch.randperm(300, generator=g)[:40]).tolist()
    p.see = [(torch.rand((40, 40), generator=g) < 0.5).numpy()]
    _both(p)


@pytest.mark.parametrize("bits", [16, 4])
def test_the_same_page_twice(bits):
    """A page that a selection names twice counts twice, as in a decode step."""
    p = Problem((1000, 400), _trees((5, 12)), budget=512, stale=10, bits=bits)
    p.sel["pages"][:, :, 1] = p.sel["pages"][:, :, 0]
    _both(p)


def test_selections_of_a_longer_sequence():
    """A selection made when there was more history than now (tokens taken back): pages that are left."""
    p = Problem((500,), _trees((7,)), budget=512)
    p.sel["lens"][0] = 640
    _both(p)


def test_heads_with_selections_of_their_own_lengths():
    p = Problem((2000, 900), _trees((6, 3)), hq=8, hkv=4, flags=[0, 0, 1, 0], budget=1024)
    p.sel["count"][0, 0], p.sel["count"][1, 1], p.sel["count"][0, 3] = 0, 1, 5
    _both(p)
