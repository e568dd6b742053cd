"""Windows of streaming heads at positions whose tile a 32-bit float does not hold."""
import numpy as np
import pytest
import torch

from tree_reference import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("first", [2 ** 30, 2 ** 30 + 128, 2 ** 31 - 64 * 40])
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("local", [64, 128])
def test_tiles_past_24_bits(first, bits, local):
    """Tile 2^24 + 1 is the first that a float rounds down: drafted keys one window behind it are no longer seen."""
    import paper_2502_14866_amd as L

    L.load_library()
    n = 6
    everything = [np.ones((n, n), dtype=bool), np.ones((3, 3), dtype=bool)]
    p = Problem((100, 0), [[-1] * n, [-1] * 3], flags=[1, 1], sink=0, local=local, see=everything, bits=bits)
    p.pos = [first + 64 * i for i in range(n)] + [first, first + 64, first + 64]
    out, lse = p.call(L)
    p.check(out, lse)
