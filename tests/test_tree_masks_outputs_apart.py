"""lserve_tree_masks refuses outputs that lie on what it reads or on each other, but for positions in the place of the parents."""
import pytest
import torch

import paper_2502_14866_amd as L
from paper_2502_14866_amd import binding as B

WORDS = {"parents": 8, "cu": 3, "lens": 2, "mask": 16, "pos": 8}


def _code(place):
    t = {k: torch.zeros(n, dtype=torch.int32) for k, n in WORDS.items()}
    t.update(place)
    with pytest.raises(B.LserveError) as e:
        L.lserve_tree_masks(t["parents"], t["cu"], t["lens"], 4, t["mask"].view(torch.int64).view(8, 1), t["pos"], stream=0)
    return e.value.code


@pytest.mark.parametrize("output,other", [(o, x) for o in ("mask", "pos") for x in WORDS if x != o])
@pytest.mark.parametrize("shift", [0, 4])
def test_overlaps(output, other, shift):
    room = torch.zeros(64, dtype=torch.int32)
    if (output, other, shift) != ("pos", "parents", 0):
        assert _code({output: room[:WORDS[output]], other: room[shift:shift + WORDS[other]]}) == -1


@pytest.mark.skipif(torch.cuda.is_available(), reason="host memory")
def test_positions_in_the_place_of_the_parents():
    """Gets as far as the launch, which needs a GPU."""
    room = torch.zeros(8, dtype=torch.int32)
    assert _code({"parents": room, "pos": room}) == -4
