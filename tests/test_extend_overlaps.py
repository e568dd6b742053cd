"""lserve_extend_tables refuses outputs that lie where its inputs or other outputs do: workgroups read the former while one writes the latter."""
import pytest
import torch

import paper_2502_14866_amd as L
from paper_2502_14866_amd import binding as B


OUTPUTS, INPUTS = ["cu", "after", "taken"], ["lens", "new", "free"]


@pytest.mark.parametrize("output,other", [(o, x) for o in OUTPUTS for x in INPUTS + OUTPUTS if o != x])
@pytest.mark.parametrize("shift", [0, 4])
def test_overlaps(output, other, shift):
    sizes = {"cu": 9, "after": 8, "taken": 1, "lens": 8, "new": 8, "free": 12}
    t = {k: torch.zeros(n, dtype=torch.int32) for k, n in sizes.items()}
    room = torch.zeros(64, dtype=torch.int32)
    shift = min(shift, (sizes[output] - 1) // 4 * 4)  # 16-byte alignment, and an overlap
    t[output], t[other] = room[:sizes[output]], room[shift:shift + sizes[other]]
    kv = L.PagedKV(None, None, None, torch.zeros((8, 4), dtype=torch.int32), t["lens"])
    with pytest.raises(B.LserveError) as e:
        L.lserve_extend_tables(L.AttnDesc(4, 2, [1, 0]), kv, t["new"], t["free"], t["cu"], t["after"], t["taken"], total_new=8, stream=0)
    assert e.value.code == -1
