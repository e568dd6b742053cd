"""lserve_extend_tables refuses positions, slots, ring slots and a page table that lie where its inputs or other outputs do."""
import pytest
import torch

import paper_2502_14866_amd as L
from paper_2502_14866_amd import binding as B

# (int32 words: batch 8, eight new tokens, four pages a row, a ring of ten pages)
WORDS = {"cu": 9, "after": 8, "taken": 1, "table": 32, "pos": 8, "slots": 16, "ring_slots": 16, "lens": 8, "new": 8, "free": 12, "ring": 80}
LONG = ("slots", "ring_slots")
OUTPUTS = ["pos", "slots", "ring_slots", "table"]


def _call(place=None, **kw):
    t = {k: torch.zeros(n, dtype=torch.int32) for k, n in WORDS.items()}
    t.update(place or {})
    t.update(kw)
    wide = {k: None if t[k] is None else t[k].view(torch.int64) for k in LONG}
    kv = L.PagedKV(None, None, None, t["table"].view(8, 4), t["lens"], ring_table=t["ring"].view(8, 10))
    L.lserve_extend_tables(L.AttnDesc(4, 2, [1, 0]), kv, t["new"], t["free"], t["cu"], t["after"], t["taken"], t["pos"], wide["slots"],
                           wide["ring_slots"], total_new=8, stream=0)


@pytest.mark.parametrize("output,other", [(o, x) for o in OUTPUTS for x in WORDS if x != o])
@pytest.mark.parametrize("shift", [0, 4])
def test_overlaps(output, other, shift):
    room = torch.zeros(256, dtype=torch.int32)
    shift = min(shift, (WORDS[output] - 1) // 4 * 4)
    with pytest.raises(B.LserveError) as e:
        _call({output: room[:WORDS[output]], other: room[shift:shift + WORDS[other]]})
    assert e.value.code == -1


def test_arrays_of_nothing_lie_anywhere():
    """Without new tokens nothing is written through them; a call that gets as far as its launch needs a GPU."""
    if torch.cuda.is_available():
        pytest.skip("host memory")
    room = torch.zeros(64, dtype=torch.int32)
    kv = L.PagedKV(None, None, None, torch.zeros((8, 4), dtype=torch.int32), room[:8])
    with pytest.raises(B.LserveError) as e:
        L.lserve_extend_tables(L.AttnDesc(4, 2, [1, 0]), kv, room[8:16], None, room[16:28], room[28:36], room[36:37], room[4:4], room[8:8].view(torch.int64),
                               total_new=0, stream=0)
    assert e.value.code == -4


def test_more_tokens_than_a_count_holds():
    kv = L.PagedKV(None, None, None, torch.zeros((8, 4), dtype=torch.int32), torch.zeros(8, dtype=torch.int32))
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        L.lserve_extend_tables(L.AttnDesc(4, 2, [1, 0]), kv, i32(8), None, i32(9), i32(8), i32(1), total_new=2 ** 32 + 1, stream=0)
