"""lserve_sparse_decode_tree refuses outputs and workspaces that lie on what it reads or on each other."""
import pytest
import torch

import paper_2502_14866_amd as L
from paper_2502_14866_amd import binding as B

TOTAL, BATCH, PAGES, STRIDE = 8, 2, 4, 4
DESC = L.AttnDesc(4, 2, [1, 0])
BYTES = {"q": TOTAL * 4 * 256, "k": TOTAL * 2 * 256, "v": TOTAL * 2 * 256, "cu": 4 * (BATCH + 1), "mask": TOTAL * 8, "pos": TOTAL * 4, "sel": BATCH * 2 * STRIDE * 4,
         "count": BATCH * 2 * 4, "ssl": BATCH * 4, "lens": BATCH * 4, "table": BATCH * PAGES * 4, "ring": BATCH * 10 * 4, "out": TOTAL * 4 * 256,
         "lse": TOTAL * 4 * 4, "ws": L.lserve_tree_workspace_bytes(DESC, BATCH, TOTAL, 4, PAGES, STRIDE)}
WRITTEN = ["out", "lse", "ws"]


def _call(place):
    t = {k: torch.zeros(n, dtype=torch.uint8) for k, n in BYTES.items()}
    t.update(place)
    half, i32 = lambda x: x.view(torch.float16), lambda x: x.view(torch.int32)  # noqa: E731
    pool = torch.zeros((8, 2, 64, 128), dtype=torch.float16)
    bounded = torch.zeros((20, 1, 64, 128), dtype=torch.float16)
    kv = L.PagedKV(pool, pool, None, i32(t["table"]).view(BATCH, PAGES), i32(t["lens"]), k_pool_stream=bounded, v_pool_stream=bounded,
                   ring_table=i32(t["ring"]).view(BATCH, 10))
    L.lserve_sparse_decode_tree(DESC, kv, half(t["q"]).view(TOTAL, 4, 128), half(t["k"]).view(TOTAL, 2, 128), half(t["v"]).view(TOTAL, 2, 128), i32(t["cu"]), 4,
                                half(t["out"]).view(TOTAL, 4, 128), t["lse"].view(torch.float32).view(TOTAL, 4),
                                tree_mask=t["mask"].view(torch.int64).view(TOTAL, 1), positions=i32(t["pos"]), sel_pages=i32(t["sel"]).view(BATCH, 2, STRIDE),
                                sel_count=i32(t["count"]).view(BATCH, 2), sel_seq_len=i32(t["ssl"]), workspace=t["ws"], stream=0)


@pytest.mark.parametrize("output,other", [(o, x) for o in WRITTEN for x in BYTES if x != o])
@pytest.mark.parametrize("shift", [0, 16, -16])
def test_overlaps(output, other, shift):
    """At one address, and by 16 bytes off to either side."""
    if min(BYTES[output], BYTES[other]) <= 16:
        shift = 0
    room = torch.zeros(BYTES[output] + BYTES[other] + 64, dtype=torch.uint8)
    a, b = max(0, -shift), max(0, shift)
    with pytest.raises(B.LserveError) as e:
        _call({output: room[a:a + BYTES[output]], other: room[b:b + BYTES[other]]})
    assert e.value.code == -1
