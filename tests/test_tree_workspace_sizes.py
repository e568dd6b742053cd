"""lserve_tree_workspace_bytes is for the sizes of one call: what a kept workspace has to be."""
import random

import pytest

import paper_2502_14866_amd as L


def test_smaller_calls_may_need_more():
    d = L.AttnDesc(32, 8, [0] * 8)
    assert L.lserve_tree_workspace_bytes(d, 512, 512, 1, 512) == 0  # no list is cut
    # 512 pieces and 4088 lists, each 64 rows (over quantised pages) of 128 sums, a maximum and a sum; 8 bytes a list, filled up to 256
    assert L.lserve_tree_workspace_bytes(d, 511, 511, 1, 512) == (512 + 4088) * 64 * (128 + 2) * 4 + 4088 * 8 // 256 * 256 + 256
    assert L.lserve_tree_workspace_bytes(d, 16, 16 * 1024, 1024, 512) == 0
    assert L.lserve_tree_workspace_bytes(d, 1, 1024, 1024, 512) > 0


@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("hkv", [1, 2, 8, 32, 64])
def test_no_call_needs_more_than_the_bound(group, hkv):
    """The most there is: 512 pieces, a list less than the 4096 from which on none is cut, and workgroups to fill eight rows of tiles up,
    128 rows of 128 sums, a maximum and a sum each; where the pieces are, 8 bytes a list and row tile."""
    rng, most = random.Random(group * 100 + hkv), 0
    d = L.AttnDesc(group * hkv, hkv, [i % 2 for i in range(hkv)])
    for _ in range(600):
        batch, nodes = min(65535, int(2 ** rng.uniform(0, 16))), min(1024, int(2 ** rng.uniform(0, 10.01)))
        total = min(2 ** 30, rng.randint(nodes, max(nodes, batch * nodes)))
        most = max(most, L.lserve_tree_workspace_bytes(d, batch, total, nodes, int(2 ** rng.uniform(0, 17)), rng.choice([0, 0, 64, 512])))
    row_tiles = -(-1024 * group // 128)
    assert 0 < most <= (512 + 4095 + 8 * row_tiles) * 128 * (128 + 2) * 4 + 4095 * row_tiles * 8 + 256 <= L.LSERVE_TREE_WORKSPACE_MOST
