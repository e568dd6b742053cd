"""The calls on new tokens where addresses and slots pass 32 bits."""
import pytest
import torch

from tree_reference import Problem, random_tree

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _lib():
    import paper_2502_14866_amd as L

    L.load_library()
    return L


@pytest.mark.parametrize("bits,pages", [(16, 140000), (4, 500000)])
def test_pages_past_four_gigabytes(bits, pages):
    g = torch.Generator().manual_seed(1)
    p = Problem((700, 90), [random_tree(9, g), random_tree(40, g)], bits=bits, flags=[0, 1])
    for which in "kv":
        pool = p.pools[which]
        big = torch.empty((pages,) + tuple(pool.shape[1:]), dtype=pool.dtype, device=DEV)
        assert big.numel() * big.element_size() > 2 ** 32
        big[pages - len(pool):] = pool.to(DEV)
        p.pools[which] = big
        moved = pages - len(pool)
    p.table = torch.where(p.table >= 0, p.table + moved, p.table)
    out, lse = p.call(_lib())
    p.check(out, lse)


def test_rows_past_four_gigabytes():
    L = _lib()
    n, last = 600000, 300
    desc, rot = L.AttnDesc(32, 8, [0] * 8, dtype=torch.bfloat16), L.RotaryDesc(rotary_dim=96)
    q = torch.empty((n, 32, 128), dtype=torch.bfloat16, device=DEV)
    assert q.numel() > 2 ** 31
    q[-last:] = torch.randn((last, 32, 128), generator=torch.Generator().manual_seed(2)).bfloat16().to(DEV)
    pos = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    pos[-last:] = torch.arange(last, dtype=torch.int32, device=DEV) * 37
    want = torch.empty_like(q[-last:])
    L.lserve_rotary(desc, rot, q[-last:].clone(), None, pos[-last:].clone(), want, None)
    L.lserve_rotary(desc, rot, q, None, pos, q, None)
    torch.cuda.synchronize()
    got = q[-last:]
    off = (got.double() - want.double()).abs() - 2.0 ** -8 * (got.double().abs() + want.double().abs()) - 2.0 ** -20
    assert off.max() <= 0  # one rounding each, of numbers that differ in their last bits of 24 at most


def test_slots_past_32_bits():
    L = _lib()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    desc = L.AttnDesc(4, 2, [1, 0])
    kv = L.PagedKV(None, None, None, i32([[5, -1, -1, -1]]), i32([60, 0, 0, 0])[:1], ring_table=i32([list(range(2 ** 30, 2 ** 30 + 10))]))
    cu, new, taken, pos = i32([0, 0]), i32([0]), i32([0]), i32([0] * 80)
    slots, ring = torch.zeros(80, dtype=torch.int64, device=DEV), torch.zeros(80, dtype=torch.int64, device=DEV)
    L.lserve_extend_tables(desc, kv, i32([80]), i32([2 ** 31 - 1, 2 ** 30]), cu, new, taken, pos, slots, ring)
    torch.cuda.synchronize()
    page = [5, 2 ** 31 - 1, 2 ** 30]
    assert slots.tolist() == [page[t // 64] * 64 + t % 64 for t in range(60, 140)]
    assert ring.tolist() == [(2 ** 30 + t // 64) * 64 + t % 64 for t in range(60, 140)]
    assert kv.page_table.tolist() == [[5, 2 ** 31 - 1, 2 ** 30, -1]] and int(taken) == 2 and int(new) == 140
