"""lserve_extend_tables with as many new tokens as a 32-bit count holds: the last ones, and nothing behind them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("total", [2 ** 31 - 1, 2 ** 31 - 1024, 2 ** 31 - 1025])
def test_tokens_next_to_31_bits(total):
    import paper_2502_14866_amd as L

    L.load_library()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    kv = L.PagedKV(None, None, None, i32([[-7, -7]]), i32([0]))
    cu, lens, taken = i32([0, 0]), i32([0]), i32([0])
    room = torch.full((2 ** 31 + 8,), -9, dtype=torch.int32, device=DEV)
    held = total - 3  # the last three belong to nobody
    L.lserve_extend_tables(L.AttnDesc(4, 2, [1, 0]), kv, i32([held]), i32([41, 40, 39]), cu, lens, taken, positions=room[:total])
    torch.cuda.synchronize()
    assert cu.tolist() == [0, held] and lens.tolist() == [held] and taken.tolist() == [2] and kv.page_table.tolist() == [[41, 40]]
    step = 1 << 26
    for at in range(0, held, step):
        n = min(step, held - at)
        assert torch.equal(room[at:at + n], torch.arange(at, at + n, dtype=torch.int64, device=DEV).to(torch.int32)), at
    assert room[held:total].tolist() == [-1] * 3
    assert bool((room[total:] == -9).all())

