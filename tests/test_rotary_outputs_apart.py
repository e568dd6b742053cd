"""lserve_rotary refuses outputs that lie on what it reads or on each other, but for rows in their own place; gaps between rows are free."""
import pytest
import torch

import paper_2502_14866_amd as L
from paper_2502_14866_amd import binding as B

DESC = L.AttnDesc(4, 2, [1, 0])
HEADS = {"q": 4, "k": 2, "q_out": 4, "k_out": 2}
N = 5


def _code(place, positions=None, freq=None):
    t = {x: torch.zeros((N, h, 128), dtype=torch.float16) for x, h in HEADS.items()}
    t.update(place)
    rot = L.RotaryDesc(device="cpu", inv_freq=freq) if freq is not None else L.RotaryDesc(device="cpu")
    with pytest.raises(B.LserveError) as e:
        L.lserve_rotary(DESC, rot, t["q"], t["k"], positions if positions is not None else torch.zeros(N, dtype=torch.int32), t["q_out"], t["k_out"], stream=0)
    return e.value.code


def _rows(room, at, heads, apart):
    """N rows of heads from element `at` of a buffer on, `apart` elements from one to the next."""
    return room.as_strided((N, heads, 128), (apart, 128, 1), at)


@pytest.mark.parametrize("output,other", [("q_out", "k"), ("q_out", "k_out"), ("k_out", "q"), ("q_out", "q"), ("k_out", "k")])
@pytest.mark.parametrize("shift", [0, 8, -8])
def test_overlaps(output, other, shift):
    if shift == 0 and output[0] == other:
        return  # in place
    room = torch.zeros(8192, dtype=torch.float16)
    a, b = 64, 64 + shift
    assert _code({output: _rows(room, a, HEADS[output], HEADS[output] * 128), other: _rows(room, b, HEADS[other], HEADS[other] * 128)}) == -1


@pytest.mark.parametrize("output,wide", [("q_out", "q"), ("q_out", "k"), ("k_out", "q"), ("k_out", "k")])
def test_outputs_among_rows_that_lie_apart(output, wide):
    """An output between two rows is refused where it reaches one of them, and taken where it does not."""
    n, w, apart = N * HEADS[output] * 128, HEADS[wide] * 128, 8192
    room = torch.zeros(5 * apart, dtype=torch.float16)
    for row in range(4):
        free = row * apart + w, (row + 1) * apart - n
        for at, code in ((free[0], -4), (free[0] - 8, -1), (free[1], -4), (free[1] + 8, -1)):
            if torch.cuda.is_available() and code == -4:
                continue  # gets as far as a launch, on host memory
            assert _code({output: _rows(room, at, HEADS[output], HEADS[output] * 128), wide: _rows(room, 0, HEADS[wide], apart)}) == code, (row, at)
    for at, code in ((4 * apart + w, -4), (4 * apart + w - 8, -1)):
        if code == -1 or not torch.cuda.is_available():
            big = torch.zeros(6 * apart, dtype=torch.float16)
            assert _code({output: _rows(big, at, HEADS[output], HEADS[output] * 128), wide: _rows(big, 0, HEADS[wide], apart)}) == code


@pytest.mark.parametrize("output", ["q_out", "k_out"])
def test_positions_and_frequencies(output):
    room = torch.zeros(8192, dtype=torch.float16)
    out = {output: _rows(room, 64, HEADS[output], HEADS[output] * 128)}
    assert _code(out, positions=room[128:256].view(torch.int32)[:N]) == -1
    assert _code(out, freq=room[128:512].view(torch.float64)[:64]) == -1


@pytest.mark.skipif(torch.cuda.is_available(), reason="host memory")
def test_rows_in_their_own_place():
    """Get as far as the launch, which needs a GPU."""
    q, k = torch.zeros((N, 4, 128), dtype=torch.float16), torch.zeros((N, 2, 128), dtype=torch.float16)
    assert _code({"q": q, "q_out": q, "k": k, "k_out": k}) == -4
    wide = torch.zeros((N, 1024), dtype=torch.float16)  # a fused projection into tensors of their own
    assert _code({"q": wide[:, :512].view(N, 4, 128), "k": wide[:, 512:768].view(N, 2, 128)}) == -4
