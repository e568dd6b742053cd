"""lserve_rotary on large batches, whose rows are worked on in pieces of eight channels where the channels that turn come in such."""
import math

import pytest
import torch

from test_gpu_rotary import DEV, _lib, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [2, 6, 8, 16, 20, 32, 48, 64, 96, 112, 120, 128])
def test_parts_of_a_head(dtype, interleaved, R):
    _run(dtype, 2003, R, interleaved, seed=R)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (8, 1), (32, 8), (64, 64), (40, 5)])
@pytest.mark.parametrize("interleaved,R", [(False, 128), (False, 48), (True, 72)])
def test_heads(hq, hkv, interleaved, R):
    _run(torch.float16, 13000 // (hq + hkv) + 1, R, interleaved, hq=hq, hkv=hkv, fused=hq == 8)


@pytest.mark.parametrize("interleaved,R", [(False, 128), (True, 128), (False, 64), (True, 8)])
def test_in_place_with_rows_that_fill_up_a_batch(interleaved, R):
    positions = torch.arange(1700) % 900
    positions[::7] = -1
    _run(torch.bfloat16, 1700, R, interleaved, in_place=True, positions=positions)
    _run(torch.bfloat16, 1700, R, interleaved, fused=True, positions=positions)


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_same_with_few_tokens_and_with_many(interleaved):
    """A token's rows do not depend on how many others there are."""
    L = _lib()
    desc, rot = L.AttnDesc(8, 2, [1, 0], dtype=torch.float16), L.RotaryDesc(rotary_dim=96, interleaved=interleaved, base=500000.0)
    g = torch.Generator().manual_seed(3)
    q, k = (torch.randn((4000, h, 128), generator=g).half().to(DEV) for h in (8, 2))
    pos = torch.randint(0, 100000, (4000,), generator=g).to(torch.int32).to(DEV)
    outs = []
    for n in (4000, 50):
        qo, ko = torch.empty_like(q[:n]), torch.empty_like(k[:n])
        L.lserve_rotary(desc, rot, q[:n], k[:n], pos[:n], qo, ko)
        outs.append((qo, ko))
    torch.cuda.synchronize()
    for many, few in zip(*outs):
        off = (many[:50].double() - few.double()).abs() - 2.0 ** -11 * (many[:50].double().abs() + few.double().abs()) - 2.0 ** -20
        assert off.max() <= 0  # one rounding each, of numbers that differ in their last bits of 24 at most


@pytest.mark.parametrize("interleaved", [False, True])
def test_not_a_number_stays_in_its_pair(interleaved):
    L = _lib()
    R, n = 64, 1500
    desc, rot = L.AttnDesc(8, 2, [1, 0], dtype=torch.float16), L.RotaryDesc(rotary_dim=R, interleaved=interleaved)
    q = torch.ones((n, 8, 128), dtype=torch.float16)
    q[:, 3, 10], q[:, 5, 100] = math.nan, math.inf
    qo = torch.zeros_like(q).to(DEV)
    L.lserve_rotary(desc, rot, q.to(DEV), None, torch.arange(n, dtype=torch.int32, device=DEV), qo, None)
    bad = ~torch.isfinite(qo.cpu())
    want = torch.zeros_like(bad)
    want[:, 3, [10, 11] if interleaved else [10, 42]] = True
    want[:, 5, 100] = True
    assert torch.equal(bad, want) and bool((qo[:, 5, 100] == math.inf).all())
