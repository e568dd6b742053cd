"""Rotary positions against the formula in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _lib():
    import paper_2502_14866_amd as L

    L.load_library()
    return L


def _reference(x, positions, freq, R, interleaved, scale):
    """(turned rows, |a| + |b| of every channel's pair, |angle| of it) in 64 bits."""
    y = x.double()
    angle = positions.double()[:, None] * freq
    c, s = angle.cos()[:, None] * scale, angle.sin()[:, None] * scale
    out, size, far = y.clone(), torch.zeros_like(y), torch.zeros_like(y)
    ia = torch.arange(0, R, 2) if interleaved else torch.arange(R // 2)
    ib = ia + (1 if interleaved else R // 2)
    a, b = y[..., ia], y[..., ib]
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    for i in (ia, ib):
        size[..., i] = a.abs() + b.abs()
        far[..., i] = angle.abs()[:, None].expand_as(a)
    return out, size, far


def _close(got, want, dtype, scale):
    """One rounding to the type (half a step, or half the smallest number).  Before it, in fp32: the part of a turn off by 2^-26, so
    the angle by 2 pi 2^-26 = 0.94e-7; sine and cosine by two steps of 2^-24 each of which 1.2e-7; scale, two products and their sum by 2^-24
    each, 2.4e-7: 4.6e-7 of |a| + |b|, and what an angle in 64 bits loses (2^-52 of it, in either computation)."""
    ref, size, far = want
    g = got.cpu().double()
    half = torch.finfo(dtype).eps / 2
    tol = ref.abs() * half + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2 + \
        size * scale * (4.6e-7 + 2 * far * 2.0 ** -52) * (1 + half)
    worst = ((g - ref).abs() - tol).max()
    assert worst <= 0, float(worst)


def _run(dtype, tokens, R, interleaved, hq=8, hkv=2, far=5000, fused=False, in_place=False, scaling="none", positions=None, seed=0, **kw):
    L = _lib()
    g = torch.Generator().manual_seed(seed)
    desc = L.AttnDesc(hq, hkv, [1] * (hkv // 2) + [0] * (hkv - hkv // 2), dtype=dtype)
    rot = L.RotaryDesc(rotary_dim=R, interleaved=interleaved, base=500000.0, scaling=scaling, **kw)
    rows = torch.randn((tokens, (hq + 2 * hkv) * 128), generator=g).to(dtype)
    q, k = rows[:, :hq * 128].view(tokens, hq, 128), rows[:, hq * 128:(hq + hkv) * 128].view(tokens, hkv, 128)
    if positions is None:
        positions = torch.randint(0, far, (tokens,), generator=g)
    positions = torch.as_tensor(positions).to(torch.int32)
    dev = rows.to(DEV)
    qd, kd = dev[:, :hq * 128].view(tokens, hq, 128), dev[:, hq * 128:(hq + hkv) * 128].view(tokens, hkv, 128)
    if not fused:
        qd, kd = qd.contiguous(), kd.contiguous()
    qo = qd if in_place else torch.full((tokens, hq, 128), 7.0, dtype=dtype, device=DEV)
    ko = kd if in_place else torch.full((tokens, hkv, 128), 7.0, dtype=dtype, device=DEV)
    L.lserve_rotary(desc, rot, qd, kd, positions.to(DEV), qo, ko)
    torch.cuda.synchronize()
    freq, scale = rot.inv_freq.cpu(), rot.scale or 1.0
    there = positions >= 0
    for x, got in ((q, qo), (k, ko)):
        ref, size, angle = _reference(x, positions, freq, R, interleaved, scale)
        _close(got[there.to(DEV)], (ref[there], size[there], angle[there]), dtype, scale)
        assert torch.equal(got[..., R:].cpu()[there], x[..., R:][there])  # channels that do not turn
        gone = got.cpu()[~there]
        assert torch.equal(gone, x[~there] if in_place else torch.full_like(gone, 7.0))
    return qo, ko


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [2, 6, 8, 16, 20, 32, 48, 64, 96, 112, 120, 126, 128])
def test_parts_of_a_head(dtype, interleaved, R):
    _run(dtype, 37, R, interleaved)


@pytest.mark.parametrize("tokens", [1, 2, 5, 64, 511, 2100, 9001])
@pytest.mark.parametrize("interleaved,R", [(False, 128), (True, 128), (False, 20), (True, 20)])
def test_numbers_of_tokens(tokens, interleaved, R):
    _run(torch.bfloat16, tokens, R, interleaved, fused=tokens % 2 == 1, seed=tokens)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (8, 1), (32, 8), (64, 64), (64, 8), (40, 5)])
def test_heads(hq, hkv):
    _run(torch.float16, 19, 128, False, hq=hq, hkv=hkv)
    _run(torch.float16, 19, 12, True, hq=hq, hkv=hkv, fused=True)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [128, 64, 36])
def test_in_place(interleaved, R):
    _run(torch.float16, 77, R, interleaved, in_place=True)


def test_far_positions():
    _run(torch.float16, 6, 128, False, positions=[0, 1, 131071, 1000003, 16777217, 2 ** 31 - 1])
    _run(torch.bfloat16, 500, 128, True, far=2000000)


@pytest.mark.parametrize("scaling,kw", [("linear", dict(factor=4.0)), ("wavelength", dict(factor=8.0)), ("ramp", dict(factor=16.0, low=1.0, high=32.0))])
def test_stretched_positions(scaling, kw):
    _run(torch.float16, 100, 128, False, far=100000, scaling=scaling, **kw)


def test_rows_that_fill_up_a_batch():
    positions = [5, -1, 7, -2 ** 31, 0, -1]
    _run(torch.float16, 6, 128, False, positions=positions)
    _run(torch.float16, 6, 128, False, positions=positions, in_place=True)
    _run(torch.float16, 6, 20, True, positions=positions, in_place=True)


def test_queries_or_keys_alone():
    L = _lib()
    desc, rot = L.AttnDesc(8, 2, [1, 0]), L.RotaryDesc()
    q, k = _run(torch.float16, 9, 128, False, seed=3)
    g = torch.Generator().manual_seed(3)
    rows = torch.randn((9, 12 * 128), generator=g).half()
    pos = torch.randint(0, 5000, (9,), generator=g).to(torch.int32).to(DEV)
    rot = L.RotaryDesc(base=500000.0)
    qi, ki = rows[:, :1024].view(9, 8, 128).contiguous().to(DEV), rows[:, 1024:1280].view(9, 2, 128).contiguous().to(DEV)
    qo, ko = torch.zeros_like(qi), torch.zeros_like(ki)
    L.lserve_rotary(desc, rot, qi, None, pos, qo, None)
    L.lserve_rotary(desc, rot, None, ki, pos, None, ko)
    torch.cuda.synchronize()
    assert torch.equal(qo, q) and torch.equal(ko, k)


def test_what_does_not_turn_keeps_its_bits():
    L = _lib()
    desc, rot = L.AttnDesc(8, 2, [1, 0]), L.RotaryDesc(rotary_dim=32)
    bits = torch.arange(9 * 8 * 128, dtype=torch.int32).mul(7919).to(torch.int16).view(9, 8, 128).to(DEV)
    q = bits.view(torch.float16)
    out = torch.zeros_like(q)
    L.lserve_rotary(desc, rot, q, None, torch.arange(9, dtype=torch.int32, device=DEV), out, None)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16)[..., 32:], bits[..., 32:])


def test_not_a_number_stays_in_its_pair():
    L = _lib()
    desc, rot = L.AttnDesc(8, 2, [1, 0]), L.RotaryDesc()
    q = torch.randn((3, 8, 128), generator=torch.Generator().manual_seed(1)).half().to(DEV)
    pos = torch.tensor([4, 5, 6], dtype=torch.int32, device=DEV)
    clean, spoiled = torch.zeros_like(q), torch.zeros_like(q)
    L.lserve_rotary(desc, rot, q, None, pos, clean, None)
    q[1, 2, 70] = math.nan
    q[2, 0, 3] = math.inf
    L.lserve_rotary(desc, rot, q, None, pos, spoiled, None)
    torch.cuda.synchronize()
    changed = (clean != spoiled).nonzero().tolist()
    assert sorted(changed) == [[1, 2, 6], [1, 2, 70], [2, 0, 3], [2, 0, 67]]


def test_on_a_stream_of_its_own_and_captured():
    L = _lib()
    L.lserve_init()
    desc, rot = L.AttnDesc(8, 2, [1, 0]), L.RotaryDesc()
    q = torch.randn((33, 8, 128), generator=torch.Generator().manual_seed(2)).half().to(DEV)
    pos = torch.arange(33, dtype=torch.int32, device=DEV)
    want, out = torch.zeros_like(q), torch.zeros_like(q)
    L.lserve_rotary(desc, rot, q, None, pos, want, None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    L.lserve_rotary(desc, rot, q, None, pos, out, None, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.lserve_rotary(desc, rot, q, None, pos, out, None)
    for i in range(3):
        pos.add_(100)
        graph.replay()
        L.lserve_rotary(desc, rot, q, None, pos, want, None)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
