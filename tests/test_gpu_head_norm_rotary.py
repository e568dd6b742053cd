"""Rotary positions of several axes, and head norms with the rotation, against the formulas in 64 bits."""
import math

import pytest
import torch

from turn_reference import assert_close, reference

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BASE = 500000.0


def _lib():
    import paper_2502_14866_amd as L

    L.load_library()
    return L


def _weights(g, norm, weights, hq, hkv):
    if not norm or not weights:
        return None, None
    return tuple(1 + 0.3 * torch.randn((h, 128) if weights == "heads" else (128,), generator=g) for h in (hq, hkv))


def _run(dtype, tokens, R, interleaved, pair_axis=None, norm=None, weights="shared", hq=8, hkv=2, far=5000, fused=False, in_place=False,
         positions=None, seed=0, eps=1e-6, rows=None, scale=0.0, apart=0):
    L = _lib()
    g = torch.Generator().manual_seed(seed)
    desc = L.AttnDesc(hq, hkv, [1] * (hkv // 2) + [0] * (hkv - hkv // 2), dtype=dtype)
    rot = L.RotaryDesc(rotary_dim=R, interleaved=interleaved, base=BASE, scale=scale) if R else None
    A = max(pair_axis) + 1 if pair_axis else 1
    if rows is None:
        rows = torch.randn((tokens, (hq + 2 * hkv) * 128), generator=g)
    rows = rows.to(dtype)
    q, k = rows[:, :hq * 128].view(tokens, hq, 128), rows[:, hq * 128:(hq + hkv) * 128].view(tokens, hkv, 128)
    if positions is None:
        positions = torch.randint(0, far, (A, tokens), generator=g)
    positions = torch.as_tensor(positions).to(torch.int32).view(A, tokens)
    wq, wk = _weights(g, norm, weights, hq, hkv)
    dev = rows.to(DEV)
    qd, kd = dev[:, :hq * 128].view(tokens, hq, 128), dev[:, hq * 128:(hq + hkv) * 128].view(tokens, hkv, 128)
    if not fused:
        qd, kd = qd.contiguous(), kd.contiguous()
    qo = qd if in_place else torch.full((tokens, hq, 128), 7.0, dtype=dtype, device=DEV)
    ko = kd if in_place else torch.full((tokens, hkv, 128), 7.0, dtype=dtype, device=DEV)
    axes = L.PositionAxes(pair_axis, A) if pair_axis else None
    pd = positions.to(DEV)
    if apart:  # axes of a longer buffer
        wide = torch.full((A, tokens + apart), -5, dtype=torch.int32, device=DEV)
        wide[:, :tokens] = pd
        pd = wide[:, :tokens]
    if norm:
        hn = L.HeadNorm(*(w.to(DEV) if w is not None else None for w in (wq, wk)), eps=eps, centred=norm == "centred")
        L.lserve_norm_rotary(desc, hn, rot, qd, kd, pd if axes else pd[0] if R else None, qo, ko, axes=axes)
    else:
        L.lserve_rotary_axes(desc, rot, axes, qd, kd, pd, qo, ko)
    torch.cuda.synchronize()
    there = positions[0] >= 0 if R else torch.ones(tokens, dtype=torch.bool)
    for x, got, w in ((q, qo, wq), (k, ko, wk)):
        ref, bound = reference(x, R, interleaved, positions, pair_axis or [0] * 64, rot.inv_freq.cpu() if R else None,
                               (rot.scale or 1.0) if R else 1.0, norm, w, eps)
        assert_close(got[there.to(DEV)], (ref[there], bound[there]), dtype)
        if not norm:
            assert torch.equal(got[..., R:].cpu()[there], x[..., R:][there])  # channels that do not turn
        gone = got.cpu()[~there]
        assert torch.equal(gone, x[~there] if in_place else torch.full_like(gone, 7.0))
    return qo, ko


def _axes(R, A, turns):
    n = R // 2
    return [i % A if turns else min(A - 1, i * A // n) for i in range(n)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [2, 6, 8, 16, 20, 32, 48, 64, 96, 112, 120, 126, 128])
def test_axes_of_parts_of_a_head(dtype, interleaved, R):
    A = min(3, R // 2)
    _run(dtype, 37, R, interleaved, _axes(R, A, True))
    _run(dtype, 1400, R, interleaved, _axes(R, A, False), seed=1)  # enough rows for lanes of eight pairs


@pytest.mark.parametrize("A", [1, 2, 3, 4])
@pytest.mark.parametrize("turns", [False, True])
@pytest.mark.parametrize("tokens", [1, 2, 63, 1300, 2051])
def test_numbers_of_axes(A, turns, tokens):
    axes = _axes(128, A, turns)
    axes[-1] = A - 1
    _run(torch.bfloat16, tokens, 128, tokens % 2 == 0, axes, fused=tokens % 2 == 1, seed=tokens, apart=tokens % 7)


def test_the_last_axis_may_have_no_pair():
    L = _lib()
    desc, rot = L.AttnDesc(8, 2, [1, 0]), L.RotaryDesc()
    q = torch.randn((5, 8, 128), generator=torch.Generator().manual_seed(1)).half().to(DEV)
    pos = torch.arange(20, dtype=torch.int32, device=DEV).view(4, 5)
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    L.lserve_rotary_axes(desc, rot, L.PositionAxes([0, 1] * 32, 4), q, None, pos, a, None)
    L.lserve_rotary_axes(desc, rot, L.PositionAxes([0, 1] * 32), q, None, pos[:2], b, None)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


@pytest.mark.parametrize("tokens", [40, 2000])
@pytest.mark.parametrize("interleaved,R", [(False, 128), (True, 128), (False, 64), (True, 20), (False, 20)])
def test_equal_positions_on_all_axes_are_one_axis(tokens, interleaved, R):
    """Within what two sums of the same formula may differ by: both against the same 64 bits."""
    positions = torch.randint(0, 9000, (1, tokens), generator=torch.Generator().manual_seed(4)).expand(3, tokens)
    a = _run(torch.float16, tokens, R, interleaved, _axes(R, 3, True), positions=positions, seed=9)
    b = _run(torch.float16, tokens, R, interleaved, [0] * (R // 2), positions=positions[:1], seed=9)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_far_and_negative_positions():
    far = [0, 1, 131071, 1000003, 16777217, 2 ** 31 - 1]
    _run(torch.float16, 6, 128, False, _axes(128, 2, True), positions=[far, [-x for x in far]])
    _run(torch.bfloat16, 6, 128, True, _axes(128, 2, True), positions=[far, [-2 ** 31] * 6])


@pytest.mark.parametrize("interleaved,R", [(False, 128), (True, 128), (False, 20), (True, 20)])
def test_rows_that_fill_up_a_batch(interleaved, R):
    """By axis 0 alone."""
    positions = [[5, -1, 7, -2 ** 31, 0, -1], [1, 2, -3, 4, 5, -6]]
    for in_place in (False, True):
        _run(torch.float16, 6, R, interleaved, _axes(R, 2, True), positions=positions, in_place=in_place)
        _run(torch.float16, 6, R, interleaved, _axes(R, 2, True), norm="rms", positions=positions, in_place=in_place)
    many = torch.randint(-40, 400, (2, 1500), generator=torch.Generator().manual_seed(2))
    _run(torch.float16, 1500, R, interleaved, _axes(R, 2, True), norm="rms", positions=many, in_place=True)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("norm", ["rms", "centred"])
@pytest.mark.parametrize("weights", [None, "shared", "heads"])
@pytest.mark.parametrize("interleaved,R", [(False, 128), (True, 128), (False, 64), (True, 36), (False, 20), (False, 0)])
@pytest.mark.parametrize("tokens", [3, 1337])
def test_norms(dtype, norm, weights, interleaved, R, tokens):
    _run(dtype, tokens, R, interleaved, norm=norm, weights=weights, fused=R == 64, seed=tokens)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (8, 1), (32, 8), (64, 64), (64, 8), (40, 5)])
@pytest.mark.parametrize("norm", [None, "rms"])
def test_heads(hq, hkv, norm):
    axes = _axes(128, 3, True)
    _run(torch.float16, 19, 128, False, axes, norm=norm, weights="heads", hq=hq, hkv=hkv)
    _run(torch.float16, 19, 12, True, axes[:6], norm=norm, hq=hq, hkv=hkv, fused=True)
    tokens = 13000 // (hq + hkv)
    _run(torch.bfloat16, tokens, 128, False, axes, norm=norm, weights="heads", hq=hq, hkv=hkv, fused=True)


@pytest.mark.parametrize("norm", [None, "rms", "centred"])
@pytest.mark.parametrize("interleaved,R", [(False, 128), (True, 64), (False, 36)])
@pytest.mark.parametrize("tokens", [77, 1700])
def test_in_place(norm, interleaved, R, tokens):
    _run(torch.float16, tokens, R, interleaved, _axes(R, 2, True), norm=norm, in_place=True)


def test_scaled_and_stretched():
    _run(torch.float16, 100, 64, False, norm="rms", scale=1.25)
    _run(torch.float16, 1500, 64, True, _axes(64, 3, True), scale=0.75)


@pytest.mark.parametrize("norm", ["rms", "centred"])
def test_rows_of_all_sizes(norm):
    """Zeros, the smallest numbers, large ones, a mean that is large against what is around it."""
    g = torch.Generator().manual_seed(3)
    for tokens in (8, 1400):
        rows = torch.randn((tokens, 12 * 128), generator=g)
        kind = torch.arange(tokens)[:, None] % 7
        rows = torch.where(kind == 0, torch.zeros(()), rows)
        rows = torch.where(kind == 1, rows * 1e-6, rows)
        rows = torch.where(kind == 2, rows * 8000, rows)
        rows = torch.where(kind == 3, rows * 0.1 + 50, rows)
        for eps in (1e-6, 1e-5, 0.1):
            _run(torch.float16, tokens, 128, False, norm=norm, rows=rows, eps=eps)
        _run(torch.bfloat16, tokens, 128, True, norm=norm, rows=rows * 1e12)
        _run(torch.bfloat16, tokens, 64, False, norm=norm, rows=rows * 1e-12, eps=1e-30)
        _run(torch.float16, tokens, 128, False, norm=norm, rows=rows, eps=2e-38)


def test_infinite_and_missing_numbers_stay_in_their_row():
    L = _lib()
    desc, rot = L.AttnDesc(8, 2, [1, 0]), L.RotaryDesc(rotary_dim=64)
    for tokens in (3, 2000):
        q = torch.randn((tokens, 8, 128), generator=torch.Generator().manual_seed(1)).half().to(DEV)
        pos = torch.arange(tokens, dtype=torch.int32, device=DEV)
        clean, spoiled = torch.zeros_like(q), torch.zeros_like(q)
        hn = L.HeadNorm()
        L.lserve_norm_rotary(desc, hn, rot, q, None, pos, clean, None)
        q[1, 2, 70] = math.nan
        q[2, 0, 3] = math.inf
        L.lserve_norm_rotary(desc, hn, rot, q, None, pos, spoiled, None)
        torch.cuda.synchronize()
        assert spoiled[1, 2].isnan().all()
        # of an infinite channel the norm makes no number, of the others zeros; the channel's pair turns with it
        assert spoiled[2, 0].isnan().nonzero().flatten().tolist() == [3, 35]
        assert (spoiled[2, 0][~spoiled[2, 0].isnan()] == 0).all()
        same = (clean == spoiled).all(-1)
        assert (~same).nonzero().tolist() == [[1, 2], [2, 0]]


def test_what_does_not_turn_keeps_its_bits():
    L = _lib()
    desc, rot = L.AttnDesc(8, 2, [1, 0]), L.RotaryDesc(rotary_dim=32)
    for tokens in (9, 1600):
        bits = torch.arange(tokens * 8 * 128, dtype=torch.int32).mul(7919).to(torch.int16).view(tokens, 8, 128).to(DEV)
        q = bits.view(torch.float16)
        out = torch.zeros_like(q)
        L.lserve_rotary_axes(desc, rot, L.PositionAxes([0, 1] * 8), q, None, torch.arange(2 * tokens, dtype=torch.int32, device=DEV).view(2, tokens), out, None)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16)[..., 32:], bits[..., 32:])


def test_queries_or_keys_alone():
    L = _lib()
    desc, rot, axes = L.AttnDesc(8, 2, [1, 0]), L.RotaryDesc(), L.PositionAxes.sections(16, 24, 24)
    g = torch.Generator().manual_seed(3)
    q, k = torch.randn((9, 8, 128), generator=g).half().to(DEV), torch.randn((9, 2, 128), generator=g).half().to(DEV)
    pos = torch.randint(0, 5000, (3, 9), generator=g).to(torch.int32).to(DEV)
    norm = L.HeadNorm(torch.rand(128, generator=g).to(DEV), torch.rand(128, generator=g).to(DEV))
    both = torch.zeros_like(q), torch.zeros_like(k)
    L.lserve_norm_rotary(desc, norm, rot, q, k, pos, *both, axes=axes)
    alone = torch.zeros_like(q), torch.zeros_like(k)
    L.lserve_norm_rotary(desc, norm, rot, q, None, pos, alone[0], None, axes=axes)
    L.lserve_norm_rotary(desc, norm, rot, None, k, pos, None, alone[1], axes=axes)
    torch.cuda.synchronize()
    assert torch.equal(both[0], alone[0]) and torch.equal(both[1], alone[1])


@pytest.mark.parametrize("tokens", [33, 1500])
def test_on_a_stream_of_its_own_and_captured(tokens):
    L = _lib()
    L.lserve_init()
    desc, rot, axes, norm = L.AttnDesc(8, 2, [1, 0]), L.RotaryDesc(), L.PositionAxes.in_turn(24, 20, 20), L.HeadNorm()
    q = torch.randn((tokens, 8, 128), generator=torch.Generator().manual_seed(2)).half().to(DEV)
    pos = torch.arange(3 * tokens, dtype=torch.int32, device=DEV).view(3, tokens)
    want, out = torch.zeros_like(q), torch.zeros_like(q)

    def call(to, **kw):
        L.lserve_norm_rotary(desc, norm, rot, q, None, pos, to, None, axes=axes, **kw)
        L.lserve_rotary_axes(desc, rot, axes, to, None, pos, to, None, **kw)

    call(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call(out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in range(3):
        pos.add_(100)
        graph.replay()
        call(want)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
