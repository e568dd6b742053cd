"""What lserve_rotary_axes, lserve_norm_rotary and lserve_rotary_append_kv refuse, on the host and before anything is launched."""
import ctypes
import math

import pytest
import torch

import paper_2502_14866_amd as L
from paper_2502_14866_amd import binding as B

i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
f16 = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731


def _code(f, *a, **k):
    with pytest.raises(B.LserveError) as e:
        f(*a, **k)
    return e.value.code


def _c_rotary(dim=128, interleaved=0, scale=0.0, freq=True):
    d = L.RotaryDesc(device="cpu")
    d._c = B._CRotaryDesc(dim, interleaved, d.inv_freq.data_ptr() if freq else None, scale)
    return d


def _c_norm(kind=0, per_head=0, eps=1e-6):
    n = L.HeadNorm(torch.ones(4, 128), torch.ones(2, 128))
    n._c.kind, n._c.per_head, n._c.eps = kind, per_head, eps
    return n


def _off_by(numel, shape, dtype=torch.float32):
    """A tensor whose address is no multiple of 16 bytes."""
    return torch.zeros(numel + 1, dtype=dtype)[1:].view(shape)


AXES = L.PositionAxes.sections(16, 24, 24)


def _axes(**kw):
    q, k = f16(3, 4, 128), f16(3, 2, 128)
    a = dict(desc=L.AttnDesc(4, 2, [1, 0]), rotary=L.RotaryDesc(device="cpu"), axes=AXES, q=q, k=k, positions=i32(3, 3), q_out=torch.zeros_like(q),
             k_out=torch.zeros_like(k), stream=0)
    a.update(kw)
    return a


ROTARY = [(_c_rotary(0), -1), (_c_rotary(7), -1), (_c_rotary(130), -2), (_c_rotary(interleaved=2), -1), (_c_rotary(scale=-1.0), -1),
          (_c_rotary(scale=math.inf), -1), (_c_rotary(scale=math.nan), -1), (_c_rotary(freq=False), -1)]


@pytest.mark.parametrize("bad,code", [(dict(rotary=r), c) for r, c in ROTARY] + [
    (dict(q=None), -1), (dict(q_out=None), -1), (dict(q=None, q_out=None, k=None, k_out=None), -1),
    (dict(axes=L.PositionAxes([0, 1, 2, 3, 4] * 13, 5), positions=i32(5, 3)), -2), (dict(axes=L.PositionAxes([0, 1] * 31 + [2, 0], 2), positions=i32(2, 3)), -1),
    (dict(axes=L.PositionAxes([0, 1] * 31, 2), positions=i32(2, 3)), -1),  # 62 of 64 pairs
    (dict(q=f16(3, 4 * 128 + 4)[:, :512].view(3, 4, 128)), -1),   # rows not a multiple of 16 bytes apart
    (dict(q=f16(3, 512).as_strided((3, 4, 128), (256, 128, 1))), -1),  # rows that overlap
    (dict(positions=_off_by(9, (3, 3), torch.int32)), -1), (dict(desc=L.AttnDesc(4, 2, [1, 0], head_dim=64), q=f16(3, 4, 64), k=f16(3, 2, 64),
                                                                 q_out=f16(3, 4, 64), k_out=f16(3, 2, 64)), -2),
    (dict(positions=i32(6, 3).as_strided((3, 3), (2, 1))), -1),  # axes that overlap
])
def test_rotary_axes(bad, code):
    assert _code(L.lserve_rotary_axes, **_axes(**bad)) == code


@pytest.mark.parametrize("bad", [
    dict(q=torch.zeros((3, 4, 128), dtype=torch.bfloat16)), dict(q=f16(3, 5, 128)), dict(q=f16(3, 128, 4).transpose(1, 2)), dict(q=f16(2, 4, 128)),
    dict(q_out=f16(2, 4, 128)), dict(positions=torch.zeros((3, 3), dtype=torch.int64)), dict(positions=i32(3)), dict(positions=i32(2, 3)),
    dict(positions=i32(3, 6)[:, ::2]), dict(k_out=f16(3, 128, 2).transpose(1, 2)), dict(positions=None), dict(positions=i32(3, 0)),
])
def test_rotary_axes_tensors(bad):
    with pytest.raises(ValueError):
        L.lserve_rotary_axes(**_axes(**bad))


def test_rotary_axes_in_c():
    a, lib = _axes(), L.load_library()
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731

    def call(axes, stride=3, rotary=a["rotary"].c(), positions=p(a["positions"])):
        return lib.lserve_rotary_axes(a["desc"].c(), rotary, axes, p(a["q"]), p(a["k"]), positions, stride, 3, 512, 256, p(a["q_out"]), p(a["k_out"]), None)

    none = B._CPositionAxes(2, None)
    few = B._CPositionAxes(0, AXES._c.pair_axis)
    assert call(ctypes.byref(none)) == -1 and call(ctypes.byref(few)) == -1 and call(None) == -1
    assert call(ctypes.byref(AXES._c), stride=2) == -1
    assert call(ctypes.byref(AXES._c), rotary=None) == -1
    assert call(ctypes.byref(AXES._c), positions=None) == -1


def _norm(**kw):
    q, k = f16(3, 4, 128), f16(3, 2, 128)
    a = dict(desc=L.AttnDesc(4, 2, [1, 0]), norm=L.HeadNorm(torch.ones(128), torch.ones(128)), rotary=L.RotaryDesc(device="cpu"), q=q, k=k, positions=i32(3),
             q_out=torch.zeros_like(q), k_out=torch.zeros_like(k), stream=0)
    a.update(kw)
    return a


@pytest.mark.parametrize("bad,code", [(dict(rotary=r), c) for r, c in ROTARY] + [
    (dict(norm=_c_norm(kind=2)), -1), (dict(norm=_c_norm(kind=-1)), -1), (dict(norm=_c_norm(per_head=2)), -1), (dict(norm=L.HeadNorm(eps=0.0)), -1),
    (dict(norm=L.HeadNorm(eps=-1e-6)), -1), (dict(norm=L.HeadNorm(eps=math.nan)), -1), (dict(norm=L.HeadNorm(eps=math.inf)), -1),
    (dict(norm=L.HeadNorm(eps=1e-50)), -1), (dict(norm=L.HeadNorm(eps=1e-39)), -1),  # zero in 32 bits, a subnormal number
    (dict(norm=L.HeadNorm(_off_by(128, (128,)), None)), -1), (dict(norm=L.HeadNorm(None, _off_by(128, (128,)))), -1),
    (dict(positions=None), -1), (dict(rotary=None, axes=AXES, positions=i32(3, 3)), -1), (dict(q=None), -1), (dict(k_out=None), -1),
])
def test_norm_rotary(bad, code):
    assert _code(L.lserve_norm_rotary, **_norm(**bad)) == code


@pytest.mark.parametrize("bad", [
    dict(norm=L.HeadNorm(torch.ones(64), None)), dict(norm=L.HeadNorm(torch.ones(2, 128), None)), dict(norm=L.HeadNorm(None, torch.ones(1, 128))),
    dict(positions=i32(1, 3)), dict(positions=torch.zeros(3, dtype=torch.int64)), dict(axes=AXES), dict(q=f16(2, 4, 128)), dict(k_out=f16(2, 2, 128)),
    dict(positions=i32(6)[::2]),
])
def test_norm_rotary_tensors(bad):
    with pytest.raises(ValueError):
        L.lserve_norm_rotary(**_norm(**bad))


def test_descriptions():
    for bad in (dict(q_weight=torch.ones(128, dtype=torch.float16)), dict(q_weight=torch.ones(128), k_weight=torch.ones(2, 128)),
                dict(q_weight=torch.ones(1, 1, 128)), dict(q_weight=torch.ones(256)[::2])):
        with pytest.raises(ValueError):
            L.HeadNorm(**bad)
    for bad in ([], [-1, 0], [256]):
        with pytest.raises(ValueError):
            L.PositionAxes(bad)
    with pytest.raises(ValueError):
        L.PositionAxes.in_turn(2, 20, 20)
    assert L.PositionAxes.sections(2, 0, 3).pair_axis == [0, 0, 2, 2, 2] and L.PositionAxes.sections(2, 0, 3).num_axes == 3
    assert L.PositionAxes.in_turn(4, 2, 1).pair_axis == [0, 1, 2, 0, 1, 0, 0]
    assert L.PositionAxes.in_turn(24, 20, 20).pair_axis[:7] == [0, 1, 2, 0, 1, 2, 0] and L.PositionAxes.in_turn(24, 20, 20).pair_axis[-4:] == [0, 0, 0, 0]
    assert [L.PositionAxes.in_turn(24, 20, 20).pair_axis.count(a) for a in range(3)] == [24, 20, 20]


def _append(**kw):
    q, k, v = f16(6, 4, 128), f16(6, 2, 128), f16(6, 2, 128)
    kv = L.PagedKV(f16(8, 2, 64, 128), f16(8, 2, 64, 128), f16(8, 2, 4, 2, 128), i32(2, 4), i32(4)[:2])
    a = dict(desc=L.AttnDesc(4, 2, [1, 0]), kv=kv, rotary=L.RotaryDesc(device="cpu"), q=q, k=k, v=v, cu_new=i32(4)[:3], start_pos=i32(4)[:2], max_new_per_seq=3,
             q_out=torch.zeros_like(q), stream=0)
    a.update(kw)
    return a


def _kv(**kw):
    a = dict(k_pool=f16(8, 2, 64, 128), v_pool=f16(8, 2, 64, 128), stats=f16(8, 2, 4, 2, 128), page_table=i32(2, 4), seq_lens=i32(4)[:2])
    a.update(kw)
    return L.PagedKV(**a)


@pytest.mark.parametrize("bad,code", [(dict(rotary=r), c) for r, c in ROTARY] + [
    (dict(k=None), -1), (dict(v=None), -1), (dict(q=None), -1), (dict(q_out=None), -1), (dict(cu_new=None), -1), (dict(start_pos=None), -1),
    (dict(max_new_per_seq=0), -1), (dict(max_new_per_seq=-1), -1), (dict(kv=_kv(k_pool=None)), -1), (dict(kv=_kv(stats=None)), -1),
    (dict(kv=_kv(pool_heads=1)), -1),  # the streaming head has no pool
    (dict(kv=_kv(kv_bits=5)), -1), (dict(norm=_c_norm(kind=3)), -1), (dict(rotary=None, axes=AXES), -1),
    (dict(axes=L.PositionAxes([0, 1, 2, 3, 4] * 13, 5)), -2), (dict(axes=L.PositionAxes([0, 1] * 31 + [2, 0], 2)), -1),
    (dict(k=f16(6, 260)[:, :256].view(6, 2, 128)), -1), (dict(v=f16(6, 260)[:, :256].view(6, 2, 128)), -1),
    (dict(cu_new=i32(4)[1:]), -1), (dict(start_pos=i32(3)[1:]), -1),
    (dict(desc=L.AttnDesc(4, 2, [1, 0], page_size=48)), -2),
    (dict(desc=L.AttnDesc(4, 2, [1, 0], page_size=32, logical_page_size=16), kv=L.PagedKV(torch.zeros(8, 2, 8448, dtype=torch.uint8), torch.zeros(8, 2, 8448, dtype=torch.uint8),
          f16(8, 2, 4, 2, 128), i32(2, 4), i32(4)[:2], kv_bits=8)), -2),  # quantised pages hold 64 tokens
])
def test_rotary_append(bad, code):
    assert _code(L.lserve_rotary_append_kv, **_append(**bad)) == code


@pytest.mark.parametrize("bad", [
    dict(q=f16(5, 4, 128)), dict(q=torch.zeros((6, 4, 128), dtype=torch.bfloat16)), dict(k=f16(6, 3, 128)), dict(v=f16(5, 2, 128)), dict(q_out=f16(5, 4, 128)),
    dict(k_out=f16(5, 2, 128)), dict(v_out=f16(6, 2, 64)), dict(cu_new=i32(2)), dict(cu_new=torch.zeros(3, dtype=torch.int64)), dict(start_pos=i32(1)),
    dict(positions=i32(5)), dict(positions=i32(3, 6)), dict(positions=i32(2, 6), axes=AXES), dict(kv=_kv(v_pool=f16(7, 2, 64, 128))),
    dict(kv=_kv(stats=f16(8, 1, 4, 2, 128))), dict(kv=_kv(k_pool=torch.zeros(8, 2, 64, 128))), dict(norm=L.HeadNorm(torch.ones(3, 128), None)),
    dict(kv=_kv(k_pool=f16(8, 1, 64, 128), v_pool=f16(8, 1, 64, 128), pool_heads=1, stats=f16(8, 1, 4, 2, 128), k_pool_stream=f16(20, 1, 64, 128),
                v_pool_stream=f16(20, 1, 64, 128), ring_table=i32(2, 9))),
])
def test_rotary_append_tensors(bad):
    with pytest.raises(ValueError):
        L.lserve_rotary_append_kv(**_append(**bad))


ROOM = 1 << 15
SIZES = {"q": 4 * 128, "k": 2 * 128, "v": 2 * 128, "q_out": 4 * 128, "k_out": 2 * 128, "v_out": 2 * 128}


def _at(room, at, name, n=6, apart=None):
    row = SIZES[name]
    return room.as_strided((n, row // 128, 128), (apart or row, 128, 1), at)


@pytest.mark.parametrize("output", ["q_out", "k_out", "v_out"])
@pytest.mark.parametrize("other", ["q", "k", "v", "q_out", "k_out", "v_out"])
@pytest.mark.parametrize("shift", [0, 8, -8])
def test_outputs_on_rows_or_on_each_other(output, other, shift):
    """But for queries and keys in their own place."""
    if output == other or (shift == 0 and output[0] == other and other != "v"):
        return
    room = f16(ROOM)
    place = {output: _at(room, 64, output), other: _at(room, 64 + shift, other)}
    assert _code(L.lserve_rotary_append_kv, **_append(**place)) == -1
    if "v" not in (output[0], other[0]):
        a = _norm(q=f16(6, 4, 128), k=f16(6, 2, 128), q_out=f16(6, 4, 128), k_out=f16(6, 2, 128), positions=i32(6))
        assert _code(L.lserve_norm_rotary, **{**a, **place}) == -1


@pytest.mark.parametrize("output", ["q_out", "k_out", "v_out"])
@pytest.mark.parametrize("other", ["k_pool", "v_pool", "stats", "page_table", "cu_new", "start_pos", "positions", "inv_freq", "q_weight", "k_weight"])
def test_outputs_on_the_cache_or_what_is_read(output, other):
    room = torch.zeros(1 << 19, dtype=torch.uint8)
    place, n = {output: room[:6 * SIZES[output] * 2].view(torch.float16).view(6, -1, 128)}, 6 * SIZES[output] * 2
    behind = room[n - 16:]  # whose first sixteen bytes are the output's last
    kinds = {"k_pool": (torch.float16, (8, 2, 64, 128)), "v_pool": (torch.float16, (8, 2, 64, 128)), "stats": (torch.float16, (8, 2, 4, 2, 128)), "page_table": (torch.int32, (2, 4)),
             "cu_new": (torch.int32, (3,)), "start_pos": (torch.int32, (2,)), "positions": (torch.int32, (6,)), "inv_freq": (torch.float64, (64,)),
             "q_weight": (torch.float32, (128,)), "k_weight": (torch.float32, (128,))}
    kind, shape = kinds[other]
    t = behind[:math.prod(shape) * torch.empty(0, dtype=kind).element_size()].view(kind).view(shape)
    if other in ("k_pool", "v_pool", "stats", "page_table"):
        place["kv"] = _kv(**{other: t})
    elif other == "inv_freq":
        place["rotary"] = L.RotaryDesc(inv_freq=t, device="cpu")
    elif other in ("q_weight", "k_weight"):
        place["norm"] = L.HeadNorm(**{other: t})
    else:
        place[other] = t
    assert _code(L.lserve_rotary_append_kv, **_append(**place)) == -1


def test_pools_on_each_other():
    k = f16(8, 2, 64, 128)
    assert _code(L.lserve_rotary_append_kv, **_append(kv=_kv(k_pool=k, v_pool=k))) == -1
    ring = dict(pool_heads=1, k_pool=f16(8, 1, 64, 128), stats=f16(8, 1, 4, 2, 128), ring_table=i32(2, 10))
    pool = f16(20, 1, 64, 128)
    assert _code(L.lserve_rotary_append_kv, **_append(kv=_kv(v_pool=f16(8, 1, 64, 128), k_pool_stream=pool, v_pool_stream=pool, **ring))) == -1
    assert _code(L.lserve_rotary_append_kv, **_append(kv=_kv(v_pool=pool[:8], k_pool_stream=f16(20, 1, 64, 128), v_pool_stream=pool, **ring))) == -1


def test_rows_in_place_are_dense():
    lib, a = L.load_library(), _append()
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    wide = f16(6, 1024)
    code = lib.lserve_rotary_append_kv(a["desc"].c(), a["kv"].c(), None, a["rotary"].c(), None, p(wide), p(a["k"]), p(a["v"]), 1024, 256, 256, None, 0, p(a["cu_new"]),
                                       p(a["start_pos"]), 6, 3, p(wide), None, None, None)
    assert code == -1
