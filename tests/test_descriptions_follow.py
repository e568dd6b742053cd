"""Descriptions of how heads are normed and turned, changed after they were made: the next call works with what they say now, or the change is refused.  And
a session's call of the same arguments."""
import ctypes

import pytest
import torch

import paper_2502_14866_amd as L
from paper_2502_14866_amd import binding as B
from test_turned_calls_native import _stand_in, _tensors

ROUTES = pytest.mark.parametrize("route", ["native", "ctypes"])


def _called(monkeypatch, route, t, norm):
    """What both calls that take a norm hand over of it."""
    kv = L.PagedKV(t["k"], t["v"], t["stats"], t["table"], t["lens"], pool_heads=1, k_pool_stream=t["ks"], v_pool_stream=t["vs"], ring_table=t["ring"])
    desc, rot = L.AttnDesc(4, 2, [1, 0]), L.RotaryDesc(rotary_dim=64, inv_freq=t["freq"], device="cpu")
    with _stand_in(monkeypatch, route) as seen:
        L.lserve_norm_rotary(desc, norm, rot, t["qn"], t["kn"], t["pos"], t["qo"], t["ko"], 0x10)
        L.lserve_rotary_append_kv(desc, kv, rot, None, t["kn"], t["vn"], t["cu"], t["lens"], 1, None, norm=norm, stream=0x20)
    return [s[2] for s in seen[:1]] + [s[3] for s in seen[1:]]


def _says(norm, t_q, t_k, per_head, eps, kind):
    where = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
    return (norm.q_weight, norm.k_weight, norm.per_head, round(norm.eps, 9), norm.kind) == (where(t_q), where(t_k), per_head, eps, kind)


@ROUTES
def test_weights_assigned_anew(monkeypatch, route):
    t = _tensors()
    norm = L.HeadNorm(t["wq"], t["wk"], eps=1e-5)
    q, k = torch.ones(4, 128), torch.ones(2, 128)
    norm.q_weight, norm.k_weight = q, k
    assert all(_says(n, q, k, 1, 1e-5, 0) for n in _called(monkeypatch, route, t, norm))
    norm.k_weight = None
    assert all(_says(n, q, None, 1, 1e-5, 0) for n in _called(monkeypatch, route, t, norm))
    norm.q_weight = None
    norm.k_weight = torch.ones(128)  # from weights a head to shared ones
    assert all(_says(n, None, norm.k_weight, 0, 1e-5, 0) for n in _called(monkeypatch, route, t, norm))


@ROUTES
def test_weights_whose_memory_is_another(monkeypatch, route):
    """What a module that is moved, or loaded by its tensors' data, does."""
    t = _tensors()
    norm = L.HeadNorm(torch.nn.Parameter(torch.ones(4, 128)), torch.nn.Parameter(torch.ones(2, 128)))
    moved = torch.ones(4, 128), torch.ones(2, 128)
    norm.q_weight.data, norm.k_weight.data = moved
    assert all(_says(n, *moved, 1, 1e-6, 0) for n in _called(monkeypatch, route, t, norm))
    # (the type and the size are those of the new memory)
    norm.q_weight.data = torch.ones(3, 128)
    with pytest.raises(ValueError):
        _called(monkeypatch, route, t, norm)


@ROUTES
def test_eps_and_kind(monkeypatch, route):
    t = _tensors()
    norm = L.HeadNorm(t["wq"], t["wk"])
    norm.eps, norm.centred = 1e-3, True
    assert all(_says(n, t["wq"], t["wk"], 1, 1e-3, 1) for n in _called(monkeypatch, route, t, norm))


def test_a_change_that_is_refused_leaves_it_as_it_was(monkeypatch):
    t = _tensors()
    norm = L.HeadNorm(t["wq"], t["wk"])
    for bad in (torch.ones(128), torch.ones(4, 128, dtype=torch.float16), torch.ones(1, 4, 128), torch.ones(4, 256)[:, ::2]):
        with pytest.raises(ValueError):
            norm.q_weight = bad
        assert norm.q_weight is t["wq"]
    assert all(_says(n, t["wq"], t["wk"], 1, 1e-6, 0) for n in _called(monkeypatch, "ctypes", t, norm))


def test_axes_stay_as_they_were_made():
    """The library's copy of the list is the only one: nothing that looks like a change goes unseen."""
    given = [0, 1, 2, 0] * 16
    axes = L.PositionAxes(given)
    given[0] = 2
    axes.pair_axis[1] = 2
    assert axes.pair_axis == [0, 1, 2, 0] * 16 and list(axes._c.pair_axis[:64]) == axes.pair_axis and axes.num_axes == axes._c.num_axes == 3
    for name, value in (("pair_axis", [0] * 64), ("num_axes", 4)):
        with pytest.raises(AttributeError):
            setattr(axes, name, value)
    assert axes == L.PositionAxes([0, 1, 2, 0] * 16) and axes != L.PositionAxes([0] * 64, 3) and axes != L.PositionAxes([0, 1, 2, 0] * 16, 4)
    assert repr(L.PositionAxes([0, 1], 3)) == "PositionAxes(pair_axis=[0, 1], num_axes=3)"
    assert L.PositionAxes(pair_axis=range(70), num_axes=2).pair_axis == list(range(70))


@ROUTES
def test_frequencies_whose_memory_is_another(monkeypatch, route):
    from test_new_calls_native import _stand_in as stand_in_of_lserve_rotary

    t = _tensors()
    rot = L.RotaryDesc(rotary_dim=64, inv_freq=t["freq"], device="cpu")
    desc, axes = L.AttnDesc(4, 2, [1, 0]), L.PositionAxes([0, 1, 2, 0] * 8)
    for other in (torch.ones(32, dtype=torch.float64), torch.ones(40, dtype=torch.float64)):
        if other.numel() == 32:
            rot.inv_freq.data = other
        else:
            rot.inv_freq = other
        with _stand_in(monkeypatch, route) as seen:
            L.lserve_rotary_axes(desc, rot, axes, t["qn"], t["kn"], t["wide"][:, :6], t["qo"], t["ko"], 0x10)
        assert seen[0][2].inv_freq == other.data_ptr() and seen[0][2].rotary_dim == 64
        with stand_in_of_lserve_rotary(monkeypatch, route) as seen:
            L.lserve_rotary(desc, rot, t["qn"], t["kn"], t["pos"], t["qo"], t["ko"], 0x20)
        assert B._CRotaryDesc.from_buffer_copy(seen[0][2]).inv_freq == other.data_ptr()
    rot.inv_freq = torch.ones(31, dtype=torch.float64)
    with _stand_in(monkeypatch, route), pytest.raises(ValueError):
        L.lserve_rotary_axes(desc, rot, axes, t["qn"], t["kn"], t["wide"][:, :6], t["qo"], t["ko"], 0x10)


@ROUTES
def test_a_session_s_rows_without_queries(monkeypatch, route):
    """Queries that are somebody else's: nothing comes back of them."""
    from paper_2502_14866_amd.session import DecodeSession

    t = _tensors()
    pool = lambda n: torch.zeros((n, 1, 64, 128), dtype=torch.float16)  # noqa: E731
    s = DecodeSession(pool(8), pool(8), t["table"], 4, [1, 0], 128, 512, budget_tokens=256, k_pool_stream=pool(20), v_pool_stream=pool(20), ring_table=t["ring"])
    rot = L.RotaryDesc(rotary_dim=64, inv_freq=t["freq"], device="cpu")
    with _stand_in(monkeypatch, route) as seen:
        monkeypatch.setattr(B, "_stream", lambda stream: 0)
        assert s.append_rotary(rot, None, t["kn"], t["vn"], t["cu"], t["start"], 3, k_out=t["ko"]) is None
        out = s.append_rotary(rot, t["qn"], t["kn"], t["vn"], t["cu"], t["start"], 3)
    assert out.shape == t["qn"].shape and [x[0] for x in seen] == ["lserve_rotary_append_kv"] * 2
    assert seen[0][6] is None and seen[0][18:20] == (None, t["ko"].data_ptr()) and seen[1][6] == t["qn"].data_ptr() and seen[1][18] == out.data_ptr()


def test_a_list_of_axes_outlives_its_description():
    """What was handed over of a description made for one call alone is still the list when that description is gone."""
    import gc

    where = ctypes.cast(L.PositionAxes([2, 1, 0, 1] * 8)._c.pair_axis, ctypes.c_void_p).value
    gc.collect()
    others = [L.PositionAxes([1] * n) for n in range(1, 65)]
    assert list((ctypes.c_uint8 * 33).from_address(where)) == [2, 1, 0, 1] * 8 + [255]
    assert all(a.pair_axis == [1] * n for n, a in enumerate(others, 1))
