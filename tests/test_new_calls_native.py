"""The calls on new tokens hand the library the same natively and by ctypes, and refuse the same."""
import contextlib
import ctypes
import types

import pytest
import torch

import paper_2502_14866_amd as L
from paper_2502_14866_amd import binding as B

vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
dp, kp, rp = ctypes.POINTER(B._CAttnDesc), ctypes.POINTER(B._CPagedKV), ctypes.POINTER(B._CRotaryDesc)
TYPES = {"lserve_append_kv": [dp, kp, vp, vp, vp, vp, i32, vp], "lserve_select_pages": [dp, kp, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp],
         "lserve_sparse_decode": [dp, kp, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp],
         "lserve_extend_tables": [dp, kp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp], "lserve_tree_masks": [vp, vp, vp, i32, i32, i32, i32, vp, vp, vp],
         "lserve_rotary": [dp, rp, vp, vp, vp, i32, i64, i64, vp, vp, vp],
         "lserve_sparse_decode_tree": [dp, kp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]}


def _bind(lib):
    calls = B._native()
    if calls is not B._CtypesCalls:
        at = [ctypes.cast(getattr(lib, f), vp).value for f in TYPES]
        calls.bind(*at[:3])
        calls.bind_new(*at[3:])


def _tensors():
    half, ints = lambda *s: torch.zeros(s, dtype=torch.float16), lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    k = half(8, 1, 64, 128)
    t = {"k": k, "v": k.clone(), "ks": half(5, 1, 64, 128), "vs": half(5, 1, 64, 128), "table": ints(2, 4), "ring": ints(2, 10), "lens": ints(4)[:2],
         "new": ints(2), "free": ints(9)[3:], "cu": ints(3), "after": ints(2), "taken": ints(1), "pos": ints(6), "slots": torch.zeros(6, dtype=torch.int64),
         "ring_slots": torch.zeros(6, dtype=torch.int64), "parents": ints(6), "mask": torch.zeros((6, 2), dtype=torch.int64),
         "rows": half(6, 8 * 128), "qo": half(6, 4, 128), "ko": half(6, 2, 128), "q": half(6, 4, 128), "kn": half(6, 2, 128), "vn": half(6, 2, 128),
         "out": half(6, 4, 128), "lse": torch.zeros(6, 4), "sel": ints(2, 2, 4), "cnt": ints(2, 2), "ssl": ints(2),
         "ws": torch.zeros(24, dtype=torch.float32), "freq": torch.zeros(32, dtype=torch.float64)}
    return t


def _calls(t):
    kv = L.PagedKV(t["k"], t["v"], None, t["table"], t["lens"], pool_heads=1, k_pool_stream=t["ks"], v_pool_stream=t["vs"], ring_table=t["ring"])
    desc = L.AttnDesc(4, 2, [1, 0])
    rot = L.RotaryDesc(rotary_dim=64, inv_freq=t["freq"], device="cpu")
    qf, kf = t["rows"][:, :512].view(6, 4, 128), t["rows"][:, 512:768].view(6, 2, 128)
    return [
        lambda: L.lserve_extend_tables(desc, kv, t["new"], t["free"], t["cu"], t["after"], t["taken"], t["pos"], t["slots"], t["ring_slots"], 0x10),
        lambda: L.lserve_extend_tables(desc, kv, t["new"], None, t["cu"], t["after"], t["taken"], total_new=77, stream=0x20),
        lambda: L.lserve_tree_masks(t["parents"], t["cu"], t["lens"], 70, t["mask"], t["pos"], 0x30),
        lambda: L.lserve_rotary(desc, rot, qf, kf, t["pos"], t["qo"], t["ko"], 0x40),
        lambda: L.lserve_rotary(desc, rot, None, t["kn"], t["pos"], None, t["kn"], 0x50),
        lambda: L.lserve_sparse_decode_tree(desc, kv, t["q"], t["kn"], t["vn"], t["cu"], 5, t["out"], t["lse"], t["mask"], t["pos"], t["sel"], t["cnt"],
                                            t["ssl"], t["ws"], 0x60),
        lambda: L.lserve_sparse_decode_tree(desc, kv, t["q"], t["kn"], t["vn"], t["cu"], 5, t["out"], None, workspace=None, stream=0x70),
    ]


@contextlib.contextmanager
def _stand_in(monkeypatch, route):
    """A library that notes what it is handed; yields the notes."""
    seen, lib = [], types.SimpleNamespace()
    for name, args in TYPES.items():
        def body(*a, name=name):
            seen.append((name, *[bytes(x.contents) if isinstance(x, (dp, rp)) else B._CPagedKV.from_buffer_copy(x.contents) if isinstance(x, kp) else x
                                 for x in a]))
            return 0
        setattr(lib, name, ctypes.CFUNCTYPE(ctypes.c_int, *args)(body))
    real = B.load_library()
    try:
        monkeypatch.setattr(B, "_lib", lib)
        monkeypatch.setattr(B, "_calls", None if route == "native" else B._CtypesCalls)
        if route == "native":
            _bind(lib)
        yield seen
    finally:
        monkeypatch.undo()
        _bind(real)


def _seen(monkeypatch, route):
    t = _tensors()
    calls = _calls(t)
    with _stand_in(monkeypatch, route) as seen:
        for call in calls:
            call()
    base = {x.data_ptr(): k for k, x in t.items()}
    out = []
    for s in seen:
        row = []
        for x in s:
            if isinstance(x, B._CPagedKV):
                row.append(tuple(base.get(getattr(x, f), getattr(x, f)) for f, _ in B._CPagedKV._fields_))
            elif isinstance(x, bytes) and len(x) == ctypes.sizeof(B._CRotaryDesc):
                r = B._CRotaryDesc.from_buffer_copy(x)
                row.append(tuple(base.get(getattr(r, f), getattr(r, f)) for f, _ in B._CRotaryDesc._fields_))
            elif isinstance(x, bytes):
                row.append(x[:24])
            else:
                row.append(base.get(x, x) if isinstance(x, int) else x)
        out.append(tuple(row))
    return out


def test_both_routes_hand_over_the_same(monkeypatch):
    native, ctyped = _seen(monkeypatch, "native"), _seen(monkeypatch, "ctypes")
    assert len(native) == 7 and native == ctyped


@pytest.mark.parametrize("route", ["native", "ctypes"])
@pytest.mark.parametrize("wrong", [
    {"new": torch.zeros(2, dtype=torch.int64)}, {"cu": torch.zeros(2, dtype=torch.int32)}, {"pos": torch.zeros(5, dtype=torch.int32)},
    {"slots": torch.zeros(6, dtype=torch.int32)}, {"ring": torch.zeros((2, 9), dtype=torch.int32)}, {"mask": torch.zeros((5, 2), dtype=torch.int64)},
    {"kn": torch.zeros((6, 2, 128), dtype=torch.bfloat16)}, {"q": torch.zeros((6, 4, 64), dtype=torch.float16)}, {"lse": torch.zeros(6, 3)},
    {"sel": torch.zeros((1, 2, 4), dtype=torch.int32)}, {"lens": torch.zeros(1, dtype=torch.int32)}, {"ko": torch.zeros((5, 2, 128), dtype=torch.float16)},
    {"q": torch.zeros((6, 4, 256), dtype=torch.float16)[..., ::2]},
], ids=lambda w: next(iter(w)))
def test_both_routes_refuse_the_same(monkeypatch, route, wrong):
    """By one of the calls at least; none reaches a library."""
    calls, refused = _calls({**_tensors(), **wrong}), 0
    with _stand_in(monkeypatch, route):
        for call in calls:
            try:
                call()
            except ValueError:
                refused += 1
    assert refused > 0
