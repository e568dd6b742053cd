"""lserve_rotary_axes, lserve_norm_rotary and lserve_rotary_append_kv hand the library the same natively and by ctypes, and refuse the same."""
import contextlib
import ctypes
import types

import pytest
import torch

import paper_2502_14866_amd as L
from paper_2502_14866_amd import binding as B

vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
dp, kp, rp = ctypes.POINTER(B._CAttnDesc), ctypes.POINTER(B._CPagedKV), ctypes.POINTER(B._CRotaryDesc)
ap, np_ = ctypes.POINTER(B._CPositionAxes), ctypes.POINTER(B._CHeadNorm)
TURNED = {"lserve_rotary_axes": [dp, rp, ap, vp, vp, vp, i64, i32, i64, i64, vp, vp, vp],
          "lserve_norm_rotary": [dp, np_, rp, ap, vp, vp, vp, i64, i32, i64, i64, vp, vp, vp],
          "lserve_rotary_append_kv": [dp, kp, np_, rp, ap, vp, vp, vp, i64, i64, i64, vp, i64, vp, vp, i32, i32, vp, vp, vp, vp]}
STRUCTS = (dp, rp, ap, np_)


def _tensors():
    half, ints = lambda *s: torch.zeros(s, dtype=torch.float16), lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    return {"k": half(8, 1, 64, 128), "v": half(8, 1, 64, 128), "ks": half(20, 1, 64, 128), "vs": half(20, 1, 64, 128), "stats": half(8, 1, 4, 2, 128),
            "table": ints(2, 4), "ring": ints(2, 10), "lens": ints(4)[:2], "cu": ints(3), "start": ints(2), "pos": ints(6), "wide": ints(3, 9), "rows": half(6, 8 * 128),
            "qn": half(6, 4, 128), "kn": half(6, 2, 128), "vn": half(6, 2, 128), "qo": half(6, 4, 128), "ko": half(6, 2, 128), "vo": half(6, 2, 128),
            "freq": torch.zeros(32, dtype=torch.float64), "wq": torch.ones(4, 128), "wk": torch.ones(2, 128)}


def _calls(t):
    kv = L.PagedKV(t["k"], t["v"], t["stats"], t["table"], t["lens"], pool_heads=1, k_pool_stream=t["ks"], v_pool_stream=t["vs"], ring_table=t["ring"])
    desc, rot, axes = L.AttnDesc(4, 2, [1, 0]), L.RotaryDesc(rotary_dim=64, inv_freq=t["freq"], device="cpu"), L.PositionAxes([0, 1, 2, 0] * 8)
    norm, plain = L.HeadNorm(t["wq"], t["wk"], eps=1e-5, centred=True), L.HeadNorm()
    qf, kf, vf = t["rows"][:, :512].view(6, 4, 128), t["rows"][:, 512:768].view(6, 2, 128), t["rows"][:, 768:].view(6, 2, 128)
    return [
        lambda: L.lserve_rotary_axes(desc, rot, axes, qf, kf, t["wide"][:, :6], t["qo"], t["ko"], 0x10),
        lambda: L.lserve_rotary_axes(desc, rot, L.PositionAxes([0] * 32), None, t["kn"], t["pos"].view(1, -1), None, t["kn"], 0x20),
        lambda: L.lserve_norm_rotary(desc, norm, rot, qf, kf, t["pos"], t["qo"], t["ko"], 0x30),
        lambda: L.lserve_norm_rotary(desc, norm, rot, t["qn"], None, t["wide"][:, :6], t["qn"], None, 0x40, axes=axes),
        lambda: L.lserve_norm_rotary(desc, plain, None, t["qn"], t["kn"], None, t["qo"], t["ko"], 0x50),
        lambda: L.lserve_rotary_append_kv(desc, kv, rot, qf, kf, vf, t["cu"], t["start"], 5, t["qo"], t["ko"], t["vo"], norm, axes, t["wide"], 0x60),
        lambda: L.lserve_rotary_append_kv(desc, kv, rot, None, t["kn"], t["vn"], t["cu"], t["lens"], 1, None, stream=0x70),
        lambda: L.lserve_rotary_append_kv(desc, kv, None, t["qn"], t["kn"], t["vn"], t["cu"], t["lens"], 1, t["qn"], norm=plain, positions=t["pos"], stream=0x80),
    ]


@contextlib.contextmanager
def _stand_in(monkeypatch, route):
    """A library that notes what it is handed; yields the notes."""
    seen, real = [], B.load_library()
    lib = types.SimpleNamespace(**{f: getattr(real, f) for f in ("lserve_append_kv", "lserve_select_pages", "lserve_sparse_decode")})
    for name, args in TURNED.items():
        def body(*a, name=name):
            seen.append((name, *[type(x.contents).from_buffer_copy(x.contents) if isinstance(x, STRUCTS + (kp,)) and x else x for x in a]))
            return 0
        setattr(lib, name, ctypes.CFUNCTYPE(ctypes.c_int, *args)(body))
    calls = B._native()
    address = lambda of: [ctypes.cast(getattr(of, f), vp).value for f in TURNED]  # noqa: E731
    try:
        monkeypatch.setattr(B, "_lib", lib)
        if route == "native":
            assert calls is not B._CtypesCalls
            calls.bind_turned(*address(lib))
        else:
            monkeypatch.setattr(B, "_calls", B._CtypesCalls)
        yield seen
    finally:
        monkeypatch.undo()
        if calls is not B._CtypesCalls:
            calls.bind_turned(*address(real))


def _seen(monkeypatch, route, t):
    with _stand_in(monkeypatch, route) as seen:
        for call in _calls(t):
            call()
    out = []
    for s in seen:
        row = []
        for x in s:
            if isinstance(x, B._CPositionAxes):
                row.append((x.num_axes, tuple(x.pair_axis[:32])))
            elif isinstance(x, B._CAttnDesc):
                row.append((x.num_q_heads, x.num_kv_heads, x.dtype))
            elif isinstance(x, ctypes.Structure):
                row.append(tuple(getattr(x, f) for f, _ in x._fields_))
            else:  # (a null pointer to a struct is one of its own each time)
                row.append(None if isinstance(x, STRUCTS) else x)
        out.append(tuple(row))
    return out


def test_both_routes_hand_over_the_same(monkeypatch):
    t = _tensors()
    native, ctyped = _seen(monkeypatch, "native", t), _seen(monkeypatch, "ctypes", t)
    assert len(native) == 8 and native == ctyped
    rows = t["rows"].data_ptr()
    assert native[0][4:10] == (rows, rows + 1024, t["wide"].data_ptr(), 9, 6, 1024)
    assert native[5][6:12] == (rows, rows + 1024, rows + 1536, 1024, 1024, 1024) and native[5][12:18] == (t["wide"].data_ptr(), 9, t["cu"].data_ptr(), t["start"].data_ptr(), 6, 5)
    assert native[6][3] is None and native[6][5:7] == (None, None) and native[6][12:14] == (None, 0)


@pytest.mark.parametrize("route", ["native", "ctypes"])
@pytest.mark.parametrize("wrong", [
    {"cu": torch.zeros(2, dtype=torch.int32)}, {"start": torch.zeros(2, dtype=torch.int64)}, {"pos": torch.zeros(5, dtype=torch.int32)},
    {"wide": torch.zeros((2, 9), dtype=torch.int32)}, {"wide": torch.zeros((3, 18), dtype=torch.int32)[:, ::2]}, {"ring": torch.zeros((2, 9), dtype=torch.int32)},
    {"kn": torch.zeros((6, 2, 128), dtype=torch.bfloat16)}, {"qn": torch.zeros((6, 4, 64), dtype=torch.float16)}, {"vn": torch.zeros((5, 2, 128), dtype=torch.float16)},
    {"stats": torch.zeros((8, 1, 3, 2, 128), dtype=torch.float16)}, {"vs": torch.zeros((19, 1, 64, 128), dtype=torch.float16)}, {"wk": torch.ones(1, 128)},
    {"vo": torch.zeros((6, 2, 256), dtype=torch.float16)[..., ::2]}, {"qo": torch.zeros((5, 4, 128), dtype=torch.float16)},
], ids=lambda w: next(iter(w)))
def test_both_routes_refuse_the_same(monkeypatch, route, wrong):
    refused = []
    with _stand_in(monkeypatch, route):
        for i, call in enumerate(_calls({**_tensors(), **wrong})):
            try:
                call()
            except ValueError:
                refused.append(i)
    assert refused
    with _stand_in(monkeypatch, "ctypes" if route == "native" else "native"):
        for i, call in enumerate(_calls({**_tensors(), **wrong})):
            if i in refused:
                with pytest.raises(ValueError):
                    call()
            else:
                call()
