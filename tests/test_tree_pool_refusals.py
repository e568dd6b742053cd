"""What of a cache lserve_sparse_decode_tree refuses in both routes of the binding, before the library is called: tables and pools that are too short
or of another type lead the kernels to addresses outside them."""
import pytest
import torch

from test_new_calls_native import _calls, _stand_in, _tensors

i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
half = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
EXTEND, EXTEND_NO_SLOTS, MASKS, ROTARY, ROTARY_KEYS, TREE, TREE_ALL = range(7)  # what _calls makes


@pytest.mark.parametrize("route", ["native", "ctypes"])
@pytest.mark.parametrize("name,wrong,refusing", [
    ("ring", i32(2, 9), {EXTEND, TREE, TREE_ALL}),
    ("ring", torch.zeros((2, 10), dtype=torch.int64), {EXTEND, EXTEND_NO_SLOTS, TREE, TREE_ALL}),
    ("k", half(7, 1, 64, 128), {TREE, TREE_ALL}),
    ("k", torch.zeros((8, 1, 64, 128)), {TREE, TREE_ALL}),
    ("v", half(8, 1, 32, 128), {TREE, TREE_ALL}),
    ("v", torch.zeros((8, 1, 64, 128), dtype=torch.uint8), {TREE, TREE_ALL}),
    ("ks", half(5, 1, 63, 128), {TREE, TREE_ALL}),
    ("vs", half(4, 1, 64, 128), {TREE, TREE_ALL}),
    ("vs", torch.zeros((5, 1, 64, 128), dtype=torch.bfloat16), {TREE, TREE_ALL}),
    ("new", torch.zeros(2, dtype=torch.int64), {EXTEND, EXTEND_NO_SLOTS}),
    ("cu", i32(2), {EXTEND, EXTEND_NO_SLOTS, TREE, TREE_ALL}),
    ("lens", i32(1), {EXTEND, EXTEND_NO_SLOTS, MASKS, TREE, TREE_ALL}),
    ("pos", i32(5), {MASKS, TREE}),
    ("slots", i32(6), {EXTEND}),
    ("mask", torch.zeros((5, 2), dtype=torch.int64), {MASKS, TREE}),
    ("kn", torch.zeros((6, 2, 128), dtype=torch.bfloat16), {ROTARY_KEYS, TREE, TREE_ALL}),
    ("ko", half(5, 2, 128), {ROTARY}),
    ("q", half(6, 4, 64), {TREE, TREE_ALL}),
    ("q", half(6, 4, 256)[..., ::2], {TREE, TREE_ALL}),
    ("lse", torch.zeros(6, 3), {TREE}),
    ("sel", i32(1, 2, 4), {TREE}),
])
def test_which_calls_refuse_what(monkeypatch, route, name, wrong, refusing):
    """These and no others, and what is refused does not reach the library."""
    refused = set()
    with _stand_in(monkeypatch, route) as seen:
        for i, call in enumerate(_calls({**_tensors(), name: wrong})):
            before = len(seen)
            try:
                call()
            except ValueError:
                refused.add(i)
            assert len(seen) == before + (i not in refused)
    assert refused == refusing


@pytest.mark.parametrize("route", ["native", "ctypes"])
@pytest.mark.parametrize("name,refusing", [("ws", {TREE}), ("ring", {EXTEND, EXTEND_NO_SLOTS, TREE, TREE_ALL}), ("vs", {TREE, TREE_ALL}),
                                           ("freq", {ROTARY, ROTARY_KEYS}), ("parents", {MASKS}), ("free", {EXTEND})])
def test_tensors_on_another_device(monkeypatch, route, name, refusing):
    t, refused = _tensors(), set()
    if name == "freq":  # (its address is taken when the description is made)
        calls = _calls(t)
        _rotary_of(calls[ROTARY]).inv_freq = t[name].to("meta")
    else:
        calls = _calls({**t, name: t[name].to("meta")})
    with _stand_in(monkeypatch, route) as seen:
        for i, call in enumerate(calls):
            before = len(seen)
            try:
                call()
            except ValueError:
                refused.add(i)
            assert len(seen) == before + (i not in refused)
    assert refused == refusing


def _rotary_of(call):
    return next(c.cell_contents for c in call.__closure__ if type(c.cell_contents).__name__ == "RotaryDesc")


@pytest.mark.parametrize("route", ["native", "ctypes"])
def test_a_main_pool_that_nobody_reads(monkeypatch, route):
    """Where all heads are in the bounded pool the main one may be anything of the right type."""
    import paper_2502_14866_amd as L

    t = _tensors()
    desc = L.AttnDesc(4, 2, [1, 1])
    for streams, ok in ((half(5, 2, 64, 128), True), (half(5, 1, 64, 128), False)):
        kv = L.PagedKV(half(1, 1, 1, 128), half(1, 1, 1, 128), None, t["table"], t["lens"], k_pool_stream=streams, v_pool_stream=streams.clone(), ring_table=t["ring"])
        with _stand_in(monkeypatch, route) as seen:
            call = lambda: L.lserve_sparse_decode_tree(desc, kv, t["q"], t["kn"], t["vn"], t["cu"], 5, t["out"], None, stream=1)  # noqa: E731
            if ok:
                call()
            else:
                with pytest.raises(ValueError):
                    call()
        assert len(seen) == int(ok)
