"""What the calls on new tokens refuse, on the host and before anything is launched."""
import ctypes
import math

import pytest
import torch

import paper_2502_14866_amd as L
from paper_2502_14866_amd import binding as B

i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
i64 = lambda *s: torch.zeros(s, dtype=torch.int64)  # noqa: E731


def _code(f, *a, **k):
    with pytest.raises(B.LserveError) as e:
        f(*a, **k)
    return e.value.code


def _extend(**kw):
    a = dict(desc=L.AttnDesc(4, 2, [1, 0]), kv=L.PagedKV(None, None, None, i32(2, 8), i32(4)[:2], ring_table=i32(2, 10)), new_lens=i32(2),
             free_pages=i32(8), cu_new=i32(4), new_seq_lens=i32(4), pages_taken=i32(1), positions=i32(8), slots=i64(8), ring_slots=i64(8),
             stream=0)
    a.update(kw)
    return a


@pytest.mark.parametrize("bad,code", [
    (dict(new_lens=None), -1), (dict(cu_new=None), -1), (dict(new_seq_lens=None), -1), (dict(pages_taken=None), -1),
    (dict(total_new=-1), -1), (dict(kv=L.PagedKV(None, None, None, i32(2, 8), i32(4)[:2])), -1),  # ring slots without a ring
    (dict(desc=L.AttnDesc(4, 2, [1, 0], page_size=48), ring_slots=None), -2), (dict(desc=L.AttnDesc(4, 2, [1, 0], local_tokens=0)), -1),
    (dict(positions=i32(16)[1:9]), -1),  # misaligned
    (dict(kv=L.PagedKV(None, None, None, i32(65536, 1), i32(65536)), ring_slots=None, new_lens=i32(65536), cu_new=i32(65537),
          new_seq_lens=i32(65536)), -2),
])
def test_extend_tables(bad, code):
    assert _code(L.lserve_extend_tables, **_extend(**bad)) == code


def test_extend_tables_lengths_are_not_overwritten_while_they_are_read():
    a = _extend()
    a["new_seq_lens"] = a["kv"].seq_lens
    assert _code(L.lserve_extend_tables, **a) == -1


@pytest.mark.parametrize("bad", [
    dict(new_lens=i32(1)), dict(cu_new=i32(2)), dict(slots=i64(7)), dict(slots=i32(8)), dict(positions=i64(8)), dict(new_lens=i64(2)),
    dict(positions=None, slots=None, ring_slots=None), dict(positions=torch.zeros(16, dtype=torch.int32)[::2]),
    dict(kv=L.PagedKV(None, None, None, i32(2, 8), i32(4)[:2], ring_table=i32(2, 9))),
])
def test_extend_tables_tensors(bad):
    with pytest.raises(ValueError):
        L.lserve_extend_tables(**_extend(**bad))


def _rotary(**kw):
    q, k = torch.zeros((3, 4, 128), dtype=torch.float16), torch.zeros((3, 2, 128), dtype=torch.float16)
    a = dict(desc=L.AttnDesc(4, 2, [1, 0]), rotary=L.RotaryDesc(device="cpu"), q=q, k=k, positions=i32(3), q_out=torch.zeros_like(q),
             k_out=torch.zeros_like(k), stream=0)
    a.update(kw)
    return a


def _c_rotary(dim=128, interleaved=0, scale=0.0, freq=True):
    d = L.RotaryDesc(device="cpu")
    d._c = B._CRotaryDesc(dim, interleaved, d.inv_freq.data_ptr() if freq else None, scale)
    return d


@pytest.mark.parametrize("bad,code", [
    (dict(rotary=_c_rotary(0)), -1), (dict(rotary=_c_rotary(7)), -1), (dict(rotary=_c_rotary(130)), -2), (dict(rotary=_c_rotary(interleaved=2)), -1),
    (dict(rotary=_c_rotary(scale=-1.0)), -1), (dict(rotary=_c_rotary(scale=math.inf)), -1), (dict(rotary=_c_rotary(scale=math.nan)), -1),
    (dict(rotary=_c_rotary(freq=False)), -1), (dict(q=None), -1), (dict(q_out=None), -1), (dict(q=None, q_out=None, k=None, k_out=None), -1),
    (dict(q=torch.zeros((3, 4 * 128 + 4), dtype=torch.float16)[:, :512].view(3, 4, 128)), -1),   # rows not a multiple of 16 bytes apart
    (dict(q=torch.zeros((3, 512), dtype=torch.float16).as_strided((3, 4, 128), (256, 128, 1))), -1),  # rows that overlap
])
def test_rotary(bad, code):
    assert _code(L.lserve_rotary, **_rotary(**bad)) == code


def test_rotary_in_place_takes_dense_rows():
    wide = torch.zeros((3, 1024), dtype=torch.float16)
    q = wide[:, :512].view(3, 4, 128)
    a = _rotary(q=q)
    lib, d = L.load_library(), a["desc"]
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    assert lib.lserve_rotary(d.c(), a["rotary"].c(), p(q), None, p(a["positions"]), 3, 1024, 0, p(q), None, None) == -1


@pytest.mark.parametrize("bad", [
    dict(q=torch.zeros((3, 4, 128), dtype=torch.bfloat16)), dict(q=torch.zeros((3, 5, 128), dtype=torch.float16)),
    dict(q=torch.zeros((3, 128, 4), dtype=torch.float16).transpose(1, 2)), dict(q=torch.zeros((2, 4, 128), dtype=torch.float16)),
    dict(q_out=torch.zeros((2, 4, 128), dtype=torch.float16)), dict(positions=i64(3)), dict(positions=torch.zeros(6, dtype=torch.int32)[::2]),
    dict(k_out=torch.zeros((3, 128, 2), dtype=torch.float16).transpose(1, 2)),
])
def test_rotary_tensors(bad):
    with pytest.raises(ValueError):
        L.lserve_rotary(**_rotary(**bad))


def test_frequencies():
    f, loud = L.lserve_rotary_frequencies(128, 500000.0)
    want = torch.tensor([500000.0 ** (-2 * i / 128) for i in range(64)], dtype=torch.float64)
    assert loud == 1.0 and torch.allclose(f, want, rtol=1e-15, atol=0)
    f, loud = L.lserve_rotary_frequencies(64, 10000.0, "linear", 4.0)
    assert loud == 1.0 and torch.allclose(f, torch.tensor([10000.0 ** (-2 * i / 64) / 4 for i in range(32)], dtype=torch.float64), rtol=1e-15, atol=0)


def test_frequencies_by_wavelength():
    """Worked by hand: base 10^4, R = 8, so f = 1, 0.1, 0.01, 0.001; over 2000 positions these are 318, 31.8, 3.18 and 0.318 turns."""
    f, _ = L.lserve_rotary_frequencies(8, 10000.0, "wavelength", 8.0, 2000.0, 1.0, 4.0)
    turns = 2000 * 0.01 / (2 * math.pi)
    share = (turns - 1) / 3
    want = [1.0, 0.1, 0.01 * share + 0.01 / 8 * (1 - share), 0.001 / 8]
    assert torch.allclose(f, torch.tensor(want, dtype=torch.float64), rtol=1e-14, atol=0)


def test_frequencies_on_a_ramp():
    """The same; i(n) = log_10(2000 / (2 pi n)), as the frequency of pair i is 10^-i: i(32) = 0.998 and i(1) = 2.503, a ramp from 0 to 3."""
    f, loud = L.lserve_rotary_frequencies(8, 10000.0, "ramp", 16.0, 2000.0, 1.0, 32.0)
    want = [10.0 ** -i * (1 - i / 3 + i / 3 / 16) for i in range(4)]
    assert torch.allclose(f, torch.tensor(want, dtype=torch.float64), rtol=1e-14, atol=0)
    assert loud == pytest.approx(0.1 * math.log(16) + 1, rel=1e-7)
    assert L.RotaryDesc(rotary_dim=8, scaling="ramp", factor=16.0, low=1.0, high=32.0, device="cpu").scale == loud


@pytest.mark.parametrize("kw,code", [
    (dict(rotary_dim=0), -1), (dict(rotary_dim=9), -1), (dict(rotary_dim=256), -2), (dict(base=1.0), -1), (dict(base=math.nan), -1),
    (dict(scaling="linear", factor=0.5), -1), (dict(scaling="ramp", factor=2.0, low=4.0, high=4.0), -1),
    (dict(scaling="wavelength", factor=2.0, low=0.0), -1), (dict(scaling="wavelength", factor=2.0, original_positions=0.0), -1),
    (dict(scaling="wavelength", factor=math.inf), -1),
])
def test_frequencies_refused(kw, code):
    kw = {"rotary_dim": 128, **kw}
    assert _code(L.lserve_rotary_frequencies, **kw) == code


def test_frequencies_of_an_unknown_scaling():
    with pytest.raises(ValueError):
        L.lserve_rotary_frequencies(128, scaling="other")
    with pytest.raises(ValueError):
        L.RotaryDesc(inv_freq=torch.zeros(64), device="cpu")


def _masks(**kw):
    a = dict(parents=i32(8), cu_new=i32(4)[:3], seq_lens=i32(2), max_new_per_seq=4, tree_mask=i64(8, 1), positions=i32(8), stream=0)
    a.update(kw)
    return a


@pytest.mark.parametrize("bad,code", [
    (dict(max_new_per_seq=0), -1), (dict(max_new_per_seq=9), -1), (dict(parents=i32(12)[1:9]), -1),
    (dict(parents=i32(128), max_new_per_seq=65, tree_mask=i64(128, 1), positions=i32(128)), -1),  # two words needed
    (dict(parents=i32(1025), max_new_per_seq=1025, tree_mask=i64(1025, 17), positions=i32(1025)), -2),
    (dict(cu_new=i32(65537), seq_lens=i32(65536)), -2),
])
def test_tree_masks(bad, code):
    assert _code(L.lserve_tree_masks, **_masks(**bad)) == code


@pytest.mark.parametrize("bad", [dict(tree_mask=i64(7, 1)), dict(tree_mask=i32(8, 1)), dict(positions=i32(7)), dict(seq_lens=i32(1)),
                                 dict(parents=i64(8)), dict(cu_new=i32(1))])
def test_tree_masks_tensors(bad):
    with pytest.raises(ValueError):
        L.lserve_tree_masks(**_masks(**bad))
