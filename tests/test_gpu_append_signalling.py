"""Signalling not-a-numbers of rows on their way into pages: like any other they take no part in a row's range or in statistics, through lserve_append_kv as through
lserve_rotary_append_kv, which leave the same bytes."""
import numpy as np
import pytest
import torch

from test_gpu_append_special import SIGNALLING, _append, _expected
from test_gpu_quant import _unpack_rows
from test_gpu_rotary_append import _assert_same_cache, _cache, _twin

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _numbers(x):
    """In 32 bits, every not-a-number a quiet one: numpy's own reductions would take a signalling one for what came before it."""
    f = x.float().numpy()
    return np.where(np.isnan(f), np.float32(np.nan), f)


@pytest.mark.parametrize("one_by_one", [False, True])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("seed", [8, 9, 10])
def test_extremes_next_to_signalling_not_a_numbers(dtype, bits, one_by_one, seed):
    """The extremes of a row in front of one, behind one and between two, at every place of the eight channels that a lane has."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((40, 128), generator=g).to(torch.float16 if dtype == "fp16" else torch.bfloat16)
    raw = x.view(torch.int16)
    for i in range(32):  # lane i / 2's channels: the row's extremes at two of them, not-a-numbers at the others, or at half of the others
        first = 8 * (i // 2)
        for c in range(first, first + 8):
            if i % 2 or c % 2:
                raw[i, c] = SIGNALLING[dtype] - (0x8000 if c % 3 else 0)
        low, high = first + (seed + i) % 8, first + (seed + 3 * i + 5) % 8
        x[i, low] = -40.0
        x[i, high if high != low else first + (low + 1) % 8] = 50.0
    raw[39] = SIGNALLING[dtype]  # nothing but
    k, v, stats = _append(x, bits, dtype, one_by_one)
    codes, scale, zero = _expected(_numbers(x), bits)
    size = 64 * 128 * bits // 8
    for pool in (k, v):
        slab = pool.numpy()[0, 0]
        pair = np.ascontiguousarray(slab[size:]).view(np.float16).reshape(64, 2)[:40]
        assert np.array_equal(pair[:, 0], scale, equal_nan=True) and np.array_equal(pair[:, 1], zero, equal_nan=True)
        assert np.array_equal(_unpack_rows(slab[:size].reshape(64, 128 * bits // 8), bits)[:40], codes)
    for page in range(3):
        part = _numbers(x)[16 * page:16 * page + 16]
        high, low = np.fmax(np.fmax.reduce(part, axis=0), -np.inf), np.fmin(np.fmin.reduce(part, axis=0), np.inf)
        assert np.array_equal(stats[0, 0, page, 0].float().numpy(), high) and np.array_equal(stats[0, 0, page, 1].float().numpy(), low)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("two_way", [False, True])
@pytest.mark.parametrize("counts", [[1, 1, 1], [2, 1, 2], [40, 19, 64]])
def test_both_calls_leave_the_same_bytes(dtype, bits, two_way, counts):
    import paper_2502_14866_amd as L

    L.load_library()
    g = torch.Generator().manual_seed(sum(counts) + bits)
    desc = L.AttnDesc(4, 4, [1, 0, 1, 0], dtype=dtype)
    kv = _cache(L, g, dtype, desc, [7, 100, 64], counts, bits, two_way, 64)
    twin = _twin(L, kv)
    k, v = (torch.randn((sum(counts), 4, 128), generator=g).to(dtype) for _ in range(2))
    odd = torch.tensor([0x7c00, 0xfc00, 0x7e00, 0x7c01, 0x7d01, 0x7f80, 0xff80, 0x7fc0, 0x7f81, 0x7fa1, 0xffa1], dtype=torch.int32).to(torch.int16)
    for t in (k, v):
        row = t.view(torch.int16).view(-1)
        at = torch.randint(0, row.numel(), (row.numel() // 12,), generator=g)
        row[at] = odd[torch.randint(0, len(odd), at.shape, generator=g)]
    k, v = k.to(DEV), v.to(DEV)
    cu = torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32, device=DEV)
    L.lserve_rotary_append_kv(desc, kv, None, None, k, v, cu, kv.seq_lens, max(counts), None)
    L.lserve_append_kv(desc, twin, k, v, cu, kv.seq_lens, max(counts))
    torch.cuda.synchronize()
    _assert_same_cache(kv, twin)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("at", [0, 16, 47])
def test_a_token_of_nothing_but_not_a_numbers(dtype, at):
    """Statistics of a logical page whose first token, or last of three, has no number: infinities, or what the others left."""
    import paper_2502_14866_amd as L

    L.load_library()
    desc = L.AttnDesc(1, 1, [0], dtype=dtype)
    i32 = lambda *a: torch.tensor(a + (0,) * 4, dtype=torch.int32, device=DEV)[:len(a)]  # noqa: E731
    pool = torch.zeros((1, 1, 64, 128), dtype=dtype, device=DEV)
    stats = torch.full((1, 1, 4, 2, 128), 3.0, dtype=dtype, device=DEV)
    kv = L.PagedKV(pool, pool.clone(), stats, i32(0).reshape(1, 1), i32(at + 1))
    row = torch.full((1, 1, 128), float("nan"), dtype=dtype, device=DEV)
    for kind in ("bf16" if dtype == torch.bfloat16 else "fp16", None):
        if kind:
            row.view(torch.int16)[:] = SIGNALLING[kind]
        else:
            row.fill_(float("nan"))
        L.lserve_append_kv(desc, kv, row, row, i32(0, 1), i32(at), 1)
        torch.cuda.synchronize()
        got = stats[0, 0, at // 16].float().cpu()
        if at % 16 == 0:
            assert (got[0] == -float("inf")).all() and (got[1] == float("inf")).all()
        else:
            assert (got == 3.0).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("logical", [8, 16, 64])
def test_statistics_from_the_pages(dtype, logical):
    """lserve_build_page_stats and the selector's own rebuild find what lserve_append_kv left."""
    import paper_2502_14866_amd as L

    L.load_library()
    g = torch.Generator().manual_seed(logical)
    desc = L.AttnDesc(4, 2, [0, 0], dtype=dtype, logical_page_size=logical)
    counts = [130, 1, 64, 77]
    kv = _cache(L, g, dtype, desc, [0] * 4, counts, 16, False, 64)
    k = torch.randn((sum(counts), 2, 128), generator=g).to(dtype)
    row = k.view(torch.int16).view(-1)
    odd = torch.tensor([0x7c00, 0xfc00, 0x7e00, 0x7c01, 0x7d01, 0x7f80, 0xff80, 0x7fc0, 0x7f81, 0x7fa1, 0xffa1], dtype=torch.int32).to(torch.int16)
    at = torch.randint(0, row.numel(), (row.numel() // 12,), generator=g)
    row[at] = odd[torch.randint(0, len(odd), at.shape, generator=g)]
    cu = torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32, device=DEV)
    L.lserve_append_kv(desc, kv, k.to(DEV), k.to(DEV), cu, kv.seq_lens, max(counts))
    torch.cuda.synchronize()
    want = kv.stats.clone()
    kv.seq_lens = torch.tensor(counts, dtype=torch.int32, device=DEV)
    used = torch.zeros(kv.stats.shape[:3], dtype=torch.bool, device=DEV)
    for b, n in enumerate(counts):
        for first in range(0, n, logical):
            used[kv.page_table[b, first // 64].long(), :, first % 64 // logical] = True
    none = torch.zeros(4, dtype=torch.int32, device=DEV)
    q = torch.randn((4, 4, 128), generator=g).to(dtype).to(DEV)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    workspace = torch.zeros(L.lserve_workspace_bytes(1, desc, 4, kv.page_table.shape[1], 2, 0) + 16, dtype=torch.uint8, device=DEV)
    for rebuild in ("call", "selector"):
        kv.stats.zero_()
        if rebuild == "call":
            L.lserve_build_page_stats(desc, kv, None, 0)
        else:
            L.lserve_select_pages(desc, kv, q, 128, i32(4, 2, 2), i32(4, 2), i32(4), None, workspace, stats_valid_len=none)
        torch.cuda.synchronize()
        # (as numbers: the larger of zeros of both signs is either)
        assert torch.equal(kv.stats[used].float(), want[used].float()), rebuild
