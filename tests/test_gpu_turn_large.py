"""Rows, outputs and pages past 32-bit offsets, and the largest batch."""
import pytest
import torch

from turn_reference import assert_close, reference

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _lib():
    import paper_2502_14866_amd as L

    L.load_library()
    return L


@pytest.mark.parametrize("norm", [None, "rms"])
def test_rows_far_apart(norm):
    """Three rows 2^30 elements (2 GiB) and more from one to the next."""
    L = _lib()
    g = torch.Generator().manual_seed(1)
    apart = (1 << 30) + 8
    room = torch.empty(2 * apart + 12 * 128, dtype=torch.float16, device=DEV)
    rows = torch.randn((3, 12 * 128), generator=g).half()
    for i in range(3):
        room[i * apart:i * apart + 12 * 128] = rows[i].to(DEV)
    q, k = room.as_strided((3, 8, 128), (apart, 128, 1)), room.as_strided((3, 2, 128), (apart, 128, 1), 1024)
    desc, rot, axes = L.AttnDesc(8, 2, [1, 0]), L.RotaryDesc(), L.PositionAxes.sections(32, 32)
    pos = torch.tensor([[4, 5, 6], [1, 2, 3]], dtype=torch.int32)
    qo, ko = (torch.zeros((3, h, 128), dtype=torch.float16, device=DEV) for h in (8, 2))
    if norm:
        L.lserve_norm_rotary(desc, L.HeadNorm(), rot, q, k, pos.to(DEV), qo, ko, axes=axes)
    else:
        L.lserve_rotary_axes(desc, rot, axes, q, k, pos.to(DEV), qo, ko)
    torch.cuda.synchronize()
    for x, got in ((rows[:, :1024].view(3, 8, 128), qo), (rows[:, 1024:1280].view(3, 2, 128), ko)):
        assert_close(got, reference(x, 128, False, pos, axes.pair_axis, rot.inv_freq.cpu(), norm=norm), torch.float16)
    v = room.as_strided((3, 2, 128), (apart, 128, 1), 1280)
    kv = L.PagedKV(*(torch.zeros((2, 2, 64, 128), dtype=torch.float16, device=DEV) for _ in range(2)), torch.zeros((2, 2, 4, 2, 128), dtype=torch.float16, device=DEV),
                   torch.tensor([[1]], dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)[:1])
    cu = torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    qo.zero_()
    L.lserve_rotary_append_kv(desc, kv, rot, q, k, v, cu, kv.seq_lens, 3, qo, axes=axes, positions=pos.to(DEV), norm=L.HeadNorm() if norm else None)
    torch.cuda.synchronize()
    assert_close(qo, reference(rows[:, :1024].view(3, 8, 128), 128, False, pos, axes.pair_axis, rot.inv_freq.cpu(), norm=norm), torch.float16)
    assert_close(kv.k_pool[1, :, :3].transpose(0, 1), reference(rows[:, 1024:1280].view(3, 2, 128), 128, False, pos, axes.pair_axis, rot.inv_freq.cpu(), norm=norm), torch.float16)
    assert torch.equal(kv.v_pool[1, :, :3].transpose(0, 1).cpu(), rows[:, 1280:].view(3, 2, 128))


@pytest.mark.parametrize("norm", [None, "rms"])
def test_more_than_2_31_elements(norm):
    """Queries of 64 heads of 270000 tokens, in place, in one sequence of the cache too."""
    L = _lib()
    n = 270000
    desc, rot = L.AttnDesc(64, 8, [0] * 8, dtype=torch.bfloat16), L.RotaryDesc()
    g = torch.Generator(device=DEV).manual_seed(1)
    q = torch.randn((n, 64, 128), generator=g, device=DEV, dtype=torch.bfloat16)
    k = torch.randn((n, 8, 128), generator=g, device=DEV, dtype=torch.bfloat16)
    some = torch.tensor([0, 1, 131071, 262143, 262144, 262145, n - 1])
    before, before_k = q[some.to(DEV)].cpu(), k[some.to(DEV)].cpu()
    pages = -(-n // 64)
    kv = L.PagedKV(*(torch.zeros((pages, 8, 64, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)),
                   torch.zeros((pages, 8, 4, 2, 128), dtype=torch.bfloat16, device=DEV), torch.arange(pages - 1, -1, -1, dtype=torch.int32, device=DEV).view(1, pages),
                   torch.zeros(4, dtype=torch.int32, device=DEV)[:1])
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    out = torch.empty_like(q)
    hn = L.HeadNorm() if norm else None
    L.lserve_rotary_append_kv(desc, kv, rot, q, k, k, cu, kv.seq_lens, n, out, norm=hn)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    if norm:
        L.lserve_norm_rotary(desc, hn, rot, q, None, pos, q, None)
    else:
        L.lserve_rotary_axes(desc, rot, L.PositionAxes([0] * 64), q, None, pos.view(1, n), q, None)
    torch.cuda.synchronize()
    want = reference(before, 128, False, some[None].int(), [0] * 64, rot.inv_freq.cpu(), norm=norm)
    assert_close(q[some.to(DEV)], want, torch.bfloat16)
    assert_close(out[some.to(DEV)], want, torch.bfloat16)
    page, slot = kv.page_table[0, (some // 64).to(DEV)].long(), (some % 64).to(DEV)
    assert_close(kv.k_pool[page, :, slot], reference(before_k, 128, False, some[None].int(), [0] * 64, rot.inv_freq.cpu(), norm=norm), torch.bfloat16)
    assert torch.equal(kv.v_pool[page, :, slot].cpu(), before_k)


@pytest.mark.parametrize("most", [1, 2])
@pytest.mark.parametrize("bits", [16, 4])
def test_pages_past_2_31_elements(most, bits):
    """A pool whose last pages start past 2^31 elements (16 bits) or 2^32 bytes (4)."""
    L = _lib()
    per = 64 * 64 * 128 * 2 if bits == 16 else 64 * 4352
    pages = ((1 << 32) + (1 << 20)) // per + 2
    desc = L.AttnDesc(64, 64, [0] * 64)
    kind, shape = (torch.float16, (pages, 64, 64, 128)) if bits == 16 else (torch.uint8, (pages, 64, 4352))
    kv = L.PagedKV(torch.zeros(shape, dtype=kind, device=DEV), torch.zeros(shape, dtype=kind, device=DEV), torch.zeros((pages, 64, 4, 2, 128), dtype=torch.float16, device=DEV),
                   torch.tensor([[pages - 1], [pages - 2]], dtype=torch.int32, device=DEV), torch.tensor([5, 9, 0, 0], dtype=torch.int32, device=DEV)[:2], kv_bits=bits)
    g = torch.Generator().manual_seed(2)
    k, v = torch.randn((2 * most, 64, 128), generator=g).half().to(DEV), torch.randn((2 * most, 64, 128), generator=g).half().to(DEV)
    cu = torch.tensor([0, most, 2 * most], dtype=torch.int32, device=DEV)
    turned = torch.empty_like(k)
    L.lserve_rotary_append_kv(desc, kv, L.RotaryDesc(), None, k, v, cu, kv.seq_lens, most, None, k_out=turned)
    torch.cuda.synchronize()
    ends = lambda t: t[pages - 2:].clone()  # noqa: E731
    got = [ends(t) for t in (kv.k_pool, kv.v_pool, kv.stats)]
    for t in (kv.k_pool, kv.v_pool, kv.stats):
        assert not t[:pages - 2].view(torch.int64).any()
        t.zero_()
    L.lserve_append_kv(desc, kv, turned, v, cu, kv.seq_lens, most)
    torch.cuda.synchronize()
    assert got[0].any() and got[2].any()
    for x, t in zip(got, (kv.k_pool, kv.v_pool, kv.stats)):
        assert torch.equal(x.view(torch.uint8), ends(t).view(torch.uint8))


@pytest.mark.parametrize("most", [1, 7])
def test_the_largest_batch(most):
    """65535 sequences of none, one or a few tokens."""
    L = _lib()
    batch = 65535
    g = torch.Generator().manual_seed(3)
    counts = torch.randint(0, most + 1, (batch,), generator=g)
    lens = torch.randint(0, 10, (batch,), generator=g).to(torch.int32).to(DEV)
    n = int(counts.sum())
    cu = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)]).to(torch.int32).to(DEV)
    desc = L.AttnDesc(1, 1, [0], page_size=16)
    table = torch.randperm(batch, generator=g).to(torch.int32).view(batch, 1).to(DEV)
    pool = lambda: torch.zeros((batch, 1, 16, 128), dtype=torch.float16, device=DEV)  # noqa: E731
    kv = L.PagedKV(pool(), pool(), torch.zeros((batch, 1, 1, 2, 128), dtype=torch.float16, device=DEV), table, lens)
    twin = L.PagedKV(pool(), pool(), torch.zeros_like(kv.stats), table, lens)
    q, k, v = (torch.randn((n, 1, 128), generator=g).half().to(DEV) for _ in range(3))
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    rot = L.RotaryDesc()
    L.lserve_rotary_append_kv(desc, kv, rot, q, k, v, cu, lens, most, qo, k_out=ko)
    L.lserve_append_kv(desc, twin, ko, v, cu, lens, most)
    torch.cuda.synchronize()
    for name in ("k_pool", "v_pool", "stats"):
        assert torch.equal(getattr(kv, name), getattr(twin, name)), name
    at = torch.repeat_interleave(lens.cpu().long(), counts) + torch.arange(n) - torch.repeat_interleave(cu[:-1].cpu().long(), counts)
    for x, got in ((q, qo), (k, ko)):
        assert_close(got, reference(x.cpu(), 128, False, at[None].int(), [0] * 64, rot.inv_freq.cpu()), torch.float16)
