"""Tokens written at the last positions that 32 bits hold: the bytes of the same tokens as far into their pages, the ring and the logical pages, at lower positions."""
import pytest
import torch

from turn_reference import assert_close, reference

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
END = 2 ** 31 - 1


def _lib():
    import paper_2502_14866_amd as L

    L.load_library()
    return L


def _cache(L, desc, bits, ring_only, width, pages, last):
    """A cache whose sequence has its last `pages` pages in front of page `last` of a table `width` wide; a ring alone, or every head in the main pool."""
    page, hkv = desc.page_size, desc.num_kv_heads
    g = torch.Generator().manual_seed(1)

    def pool(n):
        if bits == 16:
            return torch.randn((n, hkv, page, 128), generator=g).half().to(DEV)
        return torch.randint(0, 256, (n, hkv, 64 * 128 * bits // 8 + 256), generator=g).to(torch.uint8).to(DEV)

    lens = torch.zeros(4, dtype=torch.int32, device=DEV)[:1]
    stats = torch.randn((pages, hkv, page // desc.logical_page_size, 2, 128), generator=g).half().to(DEV)
    if ring_only:
        ring = -(-desc.sink_tokens // page) - (-desc.local_tokens // page)
        return L.PagedKV(pool(1), pool(1), stats[:1].clone(), torch.zeros((1, 1), dtype=torch.int32, device=DEV), lens, k_pool_stream=pool(ring), v_pool_stream=pool(ring),
                         ring_table=torch.randperm(ring, generator=g).to(torch.int32).view(1, ring).to(DEV), kv_bits=bits)
    table = torch.zeros((1, width), dtype=torch.int32, device=DEV)
    table[0, last - pages:last] = torch.randperm(pages, generator=g).to(torch.int32).to(DEV)
    return L.PagedKV(pool(pages), pool(pages), stats, table, lens, kv_bits=bits)


def _same(a, b):
    for name in ("k_pool", "v_pool", "stats", "k_pool_stream", "v_pool_stream"):
        x, y = getattr(a, name), getattr(b, name)
        if x is not None:
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), name


CASES = [(64, 16, 16), (64, 16, 4), (64, 64, 8), (16, 2, 16), (16, 16, 16), (128, 128, 16)]


def _at(page, ring_only, n, short, sink=64, local=128):
    """A start whose tokens end `short` ones ahead of the last position, a lower one as far into its page and turn of the ring, pages, page behind the last."""
    start = END - short - n
    if ring_only:
        turn = page * -(-local // page)
        lower = start - turn * ((start - 4 * turn - sink - 128) // turn)
    else:
        lower = start - 128 * ((start - 4096) // 128)
    last, last_lower = (start + n - 1) // page + 1, (lower + n - 1) // page + 1
    assert last - last_lower == (start - lower) // page
    return start, lower, last_lower - lower // page + 1, last, last_lower


@pytest.mark.parametrize("page,logical,bits", CASES)
@pytest.mark.parametrize("ring_only", [False, True])
@pytest.mark.parametrize("n", [1, 2, 7, 40, 333])
@pytest.mark.parametrize("short", [0, 1, 14, 70])
def test_append_kv(page, logical, bits, ring_only, n, short):
    L = _lib()
    desc = L.AttnDesc(2, 2, [1, 1] if ring_only else [0, 1], page_size=page, logical_page_size=logical, sink_tokens=64, local_tokens=128)
    start, lower, pages, last, last_lower = _at(page, ring_only, n, short)
    far, near = (_cache(L, desc, bits, ring_only, (END + page) // page, pages, at) for at in (last, last_lower))
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn((n, 2, 128), generator=g).half().to(DEV) for _ in range(2))
    i32 = lambda *a: torch.tensor(a + (0,) * 4, dtype=torch.int32, device=DEV)[:len(a)]  # noqa: E731
    cu, most = i32(0, n), n if short else n + 3
    before = (near.k_pool_stream if ring_only else near.k_pool).clone()
    L.lserve_append_kv(desc, near, k, v, cu, i32(lower), most)
    L.lserve_append_kv(desc, far, k, v, cu, i32(start), most)
    torch.cuda.synchronize()
    assert not torch.equal(before, near.k_pool_stream if ring_only else near.k_pool)
    _same(far, near)


@pytest.mark.parametrize("page,logical,bits", CASES)
@pytest.mark.parametrize("ring_only", [False, True])
@pytest.mark.parametrize("n", [1, 2, 7, 40, 333])
@pytest.mark.parametrize("short", [0, 1, 14, 70])
@pytest.mark.parametrize("R,norm", [(128, None), (20, "rms")])
def test_rotary_append_kv(page, logical, bits, ring_only, n, short, R, norm):
    """Turned by the positions that were given: the same bytes at either place, and lserve_append_kv's of the turned keys."""
    L = _lib()
    desc = L.AttnDesc(6, 2, [1, 1] if ring_only else [0, 1], page_size=page, logical_page_size=logical, sink_tokens=64, local_tokens=128)
    start, lower, pages, last, last_lower = _at(page, ring_only, n, short)
    far, near, apart = (_cache(L, desc, bits, ring_only, (END + page) // page, pages, at) for at in (last, last_lower, last))
    g = torch.Generator().manual_seed(n)
    q, k, v = (torch.randn((n, h, 128), generator=g).half().to(DEV) for h in (6, 2, 2))
    i32 = lambda *a: torch.tensor(a + (0,) * 4, dtype=torch.int32, device=DEV)[:len(a)]  # noqa: E731
    cu, most = i32(0, n), n if short else n + 3
    pos = torch.randint(0, 5000, (n + 4,), generator=g).to(torch.int32).to(DEV)[:n]
    rot, hn = L.RotaryDesc(rotary_dim=R), L.HeadNorm() if norm else None
    out = [[torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)] for _ in range(2)]
    for kv, at, o in ((near, lower, out[0]), (far, start, out[1])):
        L.lserve_rotary_append_kv(desc, kv, rot, q, k, v, cu, i32(at), most, o[0], k_out=o[1], v_out=o[2], norm=hn, positions=pos)
    L.lserve_append_kv(desc, apart, out[0][1], v, cu, i32(start), most)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*out)) and torch.equal(out[0][2], v)
    _same(far, near)
    _same(far, apart)


@pytest.mark.parametrize("n", [1, 2, 40, 333])
@pytest.mark.parametrize("interleaved", [False, True])
def test_places_as_positions(n, interleaved):
    """A token's place is its position up to the last one."""
    L = _lib()
    desc = L.AttnDesc(6, 2, [1, 1], sink_tokens=64, local_tokens=128)
    start, _, pages, last, _ = _at(64, True, n, 0)
    kv = _cache(L, desc, 16, True, 0, pages, last)
    g = torch.Generator().manual_seed(n)
    q, k, v = (torch.randn((n, h, 128), generator=g).half() for h in (6, 2, 2))
    i32 = lambda *a: torch.tensor(a + (0,) * 4, dtype=torch.int32, device=DEV)[:len(a)]  # noqa: E731
    rot = L.RotaryDesc(interleaved=interleaved)
    qo, ko = torch.empty_like(q, device=DEV), torch.empty_like(k, device=DEV)
    L.lserve_rotary_append_kv(desc, kv, rot, q.to(DEV), k.to(DEV), v.to(DEV), i32(0, n), i32(start), n, qo, k_out=ko)
    torch.cuda.synchronize()
    places = torch.arange(start, start + n, dtype=torch.int64)[None]
    for x, got in ((q, qo), (k, ko)):
        assert_close(got, reference(x, 128, interleaved, places, [0] * 64, rot.inv_freq.cpu()), torch.float16)
