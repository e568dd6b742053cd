"""Both kernels of lserve_rotary_append_kv past 32-bit offsets and at the largest batch.  The bound on a sequence's tokens chooses between them, and may be wider than
the tokens that there are: from nine on the tokens go by blocks, up to eight and in batches large enough one after the other."""
import pytest
import torch

from turn_reference import assert_close, reference

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BLOCKS = 9


def _lib():
    import paper_2502_14866_amd as L

    L.load_library()
    return L


@pytest.mark.parametrize("n", [1, 3, 40])
@pytest.mark.parametrize("bits,logical", [(16, 16), (8, 16), (4, 8)])
def test_blocks_into_pages_past_2_31_elements(n, bits, logical):
    """A pool whose last pages start past 2^31 elements (16 bits) or 2^32 bytes; with logical pages of eight the last statistics too lie past 2^31 elements."""
    L = _lib()
    per, g = 64 * 64 * 128 * 2 if bits == 16 else 64 * (64 * 128 * bits // 8 + 256), 64 // logical
    pages = max(((1 << 32) + (1 << 20)) // per + 2, (1 << 31) // (64 * g * 256) + 3 if logical == 8 else 0)
    desc = L.AttnDesc(64, 64, [0] * 64, logical_page_size=logical)
    kind, shape = (torch.float16, (pages, 64, 64, 128)) if bits == 16 else (torch.uint8, (pages, 64, 64 * 128 * bits // 8 + 256))
    kv = L.PagedKV(torch.zeros(shape, dtype=kind, device=DEV), torch.zeros(shape, dtype=kind, device=DEV), torch.zeros((pages, 64, g, 2, 128), dtype=torch.float16, device=DEV),
                   torch.tensor([[pages - 1], [pages - 2]], dtype=torch.int32, device=DEV), torch.tensor([5, 9, 0, 0], dtype=torch.int32, device=DEV)[:2], kv_bits=bits)
    numbers = torch.Generator().manual_seed(2)
    k, v = (torch.randn((2 * n, 64, 128), generator=numbers).half().to(DEV) for _ in range(2))
    cu = torch.tensor([0, n, 2 * n], dtype=torch.int32, device=DEV)
    turned = torch.empty_like(k)
    L.lserve_rotary_append_kv(desc, kv, L.RotaryDesc(), None, k, v, cu, kv.seq_lens, max(n, BLOCKS), None, k_out=turned)
    torch.cuda.synchronize()
    got = [t[pages - 2:].clone() for t in (kv.k_pool, kv.v_pool, kv.stats)]
    for t in (kv.k_pool, kv.v_pool, kv.stats):
        assert not t[:pages - 2].view(torch.int64).any()
        t.zero_()
    L.lserve_append_kv(desc, kv, turned, v, cu, kv.seq_lens, n)
    torch.cuda.synchronize()
    for x, t in zip(got, (kv.k_pool, kv.v_pool, kv.stats)):
        assert x.any() and torch.equal(x.view(torch.uint8), t[pages - 2:].view(torch.uint8))


@pytest.mark.parametrize("most", [1, 7])
def test_blocks_of_the_largest_batch(most):
    """65535 sequences of none, one or a few tokens: the search of a block's sequence takes three rounds of 64 candidates."""
    L = _lib()
    batch = 65535
    g = torch.Generator().manual_seed(3)
    counts = torch.randint(0, most + 1, (batch,), generator=g)
    counts[0], counts[-1] = 0, most
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
    L.lserve_rotary_append_kv(desc, kv, rot, q, k, v, cu, lens, BLOCKS, qo, k_out=ko)
    L.lserve_append_kv(desc, twin, ko, v, cu, lens, most)
    torch.cuda.synchronize()
    for name in ("k_pool", "v_pool", "stats"):
        assert torch.equal(getattr(kv, name), getattr(twin, name)), name
    at = torch.repeat_interleave(lens.cpu().long(), counts) + torch.arange(n) - torch.repeat_interleave(cu[:-1].cpu().long(), counts)
    for x, got in ((q, qo), (k, ko)):
        assert_close(got, reference(x.cpu(), 128, False, at[None].int(), [0] * 64, rot.inv_freq.cpu()), torch.float16)


@pytest.mark.parametrize("bound", [3, BLOCKS])
@pytest.mark.parametrize("norm", [None, "rms"])
def test_rows_far_apart(bound, norm):
    """Three rows 2^30 elements and more from one to the next, the second and third reached from the first one's and from the tensor's start."""
    L = _lib()
    g = torch.Generator().manual_seed(1)
    apart, batch = (1 << 30) + 8, 64
    room = torch.empty(2 * apart + 12 * 128, dtype=torch.float16, device=DEV)
    rows = torch.randn((3, 12 * 128), generator=g).half()
    for i in range(3):
        room[i * apart:i * apart + 12 * 128] = rows[i].to(DEV)
    q, k, v = (room.as_strided((3, h, 128), (apart, 128, 1), at) for h, at in ((8, 0), (2, 1024), (2, 1280)))
    desc, rot = L.AttnDesc(8, 2, [1, 0]), L.RotaryDesc()
    for counts in ([3] + [0] * 63, [2] + [0] * 62 + [1]):
        lens = torch.full((batch,), 5, dtype=torch.int32, device=DEV)
        kv = L.PagedKV(*(torch.zeros((batch, 2, 64, 128), dtype=torch.float16, device=DEV) for _ in range(2)), torch.zeros((batch, 2, 4, 2, 128), dtype=torch.float16, device=DEV),
                       torch.arange(batch, dtype=torch.int32, device=DEV).view(batch, 1), lens)
        cu = torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32, device=DEV)
        qo, ko, vo = (torch.zeros((3, h, 128), dtype=torch.float16, device=DEV) for h in (8, 2, 2))
        L.lserve_rotary_append_kv(desc, kv, rot, q, k, v, cu, lens, bound, qo, k_out=ko, v_out=vo, norm=L.HeadNorm() if norm else None)
        torch.cuda.synchronize()
        where = [(b, 5 + j) for b, n in enumerate(counts) for j in range(n)]
        places = torch.tensor([[p for _, p in where]], dtype=torch.int32)
        want = [reference(rows[:, at:at + h * 128].view(3, h, 128), 128, False, places, [0] * 64, rot.inv_freq.cpu(), norm=norm) for h, at in ((8, 0), (2, 1024))]
        assert_close(qo, want[0], torch.float16)
        assert_close(ko, want[1], torch.float16)
        assert torch.equal(vo.cpu(), rows[:, 1280:].view(3, 2, 128))
        for pool, dense in ((kv.k_pool, ko), (kv.v_pool, vo)):
            assert torch.equal(torch.stack([pool[b, :, p] for b, p in where]), dense)
