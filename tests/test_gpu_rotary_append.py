"""Rows of a projection into the paged cache: queries and dense keys against the formulas in 64 bits, the cache against the write-back of these keys,
byte for byte."""
import numpy as np
import pytest
import torch

from test_gpu_append_special import _expected
from test_gpu_quant import _unpack_rows
from turn_reference import assert_close, reference

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BASE = 500000.0


def _lib():
    import paper_2502_14866_amd as L

    L.load_library()
    return L


def _rows(g, dtype, total, hq, hkv, fused):
    rows = torch.randn((total, (hq + 2 * hkv) * 128), generator=g).to(dtype)
    cut = lambda t: (t[:, :hq * 128].view(total, hq, 128), t[:, hq * 128:(hq + hkv) * 128].view(total, hkv, 128),  # noqa: E731
                     t[:, (hq + hkv) * 128:].view(total, hkv, 128))
    dev = cut(rows.to(DEV))
    return cut(rows), dev if fused else tuple(t.contiguous() for t in dev)


def _cache(L, g, dtype, desc, lens, counts, bits, two_way, page, width=0):
    """A cache with a history, bytes and statistics of any kind, and pages that nobody has."""
    hkv, B = desc.num_kv_heads, len(lens)
    pages = [max(1, -(-(s + n) // page)) for s, n in zip(lens, counts)]
    n_pages = sum(pages) + 3
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((B, max(max(pages), width)), 0, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    streaming = [bool(f) for f in desc.streaming_flags]
    main = hkv - sum(streaming) if two_way else hkv

    def pool(n, heads):
        if bits == 16:
            return torch.randn((n, heads, page, 128), generator=g).to(dtype).to(DEV)
        return torch.randint(0, 256, (n, heads, 64 * 128 * bits // 8 + 256), generator=g).to(torch.uint8).to(DEV)

    ring = -(-desc.sink_tokens // page) + -(-desc.local_tokens // page)
    stats = torch.randn((n_pages, main, page // desc.logical_page_size, 2, 128), generator=g).to(dtype).to(DEV)
    extra = {}
    if two_way:
        extra = dict(k_pool_stream=pool(B * ring, sum(streaming)), v_pool_stream=pool(B * ring, sum(streaming)),
                     ring_table=torch.randperm(B * ring, generator=g).to(torch.int32).view(B, ring).to(DEV))
    lens_d = torch.tensor(lens + [0] * 4, dtype=torch.int32, device=DEV)[:B]
    return L.PagedKV(pool(n_pages, main), pool(n_pages, main), stats, table.to(DEV), lens_d, pool_heads=0 if main == hkv else main, kv_bits=bits, **extra)


def _twin(L, kv):
    same = lambda t: None if t is None else t.clone()  # noqa: E731
    return L.PagedKV(same(kv.k_pool), same(kv.v_pool), same(kv.stats), kv.page_table, kv.seq_lens, pool_heads=kv.pool_heads,
                     k_pool_stream=same(kv.k_pool_stream), v_pool_stream=same(kv.v_pool_stream), ring_table=kv.ring_table, kv_bits=kv.kv_bits)


def _assert_same_cache(a, b):
    for name in ("k_pool", "v_pool", "stats", "k_pool_stream", "v_pool_stream"):
        x, y = getattr(a, name), getattr(b, name)
        if x is not None:
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), name


def _run(dtype, lens, counts, R=128, interleaved=False, bits=16, two_way=False, norm=None, weights=False, A=1, positions=None, hq=8, hkv=4,
         flags=None, page=64, logical=16, sink=128, local=512, fused=True, spare=0, most=None, dense=True, in_place=False, with_q=True, seed=0,
         far=3000):
    L = _lib()
    g = torch.Generator().manual_seed(seed)
    flags = flags if flags is not None else [1] * (hkv // 2) + [0] * (hkv - hkv // 2)
    desc = L.AttnDesc(hq, hkv, flags, dtype=dtype, page_size=page, logical_page_size=logical, sink_tokens=sink, local_tokens=local)
    kv = _cache(L, g, dtype, desc, lens, counts, bits, two_way, page)
    n = sum(counts)
    total = max(1, n + spare)
    (q, k, v), (qd, kd, vd) = _rows(g, dtype, total, hq, hkv, fused and not in_place)
    cu = torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32)
    place = torch.cat([torch.arange(s, s + c) for s, c in zip(lens, counts)] + [torch.zeros(spare, dtype=torch.long)]).to(torch.int32)
    rot = L.RotaryDesc(rotary_dim=R, interleaved=interleaved, base=BASE) if R else None
    pair_axis = [i % A for i in range(max(1, R // 2))]
    axes = L.PositionAxes(pair_axis, A) if A > 1 else None
    given = None
    if positions == "given" or A > 1 and positions != "own":
        given = torch.randint(-20, far, (A, total), generator=g).to(torch.int32)
    where = given if given is not None else place[None].expand(A, total)
    wq = wk = None
    if weights:
        wq, wk = (1 + 0.3 * torch.randn((h, 128) if weights == "heads" else (128,), generator=g) for h in (hq, hkv))
    hn = L.HeadNorm(*(w.to(DEV) if w is not None else None for w in (wq, wk)), centred=norm == "centred") if norm else None
    mark = lambda h: torch.full((total, h, 128), 7.0, dtype=dtype, device=DEV)  # noqa: E731
    qo = None if not with_q else qd if in_place else mark(hq)
    ko = kd if in_place else mark(hkv) if dense else None
    vo = mark(hkv) if dense else None
    twin, k_turned = _twin(L, kv), mark(hkv)
    keys = kd.clone()
    L.lserve_rotary_append_kv(desc, kv, rot, qd if with_q else None, kd, vd, cu.to(DEV), kv.seq_lens, most or max(counts), qo, k_out=ko, v_out=vo,
                              norm=hn, axes=axes, positions=None if given is None else given.to(DEV) if axes else given[0].to(DEV))
    torch.cuda.synchronize()
    freq = rot.inv_freq.cpu() if R else None

    def want(x, w):
        ref, bound = reference(x[:n], R, interleaved, where[:, :n], pair_axis, freq, 1.0, norm, w)
        return ref, bound

    if with_q:
        assert_close(qo[:n], want(q, wq), dtype)
        assert torch.equal(qo[n:].cpu(), q[n:] if in_place else torch.full_like(q[n:], 7.0))
    if ko is None:  # the same call again, on the same cache as it was before, with the keys kept
        again = _twin(L, twin)
        L.lserve_rotary_append_kv(desc, again, rot, None, keys, vd, cu.to(DEV), kv.seq_lens, most or max(counts), None, k_out=k_turned, norm=hn, axes=axes,
                                  positions=None if given is None else given.to(DEV) if axes else given[0].to(DEV))
        torch.cuda.synchronize()
        _assert_same_cache(kv, again)
        ko = k_turned
    assert_close(ko[:n], want(k, wk), dtype)
    if vo is not None:
        assert torch.equal(vo[:n].cpu(), v[:n]) and (vo[n:] == 7.0).all()
        if not in_place:
            assert (ko[n:] == 7.0).all()
    L.lserve_append_kv(desc, twin, ko.contiguous(), vd.contiguous(), cu.to(DEV), kv.seq_lens, most or max(counts))
    torch.cuda.synchronize()
    _assert_same_cache(kv, twin)
    return kv


RAGGED = ([0, 5, 70, 130, 16, 900, 64, 33], [200, 17, 1, 0, 16, 150, 64, 3])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("two_way", [False, True])
@pytest.mark.parametrize("R,interleaved", [(128, False), (128, True), (64, False), (20, True), (20, False), (0, False)])
def test_ragged_batches(dtype, bits, two_way, R, interleaved):
    _run(dtype, *RAGGED, R=R, interleaved=interleaved, bits=bits, two_way=two_way, norm="rms" if R == 64 else None)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("two_way", [False, True])
@pytest.mark.parametrize("R,interleaved", [(128, False), (128, True), (64, False), (20, True), (20, False), (0, False)])
def test_decode_steps(dtype, bits, two_way, R, interleaved):
    """A token each, or none; first and later tokens of logical and physical pages."""
    lens = [0, 5, 15, 16, 63, 64, 127, 700, 701, 3000, 1, 31]
    _run(dtype, lens, [1, 1, 1, 1, 1, 1, 1, 0, 1, 1, 0, 1], R=R, interleaved=interleaved, bits=bits, two_way=two_way, norm="centred" if R == 64 else None)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("two_way", [False, True])
@pytest.mark.parametrize("R,interleaved,norm", [(128, False, None), (64, True, "rms"), (20, False, "centred"), (0, False, None)])
def test_a_few_tokens_each(dtype, bits, two_way, R, interleaved, norm):
    """Up to two, three, four and eight of as many sequences as take them one after the other, across the ends of logical and physical pages."""
    g = torch.Generator().manual_seed(R + bits)
    for batch, most in ((5, 2), (64, 3), (130, 4), (390, 8)):
        counts = torch.randint(0, most + 1, (batch,), generator=g).tolist()
        counts[0], counts[-1] = most, 1
        lens = torch.randint(0, 200, (batch,), generator=g).tolist()
        lens[:4] = [63, 15, 0, 64]
        _run(dtype, lens, counts, R=R, interleaved=interleaved, norm=norm, bits=bits, two_way=two_way, sink=64, local=64, hq=2, hkv=2, dense=batch != 64, spare=batch % 3,
             weights="heads" if norm else False)


@pytest.mark.parametrize("two_way", [False, True])
@pytest.mark.parametrize("page,logical", [(16, 2), (16, 4), (32, 32), (128, 128)])
def test_a_few_tokens_each_in_pages_of_other_sizes(two_way, page, logical):
    """One local page of sixteen tokens: some of the call's own are gone by its end."""
    g = torch.Generator().manual_seed(page + logical)
    counts, lens = torch.randint(0, 9, (400,), generator=g).tolist(), torch.randint(0, 300, (400,), generator=g).tolist()
    _run(torch.bfloat16, lens, counts, page=page, logical=logical, two_way=two_way, sink=16, local=1, hq=4, hkv=2, in_place=page == 32)


@pytest.mark.parametrize("page,logical", [(16, 16), (16, 2), (32, 16), (32, 4), (64, 64), (64, 32), (64, 8), (128, 16), (128, 128), (128, 64)])
@pytest.mark.parametrize("two_way", [False, True])
def test_pages(page, logical, two_way):
    _run(torch.float16, *RAGGED, page=page, logical=logical, two_way=two_way, sink=16, local=48)
    _run(torch.bfloat16, [0, 5, 70, 15, 127], [1, 1, 0, 1, 1], page=page, logical=logical, two_way=two_way, sink=16, local=48)
    _run(torch.bfloat16, *RAGGED, R=20, page=page, logical=logical, two_way=two_way)


@pytest.mark.parametrize("norm", [None, "rms", "centred"])
@pytest.mark.parametrize("weights", [False, "shared", "heads"])
@pytest.mark.parametrize("A,positions", [(1, "own"), (1, "given"), (3, "given"), (2, "own")])
def test_norms_and_positions(norm, weights, A, positions):
    _run(torch.float16, *RAGGED, norm=norm, weights=weights, A=A, positions=positions)
    _run(torch.bfloat16, [5, 800, 64], [1, 1, 1], norm=norm, weights=weights, A=A, positions=positions, interleaved=True)
    _run(torch.bfloat16, *RAGGED, R=20, norm=norm, weights=weights, A=A, positions=positions, bits=8)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (8, 1), (32, 8), (64, 64), (64, 8), (40, 5)])
def test_heads(hq, hkv):
    flags = [i % 2 for i in range(hkv)]
    _run(torch.float16, [7, 100], [40, 19], hq=hq, hkv=hkv, flags=flags, norm="rms", weights="heads")
    _run(torch.float16, [7, 100], [1, 1], hq=hq, hkv=hkv, flags=flags, norm="rms", weights="heads", bits=4)


@pytest.mark.parametrize("flags", [[0, 0, 0, 0], [1, 1, 1, 1], [0, 1, 0, 1]])
def test_kinds_of_heads(flags):
    for counts in ([40, 0, 190], [1, 0, 1]):
        _run(torch.bfloat16, [7, 100, 333], counts, flags=flags)
        _run(torch.bfloat16, [7, 100, 333], counts, flags=flags, two_way=0 < sum(flags) < 4, bits=8)


def test_rows_past_the_last_sequence_are_left_alone():
    _run(torch.float16, [7, 100], [40, 19], spare=37)
    _run(torch.float16, [7, 100], [1, 1], spare=5)
    _run(torch.float16, [7, 100], [40, 19], spare=37, in_place=True)


@pytest.mark.parametrize("counts", [[40, 19, 64], [1, 1, 1]])
def test_in_place_and_parts_of_the_call(counts):
    lens = [7, 100, 64]
    _run(torch.float16, lens, counts, in_place=True, norm="rms")
    _run(torch.float16, lens, counts, with_q=False)
    _run(torch.float16, lens, counts, dense=False, two_way=True)
    _run(torch.float16, lens, counts, dense=False, bits=4, norm="rms")
    _run(torch.float16, lens, counts, fused=False, R=20)


@pytest.mark.parametrize("batch", [1, 63, 64, 65, 200, 5000])
def test_batches(batch):
    """The search for a block's sequence, 64 candidates at a time; sequences without tokens among them."""
    g = torch.Generator().manual_seed(batch)
    lens = torch.randint(0, 40, (batch,), generator=g).tolist()
    counts = torch.randint(0, 6, (batch,), generator=g).tolist()
    counts[-1] = 3
    counts[0] = 0 if batch > 1 else 3
    _run(torch.float16, lens, counts, hq=2, hkv=1, flags=[0], page=16, seed=batch, most=40)
    _run(torch.float16, lens, [min(c, 1) for c in counts], hq=2, hkv=1, flags=[0], page=16, seed=batch)


def test_one_long_prompt():
    _run(torch.bfloat16, [0], [9001], hq=32, hkv=8, norm="rms", weights="shared")
    _run(torch.bfloat16, [77], [5000], hq=8, hkv=2, bits=4, two_way=True, dense=False)


def test_a_step_written_as_more_than_one_token_at_most():
    """max_new_per_seq is a bound: single tokens under a larger one go another way to the same bytes."""
    a = _run(torch.float16, [5, 64, 200], [1, 1, 1], norm=None)
    b = _run(torch.float16, [5, 64, 200], [1, 1, 1], norm=None, most=3)
    _assert_same_cache(a, b)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("counts", [[1, 1, 1], [40, 19, 64]])
def test_rows_of_any_bits(dtype, bits, counts):
    """Infinities, what is not a number, signalling or not, zeros of both signs: where nothing turns, the bytes that the formulas in numpy make of the same
    rows.  A not-a-number takes no part in ranges and gets code 0."""
    L = _lib()
    g = torch.Generator().manual_seed(sum(counts))
    desc = L.AttnDesc(4, 2, [0, 0], dtype=dtype)
    lens = [7, 100, 64]
    kv = _cache(L, g, dtype, desc, lens, counts, bits, False, 64)
    before = kv.stats.float().cpu().numpy()
    n = sum(counts)
    k, v = (torch.randn((n, 2, 128), generator=g).to(dtype) for _ in range(2))
    odd = torch.tensor([0x7c00, 0xfc00, 0x7e00, 0x7c01, 0xfe00, 0x8000, 0x0000, 0x0001, 0x7f80, 0xff80, 0x7fc0, 0x7f81, 0xffc0], dtype=torch.int32).to(torch.int16)
    for t in (k, v):
        bits_of = t.view(torch.int16).view(-1)
        at = torch.randint(0, bits_of.numel(), (bits_of.numel() // 50,), generator=g)
        bits_of[at] = odd[torch.randint(0, len(odd), at.shape, generator=g)]
        t[0, 0] = 0.0
        t[0, 0, ::2] = -0.0
    cu = torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32)
    ko, vo = torch.empty_like(k, device=DEV), torch.empty_like(v, device=DEV)
    L.lserve_rotary_append_kv(desc, kv, None, None, k.to(DEV), v.to(DEV), cu.to(DEV), kv.seq_lens, max(counts), None, k_out=ko, v_out=vo)
    torch.cuda.synchronize()
    assert torch.equal(ko.view(torch.int16).cpu(), k.view(torch.int16)) and torch.equal(vo.view(torch.int16).cpu(), v.view(torch.int16))
    table, stats = kv.page_table.cpu(), kv.stats.float().cpu().numpy()

    def numbers(x):  # (a signalling not-a-number would take the place of what numpy's reductions held before it)
        f = x.float().numpy()
        return np.where(np.isnan(f), np.float32(np.nan), f)

    for rows, pool in ((k, kv.k_pool.cpu()), (v, kv.v_pool.cpu())):
        where = [(b, lens[b] + j, int(cu[b]) + j) for b in range(3) for j in range(counts[b])]
        for h in range(2):
            x = rows[[t for _, _, t in where], h]
            slabs = [(pool[table[b, p // 64], h], p % 64) for b, p, _ in where]
            if bits == 16:
                assert torch.equal(torch.stack([s[i] for s, i in slabs]).view(torch.int16), x.view(torch.int16))
                continue
            codes, scale, zero = _expected(numbers(x), bits)
            size = 128 * bits // 8
            got = np.stack([_unpack_rows(s[:64 * size].numpy().reshape(64, size)[i:i + 1], bits)[0] for s, i in slabs])
            pair = np.stack([s[64 * size:].numpy().view(np.float16).reshape(64, 2)[i] for s, i in slabs])
            # (as numbers: the smallest of zeros of both signs is either)
            assert np.array_equal(pair[:, 0], scale, equal_nan=True) and np.array_equal(pair[:, 1], zero, equal_nan=True)
            assert np.array_equal(got, codes)
    for b in range(3):  # statistics, logical page by logical page
        for first in range(lens[b] // 16 * 16, lens[b] + counts[b], 16):
            part = numbers(k[int(cu[b]) + max(first - lens[b], 0):int(cu[b]) + min(first + 16, lens[b] + counts[b]) - lens[b]])
            at = table[b, first // 64], slice(None), first % 64 // 16
            old = before[at] if first < lens[b] else np.stack([np.full((2, 128), -np.inf), np.full((2, 128), np.inf)], 1)
            high, low = np.fmax(np.fmax.reduce(part, axis=0), old[:, 0]), np.fmin(np.fmin.reduce(part, axis=0), old[:, 1])
            assert np.array_equal(stats[at][:, 0], high.astype(np.float32)) and np.array_equal(stats[at][:, 1], low.astype(np.float32)), (b, first)


@pytest.mark.parametrize("counts", [[1, 1], [40, 150]])
def test_a_page_table_narrower_than_the_ring_s_sequences(counts):
    """A layer whose heads all stream through the ring keeps no pages elsewhere."""
    L = _lib()
    g = torch.Generator().manual_seed(6)
    desc = L.AttnDesc(4, 2, [1, 1], sink_tokens=64, local_tokens=128)
    pool = lambda: torch.zeros((6, 2, 64, 128), dtype=torch.float16, device=DEV)  # noqa: E731
    start = torch.tensor([1000, 64 * 100000 + 5, 0, 0], dtype=torch.int32, device=DEV)[:2]
    ring = torch.randperm(6, generator=g).to(torch.int32).view(2, 3).to(DEV)
    none = torch.zeros((1, 2, 64, 128), dtype=torch.float16, device=DEV)
    kv, twin = (L.PagedKV(none, none.clone(), None, torch.zeros((2, 1), dtype=torch.int32, device=DEV), start, k_pool_stream=pool(), v_pool_stream=pool(), ring_table=ring)
                for _ in range(2))
    _, (q, k, v) = _rows(g, torch.float16, sum(counts), 4, 2, True)
    cu = torch.tensor([0, counts[0], sum(counts)], dtype=torch.int32, device=DEV)
    qo, ko = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)
    L.lserve_rotary_append_kv(desc, kv, L.RotaryDesc(), q, k, v, cu, start, max(counts), qo, k_out=ko)
    L.lserve_append_kv(desc, twin, ko, v.contiguous(), cu, start, max(counts))
    torch.cuda.synchronize()
    assert kv.k_pool_stream.any()
    _assert_same_cache(kv, twin)


@pytest.mark.parametrize("step", [False, True])
def test_on_a_stream_of_its_own_and_captured(step):
    L = _lib()
    L.lserve_init()
    g = torch.Generator().manual_seed(5)
    lens, counts = [7, 100, 64], [1, 1, 1] if step else [40, 19, 64]
    desc, rot, norm = L.AttnDesc(8, 4, [1, 1, 0, 0]), L.RotaryDesc(), L.HeadNorm()
    kv = _cache(L, g, torch.float16, desc, lens, [200] * 3, 8, True, 64)
    twin = _twin(L, kv)
    _, (q, k, v) = _rows(g, torch.float16, sum(counts), 8, 4, True)
    cu = torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32, device=DEV)
    start = kv.seq_lens.clone()
    out, want = torch.zeros_like(q, memory_format=torch.contiguous_format), torch.zeros_like(q, memory_format=torch.contiguous_format)

    def call(cache, to, **kw):
        L.lserve_rotary_append_kv(desc, cache, rot, q, k, v, cu, start, max(counts), to, norm=norm, **kw)

    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call(kv, out, stream=side)
    side.synchronize()
    call(twin, want)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    _assert_same_cache(kv, twin)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(kv, out)
    for i in range(3):
        start.add_(max(counts))
        q.mul_(0.9)
        k.mul_(1.1)
        graph.replay()
        call(twin, want)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        _assert_same_cache(kv, twin)
