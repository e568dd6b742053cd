"""lserve_sparse_decode_tree against its definition in 64 bits: trees and chains over paged history of every kind."""
import math

import numpy as np
import pytest
import torch

from tree_reference import Problem, random_tree

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _lib():
    import paper_2502_14866_amd as L

    L.load_library()
    return L


def _g(seed):
    return torch.Generator().manual_seed(seed)


def _trees(sizes, seed=0):
    g = _g(100 + seed)
    return [random_tree(n, g) for n in sizes]


def _both(p, **kw):
    out, lse = p.call(_lib(), **kw)
    p.check(out, lse, chain=kw.get("chain", False))
    return out, lse


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lens,sizes", [
    ((0,), (1,)), ((1,), (1,)), ((63,), (3,)), ((64,), (9,)), ((65,), (2,)), ((700,), (17,)), ((0, 300, 129), (5, 0, 33)),
    ((1000, 1, 64), (64, 7, 1)), ((2000,), (65,)), ((333, 100), (130, 3)),
])
def test_history_in_one_pool(dtype, lens, sizes):
    _both(Problem(lens, _trees(sizes), dtype=dtype), pad=3)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("two_way", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_kinds_of_cache(bits, two_way, dtype):
    _both(Problem((700, 0, 130, 1281), _trees((9, 4, 0, 21)), dtype=dtype, bits=bits, two_way=two_way))


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("hq,hkv,nodes", [(1, 1, 5), (3, 3, 40), (2, 1, 16), (2, 1, 33), (8, 1, 4), (8, 1, 5), (16, 2, 9), (8, 1, 64), (10, 2, 7), (64, 8, 3), (64, 64, 2)])
def test_heads_and_rows(bits, hq, hkv, nodes):
    _both(Problem((450, 77), _trees((nodes, max(1, nodes // 2))), hq=hq, hkv=hkv, bits=bits, flags=[0] * hkv if hkv < 2 else None))


@pytest.mark.parametrize("flags", [[0, 0], [1, 1], [0, 1], [1, 0]])
@pytest.mark.parametrize("two_way", [False, True])
def test_kinds_of_heads(flags, two_way):
    _both(Problem((900, 200), _trees((12, 30)), flags=flags, two_way=two_way and sum(flags) > 0))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("stale", [0, 1, 70, 300])
def test_selections(bits, stale):
    """Lists that leave out pages, some of them older than the history, so that pages made since follow."""
    _both(Problem((1500, 64, 333, 2), _trees((9, 3, 40, 2)), budget=256, stale=stale, bits=bits, hq=8, hkv=4))


def test_selection_without_pages():
    p = Problem((640, 100), _trees((5, 6)), budget=256)
    p.sel["count"].zero_()
    _both(p)


def test_selected_pages_that_do_not_exist_are_not_read():
    p = Problem((640, 100), _trees((5, 6)), budget=256)
    count = p.sel["count"].clone()
    for b in range(2):
        n = int(count[b, 1])
        p.sel["pages"][b, 1, n:] = torch.tensor([10 ** 6, -5][:4 - n], dtype=torch.int32)
        p.sel["count"][b, 1] = 4
    p.sel["pages"][0, 1, 3], dropped = 2 ** 31 - 1, int(p.sel["pages"][0, 1, 3])
    out, lse = p.call(_lib())
    p.sel["count"], p.sel["pages"][0, 1, 3] = count, dropped
    p.sel["count"][0, 1] = 3
    p.check(out, lse)


@pytest.mark.parametrize("local", [64, 128, 512])
@pytest.mark.parametrize("sink", [0, 64])
@pytest.mark.parametrize("two_way", [False, True])
def test_streaming_windows_move_along_the_tree(local, sink, two_way):
    """Long paths cross page borders: a deep token has lost pages, and drafted ancestors, that a shallow one still sees."""
    chain = list(range(-1, 149))
    bushy = [-1 if j == 0 else max(-1, j - 2) for j in range(100)]
    _both(Problem((1000, 190), [chain, bushy], sink=sink, local=local, two_way=two_way))
    _both(Problem((63, 64), [chain, bushy], sink=sink, local=local, two_way=two_way))


@pytest.mark.parametrize("nodes", [1, 2, 64, 65, 200])
@pytest.mark.parametrize("bits", [16, 8])
def test_chains_without_a_mask(nodes, bits):
    p = Problem((500, 64), [list(range(-1, nodes - 1)), list(range(-1, max(1, nodes // 3) - 1))], bits=bits)
    a = _both(p, chain=True)
    b = _both(p)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_the_widest_tree():
    _both(Problem((100,), [random_tree(1024, _g(5))], hq=2, hkv=1, flags=[0]))


def test_more_words_than_needed():
    _both(Problem((100, 20), _trees((70, 3)), words=5))


def test_rows_that_see_nothing():
    none = np.zeros((5, 5), dtype=bool)
    some = none.copy()
    some[1, 0] = some[3, 3] = True
    _both(Problem((0, 0, 90), [[-1] * 5] * 3, see=[none, some, none]))


def test_any_mask():
    g = _g(9)
    _both(Problem((100, 0), [[-1] * 100, [-1] * 40], see=[torch.rand((n, n), generator=g).numpy() < 0.3 for n in (100, 40)]))


@pytest.mark.parametrize("budget", [0, 1024])
@pytest.mark.parametrize("nodes", [3, 14, 40])
@pytest.mark.parametrize("bits", [16, 4])
def test_long_histories_in_many_pieces(budget, nodes, bits):
    _both(Problem((20000, 301, 9000), _trees((nodes, 1, nodes // 2 + 1)), budget=budget, bits=bits, two_way=bits == 4, local=256))


def test_lists_longer_than_the_table_of_entries():
    """More lists than workgroups run at once leaves lists whole: of 300 pages each here."""
    lens = [19300] * 2 + [100] * 700
    p = Problem(lens, [[-1]] * 702, hq=8, hkv=8, flags=[0] * 8)
    out, lse = p.call(_lib())
    short = Problem(lens[:2], [[-1]] * 2, hq=8, hkv=8, flags=[0] * 8)
    short.q, short.k, short.v = p.q[:2], p.k[:2], p.v[:2]
    short.values = {w: p.values[w][:2] for w in "kv"}
    short.check(out[:2], lse[:2])


def test_loud_queries():
    _both(Problem((700, 90), _trees((9, 30)), loud=8.0))
    _both(Problem((700, 90), _trees((9, 30)), loud=8.0, bits=8, dtype=torch.bfloat16))


def test_one_token_agrees_with_a_decode_step():
    """The drafted token's K / V in the cache and counted, or alongside: the same attention."""
    L = _lib()
    p = Problem((700, 128, 65), [[-1]] * 3, budget=256, stale=5)
    out, lse = p.call(L)
    grown = Problem((701, 129, 66), [[-1]] * 3)
    for b in range(3):
        grown.table[b] = -1
    pages = [-(-n // 64) for n in (701, 129, 66)]
    kp, vp = torch.zeros((sum(pages), 2, 64, 128), dtype=torch.float16), torch.zeros((sum(pages), 2, 64, 128), dtype=torch.float16)
    table, at = torch.zeros((3, max(pages)), dtype=torch.int32), 0
    for b, n in enumerate((700, 128, 65)):
        table[b, :pages[b]] = torch.arange(at, at + pages[b])
        for pool, rows, new in ((kp, p.kh[b], p.k[b]), (vp, p.vh[b], p.v[b])):
            flat = torch.cat([rows, new[None]])
            for t in range(n + 1):
                pool[at + t // 64, :, t % 64] = flat[t]
        at += pages[b]
    lens = torch.tensor([701, 129, 66, 0], dtype=torch.int32, device=DEV)[:3]
    kv = L.PagedKV(kp.to(DEV), vp.to(DEV), None, table.to(DEV), lens)
    desc = L.AttnDesc(4, 2, p.flags, sink_tokens=p.sink, local_tokens=p.local)
    ws = torch.zeros((L.lserve_workspace_bytes(L.LSERVE_CALL_SPARSE_DECODE, desc, 3, max(pages), 4, 0),), dtype=torch.uint8, device=DEV)
    ref, ref_lse = torch.zeros((3, 4, 128), dtype=torch.float16, device=DEV), torch.zeros((3, 4), device=DEV)
    L.lserve_sparse_decode(desc, kv, p.q.to(DEV), p.sel["pages"].to(DEV), p.sel["count"].to(DEV), p.sel["lens"].to(DEV), ref, ref_lse, ws)
    torch.cuda.synchronize()
    assert float((ref.double() - out.double()).abs().max()) <= 2e-3  # two roundings of each, |out| < 2
    assert float((ref_lse - lse).abs().max()) <= 1e-4


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("nodes", [6, 30, 60])
def test_what_is_not_attended_leaves_no_trace(dtype, value, nodes):
    """Siblings do not see each other: a spoiled key or value of one reaches its descendants and nobody else."""
    L = _lib()
    trees = [random_tree(nodes, _g(3)), [-1] * 5]
    p = Problem((100, 40), trees, dtype=dtype, hq=4, hkv=2, flags=[0, 0])
    clean, lse = p.call(L)
    p.check(clean, lse)
    victim = 2
    hit = torch.from_numpy(p.see[0][:, victim].copy())
    p.v[victim, 0, 17] = value
    spoiled, lse_v = p.call(L)
    others = torch.ones((nodes + 5, 4, 128), dtype=torch.bool)
    others[:nodes][hit, 0:2, 17] = False
    assert torch.equal(spoiled.cpu()[others], clean.cpu()[others]) or \
        float((spoiled.cpu()[others].double() - clean.cpu()[others].double()).abs().max()) <= 4 * torch.finfo(dtype).eps
    got = spoiled[:nodes].cpu()[hit][:, 0:2, 17]
    assert bool(got.isnan().all()) if math.isnan(value) else bool((got == value).all())
    assert torch.equal(lse_v, lse)
    p = Problem((100, 40), trees, dtype=dtype, hq=4, hkv=2, flags=[0, 0])
    p.k[victim, 1] = math.nan
    spoiled, lse_k = p.call(L)
    others = torch.ones((nodes + 5, 4), dtype=torch.bool)
    others[:nodes][hit, 2:4] = False
    assert torch.equal(spoiled.cpu()[others], clean.cpu()[others]) and torch.equal(lse_k.cpu()[others], lse.cpu()[others])
    assert bool(spoiled.cpu()[~others].isnan().all()) and bool(lse_k.cpu()[~others].isnan().all())


def test_a_spoiled_page_that_has_left_the_window():
    """Two deep branches, one past a page border: the page that only the shallow tokens see holds an infinity."""
    L = _lib()
    chain = list(range(-1, 69))
    p = Problem((640,), [chain], flags=[1, 1], sink=64, local=128)
    clean, _ = p.call(L)
    p.check(clean)
    page = int(p.table[0, 9])  # tile 9 and the tokens' own tile 10: seen from tile 10 only
    p.pools["v"][page, 0, 5, 3] = math.inf
    out, _ = p.call(L)
    out = out.cpu()
    assert bool((out[:64, 0:2, 3] == math.inf).all()) and bool(torch.isfinite(out[64:]).all())
    assert float((out[64:].double() - clean.cpu()[64:].double()).abs().max()) <= 1e-3


def test_the_same_bits_every_time_and_on_every_stream():
    L = _lib()
    p = Problem((9000, 301), _trees((14, 5)), budget=512)
    a, la = p.call(L)
    b, lb = p.call(L)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def on_side(f):
        f(side)
        side.synchronize()

    c, lc = p.call(L, run=on_side)
    assert torch.equal(a, b) and torch.equal(a, c) and torch.equal(la, lb) and torch.equal(la, lc)
    d, _ = p.call(L, lse=False)
    assert torch.equal(a, d)


def test_captured_and_replayed_with_its_workspace_in_use_elsewhere():
    """Two graphs and eager calls of other sizes share a workspace, one after the other."""
    L = _lib()
    L.lserve_init()
    big, small = Problem((9000, 301), _trees((14, 5))), Problem((700,), _trees((30,)))
    want_big, want_small = big.call(L)[0], small.call(L)[0]
    ws = torch.full((128 << 20,), 255, dtype=torch.uint8, device=DEV)
    graphs, outs = [], []
    for p in (big, small):
        graph = torch.cuda.CUDAGraph()

        def capture(f):
            f()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                f()

        keep = {}
        out, _ = p.call(L, workspace=ws, run=lambda f: (keep.setdefault("f", f), capture(f)))
        graphs.append((graph, keep))
        outs.append(out)
    for i in range(3):
        for (graph, keep), out, want in zip(graphs, outs, (want_big, want_small)):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), i
            keep["f"]()
            torch.cuda.synchronize()
            assert torch.equal(out, want), i
