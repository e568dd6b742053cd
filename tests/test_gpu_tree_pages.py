"""lserve_sparse_decode_tree over quantised pages with unusual scales, in large batches, and as two calls at once."""
import math

import pytest
import torch

from tree_reference import NP, Problem, random_tree

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _lib():
    import paper_2502_14866_amd as L

    L.load_library()
    return L


def _trees(sizes, seed=0):
    g = torch.Generator().manual_seed(100 + seed)
    return [random_tree(n, g) for n in sizes]


def _both(p, **kw):
    out, lse = p.call(_lib(), **kw)
    p.check(out, lse)
    return out, lse


def _set_row(p, which, b, hk, t, scale, zero):
    """Token t of the history gets another scale and zero, its codes stay: in the page and in the numbers that it stands for."""
    size = 128 * p.bits // 8
    page = p.pools[which][int(p.table[b, t // NP]), hk]
    codes = page[t % NP * size:(t % NP + 1) * size]
    if p.bits == 4:
        c = codes.view(-1, 4)
        codes = torch.stack([c & 15, c >> 4], 1).reshape(-1)
    page[64 * size:].view(torch.float16).view(64, 2)[t % NP] = torch.tensor([scale, zero], dtype=torch.float16)
    sz = torch.tensor([scale, zero], dtype=torch.float16).double()
    p.values[which][b][t, hk] = codes.double() * sz[0] + sz[1]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("nodes", [4, 40])
def test_scales_of_every_size(bits, dtype, nodes):
    """Constant rows (a scale of zero), the smallest numbers of the pages' scales, large values beside small ones.

    Values of 8 bits whose scale is below the smallest normal number are exact as fp16 scales still, so the bounds of any page hold."""
    p = Problem((300, 20), _trees((nodes, 3)), dtype=dtype, bits=bits, flags=[0, 0])
    g = torch.Generator().manual_seed(5)
    for hk in range(2):
        for t in range(0, 300, 3):
            kind = t // 3 % 5
            scale = (0.0, 2.0 ** -24, 2.0 ** -14, 0.75 * 2.0 ** -9, 3.0)[kind]
            zero = (1.25, -0.5, 0.0, -2.0 ** -9, -1.5 * (2 ** bits - 1))[kind]
            _set_row(p, "v", 0, hk, t, scale, zero)
        for t in torch.randperm(300, generator=g)[:40].tolist():
            _set_row(p, "k", 0, hk, t, 0.0, 0.125 * (t % 7))
    _both(p)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_unread_scales_leave_no_trace(bits, dtype):
    """Pages inside the list that only some of the tokens still see: what the others no longer see may be anything."""
    L = _lib()
    chain = list(range(-1, 69))
    p = Problem((640,), [chain], flags=[1, 1], sink=64, local=128, dtype=dtype, bits=bits)
    clean, lse = p.call(L)
    p.check(clean, lse)
    page = int(p.table[0, 9])  # tokens of tile 10 see it, those of tile 11 do not
    p.pools["v"][page, 0, 64 * 128 * bits // 8:].view(torch.float16).view(64, 2)[5, 0] = math.nan
    out, lse_v = p.call(L)
    assert bool(out[:64, 0:2].isnan().all()) and bool(torch.isfinite(out[64:]).all()) and bool(torch.isfinite(out[:64, 2:4]).all())
    assert float((out[64:].double() - clean[64:].double()).abs().max()) <= 4 * torch.finfo(dtype).eps
    assert torch.equal(lse_v, lse)


@pytest.mark.parametrize("bits", [16, 4])
def test_more_sequences_than_lanes(bits):
    """The lists of 150 sequences, one of them long enough to be cut, are laid out 64 sequences at a time."""
    g = torch.Generator().manual_seed(9)
    lens = [int(x) for x in torch.randint(0, 200, (150,), generator=g)]
    lens[100], lens[3] = 7000, 0
    sizes = [int(x) for x in torch.randint(0, 4, (150,), generator=g)]
    sizes[100] = 5
    _both(Problem(lens, _trees(sizes), bits=bits))


@pytest.mark.parametrize("bits,dtype", [(16, torch.float16), (8, torch.float16), (4, torch.bfloat16)])
def test_long_histories_under_many_rows(bits, dtype):
    """Several tiles of rows over the same pieces of a list."""
    _both(Problem((6000, 40), _trees((40, 21)), hq=16, hkv=2, bits=bits, dtype=dtype, flags=[0, 1]))


def test_two_calls_at_once():
    """On two streams with workspaces of their own, nothing waited for between them."""
    L = _lib()
    problems = [Problem((9000, 301), _trees((14, 5)), flags=[0, 0]), Problem((5000, 64, 7), _trees((30, 2, 2)), bits=8, seed=4)]
    want = [p.call(L) for p in problems]
    streams = [torch.cuda.Stream() for _ in problems]
    launches, outs = [], []
    for p in problems:
        outs.append(p.call(L, run=lambda f: (launches.append(f), f())))
    for out, lse in outs:
        out.zero_(), lse.zero_()
    torch.cuda.synchronize()
    for _ in range(6):
        for f, stream in zip(launches, streams):
            f(stream)
    torch.cuda.synchronize()
    for (out, lse), (w, wl) in zip(outs, want):
        assert torch.equal(out, w) and torch.equal(lse, wl)
