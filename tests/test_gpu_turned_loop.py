"""A serving loop whose rows go into the pages by lserve_rotary_append_kv next to one that writes the same turned keys with lserve_append_kv: the same bytes in every pool
after every call and the same attention of every head; and the attention against softmax in 64 bits over what a head attends, streaming heads among them."""
import pytest
import torch

from test_gpu_append_special import _expected
from test_gpu_turned_session import D, DEV, HKV, HQ, LOCAL, PAGE, SINK, _rows, _session

pytestmark = pytest.mark.gpu


def _kept(rows, bits):
    """What pages hold of rows [n][heads][D], in 64 bits."""
    x = rows.cpu()
    if bits == 16 or not x.shape[0]:
        return x.double()
    codes, scale, zero = _expected(x.float().numpy().reshape(-1, D), bits)
    return torch.from_numpy(codes.astype("float64") * scale.astype("float64")[:, None] + zero.astype("float64")[:, None]).view(x.shape)


def _attended(keys, values, query):
    return torch.softmax(keys @ query / D ** 0.5, 0) @ values


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits,two_way", [(16, False), (16, True), (8, False), (8, True), (4, False), (4, True)])
@pytest.mark.parametrize("A", [1, 3])
def test_two_loops(dtype, bits, two_way, A):
    import paper_2502_14866_amd as L

    L.load_library()
    g = torch.Generator().manual_seed(11)
    # a prompt, a chunk of another for some, single tokens (none for one), and a few accepted ones
    rounds = [[300, 1, 65, 517], [0, 130, 0, 7], [1, 1, 1, 1], [1, 0, 1, 1], [2, 1, 2, 2], [1, 1, 1, 1], [3, 5, 1, 4], [1, 1, 1, 1]]
    batch, width = 4, 10
    one, twin = (_session(L, dtype, bits, two_way, 40, batch, width) for _ in range(2))
    rot, norm = L.RotaryDesc(base=500000.0), L.HeadNorm(*((1 + 0.2 * torch.randn(D, generator=g)).to(DEV) for _ in range(2)))
    axes = L.PositionAxes.in_turn(24, 20, 20) if A == 3 else None
    free = torch.randperm(40, generator=g).to(torch.int32).to(DEV)
    i32 = lambda n: torch.zeros((n,), dtype=torch.int32, device=DEV)  # noqa: E731
    lens, taken = i32(batch), 0
    keys, values = ([torch.zeros((0, HKV, D), dtype=torch.float64)] * batch for _ in range(2))
    stepped, half = 0, torch.finfo(dtype).eps / 2
    for counts in rounds:
        total, most = sum(counts), max(counts)
        cu, after, pages, pos = i32(batch + 1), i32(batch), i32(1), i32(total)
        for s in (one, twin):
            s.set_seq_lens(lens)
            s.extend(torch.tensor(counts, dtype=torch.int32, device=DEV), free[taken:], cu, after, pages, pos)
        taken += int(pages)
        q, k, v = _rows(g, dtype, total)
        where = torch.stack([pos, pos % 17, pos % 5]).contiguous() if axes else None
        kd, vd = (torch.empty((total, HKV, D), dtype=dtype, device=DEV) for _ in range(2))
        turned = one.append_rotary(rot, q, k, v, cu, lens, most, norm=norm, axes=axes, positions=where, k_out=kd, v_out=vd)
        twin.append(kd, vd, cu, lens, most)
        torch.cuda.synchronize()
        assert torch.equal(vd, v)
        for name in ("k_pool", "v_pool", "stats", "k_pool_stream", "v_pool_stream"):
            x, y = getattr(one.kv, name), getattr(twin.kv, name)
            assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8)), (counts, name)
        at = cu.tolist()
        for b in range(batch):
            keys[b] = torch.cat([keys[b], _kept(kd[at[b]:at[b + 1]], bits)])
            values[b] = torch.cat([values[b], _kept(vd[at[b]:at[b + 1]], bits)])
        if counts == [1] * batch:
            stepped += 1
            out = one.step(turned, after, lens).clone()
            again = twin.step(turned, after, lens)
            torch.cuda.synchronize()
            assert torch.equal(out, again) and torch.equal(one.lse, twin.lse)
            assert torch.equal(one.sel_pages, twin.sel_pages) and torch.equal(one.sel_count, twin.sel_count)
            for b in range(batch):
                n = keys[b].shape[0]
                tail = (-(-n // PAGE) - LOCAL // PAGE) * PAGE  # first token of the local pages
                for h in range(HQ):
                    hk = h // (HQ // HKV)
                    seen = torch.arange(n)
                    if hk < 2:  # sink and local pages
                        seen = seen[(seen < SINK) | (seen >= tail)]
                    elif n > 256:  # more than the budget: what is attended is the selector's choice, of the twin's statistics too
                        continue
                    # Half a step of the type: the output, a weight, the sum of the weights (of rounded ones or not), and all else: sums of 128 products in 32 bits,
                    # 128 U of 100 / sqrt(D) at most, below 1e-4 of a weight.  Codes: what they stand for may be rounded to the type on its way, in a value, and in a
                    # key, which moves a score by half a step of the sum of its products' sizes.
                    kk, vv, query = keys[b][seen, hk], values[b][seen, hk], turned[b, h].cpu().double()
                    tol = 4 * half * vv.abs().max() + 1e-5
                    if bits != 16:
                        off = half * (kk.abs() @ query.abs()).max() / D ** 0.5
                        tol = tol + (half + torch.expm1(2 * off)) * vv.abs().max()
                    got, want = out[b, h].cpu().double(), _attended(kk, vv, query)
                    assert ((got - want).abs() <= tol).all(), (b, h, float((got - want).abs().max()), float(tol))
        lens = after
    assert stepped == 3
