"""The calls on new tokens one after the other, as a server makes them: pages for a prompt, its rotation and cache; then drafted trees,
of which a path is accepted and joins the cache, against the definition in 64 bits."""
import types

import pytest
import torch

from tree_reference import NP, Problem, ancestors, random_tree

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
D, HQ, HKV, SINK, LOCAL = 128, 4, 2, 64, 128


def _i32(x):
    return torch.tensor(x + [0] * 4, dtype=torch.int32, device=DEV)[:len(x)]


def _numbers(pages, bits):
    """[pages][heads][bytes] -> [tokens][heads][D] in 64 bits."""
    size = NP * D * bits // 8
    code = pages[..., :size]
    if bits == 4:
        code = code.reshape(-1, 4)
        code = torch.stack([code & 15, code >> 4], 1)
    sz = pages[..., size:].contiguous().view(torch.float16).view(pages.shape[0], -1, NP, 2).double()
    x = code.reshape(pages.shape[0], -1, NP, D).double() * sz[..., :1] + sz[..., 1:]
    return x.transpose(1, 2).reshape(-1, x.shape[1], D)


class Server:
    """A session, its free pages and, on the host, every token that the cache should hold."""

    def __init__(self, batch, dtype, two_way, seed=0, width=12, bits=16):
        import paper_2502_14866_amd as L
        from paper_2502_14866_amd.session import DecodeSession

        L.load_library()
        self.L, self.dtype, self.two_way, self.batch, self.bits = L, dtype, two_way, batch, bits
        self.g = torch.Generator().manual_seed(seed)
        pages = batch * width
        shape, kind = ((NP, D), dtype) if bits == 16 else ((NP * D * bits // 8 + 256,), torch.uint8)
        zeros = lambda n, h: torch.zeros((n, h) + shape, dtype=kind, device=DEV)  # noqa: E731
        heads = 1 if two_way else 2
        ring = SINK // NP + LOCAL // NP
        bounded = dict(k_pool_stream=zeros(batch * ring, 1), v_pool_stream=zeros(batch * ring, 1),
                       ring_table=torch.randperm(batch * ring, generator=self.g).to(torch.int32).view(batch, ring).to(DEV)) if two_way else {}
        self.s = DecodeSession(zeros(pages, heads), zeros(pages, heads), torch.full((batch, width), -1, dtype=torch.int32, device=DEV), HQ, [1, 0],
                                 SINK, LOCAL, 128, kv_bits=bits, dtype=dtype, **bounded)
        self.free = torch.randperm(pages, generator=self.g).to(torch.int32).to(DEV)
        self.rotary = L.RotaryDesc(rotary_dim=64)
        self.lens = [0] * batch
        self.s.set_seq_lens(_i32(self.lens))
        self.rows = {w: [torch.zeros((0, HKV, D), dtype=dtype) for _ in range(batch)] for w in "kv"}

    def draw(self, n):
        return [torch.randn((n, h, D), generator=self.g).to(self.dtype).to(DEV) for h in (HQ, HKV, HKV)]

    def grow(self, counts, k=None, v=None):
        """counts new tokens a sequence: their pages, their rotation if they come without, and their rows of the cache."""
        total = sum(counts)
        cu, new, taken, pos = _i32([0] * (self.batch + 1)), _i32([0] * self.batch), _i32([0]), _i32([0] * total)
        self.s.extend(_i32(counts), self.free, cu, new, taken, positions=pos)
        if k is None:
            _, k, v = self.draw(total)
            self.L.lserve_rotary(self.s.desc, self.rotary, None, k, pos, None, k)
        self.s.append(k, v, cu, self.s.kv.seq_lens, max(counts))
        torch.cuda.synchronize()
        assert cu.tolist() == [sum(counts[:b]) for b in range(self.batch + 1)]
        assert pos.tolist() == [n + j for n, m in zip(self.lens, counts) for j in range(m)]
        self.free = self.free[int(taken):].clone()
        for b, m in enumerate(counts):
            self.lens[b] += m
            for w, x in (("k", k), ("v", v)):
                self.rows[w][b] = torch.cat([self.rows[w][b], x[int(cu[b]):int(cu[b + 1])].cpu()])
        assert new.tolist() == self.lens
        self.s.set_seq_lens(new)
        for b, n in enumerate(self.lens):  # the head of every token, page after page
            for w, pool in (("k", self.s.kv.k_pool), ("v", self.s.kv.v_pool)):
                at = [int(p) for p in self.s.kv.page_table[b, :-(-n // NP)]]
                if self.bits != 16:  # what the codes stand for
                    self.rows[w][b] = _numbers(pool[at].cpu(), self.bits)[:n]
                    continue
                assert torch.equal(pool[at, -1].reshape(-1, D)[:n].cpu(), self.rows[w][b][:, 1])

    def expect(self, trees, q, k, v, pos, selected):
        p = Problem.__new__(Problem)
        p.lens, p.trees, p.hq, p.hkv, p.dtype, p.bits, p.flags = list(self.lens), trees, HQ, HKV, self.dtype, self.bits, [1, 0]
        p.s, p.w = SINK // NP, LOCAL // NP
        p.counts = [len(t) for t in trees]
        p.most = max(p.counts)
        p.q, p.k, p.v, p.pos = q.cpu(), k.cpu(), v.cpu(), pos
        p.see = [ancestors(t)[0] for t in trees]
        p.values = {w: [x.double() for x in self.rows[w]] for w in "kv"}
        p.sel = {"pages": self.s.sel_pages.cpu(), "count": self.s.sel_count.cpu(), "lens": self.s.sel_seq_len.cpu()} if selected else None
        return p

    def drafts(self, trees):
        """What a step over drafted trees needs, and the step itself."""
        counts = [len(t) for t in trees]
        total = sum(counts)
        x = types.SimpleNamespace(trees=trees, counts=counts, most=max(counts), cu=_i32([0] + [sum(counts[:b + 1]) for b in range(self.batch)]))
        x.parents = _i32([p for t in trees for p in t])
        x.mask = torch.zeros((total, -(-x.most // 64)), dtype=torch.int64, device=DEV)
        x.pos = _i32([0] * total)
        x.q, x.k, x.v = self.draw(total)
        x.qr, x.kr = torch.empty_like(x.q), torch.empty_like(x.k)
        x.lse = torch.empty((total, HQ), device=DEV)

        def step():
            self.L.lserve_tree_masks(x.parents, x.cu, self.s.kv.seq_lens, x.most, x.mask, x.pos)
            self.L.lserve_rotary(self.s.desc, self.rotary, x.q, x.k, x.pos, x.qr, x.kr)
            return self.s.decode_tree(x.qr, x.kr, x.v, x.cu, x.most, x.mask, x.pos, x.lse)

        x.step = step
        return x


def _path(tree, g):
    j, path = int(torch.randint(0, len(tree), (1,), generator=g)), []
    while j >= 0:
        path.append(j)
        j = tree[j]
    return path[::-1]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("two_way", [False, True])
def test_prompts_drafts_and_what_is_accepted(dtype, two_way):
    s = Server(3, dtype, two_way)
    s.grow([300, 64, 1])
    for turn in range(5):
        trees = [random_tree(n, s.g) for n in ((9, 1, 33), (70, 5, 2), (1, 1, 1), (3, 64, 20), (65, 2, 7))[turn]]
        x = s.drafts(trees)
        if turn in (1, 3):  # a selection serves until the next one, tokens of the turns between count too
            s.s.select(x.q[[int(c) for c in x.cu[:-1]]].contiguous())
        out = x.step()
        torch.cuda.synchronize()
        want_pos = [n + d for n, t in zip(s.lens, trees) for d in ancestors(t)[1]]
        assert x.pos.tolist() == want_pos
        s.expect(trees, x.qr, x.kr, x.v, want_pos, turn > 0).check(out, x.lse)
        paths = [_path(t, s.g) for t in trees]
        if turn == 1:
            paths[0] = []  # nothing of one tree
        rows = torch.tensor([int(x.cu[b]) + j for b, p in enumerate(paths) for j in p], device=DEV)
        s.grow([len(p) for p in paths], x.kr[rows], x.v[rows])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_over_quantised_pages(dtype, bits):
    s = Server(2, dtype, False, seed=3, bits=bits)
    s.grow([210, 64])
    for turn in range(3):
        trees = [random_tree(n, s.g) for n in ((12, 5), (3, 40), (1, 30))[turn]]
        x = s.drafts(trees)
        if turn == 1:
            s.s.select(x.q[[int(c) for c in x.cu[:-1]]].contiguous())
        out = x.step()
        torch.cuda.synchronize()
        s.expect(trees, x.qr, x.kr, x.v, x.pos.tolist(), turn > 0).check(out, x.lse)
        paths = [_path(t, s.g) for t in trees]
        rows = torch.tensor([int(x.cu[b]) + j for b, p in enumerate(paths) for j in p], device=DEV)
        s.grow([len(p) for p in paths], x.kr[rows], x.v[rows])


def test_a_step_over_drafts_captured_and_replayed():
    """Each graph keeps its own workspace; the session's eager steps between the replays do not disturb it."""
    s = Server(2, torch.float16, False, seed=1)
    s.L.lserve_init()
    s.grow([500, 90])
    steps = [s.drafts([random_tree(n, s.g) for n in sizes]) for sizes in ((20, 40), (3, 1))]
    want = [x.step().clone() for x in steps]
    torch.cuda.synchronize()
    graphs = []
    for x in steps:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = x.step()
        graphs.append((graph, out))
    for _ in range(3):
        for (graph, out), w in zip(graphs, want):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, w)
        for x, w in zip(steps, want):
            assert torch.equal(x.step(), w)
        torch.cuda.synchronize()


def test_a_chain_of_drafts_without_a_mask():
    s = Server(2, torch.bfloat16, True, seed=2)
    s.grow([130, 1])
    chains = [list(range(-1, n - 1)) for n in (6, 3)]
    x = s.drafts(chains)
    tree = x.step()
    chain = s.s.decode_tree(x.qr, x.kr, x.v, x.cu, x.most)
    torch.cuda.synchronize()
    s.expect(chains, x.qr, x.kr, x.v, x.pos.tolist(), False).check(tree, x.lse)
    assert torch.equal(chain, tree)
