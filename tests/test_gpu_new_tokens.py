"""Page tables, positions and slots of new tokens, and the ancestors of drafted ones, against plain loops: whole numbers, all equal."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _lib():
    import paper_2502_14866_amd as L

    L.load_library()
    return L


def _extend(lens, new, page=64, width=None, num_free=None, pad=0, sink=128, local=512, seed=0, want=("positions", "slots", "ring_slots"),
            call=None):
    """(outputs of the call, outputs of the loops)."""
    L = _lib()
    g = torch.Generator().manual_seed(seed)
    batch = len(lens)
    had = [-(-n // page) for n in lens]
    will = [-(-(n + max(m, 0)) // page) for n, m in zip(lens, new)]
    width = width or max(will + [1])
    need = sum(min(w, width) - min(h, width) for h, w in zip(had, will))
    num_free = need + 3 if num_free is None else num_free
    table = torch.full((batch, width), -7, dtype=torch.int32)
    ids = torch.randperm(batch * width + num_free + 1, generator=g).to(torch.int32)
    for b, h in enumerate(had):
        table[b, :min(h, width)] = ids[b * width:b * width + min(h, width)]
    free = ids[batch * width:batch * width + num_free].clone()
    s, w = -(-sink // page), -(-local // page)
    ring = torch.randperm(batch * (s + w), generator=g).to(torch.int32).view(batch, s + w)
    total = sum(max(m, 0) for m in new)
    desc = L.AttnDesc(4, 2, [1, 0], page_size=page, logical_page_size=16, sink_tokens=sink, local_tokens=local)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    kv = L.PagedKV(None, None, None, table.to(DEV), i32(lens + [0])[:batch], ring_table=ring.to(DEV))
    out = {"cu": i32([-9] * (batch + 1)), "lens": i32([-9] * batch), "taken": i32([-9]),
           "positions": torch.full((total + pad,), -9, dtype=torch.int32, device=DEV),
           "slots": torch.full((total + pad,), -9, dtype=torch.int64, device=DEV),
           "ring_slots": torch.full((total + pad,), -9, dtype=torch.int64, device=DEV)}
    args = [desc, kv, i32(new), free.to(DEV) if num_free else None, out["cu"], out["lens"], out["taken"]]
    kw = {k: out[k] for k in want}
    (call or (lambda f: f()))(lambda: L.lserve_extend_tables(*args, total_new=total + pad, **kw))
    torch.cuda.synchronize()
    ref = {"cu": [0], "lens": [], "positions": [], "slots": [], "ring_slots": []}
    ref_table, taken = table.clone(), 0
    for b, (n, m) in enumerate(zip(lens, new)):
        m = max(m, 0)
        for p in range(min(had[b], width), min(will[b], width)):
            ref_table[b, p] = free[taken] if taken < num_free else -1
            taken += 1
        for t in range(n, n + m):
            p = t // page
            phys = int(ref_table[b, p]) if p < width else -1
            ref["positions"].append(t)
            ref["slots"].append(phys * page + t % page if phys >= 0 else -1)
            here = p < s or p > will[b] - 1 - w
            ref["ring_slots"].append(int(ring[b, p if p < s else s + (p - s) % w]) * page + t % page if here else -1)
        ref["cu"].append(ref["cu"][-1] + m)
        ref["lens"].append(n + m)
    for k in ("positions", "slots", "ring_slots"):
        ref[k] = ref[k] + [-1] * pad if k in want else [-9] * (total + pad)
    ref["taken"] = [taken]
    got = {k: v.tolist() for k, v in out.items()}
    got["table"], ref["table"] = kv.page_table.tolist(), ref_table.tolist()
    return got, ref


def _same(got_ref):
    got, ref = got_ref
    for k in ref:
        assert got[k] == ref[k], k


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("lens,new", [
    ([0], [1]), ([0], [0]), ([64], [1]), ([63, 64, 65], [1, 1, 1]), ([0, 5, 700], [1000, 0, 129]), ([127, 1, 640, 3], [0, 0, 0, 5000]),
    ([5] * 70, [1] * 70), (list(range(300)), [(7 * i) % 11 for i in range(300)]), ([3], [1023]), ([3], [1024]), ([3], [1025]),
])
def test_new_tokens_of_a_batch(page, lens, new):
    _same(_extend(lens, new, page=page, pad=5))


def test_large_batches():
    lens = [(i * 7919) % 3000 for i in range(5000)]
    _same(_extend(lens, [1] * 5000))
    _same(_extend(lens, [(i * 31) % 40 if i % 5 else 0 for i in range(5000)], seed=1))


def test_nothing_to_read_behind_the_lists():
    """A free list that ends early, or is empty, a table that is too narrow, lengths below zero."""
    _same(_extend([100, 64, 300], [500, 64, 70], num_free=4))
    _same(_extend([100, 64, 300], [500, 64, 70], num_free=0))
    _same(_extend([100, 64, 300], [500, 64, 70], width=3))
    _same(_extend([64, 64], [-5, 10], pad=3))


def test_the_rest_of_a_free_list():
    L = _lib()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    pool = i32(list(range(100, 120)))
    for used in (1, 2, 7):
        kv = L.PagedKV(None, None, None, i32([[0, -7, -7], [1, -7, -7]]), i32([64, 62]))
        cu, lens, taken, slots = i32([0, 0, 0]), i32([0, 0]), i32([0]), torch.zeros(5, dtype=torch.int64, device=DEV)
        L.lserve_extend_tables(L.AttnDesc(4, 2, [1, 0]), kv, i32([1, 4]), pool[used:], cu, lens, taken, slots=slots)
        torch.cuda.synchronize()
        p = 100 + used
        assert kv.page_table.tolist() == [[0, p, -7], [1, p + 1, -7]]
        assert slots.tolist() == [p * 64, 64 + 62, 64 + 63, (p + 1) * 64, (p + 1) * 64 + 1]


def test_outputs_that_are_not_wanted():
    _same(_extend([100, 64, 300], [500, 64, 70], want=()))
    _same(_extend([100, 64, 300], [500, 64, 70], want=("slots",)))
    _same(_extend([100, 64, 300], [500, 64, 70], want=("positions",), pad=2))


def test_lengths_past_32_bits_stay_inside_the_arrays():
    """2^31 - 10 tokens and twenty more: no page of the table is that far out."""
    L = _lib()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    kv = L.PagedKV(None, None, None, i32([[5, 6], [7, 8]]), i32([2 ** 31 - 10, 64]), ring_table=torch.zeros((2, 10), dtype=torch.int32, device=DEV))
    slots, ring = torch.zeros(24, dtype=torch.int64, device=DEV), torch.zeros(24, dtype=torch.int64, device=DEV)
    cu, lens, taken = i32([0, 0, 0]), i32([0, 0]), i32([0])
    L.lserve_extend_tables(L.AttnDesc(4, 2, [1, 0]), kv, i32([20, 4]), i32([9]), cu, lens, taken, slots=slots, ring_slots=ring)
    torch.cuda.synchronize()
    assert kv.page_table.tolist() == [[5, 6], [7, 9]] and taken.tolist() == [1] and cu.tolist() == [0, 20, 24]
    assert slots.tolist() == [-1] * 20 + [9 * 64 + i for i in range(4)]


def test_captured_and_replayed():
    """The lengths of the replay are those in memory then; the table grows as they do."""
    L = _lib()
    L.lserve_init()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    kv = L.PagedKV(None, None, None, i32([[0, -7, -7], [1, -7, -7]]), i32([63, 62]))
    new, free, cu, lens, taken = i32([1, 1]), i32([4, 5, 6]), i32([0, 0, 0]), i32([0, 0]), i32([0])
    pos, slots = i32([0, 0]), torch.zeros(2, dtype=torch.int64, device=DEV)
    desc, graph = L.AttnDesc(4, 2, [1, 0]), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        L.lserve_extend_tables(desc, kv, new, free, cu, lens, taken, pos, slots)
    seen = []
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        seen.append((lens.tolist(), taken.tolist(), slots.tolist()))
        kv.seq_lens.copy_(lens)
    assert seen == [([64, 63], [0], [63, 64 + 62]), ([65, 64], [1], [4 * 64, 64 + 63]), ([66, 65], [1], [4 * 64 + 1, 4 * 64])]


def _trees(parents_of, lens, words=None, pad=0, most=None):
    L = _lib()
    counts = [len(p) for p in parents_of]
    total, most = sum(counts), most or max(counts)
    words = words or -(-most // 64)
    flat = [p for ps in parents_of for p in ps] + [0] * pad
    cu = [0]
    for c in counts:
        cu.append(cu[-1] + c)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    mask = torch.full((total + pad, words), 77, dtype=torch.int64, device=DEV)
    pos = torch.full((total + pad,), -9, dtype=torch.int32, device=DEV)
    L.lserve_tree_masks(i32(flat), i32(cu), i32(lens), most, mask, pos)
    torch.cuda.synchronize()
    rows, positions = [], []
    for ps, n in zip(parents_of, lens):
        sets, deep = [], []
        for j, p in enumerate(ps):
            p = p if 0 <= p < j else -1
            sets.append((sets[p] if p >= 0 else 0) | 1 << j)
            deep.append(deep[p] + 1 if p >= 0 else 0)
        for x, d in zip(sets, deep):
            row = [(x >> 64 * w) & (2 ** 64 - 1) for w in range(words)]
            rows.append([r - 2 ** 64 if r >= 2 ** 63 else r for r in row])
            positions.append(n + d)
    rows += [[77] * words] * pad
    assert mask.tolist() == rows
    assert pos.tolist() == positions + [-9] * pad


def _random_tree(n, seed):
    g = torch.Generator().manual_seed(seed)
    return [int(torch.randint(-1, j, (1,), generator=g)) if j else -1 for j in range(n)]


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 128, 200, 256, 257, 700, 1024])
def test_ancestors(n):
    _trees([_random_tree(n, n)], [100])
    _trees([list(range(-1, n - 1))], [0])        # a chain
    _trees([[-1] * n], [5])                      # n alternatives to one another


def test_ancestors_of_a_ragged_batch():
    sizes = [5, 0, 1, 64, 17, 0, 33]
    _trees([_random_tree(n, i) for i, n in enumerate(sizes)], [10 * i for i in range(7)], pad=3)
    _trees([_random_tree(n, i) for i, n in enumerate(sizes)], [10 * i for i in range(7)], words=5)
    _trees([_random_tree(n, i) for i, n in enumerate([300, 2, 0, 90])], [1, 2, 3, 4], pad=1)


def test_parents_that_are_none():
    _trees([[-1, 5, -3, 3, 0, 1000, 2 ** 31 - 1, -2 ** 31, 7]], [3])
