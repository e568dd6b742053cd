"""Operators around the sparse attention path whose speed counts: what a serving layer needs in front of a decode, draft or
prefill step, and the attention that reads a tree of drafted tokens over the cache.

A case is a dict of plain values.  Its `kind` says which operator it is:

  tables  new tokens of a batch: pages off the free list, page table, running counts, positions, slots (lserve_extend_tables)
  masks   ancestors and positions of drafted tokens from their parents (lserve_tree_masks)
  rotary  rotary positions of queries and keys (lserve_rotary)
  tree    attention of a tree of drafted tokens over the paged cache and over each other (lserve_sparse_decode_tree)

Half of the KV heads stream (128 sink and 512 local tokens), the others attend the pages a selection lists or all of them.
With `own` false `run` computes the plain forms with elementary torch operations, otherwise it calls the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D = 128
PAGE = 64
SINK, LOCAL = 128, 512
RING = SINK // PAGE + LOCAL // PAGE


def _case(name, kind, **kw):
    case = {"name": name, "kind": kind, "dtype": "fp16", "q_heads": 32, "kv_heads": 8, "batch": 1, "shortest": 0, "longest": 0}
    if kind == "tables":
        # new tokens per sequence go from `new_least` to `new_most`; `scarce`: the free list is a little too short
        case.update(page=PAGE, new_least=1, new_most=1, scarce=False)
    elif kind == "masks":
        case.update(nodes=1, nodes_least=0, chain=False)
    elif kind == "rotary":
        case.update(tokens=1, rotary=D, interleaved=False, scaling="none", fused=False, far=8192)
    else:
        case.update(nodes=1, nodes_least=0, chain=False, budget=0, kv_bits=16, two_way=False)
    case.update(kw)
    if not case["shortest"]:
        case["shortest"] = case["longest"]
    if "nodes" in case and not case["nodes_least"]:
        case["nodes_least"] = case["nodes"]
    if not name:
        del case["name"]
    return case


def listed():
    return [
        # one decode step of a full serving batch: a token each, a new page now and then; latency is all there is
        _case("tables_step_64", "tables", batch=64, shortest=9001, longest=24011),
        # a scheduler admits 500 prompts of all lengths in one go
        _case("tables_prompts_500", "tables", batch=500, shortest=1, longest=700, new_least=16, new_most=8192),
        # drafted trees of 32 tokens for the benchmark's batch
        _case("masks_16x32", "masks", batch=16, nodes=32, longest=32768),
        # wide trees of a large batch
        _case("masks_256x200", "masks", batch=256, nodes=200, nodes_least=9, shortest=300, longest=16000),
        # one decode step of the benchmark's batch
        _case("rotary_step_16", "rotary", tokens=16, far=32768),
        # the queries and keys of a ragged prefill batch, as they come out of one fused projection; half of a head's channels turn
        _case("rotary_part_9k", "rotary", dtype="bf16", tokens=9217, rotary=64, interleaved=True, fused=True),
        # the longest prompt of the benchmark, positions stretched over a long context
        _case("rotary_prompt_64k", "rotary", dtype="bf16", tokens=65536, scaling="wavelength", far=65536),
        # one user, a short conversation, a small tree: latency and launches count
        _case("tree_1x4k", "tree", batch=1, nodes=8, longest=4000),
        # the benchmark's batch at 32K context over selected pages, sixteen drafted tokens each
        _case("tree_16x32k", "tree", batch=16, nodes=16, longest=32768, budget=4096),
        # few users with very long documents, a short chain of drafted tokens, dense heads over everything
        _case("tree_4x256k", "tree", dtype="bf16", batch=4, nodes=5, longest=262144, chain=True),
        # a ragged batch of a model without grouped queries, trees of all sizes
        _case("tree_mha_32_ragged", "tree", batch=32, kv_heads=32, nodes=24, nodes_least=1, shortest=4096, longest=60000, budget=2048),
        # a full serving batch over 4-bit pages, streaming heads in their bounded cache, large trees
        _case("tree_kv4_64x16k", "tree", dtype="bf16", batch=64, nodes=64, nodes_least=20, shortest=5001, longest=16011, budget=4096,
              kv_bits=4, two_way=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["tables", "masks", "rotary", "tree"], [3, 2, 4, 7])[0]
    kw = {"dtype": rng.choice(["fp16", "bf16"])}
    kw["q_heads"], kw["kv_heads"] = rng.choice([(32, 8), (32, 8), (32, 32), (8, 2), (64, 8), (32, 16)])
    if kind == "tables":
        kw["batch"] = _log(rng, 1, 2000)
        kw["longest"] = _log(rng, 1, 30000)
        kw["shortest"] = max(1, kw["longest"] // rng.randint(1, 40))
        kw["new_most"] = rng.choice([1, _log(rng, 1, max(2, 1000000 // kw["batch"]))])
        kw["new_least"] = rng.choice([0, kw["new_most"], max(1, kw["new_most"] // 30)])
        kw["page"] = rng.choice([64, 64, 16, 32, 128])
        kw["scarce"] = rng.random() < 0.2
    elif kind == "masks":
        kw["batch"] = _log(rng, 1, 256)
        kw["nodes"] = _log(rng, 1, 200)
        kw["nodes_least"] = rng.choice([0, max(1, kw["nodes"] // rng.randint(2, 20))])
        kw["chain"] = rng.random() < 0.3
        kw["longest"] = _log(rng, 1, 200000)
    elif kind == "rotary":
        kw["tokens"] = _log(rng, 1, 65536 * 40 // (kw["q_heads"] + kw["kv_heads"]))
        kw["rotary"] = rng.choice([128, 128, 128, 64, 32, 96, 20])
        kw["interleaved"] = rng.random() < 0.4
        kw["scaling"] = rng.choice(["none", "linear", "wavelength", "ramp"])
        kw["fused"] = rng.random() < 0.5
        kw["far"] = _log(rng, 1000, 1000000)
    else:
        kw["batch"] = _log(rng, 1, 64)
        kw["nodes"] = _log(rng, 1, 64)
        kw["nodes_least"] = rng.choice([0, max(1, kw["nodes"] // rng.randint(2, 20))])
        top = min(262144, (5 << 20) // (kw["batch"] * kw["kv_heads"]), (1 << 28) // (kw["batch"] * kw["q_heads"] * kw["nodes"]))
        kw["longest"] = _log(rng, 100, max(200, top))
        kw["shortest"] = rng.choice([0, max(1, kw["longest"] // rng.randint(2, 30))])
        kw["chain"] = rng.random() < 0.3
        kw["kv_bits"] = rng.choice([16, 16, 8, 4])
        kw["two_way"] = rng.random() < 0.4
        kw["budget"] = rng.choice([0, 64 * _log(rng, 4, 96)])
    return _case("", kind, **kw)


# ---- inputs ------------------------------------------------------------------------------------------------------


def _gen(seed, *which):
    x = seed & 0xFFFFFFFF
    for w in which:
        x = (x * 1000003 + w + 12345) & 0x7FFFFFFFFFFF
    g = torch.Generator(device="cuda")
    g.manual_seed(x)
    return g


def _spread(n, lo, hi, turn=0.6180339887498949):
    """n whole numbers from lo to hi, spread over their logarithm (zero counts as such), the largest first."""
    lo1, hi1 = math.log(max(lo, 0.5)), math.log(max(hi, 0.5))
    return [hi] + [int(round(math.exp(lo1 + ((i * turn) % 1.0) * (hi1 - lo1)))) if hi > lo else lo for i in range(1, n)]


def _lengths(case):
    return _spread(case["batch"], case["shortest"], case["longest"])


def _counts(case):
    """New tokens of every sequence."""
    if case["kind"] == "tables":
        return _spread(case["batch"], case["new_least"], case["new_most"], 0.7548776662466927)
    return _spread(case["batch"], case["nodes_least"], case["nodes"], 0.7548776662466927)


def _dtype(case):
    return torch.float16 if case["dtype"] == "fp16" else torch.bfloat16


def _int32(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _cu(counts):
    return [0] + np.cumsum(counts).tolist()


def _rows(gen, dtype, shape):
    """N(0, 1), made in pieces."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for r in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - r)
        flat[r:r + n] = torch.randn((n,), generator=gen, device="cuda")
    return out


def _quantise(x, bits):
    """Rows [.., 64, D] as quantised pages [.., 64 D bits / 8 + 256]: codes, then (scale, zero) of every row in fp16."""
    top = 2 ** bits - 1
    zero = x.amin(-1, keepdim=True).half()
    scale = ((x.amax(-1, keepdim=True) - zero.float()) / top).half()
    code = ((x - zero.float()) / scale.float()).round().clamp(0, top).to(torch.uint8)
    if bits == 4:  # byte j of word g: channel 8 g + j in the low half, 8 g + 4 + j in the high one
        code = code.unflatten(-1, (D // 8, 2, 4))
        code = code[..., 0, :] | code[..., 1, :] << 4
    tail = torch.cat([scale, zero], -1).contiguous().view(torch.uint8)
    return torch.cat([code.flatten(-2 if bits == 8 else -3), tail.flatten(-2)], -1)


def _pool(case, gen, pages, heads):
    shape = (pages, heads, PAGE, D)
    if case["kv_bits"] == 16:
        return _rows(gen, _dtype(case), shape)
    out = torch.empty((pages, heads, PAGE * D * case["kv_bits"] // 8 + 256), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // (heads * PAGE * D))
    for r in range(0, pages, step):
        n = min(step, pages - r)
        out[r:r + n] = _quantise(torch.randn((n,) + shape[1:], generator=gen, device="cuda"), case["kv_bits"])
    return out


def _parents(case, seed, counts):
    """Parents of the drafted tokens of all sequences: a chain, or children of earlier tokens, most of them shallow."""
    total, cu = sum(counts), _cu(counts)
    index = torch.arange(total, device="cuda") - torch.repeat_interleave(
        torch.tensor(cu[:-1], device="cuda"), torch.tensor(counts, device="cuda"))
    if case["chain"]:
        return (index - 1).to(torch.int32)
    u = torch.rand((total,), generator=_gen(seed, 5), device="cuda")
    return torch.minimum((u * u * (index + 1)).floor().long() - 1, index - 1).to(torch.int32)


def _tables(case, seed, page, pages, slack=2):
    """Page tables [batch][most pages] with pages of a shared pool in random order (-1 behind them), and the pages left."""
    used = sum(pages)
    order = torch.randperm(used + slack + 1000, generator=_gen(seed, 3), device="cuda").to(torch.int32)  # others hold the rest
    table = torch.full((len(pages), max(1, max(pages))), -1, dtype=torch.int32, device="cuda")
    keep = torch.arange(table.shape[1], device="cuda")[None, :] < torch.tensor(pages, device="cuda")[:, None]
    table[keep] = order[:used]
    return table, order[used:used + slack].contiguous()


def _prepare_tables(case, seed):
    lens, new, page = _lengths(case), _counts(case), case["page"]
    old = [-(-n // page) for n in lens]
    need = sum(-(-(n + m) // page) - o for n, m, o in zip(lens, new, old))
    table, free = _tables(case, seed, page, old, need if case["scarce"] else need + 7)
    if case["scarce"] and need > 0:
        free = free[:max(1, need * 3 // 4)].contiguous()
    width = max(-(-(n + m) // page) for n, m in zip(lens, new)) + 1
    wide = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    ring = SINK // page + LOCAL // page
    total = max(1, sum(new))
    i32 = lambda n: torch.empty((n,), dtype=torch.int32, device="cuda")  # noqa: E731
    i64 = lambda n: torch.empty((n,), dtype=torch.int64, device="cuda")  # noqa: E731
    return {"case": case, "lens": _int32(lens), "new": _int32(new), "table": wide, "free": free, "total": total,
            "ring": torch.randperm(len(lens) * ring, generator=_gen(seed, 4), device="cuda").to(torch.int32).view(len(lens), ring),
            "out": {"cu": i32(len(lens) + 1), "lens": i32(len(lens)), "positions": i32(total), "slots": i64(total),
                    "ring_slots": i64(total), "taken": i32(1)}}


def _lengths_now(case, seed):
    """Lengths that moved on by some tokens since the batch was put together."""
    return _int32(_lengths(case)) + torch.randint(0, 1000, (case["batch"],), generator=_gen(seed, 6), device="cuda").to(torch.int32)


def _prepare_masks(case, seed):
    counts = _counts(case)
    words = -(-case["nodes"] // 64)
    return {"case": case, "parents": _parents(case, seed, counts), "cu": _int32(_cu(counts)), "lens": _lengths_now(case, seed),
            "most": case["nodes"],
            "out": {"mask": torch.empty((sum(counts), words), dtype=torch.int64, device="cuda"),
                    "positions": torch.empty((sum(counts),), dtype=torch.int32, device="cuda")}}


def _prepare_rotary(case, seed):
    n, hq, hkv, dt = case["tokens"], case["q_heads"], case["kv_heads"], _dtype(case)
    if case["fused"]:  # rows of one projection: queries, keys, values
        rows = _rows(_gen(seed, 1), dt, (n, (hq + 2 * hkv) * D))
        q, k = rows[:, :hq * D].view(n, hq, D), rows[:, hq * D:(hq + hkv) * D].view(n, hkv, D)
    else:
        q, k = _rows(_gen(seed, 1), dt, (n, hq, D)), _rows(_gen(seed, 2), dt, (n, hkv, D))
    if n <= 256:  # one token of each of many sequences
        positions = torch.randint(0, case["far"], (n,), generator=_gen(seed, 3), device="cuda").to(torch.int32)
    else:  # a few prompts
        step = -(-n // 3)
        positions = ((torch.arange(n, device="cuda") % step) * max(1, case["far"] // step)).to(torch.int32)
    return {"case": case, "q": q, "k": k, "positions": positions,
            "out": {"q": torch.empty((n, hq, D), dtype=dt, device="cuda"), "k": torch.empty((n, hkv, D), dtype=dt, device="cuda")}}


def _selection(case, seed, lens):
    """A selection a few tokens old: the newest page and random others, ascending."""
    K, hkv = case["budget"] // PAGE, case["kv_heads"]
    at = [max(1, n - 3) for n in lens]
    pages = _int32([-(-n // PAGE) for n in at])
    most = -(-max(at) // PAGE)
    score = torch.rand((len(lens), hkv, most), generator=_gen(seed, 7), device="cuda")
    index = torch.arange(most, device="cuda")
    score = torch.where(index == pages[:, None, None] - 1, 2.0, score).masked_fill(index >= pages[:, None, None], -1.0)
    best = score.topk(min(K, most), -1).indices
    count = torch.clamp(pages, max=K)[:, None].expand(-1, hkv)
    best = torch.where(torch.arange(best.shape[-1], device="cuda") < count[..., None], best, most + 1).sort(-1).values
    sel = torch.full((len(lens), hkv, K), -1, dtype=torch.int32, device="cuda")
    sel[..., :best.shape[-1]] = torch.where(best > most, -1, best).to(torch.int32)
    return {"pages": sel, "count": count.to(torch.int32).contiguous(), "lens": _int32(at)}


def _ancestors(parents, counts):
    """(mask words as whole numbers per token, depth) from the parents, on the host."""
    out, depth, at = [], [], 0
    parents = parents.tolist()
    for n in counts:
        bits, deep = [], []
        for j in range(n):
            p = parents[at + j]
            bits.append((bits[p] if p >= 0 else 0) | 1 << j)
            deep.append(deep[p] + 1 if p >= 0 else 0)
        out += bits
        depth += deep
        at += n
    return out, depth


def _prepare_tree(case, seed):
    lens, counts, hq, hkv, dt = _lengths(case), _counts(case), case["q_heads"], case["kv_heads"], _dtype(case)
    total, words, n_stream = sum(counts), -(-case["nodes"] // 64), hkv // 2
    table, _ = _tables(case, seed, PAGE, [-(-n // PAGE) for n in lens], 0)
    table = table.clamp(min=0)
    pages, main = int(table.max()) + 1, hkv - n_stream if case["two_way"] else hkv
    pools = {"k": _pool(case, _gen(seed, 11), pages, main), "v": _pool(case, _gen(seed, 12), pages, main), "ks": None, "vs": None, "ring": None}
    if case["two_way"]:
        n = len(lens) * RING
        pools["ks"], pools["vs"] = _pool(case, _gen(seed, 13), n, n_stream), _pool(case, _gen(seed, 14), n, n_stream)
        pools["ring"] = torch.randperm(n, generator=_gen(seed, 4), device="cuda").to(torch.int32).view(len(lens), RING)
    bits, depth = _ancestors(_parents(case, seed, counts), counts)
    mask = [[(b >> 64 * w & (1 << 64) - 1) - (1 << 64) * (b >> 64 * w + 63 & 1) for w in range(words)] for b in bits]
    at = torch.repeat_interleave(torch.tensor(lens), torch.tensor(counts))
    return {"case": case, "pools": pools, "table": table, "lens": _int32(lens), "cu": _int32(_cu(counts)), "most": case["nodes"],
            "q": _rows(_gen(seed, 21), dt, (total, hq, D)), "k": _rows(_gen(seed, 22), dt, (total, hkv, D)),
            "v": _rows(_gen(seed, 23), dt, (total, hkv, D)), "mask": torch.tensor(mask, dtype=torch.int64, device="cuda"),
            "positions": (at + torch.tensor(depth)).to(torch.int32).cuda(),
            "sel": _selection(case, seed, lens) if case["budget"] else None,
            "out": {"out": torch.empty((total, hq, D), dtype=dt, device="cuda"),
                    "lse": torch.empty((total, hq), dtype=torch.float32, device="cuda")}}


def prepare(case, seed):
    return {"tables": _prepare_tables, "masks": _prepare_masks, "rotary": _prepare_rotary, "tree": _prepare_tree}[case["kind"]](case, seed)


# ---- the library's calls -------------------------------------------------------------------------------------------


def _flags(case):
    half = case["kv_heads"] // 2
    return [1] * half + [0] * (case["kv_heads"] - half)


def _handles(state):
    """Descriptions and workspace, made once as a program keeps them."""
    if "handles" not in state:
        import paper_2502_14866_amd as L

        case = state["case"]
        h = state["handles"] = {"L": L, "desc": L.AttnDesc(
            case["q_heads"], case["kv_heads"], _flags(case), page_size=case.get("page", PAGE), logical_page_size=16,
            dtype=_dtype(case), sink_tokens=SINK, local_tokens=LOCAL)}
        if case["kind"] == "tables":
            h["kv"] = L.PagedKV(None, None, None, state["table"], state["lens"], ring_table=state["ring"])
        elif case["kind"] == "rotary":
            h["rotary"] = L.RotaryDesc(rotary_dim=case["rotary"], interleaved=case["interleaved"], base=BASE, **SCALING[case["scaling"]])
        elif case["kind"] == "tree":
            p, main = state["pools"], state["pools"]["k"].shape[1]
            h["kv"] = L.PagedKV(p["k"], p["v"], None, state["table"], state["lens"], pool_heads=0 if main == case["kv_heads"] else main,
                                k_pool_stream=p["ks"], v_pool_stream=p["vs"], ring_table=p["ring"], kv_bits=case["kv_bits"])
            need = L.lserve_tree_workspace_bytes(h["desc"], case["batch"], state["q"].shape[0], state["most"], state["table"].shape[1],
                                                 case["budget"] // PAGE)
            h["workspace"] = torch.zeros((max(16, need),), dtype=torch.uint8, device="cuda")
    return state["handles"]


def _run_own(state):
    h, out = _handles(state), state["out"]
    L, kind = h["L"], state["case"]["kind"]
    if kind == "tables":
        L.lserve_extend_tables(h["desc"], h["kv"], state["new"], state["free"], out["cu"], out["lens"], out["taken"], out["positions"],
                               out["slots"], out["ring_slots"])
        return dict(out, table=state["table"])
    if kind == "masks":
        L.lserve_tree_masks(state["parents"], state["cu"], state["lens"], state["most"], out["mask"], out["positions"])
    elif kind == "rotary":
        L.lserve_rotary(h["desc"], h["rotary"], state["q"], state["k"], state["positions"], out["q"], out["k"])
    else:
        sel = state["sel"] or {"pages": None, "count": None, "lens": None}
        L.lserve_sparse_decode_tree(h["desc"], h["kv"], state["q"], state["k"], state["v"], state["cu"], state["most"], out["out"],
                                    out["lse"], tree_mask=state["mask"], positions=state["positions"], sel_pages=sel["pages"],
                                    sel_count=sel["count"], sel_seq_len=sel["lens"], workspace=h["workspace"])
    return out


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _plain_tables(state):
    page, lens, new, free, total = state["case"]["page"], state["lens"].long(), state["new"].long(), state["free"], state["total"]
    table = state["table"].clone()
    batch, width = table.shape
    cu = torch.cat([torch.zeros_like(new[:1]), new.cumsum(0)])
    had, will = (lens + page - 1) // page, (lens + new + page - 1) // page
    first = (will - had).cumsum(0) - (will - had)  # pages handed out to sequences before
    p = torch.arange(width, device="cuda")
    fresh = (p >= had[:, None]) & (p < will[:, None])
    index = first[:, None] + p - had[:, None]
    table = torch.where(fresh, torch.where(index < len(free), free[index.clamp(0, len(free) - 1)], -1), table)
    t = torch.arange(total, device="cuda")
    b = (torch.searchsorted(cu, t, right=True) - 1).clamp(max=batch - 1)
    held = t < cu[-1]
    pos = lens[b] + t - cu[b]
    pg = (pos // page).clamp(max=width - 1)
    phys = table[b, pg].long()
    slots = torch.where(held & (phys >= 0), phys * page + pos % page, -1)
    s, w = SINK // page, LOCAL // page
    slot = torch.where(pg < s, pg, s + (pg - s) % w)
    stays = (pg < s) | (pg > will[b] - 1 - w)
    ring = torch.where(held & stays, state["ring"][b, slot].long() * page + pos % page, -1)
    return {"cu": cu.int(), "lens": (lens + new).int(), "positions": torch.where(held, pos, -1).int(), "slots": slots,
            "ring_slots": ring, "taken": (will - had).sum(0, keepdim=True).int(), "table": table}


def _padded(cu, total, most):
    """Of every row its sequence and index, and the rows [batch][most] of the sequences (clamped) with who of them exists."""
    t = torch.arange(total, device="cuda")
    b = torch.searchsorted(cu, t, right=True) - 1
    j = torch.arange(most, device="cuda")
    return b, t - cu[b], (cu[:-1, None] + j).clamp(max=total - 1), j < (cu[1:] - cu[:-1])[:, None]


def _plain_masks(state):
    parents, cu, most = state["parents"].long(), state["cu"].long(), state["most"]
    b, j, rows, there = _padded(cu, len(parents), most)
    up = (parents[rows][:, :, None] == torch.arange(most, device="cuda")) & there[:, :, None]
    step = up.float()
    reach = step + torch.eye(most, device="cuda")
    for _ in range(max(1, (most - 1).bit_length())):  # paths of up to twice the length
        step = step @ step
        reach = reach + step @ reach
    words = state["out"]["mask"].shape[1]
    bits = torch.nn.functional.pad(reach.round().long(), (0, 64 * words - most)).unflatten(-1, (words, 64))
    mask = (bits << torch.arange(64, device="cuda")).sum(-1)
    depth = reach.sum(-1).round().long() - 1
    return {"mask": mask[b, j], "positions": (state["lens"].long()[b] + depth[b, j]).int()}


BASE = 500000.0
SCALING = {
    "none": {"scaling": "none"},
    "linear": {"scaling": "linear", "factor": 4.0},
    "wavelength": {"scaling": "wavelength", "factor": 8.0, "original_positions": 8192.0, "low": 1.0, "high": 4.0},
    "ramp": {"scaling": "ramp", "factor": 16.0, "original_positions": 4096.0, "low": 1.0, "high": 32.0},
}


def _frequencies(case):
    """(radians per position and pair, factor on the result) in 64 bits."""
    R, sc = case["rotary"], SCALING[case["scaling"]]
    i = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    f = BASE ** (-2 * i / R)
    kind, factor = sc["scaling"], sc.get("factor", 1.0)
    if kind == "linear":
        return f / factor, 1.0
    if kind == "wavelength":
        # turns over the original context: at most `low` of them: stretched, `high` or more: as they are, mixed between
        turns = sc["original_positions"] * f / (2 * math.pi)
        mix = ((turns - sc["low"]) / (sc["high"] - sc["low"])).clamp(0, 1)
        return f / factor * (1 - mix) + f * mix, 1.0
    if kind == "ramp":
        # the same idea, a ramp over the pairs' index between those of `high` and `low` turns, and a louder result
        at = lambda turns: R * math.log(sc["original_positions"] / (turns * 2 * math.pi)) / (2 * math.log(BASE))  # noqa: E731
        lo, hi = max(0, math.floor(at(sc["high"]))), min(R - 1, math.ceil(at(sc["low"])))
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f / factor * ramp + f * (1 - ramp), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _plain_rotary(state):
    case = state["case"]
    R = case["rotary"]
    f, loud = _frequencies(case)
    angle = state["positions"].double()[:, None] * f
    cos, sin = (angle.cos() * loud).float()[:, None], (angle.sin() * loud).float()[:, None]

    def turn(x):
        y = x.float()
        if case["interleaved"]:
            a, b = y[..., 0:R:2], y[..., 1:R:2]
            r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = y[..., :R // 2], y[..., R // 2:R]
            r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([r, y[..., R:]], -1).to(x.dtype)

    return {"q": turn(state["q"]), "k": turn(state["k"])}


def _unpacked(case, pages):
    """Rows [.., 64, D] that gathered pages stand for, in 32 bits."""
    bits = case["kv_bits"]
    if bits == 16:
        return pages.float()
    code, tail = pages[..., :PAGE * D * bits // 8], pages[..., PAGE * D * bits // 8:].contiguous().view(torch.float16).float()
    code = code.unflatten(-1, (PAGE, D * bits // 8))
    if bits == 4:
        code = code.unflatten(-1, (D // 8, 1, 4))
        code = torch.cat([code & 15, code >> 4], -2).flatten(-3)
    tail = tail.unflatten(-1, (PAGE, 2))
    return code.float() * tail[..., :1] + tail[..., 1:]


def _history(state, which):
    """[batch][Hkv][pages * 64][D] of the cached keys or values, rows past the length zero."""
    case, p, table = state["case"], state["pools"], state["table"].long()
    x = _unpacked(case, p[which][table])  # [batch][pages][heads][64][D]
    if case["two_way"]:
        page = torch.arange(table.shape[1], device="cuda")
        slot = torch.where(page < SINK // PAGE, page, SINK // PAGE + (page - SINK // PAGE) % (LOCAL // PAGE))
        x = torch.cat([_unpacked(case, p[which + "s"][p["ring"].long()[:, slot]]), x], 2)
    x = x.transpose(1, 2).flatten(2, 3)
    u = torch.arange(x.shape[2], device="cuda")
    return x.masked_fill((u >= state["lens"][:, None])[:, None, :, None], 0.0)


def _plain_tree(state):
    case, cu, lens = state["case"], state["cu"].long(), state["lens"].long()
    hq, hkv, most = case["q_heads"], case["kv_heads"], state["most"]
    b, j, rows, there = _padded(cu, state["q"].shape[0], most)
    batch, pages = state["table"].shape
    q = state["q"].float()[rows].unflatten(2, (hkv, hq // hkv)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [batch][Hkv][n G][D]
    fresh = lambda x: x.float()[rows].transpose(1, 2) * there[:, None, :, None]  # noqa: E731
    at = torch.cat([torch.arange(pages * PAGE, device="cuda").expand(batch, -1), state["positions"].long()[rows]], 1)  # of every key
    held = torch.cat([at[:, :pages * PAGE] < lens[:, None], there], 1)
    # [batch][n][keys]: history, then the row's ancestors
    i = torch.arange(most, device="cuda")
    tree = (state["mask"][rows][:, :, i // 64] >> (i % 64)) & 1
    seen = torch.cat([torch.ones((batch, most, pages * PAGE), dtype=torch.bool, device="cuda"), tree.bool()], 2) & held[:, None]
    mine = state["positions"].long()[rows]
    near = (at[:, None] // PAGE < SINK // PAGE) | (at[:, None] // PAGE > mine[:, :, None] // PAGE - LOCAL // PAGE)
    streams = torch.tensor(_flags(case), device="cuda").bool()
    allowed = seen[:, None] & (near[:, None] | ~streams[:, None, None])  # [batch][Hkv][n][keys]
    if state["sel"] is not None:
        sel = state["sel"]
        page = torch.arange(pages, device="cuda")
        kept = (page >= (sel["lens"][:, None, None] + PAGE - 1) // PAGE).expand(-1, hkv, -1).clone()
        index = torch.where(torch.arange(sel["pages"].shape[2], device="cuda") < sel["count"][..., None], sel["pages"].long(), pages)
        kept = torch.nn.functional.pad(kept, (0, 1)).scatter(2, index, True)[..., :pages]
        kept = torch.nn.functional.pad((kept | streams[:, None]).repeat_interleave(PAGE, -1), (0, most), value=True)
        allowed &= kept[:, :, None]
    k = torch.cat([_history(state, "k"), fresh(state["k"])], 2)
    s = ((q @ k.transpose(2, 3)) * (1 / math.sqrt(D))).unflatten(2, (most, hq // hkv))
    s = s.masked_fill(~allowed[:, :, :, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    v = torch.cat([_history(state, "v"), fresh(state["v"])], 2)
    out = (p / total.clamp(min=1e-30)).flatten(2, 3) @ v
    out = out.unflatten(2, (most, hq // hkv)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [batch][n][H][D]
    lse = (top + total.log()).squeeze(-1).permute(0, 2, 1, 3).flatten(2, 3)
    return {"out": out[b, j].to(state["q"].dtype), "lse": lse[b, j]}


def run(state):
    if own:
        return _run_own(state)
    return {"tables": _plain_tables, "masks": _plain_masks, "rotary": _plain_rotary, "tree": _plain_tree}[state["case"]["kind"]](state)


# ---- floors --------------------------------------------------------------------------------------------------------


def _attended(case):
    """(history tokens of one streaming head, of one other head) that the batch has to read."""
    stream = dense = 0
    for n in _lengths(case):
        first = max(SINK // PAGE, n // PAGE - LOCAL // PAGE + 1) * PAGE  # of the local window of the first new token
        stream += min(n, SINK) + max(0, n - first)
        if case["budget"]:
            K, then = case["budget"] // PAGE, max(1, n - 3)
            listed_pages = -(-then // PAGE)
            dense += n if listed_pages <= K else (K - 1) * PAGE + n - (listed_pages - 1) * PAGE
        else:
            dense += n
    return stream, dense


def work(case):
    counts, hq, hkv, kind = _counts(case) if case["kind"] != "rotary" else [], case["q_heads"], case["kv_heads"], case["kind"]
    total = sum(counts)
    if kind == "tables":
        page = case["page"]
        taken = sum(-(-(n + m) // page) - -(-n // page) for n, m in zip(_lengths(case), counts))
        return {"bytes": case["batch"] * 16 + taken * 8 + total * 20 + 8, "flops": total}
    if kind == "masks":
        return {"bytes": case["batch"] * 8 + total * (8 + 8 * -(-case["nodes"] // 64)), "flops": total}
    if kind == "rotary":
        n = case["tokens"]
        return {"bytes": n * ((hq + hkv) * D * 4 + 4), "flops": 3 * n * (hq + hkv) * case["rotary"]}
    row = 2 * D if case["kv_bits"] == 16 else D * case["kv_bits"] // 8 + 4
    stream, dense = _attended(case)
    n_stream = hkv // 2
    tokens = stream * n_stream + dense * (hkv - n_stream)
    share = total / case["batch"]  # drafted tokens of a sequence
    words = -(-case["nodes"] // 64)
    return {"bytes": int(2 * row * tokens + total * (hq + hkv) * D * 4 + total * (hq * 4 + 4 + 8 * words)),
            "flops": int(4 * D * (hq // hkv) * (share * tokens + total * hkv))}


# ---- the same in 64 bits -------------------------------------------------------------------------------------------


def _exact_tables(case, seed):
    st = _prepare_tables(case, seed)
    page, lens, new, total = case["page"], _lengths(case), _counts(case), st["total"]
    table, ring, free = st["table"].cpu().numpy().copy(), st["ring"].cpu().numpy(), st["free"].cpu().tolist()
    s, w, taken = SINK // page, LOCAL // page, 0
    pos, slots, rings = (np.full(total, -1, np.int64) for _ in range(3))
    at = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        end = (n + m + page - 1) // page
        for p in range((n + page - 1) // page, end):
            table[b, p] = free[taken] if taken < len(free) else -1
            taken += 1
        t = np.arange(n, n + m)
        pos[at:at + m] = t
        phys = table[b, t // page].astype(np.int64)
        slots[at:at + m] = np.where(phys < 0, -1, phys * page + t % page)
        p = t // page
        there = (p < s) | (p >= end - w)
        rings[at:at + m] = np.where(there, ring[b, np.where(p < s, p, s + (p - s) % w)].astype(np.int64) * page + t % page, -1)
        at += m
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    i64 = lambda x: torch.tensor(x, device="cuda")  # noqa: E731
    return {"cu": i32(_cu(new)), "lens": i32([n + m for n, m in zip(lens, new)]), "positions": i32(pos), "slots": i64(slots),
            "ring_slots": i64(rings), "taken": i32([taken]), "table": i32(table)}


def _exact_masks(case, seed):
    counts, lens = _counts(case), _lengths_now(case, seed).tolist()
    bits, depth = _ancestors(_parents(case, seed, counts), counts)
    words = -(-case["nodes"] // 64)
    mask = np.array([[(x >> 64 * w) & (1 << 64) - 1 for w in range(words)] for x in bits], dtype=np.uint64)
    at = np.repeat(np.array(lens), counts) + np.array(depth)
    return {"mask": torch.tensor(mask.view(np.int64), device="cuda"), "positions": torch.tensor(at, dtype=torch.int32, device="cuda")}


def _exact_rotary(case, seed):
    st, R = _prepare_rotary(case, seed), case["rotary"]
    sc = dict({"factor": 1.0}, **SCALING[case["scaling"]])
    freq = []
    for i in range(R // 2):
        f = math.exp(-2 * i / R * math.log(BASE))
        if sc["scaling"] == "linear":
            f /= sc["factor"]
        elif sc["scaling"] == "wavelength":
            wave = 2 * math.pi / f
            short, long = sc["original_positions"] / sc["high"], sc["original_positions"] / sc["low"]
            if wave > long:
                f /= sc["factor"]
            elif wave > short:
                x = (sc["original_positions"] / wave - sc["low"]) / (sc["high"] - sc["low"])
                f = (1 - x) * f / sc["factor"] + x * f
        elif sc["scaling"] == "ramp":
            pair = [R / 2 * math.log(sc["original_positions"] / (2 * math.pi * t), BASE) for t in (sc["high"], sc["low"])]
            lo, hi = max(math.floor(pair[0]), 0), min(math.ceil(pair[1]), R - 1)
            x = min(1.0, max(0.0, (i - lo) / (hi - lo)))
            f = f * (1 - x) + f / sc["factor"] * x
        freq.append(f)
    turn = torch.polar(torch.full((R // 2,), 1.0 + 0.1 * math.log(sc["factor"]) if sc["scaling"] == "ramp" else 1.0, dtype=torch.float64,
                                  device="cuda"), torch.zeros(R // 2, dtype=torch.float64, device="cuda"))
    angle = torch.tensor(freq, dtype=torch.float64, device="cuda") * st["positions"].double()[:, None]
    turn = turn * torch.polar(torch.ones_like(angle), angle)

    def rotated(x):
        y = x.double()
        pair = y[..., :R].unflatten(-1, (R // 2, 2) if case["interleaved"] else (2, R // 2))
        pair = pair if case["interleaved"] else pair.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn[:, None])
        z = z if case["interleaved"] else z.transpose(-1, -2)
        return torch.cat([z.flatten(-2), y[..., R:]], -1)

    return {"q": rotated(st["q"]), "k": rotated(st["k"])}


def _exact_rows(case, pages):
    """Rows [n * 64][D] that n pages of one head stand for."""
    bits = case["kv_bits"]
    if bits == 16:
        return pages.double().reshape(-1, D)
    size = D * bits // 8
    raw = pages[:, :PAGE * size].reshape(-1, size).long()
    if bits == 8:
        code = raw
    else:
        code = torch.empty((raw.shape[0], D), dtype=torch.int64, device="cuda")
        c = torch.arange(size, device="cuda")
        code[:, c // 4 * 8 + c % 4], code[:, c // 4 * 8 + 4 + c % 4] = raw % 16, raw // 16
    pair = pages[:, PAGE * size:].contiguous().view(torch.float16).double().reshape(-1, 2)
    return code.double() * pair[:, :1] + pair[:, 1:]


def _exact_tree(case, seed):
    st = _prepare_tree(case, seed)
    lens, counts, hq, hkv = _lengths(case), _counts(case), case["q_heads"], case["kv_heads"]
    group, flags, s, w = hq // hkv, _flags(case), SINK // PAGE, LOCAL // PAGE
    bits, _ = _ancestors(_parents(case, seed, counts), counts)
    out = torch.zeros((sum(counts), hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((sum(counts), hq), -math.inf, dtype=torch.float64, device="cuda")
    sel = {k: v.tolist() for k, v in st["sel"].items()} if st["sel"] is not None else None
    at = 0
    for b, (n, m) in enumerate(zip(lens, counts)):
        pages = -(-n // PAGE)
        rows = slice(at, at + m)
        t = st["positions"][rows].long()
        tree = torch.tensor([[x >> i & 1 for i in range(m)] for x in bits[rows]], device="cuda").bool()
        for hk in range(hkv):
            if flags[hk]:
                low = max(s, n // PAGE - w + 1)
                pick = list(range(min(s, pages))) + list(range(low, pages))
            elif sel is not None:
                pick = sel["pages"][b][hk][:sel["count"][b][hk]] + list(range(-(-sel["lens"][b] // PAGE), pages))
            else:
                pick = list(range(pages))
            index = torch.tensor(pick, dtype=torch.long, device="cuda")
            p = st["pools"]
            if flags[hk] and case["two_way"]:
                where = p["ring"][b].long()[torch.where(index < s, index, s + (index - s) % w)]
                kh, vh = p["ks"][where, hk], p["vs"][where, hk]
            else:
                where, rank = st["table"][b].long()[index], hk - (hkv // 2 if case["two_way"] else 0)
                kh, vh = p["k"][where, rank], p["v"][where, rank]
            u = (index[:, None] * PAGE + torch.arange(PAGE, device="cuda")).flatten()
            live = u < n
            k = torch.cat([_exact_rows(case, kh)[live], st["k"][rows, hk].double()])
            v = torch.cat([_exact_rows(case, vh)[live], st["v"][rows, hk].double()])
            pos = torch.cat([u[live], t])
            seen = torch.cat([torch.ones((m, int(live.sum())), dtype=torch.bool, device="cuda"), tree], 1)
            if flags[hk]:
                seen = seen & ((pos[None] // PAGE < s) | (pos[None] // PAGE + w > t[:, None] // PAGE))
            for h in range(hk * group, (hk + 1) * group):
                x = (st["q"][rows, h].double() @ k.T / math.sqrt(D)).masked_fill(~seen, -math.inf)
                lse[rows, h] = torch.logsumexp(x, -1)
                out[rows, h] = torch.exp(x - lse[rows, h, None]) @ v
        at += m
    return {"out": out, "lse": lse}


def exact(case, seed):
    if case["kind"] == "tables":
        return _exact_tables(case, seed)
    if case["kind"] == "masks":
        return _exact_masks(case, seed) if sum(_counts(case)) <= 60000 else None
    if case["kind"] == "rotary":
        return _exact_rotary(case, seed)
    return _exact_tree(case, seed) if case["batch"] * case["q_heads"] <= 2100 else None
