"""Operators between a layer's fused projection and its attention calls whose speed counts: what happens to the queries, keys and values of
new tokens before a prefill, chunk, decode or draft step reads them.

A case is a dict of plain values.  Its `kind` says which operator it is:

  axes    rotary positions with several axes (time, height, width ...) of queries and keys (lserve_rotary_axes)
  norm    norm of every query and key head and the rotary position, in one pass (lserve_norm_rotary)
  append  queries turned; keys turned and written, with the values, into the paged cache, statistics updated (lserve_rotary_append_kv)

Half of the KV heads stream (128 sink and 512 local tokens).  With `own` false `run` computes the plain forms with elementary torch
operations, otherwise it calls the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D = 128
SINK, LOCAL, LOGICAL = 128, 512, 16
BASE = 500000.0
EPS = 1e-6


def _case(name, kind, **kw):
    # axes: positions of a token; layout: pairs of an axis next to each other ("sections") or the axes in turn ("turns")
    case = {"name": name, "kind": kind, "dtype": "bf16", "q_heads": 32, "kv_heads": 8, "rotary": D, "interleaved": False, "axes": 1,
            "layout": "sections", "norm": "none", "weights": "shared", "fused": True, "far": 8192}
    if kind == "append":
        # history and new tokens of the sequences go from `.._least` to `.._most`; dense: keys and values also to tensors of their own
        case.update(batch=1, history_least=0, history_most=0, new_least=1, new_most=1, page=64, kv_bits=16, two_way=False, dense=False)
    else:
        case.update(tokens=1)
    case.update(kw)
    if not name:
        del case["name"]
    return case


def listed():
    return [
        # one decode step of the benchmark's batch, each token with a time, a height and a width; latency is all there is
        _case("axes_step_16", "axes", dtype="fp16", tokens=16, axes=3, layout="turns", fused=False, far=32768),
        # patches of pictures, two axes, half of a head's channels turn, as many KV heads as query heads
        _case("axes_patches_5k", "axes", dtype="fp16", q_heads=32, kv_heads=32, tokens=5003, axes=2, rotary=64, interleaved=True),
        # a long prompt with a film in it
        _case("axes_film_64k", "axes", tokens=65536, axes=3, fused=False, far=65536),
        # one decode step of the benchmark's batch
        _case("norm_step_16", "norm", tokens=16, norm="rms", far=32768),
        # a ragged prefill batch; heads with weights of their own, mean taken off, half of a head's channels turn
        _case("norm_ragged_4k", "norm", dtype="fp16", tokens=4097, norm="centred", weights="heads", rotary=64, interleaved=True),
        # a prompt with pictures through a layer of 64 query heads
        _case("norm_axes_20k", "norm", q_heads=64, kv_heads=8, tokens=20011, norm="rms", axes=3, layout="turns"),
        # the longest prompt of the benchmark
        _case("norm_prompt_64k", "norm", tokens=65536, norm="rms", far=65536),
        # one decode step of the benchmark's batch, 16-bit pages
        _case("append_step_16", "append", dtype="fp16", batch=16, history_least=4001, history_most=4001),
        # one decode step of a full serving batch with query and key norms, streaming heads in their bounded cache
        _case("append_step_64", "append", batch=64, norm="rms", history_least=300, history_most=4000, two_way=True),
        # chunks of 512 tokens of eight long documents, behind what is cached already
        _case("append_chunk_8x512", "append", dtype="fp16", batch=8, history_least=1000, history_most=9001, new_least=512, new_most=512),
        # prompts of all lengths into 8-bit pages of the two-way cache, keys and values kept for the prompts' own attention
        _case("append_ragged_kv8", "append", batch=8, norm="rms", new_least=512, new_most=8192, kv_bits=8, two_way=True, dense=True),
        # the longest prompt of the benchmark
        _case("append_prompt_64k", "append", batch=1, new_least=65536, new_most=65536),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["axes", "norm", "append"])
    kw = {"dtype": rng.choice(["fp16", "bf16"]), "interleaved": rng.random() < 0.4, "fused": rng.random() < 0.6}
    kw["q_heads"], kw["kv_heads"] = rng.choice([(32, 8), (32, 8), (32, 32), (8, 2), (64, 8), (32, 16)])
    kw["rotary"] = rng.choice([128, 128, 128, 64, 32, 96, 20])
    kw["far"] = _log(rng, 1000, 1000000)
    kw["axes"] = rng.choice([2, 3, 3, 4] if kind == "axes" else [1, 1, 3])
    kw["layout"] = rng.choice(["sections", "turns"])
    kw["norm"] = "none" if kind == "axes" else rng.choice(["rms", "rms", "centred"] if kind == "norm" else ["none", "rms", "centred"])
    kw["weights"] = rng.choice(["shared", "shared", "heads", "none"])
    most = 65536 * 40 // (kw["q_heads"] + (1 if kind != "append" else 2) * kw["kv_heads"])
    if kind != "append":
        kw["tokens"] = _log(rng, 1, most)
        return _case("", kind, **kw)
    kw["batch"] = _log(rng, 1, 128)
    kw["new_most"] = rng.choice([1, _log(rng, 1, max(2, most // kw["batch"]))])
    kw["new_least"] = rng.choice([0, kw["new_most"], max(1, kw["new_most"] // 30)])
    kw["history_most"] = rng.choice([0, _log(rng, 1, max(2, min(20000, (1 << 21) // (kw["batch"] * kw["kv_heads"]))))])
    kw["history_least"] = rng.choice([0, kw["history_most"], kw["history_most"] // 7])
    kw["kv_bits"] = rng.choice([16, 16, 16, 8, 4])
    kw["page"] = rng.choice([64, 64, 64, 32, 128]) if kw["kv_bits"] == 16 else 64
    kw["two_way"] = rng.random() < 0.4
    kw["dense"] = rng.random() < 0.4
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


def _dtype(case):
    return torch.float16 if case["dtype"] == "fp16" else torch.bfloat16


def _int32(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _rows(gen, dtype, shape):
    """N(0, 1), made in pieces."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for r in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - r)
        flat[r:r + n] = torch.randn((n,), generator=gen, device="cuda")
    return out


def _qkv(case, seed, n, values):
    """Queries, keys and (where wanted) values of n tokens, cut out of the rows of one projection or tensors of their own."""
    hq, hkv, dt = case["q_heads"], case["kv_heads"], _dtype(case)
    if not case["fused"]:
        return [_rows(_gen(seed, 1 + i), dt, (n, h, D)) for i, h in enumerate([hq, hkv, hkv][:3 if values else 2])]
    rows = _rows(_gen(seed, 1), dt, (n, (hq + 2 * hkv) * D))
    parts = [rows[:, :hq * D].view(n, hq, D), rows[:, hq * D:(hq + hkv) * D].view(n, hkv, D), rows[:, (hq + hkv) * D:].view(n, hkv, D)]
    return parts[:3 if values else 2]


def _pair_axis(case):
    """Axis of each of the rotary / 2 pairs."""
    n, axes = case["rotary"] // 2, case["axes"]
    if case["layout"] == "turns":  # the first axis has what is left at the end
        return [i % axes if i < n - n % axes - n // 8 else 0 for i in range(n)]
    first = max(1, n // (2 * axes - 1))  # the first section is the shortest
    return [0 if i < first else min(axes - 1, 1 + (i - first) * (axes - 1) // max(1, n - first)) for i in range(n)]


def _positions(case, seed, n):
    """[axes][n]: single tokens of many sequences anywhere; else text, then pictures or a film row by row, then nothing more."""
    axes, far = case["axes"], case["far"]
    if n <= 256:
        return torch.randint(0, far, (axes, n), generator=_gen(seed, 3), device="cuda").to(torch.int32)
    text, side = n // 8, max(2, int(round((n / 6) ** 0.5)))
    i = torch.arange(n, device="cuda")
    j = (i - text).clamp(min=0)
    stretch = max(1, far // n)
    of = [j // (side * side) * stretch, j // side % side, j % side, i % 5]
    if axes == 1:
        of = [i % -(-n // 3) * stretch]
    elif axes == 2:
        of = of[1:3]
    return torch.stack([torch.where(i < text, i, text + p) for p in of[:axes]]).to(torch.int32)


def _weights(case, seed):
    if case["norm"] == "none" or case["weights"] == "none":
        return None, None
    shapes = [(h, D) if case["weights"] == "heads" else (D,) for h in (case["q_heads"], case["kv_heads"])]
    return tuple((1 + 0.2 * torch.randn(s, generator=_gen(seed, 30 + i), device="cuda")) for i, s in enumerate(shapes))


def _prepare_rows(case, seed):
    n, hq, hkv, dt = case["tokens"], case["q_heads"], case["kv_heads"], _dtype(case)
    q, k = _qkv(case, seed, n, False)
    return {"case": case, "q": q, "k": k, "positions": _positions(case, seed, n), "axis": torch.tensor(_pair_axis(case), device="cuda"),
            "weights": _weights(case, seed),
            "out": {"q": torch.empty((n, hq, D), dtype=dt, device="cuda"), "k": torch.empty((n, hkv, D), dtype=dt, device="cuda")}}


def _ring(page):
    return -(-SINK // page) + -(-LOCAL // page)


def _streams(case):
    """(KV heads of the main pool, KV heads that stream)."""
    half = case["kv_heads"] // 2
    return list(range(half if case["two_way"] else 0, case["kv_heads"])), list(range(half))


def _pool(case, gen, pages, heads):
    if case["kv_bits"] == 16:
        return _rows(gen, _dtype(case), (pages, heads, case["page"], D))
    return torch.zeros((pages, heads, case["page"] * D * case["kv_bits"] // 8 + 256), dtype=torch.uint8, device="cuda")


def _touched(case, lens, counts):
    """Logical pages that get tokens: sequence, first position, and for each of their places the new token there or -1."""
    seq = np.repeat(np.arange(len(lens)), [(-(-(s + n) // LOGICAL) - s // LOGICAL) if n else 0 for s, n in zip(lens, counts)])
    start, end = np.array(lens), np.array(lens) + np.array(counts)
    cu = np.concatenate([[0], np.cumsum(counts)])
    nth = np.arange(len(seq)) - np.searchsorted(seq, seq)
    first = (start[seq] // LOGICAL + nth) * LOGICAL
    at = first[:, None] + np.arange(LOGICAL)
    token = np.where((at >= start[seq][:, None]) & (at < end[seq][:, None]), at + (cu[seq] - start[seq])[:, None], -1)
    return {"seq": seq, "first": first, "held": first < start[seq], "token": token}


def _prepare_append(case, seed):
    hq, hkv, dt, page = case["q_heads"], case["kv_heads"], _dtype(case), case["page"]
    lens = _spread(case["batch"], case["history_least"], case["history_most"])
    counts = _spread(case["batch"], case["new_least"], case["new_most"], 0.7548776662466927)
    total, cu = sum(counts), [0] + np.cumsum(counts).tolist()
    q, k, v = _qkv(case, seed, total, True)
    pages = [max(1, -(-(s + n) // page)) for s, n in zip(lens, counts)]
    order = torch.randperm(sum(pages) + 2, generator=_gen(seed, 4), device="cuda").to(torch.int32)
    table = torch.zeros((len(pages), max(pages)), dtype=torch.int32, device="cuda")
    table[torch.arange(max(pages), device="cuda")[None, :] < torch.tensor(pages, device="cuda")[:, None]] = order[:sum(pages)]
    main, streams = _streams(case)
    n_main = len(order)
    state = {"case": case, "q": q, "k": k, "v": v, "axis": torch.tensor(_pair_axis(case), device="cuda"), "weights": _weights(case, seed),
             "lens": _int32(lens), "cu": _int32(cu), "counts": torch.tensor(counts, device="cuda"), "most": max(counts), "table": table,
             "k_pool": _pool(case, _gen(seed, 11), n_main, len(main)), "v_pool": _pool(case, _gen(seed, 12), n_main, len(main)),
             "ks": None, "vs": None, "ring": None,
             "positions": _positions(case, seed, total) if case["axes"] > 1 else None,
             "out": {"q": torch.empty((total, hq, D), dtype=dt, device="cuda")}}
    spans = _rows(_gen(seed, 15), dt, (n_main, len(main), page // LOGICAL, 2, D)).abs()  # of earlier keys: largest, smallest
    spans[..., 1, :] *= -1
    state["stats"] = spans
    if case["dense"]:
        state["out"].update({x: torch.empty((total, hkv, D), dtype=dt, device="cuda") for x in "kv"})
    if case["two_way"]:
        n = len(lens) * _ring(page)
        state["ks"], state["vs"] = _pool(case, _gen(seed, 13), n, len(streams)), _pool(case, _gen(seed, 14), n, len(streams))
        state["ring"] = torch.randperm(n, generator=_gen(seed, 5), device="cuda").to(torch.int32).view(len(lens), -1)
    # what a scheduler, which keeps the lengths, knows of the tokens' places
    seq, at = np.repeat(np.arange(len(lens)), counts), np.concatenate([np.arange(s, s + n) for s, n in zip(lens, counts)])
    last = np.array([-(-(s + n) // page) for s, n in zip(lens, counts)])[seq]
    stays = np.nonzero((at // page < -(-SINK // page)) | (at // page >= last - -(-LOCAL // page)))[0]
    plan = _touched(case, lens, counts) | {"of": seq, "at": at, "stays": stays}
    state["plan"] = {x: torch.from_numpy(y).cuda() for x, y in plan.items()}
    return state


def prepare(case, seed):
    return (_prepare_append if case["kind"] == "append" else _prepare_rows)(case, seed)


# ---- the library's calls -------------------------------------------------------------------------------------------


def _handles(state):
    """Descriptions, made once as a program keeps them."""
    if "handles" not in state:
        import paper_2502_14866_amd as L

        case = state["case"]
        half = case["kv_heads"] // 2
        h = state["handles"] = {"L": L, "desc": L.AttnDesc(
            case["q_heads"], case["kv_heads"], [1] * half + [0] * (case["kv_heads"] - half), page_size=case.get("page", 64),
            logical_page_size=LOGICAL, dtype=_dtype(case), sink_tokens=SINK, local_tokens=LOCAL)}
        h["rotary"] = L.RotaryDesc(rotary_dim=case["rotary"], interleaved=case["interleaved"], base=BASE)
        h["axes"] = L.PositionAxes(_pair_axis(case), case["axes"]) if case["axes"] > 1 else None
        h["norm"] = None
        if case["norm"] != "none":
            h["norm"] = L.HeadNorm(*state["weights"], eps=EPS, centred=case["norm"] == "centred")
        if case["kind"] == "append":
            main = state["k_pool"].shape[1]
            h["kv"] = L.PagedKV(state["k_pool"], state["v_pool"], state["stats"], state["table"], state["lens"],
                                pool_heads=0 if main == case["kv_heads"] else main, k_pool_stream=state["ks"], v_pool_stream=state["vs"],
                                ring_table=state["ring"], kv_bits=case["kv_bits"])
    return state["handles"]


def _run_own(state):
    h, out, case = _handles(state), state["out"], state["case"]
    L, kind = h["L"], state["case"]["kind"]
    if kind == "axes":
        L.lserve_rotary_axes(h["desc"], h["rotary"], h["axes"], state["q"], state["k"], state["positions"], out["q"], out["k"])
    elif kind == "norm":
        L.lserve_norm_rotary(h["desc"], h["norm"], h["rotary"], state["q"], state["k"],
                             state["positions"] if h["axes"] else state["positions"][0], out["q"], out["k"], axes=h["axes"])
    else:
        L.lserve_rotary_append_kv(h["desc"], h["kv"], h["rotary"], state["q"], state["k"], state["v"], state["cu"], state["lens"],
                                  state["most"], out["q"], k_out=out.get("k"), v_out=out.get("v"), norm=h["norm"], axes=h["axes"],
                                  positions=state["positions"])
        return _cache(state)
    return dict(out)


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _turned(case, x, weight, positions, axis):
    """Rows [n][heads][D] normed and turned, in 32 bits, the angles [n][pairs] in 64."""
    R = case["rotary"]
    x = x.float()
    if case["norm"] != "none":
        if case["norm"] == "centred":
            x = x - x.mean(-1, keepdim=True)
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        if weight is not None:
            x = x * weight
    f = BASE ** (-2 * torch.arange(R // 2, dtype=torch.float64, device="cuda") / R)
    angle = positions[axis].t().double() * f
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = (x[..., :R:2], x[..., 1:R:2]) if case["interleaved"] else (x[..., :R // 2], x[..., R // 2:R])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., R:]], -1)


def _plain_rows(state):
    case = state["case"]
    return {x: _turned(case, state[x], w, state["positions"], state["axis"]).to(_dtype(case)) for x, w in zip("qk", state["weights"])}


def _codes(x, bits):
    """Rows [.., D] as codes, in bytes, and the four bytes of their (scale, zero) in fp16."""
    top = 2 ** bits - 1
    zero = x.amin(-1, keepdim=True).half()
    scale = ((x.amax(-1, keepdim=True) - zero.float()) / top).half()
    code = ((x - zero.float()) / scale.float()).round().clamp(0, top).to(torch.uint8)
    if bits == 4:  # byte j of word g: channel 8 g + j in the low half, 8 g + 4 + j in the high one
        code = code.unflatten(-1, (D // 8, 2, 4))
        code = (code[..., 0, :] | code[..., 1, :] << 4).flatten(-2)
    return code, torch.cat([scale, zero], -1).contiguous().view(torch.uint8)


def _write(case, pool, page, slot, x):
    """Rows [n][heads][D] to the places [n] of the pool's pages."""
    if case["kv_bits"] == 16:
        pool[page, :, slot] = x
        return
    code, tail = _codes(x.float(), case["kv_bits"])
    size = D * case["kv_bits"] // 8
    pool[..., :64 * size].unflatten(-1, (64, size))[page, :, slot] = code
    pool[..., 64 * size:].unflatten(-1, (64, 4))[page, :, slot] = tail


def _values(case, pool):
    """What the pool's pages stand for, in the layer's type."""
    bits = case["kv_bits"]
    if bits == 16 or pool is None:
        return pool
    size = D * bits // 8
    code = pool[..., :64 * size].unflatten(-1, (64, size))
    tail = pool[..., 64 * size:].contiguous().view(torch.float16).unflatten(-1, (64, 2))
    scale, zero = tail.to(torch.float16 if case["dtype"] == "fp16" else torch.float32).split(1, -1)
    if bits == 4:
        code = torch.stack([code & 15, code >> 4], -1).unflatten(-2, (D // 8, 4)).transpose(-1, -2).flatten(-3)
    return torch.addcmul(zero, scale, code.to(scale.dtype)).to(_dtype(case))


def _cache(state):
    """Everything that the call writes."""
    case = state["case"]
    made = dict(state["out"], stats=state["stats"], k_pool=_values(case, state["k_pool"]), v_pool=_values(case, state["v_pool"]))
    if case["two_way"]:
        made.update(k_stream=_values(case, state["ks"]), v_stream=_values(case, state["vs"]))
    return made


def _plain_append(state):
    case, plan, dt, page = state["case"], state["plan"], _dtype(state["case"]), state["case"]["page"]
    seq, at = plan["of"], plan["at"]
    positions = state["positions"] if state["positions"] is not None else at[None]
    q, k = (_turned(case, state[x], w, positions, state["axis"]).to(dt) for x, w in zip("qk", state["weights"]))
    state["out"]["q"] = q
    if case["dense"]:
        state["out"].update(k=k, v=state["v"].contiguous())
    half = case["kv_heads"] // 2  # the first half streams
    main = half if case["two_way"] else 0
    where, slot = state["table"][seq, at // page].long(), at % page
    _write(case, state["k_pool"], where, slot, k[:, main:])
    _write(case, state["v_pool"], where, slot, state["v"][:, main:])
    if case["two_way"]:
        stays, sink = plan["stays"], -(-SINK // page)
        p = at[stays] // page
        where = state["ring"][seq[stays], torch.where(p < sink, p, sink + (p - sink) % -(-LOCAL // page))].long()
        _write(case, state["ks"], where, slot[stays], k[stays, :half])
        _write(case, state["vs"], where, slot[stays], state["v"][stays, :half])
    # statistics of the heads that select: of the new keys, and of the stored rows where a logical page held tokens before
    keys = k[plan["token"].clamp(min=0), half:].float()
    there = (plan["token"] >= 0)[..., None, None]
    first, g = plan["first"], page // LOGICAL
    where, row = state["table"][plan["seq"], first // page].long(), first // LOGICAL % g
    held = plan["held"][:, None, None]
    old = state["stats"][where, half - main:, row].float()
    high = torch.where(there, keys, -math.inf).amax(1).maximum(torch.where(held, old[..., 0, :], -math.inf))
    low = torch.where(there, keys, math.inf).amin(1).minimum(torch.where(held, old[..., 1, :], math.inf))
    state["stats"][where, half - main:, row] = torch.stack([high, low], -2).to(dt)
    return _cache(state)


def run(state):
    if own:
        return _run_own(state)
    return _plain_append(state) if state["case"]["kind"] == "append" else _plain_rows(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------


def work(case):
    hq, hkv = case["q_heads"], case["kv_heads"]
    weight = 0 if case["norm"] == "none" or case["weights"] == "none" else 4 * D * (hq + hkv if case["weights"] == "heads" else 2)
    per_channel = 0 if case["norm"] == "none" else 4
    if case["kind"] != "append":
        n = case["tokens"]
        return {"bytes": n * ((hq + hkv) * D * 4 + 4 * case["axes"]) + weight,
                "flops": n * (hq + hkv) * (3 * case["rotary"] + per_channel * D)}
    lens = _spread(case["batch"], case["history_least"], case["history_most"])
    counts = _spread(case["batch"], case["new_least"], case["new_most"], 0.7548776662466927)
    n, page = sum(counts), case["page"]
    main, streams = _streams(case)
    # tokens of the streaming heads that stay in the ring: sink pages and the last ones
    kept = 0
    for s, m in zip(lens, counts):
        sink, local = -(-SINK // page) * page, (-(-(s + m) // page) - -(-LOCAL // page)) * page
        kept += m - max(0, min(s + m, local) - max(s, sink))
    rows = n * len(main) + (kept * len(streams) if case["two_way"] else 0)  # of keys, and as many of values, that go to pages
    read = n * hkv if case["dense"] else rows
    logical = sum(-(-(s + m) // LOGICAL) - s // LOGICAL for s, m in zip(lens, counts) if m)
    held = sum(1 for s, m in zip(lens, counts) if m and s % LOGICAL)
    selecting = hkv - len(streams)
    row = D * case["kv_bits"] // 8 + (0 if case["kv_bits"] == 16 else 4)
    return {"bytes": n * hq * D * 4 + read * D * 4 + rows * 2 * row + (n * hkv * D * 4 if case["dense"] else 0) + weight
            + (logical + held) * selecting * 4 * D + (4 * case["axes"] * n if case["axes"] > 1 else 0) + 4 * (2 * case["batch"] + sum(-(-m // page) for m in counts)),
            "flops": n * (hq + hkv) * (3 * case["rotary"] + per_channel * D) + (0 if case["kv_bits"] == 16 else rows * 2 * 4 * D) + 2 * n * selecting * D}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------


def _defined(case, rows, weight, positions):
    """Rows normed and turned one pair at a time; positions: [axes][n]."""
    x = rows.to(torch.float64)
    if case["norm"] != "none":
        middle = x.sum(-1, keepdim=True) / D if case["norm"] == "centred" else 0.0
        x = (x - middle) / torch.sqrt(((x - middle) ** 2).sum(-1, keepdim=True) / D + EPS)
        x = x if weight is None else x * weight.to(torch.float64)
    y = x.clone()
    R = case["rotary"]
    for i, a in enumerate(_pair_axis(case)):
        first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R // 2)
        by = positions[a].to(torch.float64)[:, None] * BASE ** (-2.0 * i / R)
        y[..., first] = x[..., first] * torch.cos(by) - x[..., second] * torch.sin(by)
        y[..., second] = x[..., first] * torch.sin(by) + x[..., second] * torch.cos(by)
    return y


def _stored(case, x):
    """What a page holds of rows in 64 bits: the rows, or those of the layer's type as their codes stand for them."""
    if case["kv_bits"] == 16:
        return x
    top = 2 ** case["kv_bits"] - 1
    x = x.to(_dtype(case)).to(torch.float64)
    zero = x.min(-1, keepdim=True).values.to(torch.float16).to(torch.float64)
    scale = ((x.max(-1, keepdim=True).values - zero) / top).to(torch.float16).to(torch.float64)
    return torch.clamp(torch.round((x - zero) / scale), 0, top) * scale + zero


def exact(case, seed):
    if case["kind"] != "append":
        st = _prepare_rows(case, seed)
        return {x: _defined(case, st[x], w, st["positions"]) for x, w in zip("qk", st["weights"])}
    st = _prepare_append(case, seed)
    page, g = case["page"], case["page"] // LOGICAL
    lens, cu = st["lens"].tolist(), st["cu"].tolist()
    at = torch.cat([torch.arange(s, s + cu[b + 1] - cu[b]) for b, s in enumerate(lens)]).cuda()
    positions = st["positions"] if st["positions"] is not None else at[None]
    q, k = (_defined(case, st[x], w, positions) for x, w in zip("qk", st["weights"]))
    v = st["v"].to(torch.float64)
    main, streams = _streams(case)
    whole = {x: _values(case, st[x]).to(torch.float64) for x in ["k_pool", "v_pool"] + (["ks", "vs"] if case["two_way"] else [])}
    stats = st["stats"].to(torch.float64)
    sink, local = -(-SINK // page), -(-LOCAL // page)
    table, ring = st["table"].tolist(), st["ring"].tolist() if case["two_way"] else None
    for b, s in enumerate(lens):
        e = s + cu[b + 1] - cu[b]
        for p in range(s // page, -(-e // page) if e > s else 0):  # page by page
            lo, hi = max(s, p * page), min(e, (p + 1) * page)
            new, places = slice(cu[b] + lo - s, cu[b] + hi - s), slice(lo - p * page, hi - p * page)
            phys = table[b][p]
            for rows, name in ((k, "k_pool"), (v, "v_pool")):
                whole[name][phys][:, places] = _stored(case, rows[new][:, main]).transpose(0, 1)
            if case["two_way"] and (p < sink or p >= -(-e // page) - local):
                slot = ring[b][p if p < sink else sink + (p - sink) % local]
                for rows, name in ((k, "ks"), (v, "vs")):
                    whole[name][slot][:, places] = _stored(case, rows[new][:, streams]).transpose(0, 1)
            for j in range(g):
                first, past = max(lo, p * page + j * LOGICAL), min(hi, p * page + (j + 1) * LOGICAL)
                if first >= past:
                    continue
                keys = k[cu[b] + first - s:cu[b] + past - s, len(streams):]
                row = stats[phys][len(main) + len(streams) - case["kv_heads"]:, j]
                if p * page + j * LOGICAL < s:
                    keys = torch.cat([keys, row.transpose(0, 1)])
                row[:, 0], row[:, 1] = keys.max(0).values, keys.min(0).values
    made = {"q": q, "stats": stats, "k_pool": whole["k_pool"], "v_pool": whole["v_pool"]}
    if case["dense"]:
        made.update(k=k, v=v)
    if case["two_way"]:
        made.update(k_stream=whole["ks"], v_stream=whole["vs"])
    return made
