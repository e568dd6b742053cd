"""Attention of drafted tokens over a paged cache, from its definition in 64 bits, and inputs for it."""
import math

import numpy as np
import torch

D, NP = 128, 64


def random_tree(n, g):
    return [int(torch.randint(-1, j, (1,), generator=g)) if j else -1 for j in range(n)]


def ancestors(parents):
    """(boolean [n][n]: row j sees itself and its ancestors, depth)."""
    n = len(parents)
    see, depth = np.zeros((n, n), dtype=bool), [0] * n
    for j, p in enumerate(parents):
        if p >= 0:
            see[j] = see[p]
            depth[j] = depth[p] + 1
        see[j, j] = True
    return see, depth


def pack_bits(see, words):
    out = []
    for row in see:
        x = sum(1 << i for i, on in enumerate(row) if on)
        w = [(x >> 64 * k) & (2 ** 64 - 1) for k in range(words)]
        out.append([v - 2 ** 64 if v >= 2 ** 63 else v for v in w])
    return out


def quantise(x, bits):
    """[n][D] -> (bytes [n][D bits / 8], (scale, zero) fp16 [n][2], the numbers they stand for in 64 bits)."""
    top = 2 ** bits - 1
    x = x.float()
    zero = x.amin(-1, keepdim=True).half()
    scale = ((x.amax(-1, keepdim=True) - zero.float()) / top).half()
    code = ((x - zero.float()) / scale.float()).round().clamp(0, top).to(torch.uint8)
    value = code.double() * scale.double() + zero.double()
    if bits == 4:
        c = code.view(-1, D // 8, 2, 4)
        code = (c[:, :, 0] | c[:, :, 1] << 4).reshape(-1, D // 2)
    return code, torch.cat([scale, zero], -1), value


class Problem:
    """A batch with history in pages and drafted tokens alongside.  What no token attends (slots behind the lengths, pages nobody lists,
    dropped ring pages) is not a number."""

    def __init__(self, lens, trees, hq=4, hkv=2, flags=None, dtype=torch.float16, bits=16, two_way=False, sink=64, local=128, budget=0,
                 stale=0, words=None, seed=0, loud=1.0, see=None):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.trees, self.hq, self.hkv, self.dtype, self.bits = list(lens), trees, hq, hkv, dtype, bits
        self.flags = flags if flags is not None else [1] * (hkv // 2) + [0] * (hkv - hkv // 2)
        self.sink, self.local, self.two_way = sink, local, two_way
        self.s, self.w = -(-sink // NP), -(-local // NP)
        self.counts = [len(t) for t in trees]
        B, total = len(lens), sum(self.counts)
        self.most = max(self.counts)
        self.q = (torch.randn((total, hq, D), generator=g) * loud).to(dtype)
        self.k = torch.randn((total, hkv, D), generator=g).to(dtype)
        self.v = torch.randn((total, hkv, D), generator=g).to(dtype)
        self.see, self.pos = [], []
        for b, t in enumerate(trees):
            a, depth = ancestors(t)
            self.see.append(a if see is None or see[b] is None else see[b])
            self.pos += [lens[b] + d for d in depth]
        self.words = words or -(-self.most // 64)
        pages = [-(-n // NP) for n in lens]
        self.width = max(pages + [1]) + 1
        n_pages = sum(pages) + 3
        order = torch.randperm(n_pages, generator=g)
        self.table = torch.full((B, self.width), -1, dtype=torch.int32)
        at = 0
        for b, p in enumerate(pages):
            self.table[b, :p] = order[at:at + p].to(torch.int32)
            at += p
        streams = [h for h in range(hkv) if self.flags[h]]
        dense = [h for h in range(hkv) if not self.flags[h]]
        main = dense if two_way and dense else list(range(hkv))  # (a main pool of no heads is none)
        ring = self.s + self.w
        self.ring = torch.randperm(B * ring + 1, generator=g)[:B * ring].to(torch.int32).view(B, ring)
        self.kh = [torch.randn((n, hkv, D), generator=g).to(dtype) for n in lens]
        self.vh = [torch.randn((n, hkv, D), generator=g).to(dtype) for n in lens]
        self.pool_heads = len(main) if two_way and dense else 0

        def empty(n, heads):
            if bits == 16:
                return torch.full((n, heads, NP, D), math.nan, dtype=dtype)
            raw = torch.full((n, heads, 64 * D * bits // 8 + 256), 255, dtype=torch.uint8)
            raw[..., 64 * D * bits // 8:].view(torch.float16).fill_(math.nan)
            return raw

        self.pools = {"k": empty(n_pages, len(main)), "v": empty(n_pages, len(main))}
        if two_way:
            self.pools["ks"], self.pools["vs"] = empty(B * ring + 1, len(streams)), empty(B * ring + 1, len(streams))
        self.values = {"k": [], "v": []}  # [sequence]: [n][Hkv][D] in 64 bits, as stored
        for which, rows in (("k", self.kh), ("v", self.vh)):
            for b, n in enumerate(lens):
                self.values[which].append(rows[b].double() if bits == 16 else torch.zeros((n, hkv, D), dtype=torch.float64))
                for hk in range(hkv):
                    x = rows[b][:, hk]
                    if bits != 16 and n:
                        code, sz, value = quantise(x, bits)
                        self.values[which][b][:, hk] = value
                    bounded = two_way and self.flags[hk]
                    pool = self.pools[which + "s"] if bounded else self.pools[which]
                    rank = streams.index(hk) if bounded else main.index(hk)
                    for p in range(pages[b]):
                        if bounded and not (p < self.s or p >= pages[b] - self.w):
                            continue
                        page = int(self.ring[b, p if p < self.s else self.s + (p - self.s) % self.w]) if bounded else int(self.table[b, p])
                        m = min(NP, n - p * NP)
                        if bits == 16:
                            pool[page, rank, :m] = x[p * NP:p * NP + m]
                        else:
                            size = D * bits // 8
                            pool[page, rank, :m * size] = code[p * NP:p * NP + m].reshape(-1)
                            tail = pool[page, rank, 64 * size:].view(torch.float16).view(64, 2)
                            tail[:m] = sz[p * NP:p * NP + m]
        self.sel = None
        if budget:
            K = budget // NP
            at = [max(0, n - stale) for n in lens]
            self.sel = {"pages": torch.full((B, hkv, K), -1, dtype=torch.int32), "count": torch.zeros((B, hkv), dtype=torch.int32),
                        "lens": torch.tensor(at, dtype=torch.int32)}
            for b in range(B):
                P = -(-at[b] // NP)
                for hk in dense:
                    pick = sorted(torch.randperm(P, generator=g)[:K].tolist())
                    self.sel["pages"][b, hk, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
                    self.sel["count"][b, hk] = len(pick)

    def listed(self, b, hk):
        """Pages of history that a head reads, for some token at least."""
        P = -(-self.lens[b] // NP)
        if self.flags[hk]:
            low = max(self.s, self.lens[b] // NP - self.w + 1)
            return list(range(min(self.s, P))) + list(range(low, P))
        if self.sel is None:
            return list(range(P))
        return self.sel["pages"][b, hk, :int(self.sel["count"][b, hk])].tolist() + list(range(-(-int(self.sel["lens"][b]) // NP), P))

    def reference(self, chain=False):
        """(out, lse, A = sum of weights times |value|, E = bound of the error of a score in fp32, keys) per (token, query head)."""
        G, total = self.hq // self.hkv, sum(self.counts)
        out = torch.zeros((total, self.hq, D), dtype=torch.float64)
        lse = torch.full((total, self.hq), -math.inf, dtype=torch.float64)
        A, E = torch.zeros_like(out), torch.zeros_like(lse)
        at = 0
        for b, n in enumerate(self.counts):
            see = np.tril(np.ones((n, n), dtype=bool)) if chain else self.see[b]
            pos = [self.lens[b] + j for j in range(n)] if chain else self.pos[at:at + n]
            for hk in range(self.hkv):
                u = [t for p in self.listed(b, hk) for t in range(p * NP, min(self.lens[b], (p + 1) * NP))]
                k = torch.cat([self.values["k"][b][u, hk], self.k[at:at + n, hk].double()])
                v = torch.cat([self.values["v"][b][u, hk], self.v[at:at + n, hk].double()])
                where = np.array(u + list(pos))
                for j in range(n):
                    on = np.concatenate([np.ones(len(u), dtype=bool), see[j]])
                    if self.flags[hk]:
                        on &= (where // NP < self.s) | (where // NP > pos[j] // NP - self.w)
                    on = torch.from_numpy(on)
                    if not on.any():
                        continue
                    for h in range(hk * G, (hk + 1) * G):
                        q = self.q[at + j, h].double()
                        x = k[on] @ q / math.sqrt(D)
                        lse[at + j, h] = torch.logsumexp(x, 0)
                        p = torch.exp(x - lse[at + j, h])
                        out[at + j, h] = p @ v[on]
                        A[at + j, h] = p @ v[on].abs()
                        reach = k[on].abs().amax(0) if self.bits == 16 else 2 * k[on].abs().max()  # code * scale and zero apart
                        E[at + j, h] = (q.abs() * reach).sum() / math.sqrt(D) * 132 * 2.0 ** -24
            at += n
        return out, lse, A, E

    def call(self, L, dev="cuda:0", chain=False, pad=0, lse=True, workspace=None, run=None, most=None):
        put = lambda t: None if t is None else t.to(dev)  # noqa: E731
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
        desc = L.AttnDesc(self.hq, self.hkv, self.flags, dtype=self.dtype, sink_tokens=self.sink, local_tokens=self.local)
        total = sum(self.counts)
        kv = L.PagedKV(put(self.pools["k"]), put(self.pools["v"]), None, put(self.table), i32(self.lens + [0] * 4)[:len(self.lens)],
                       pool_heads=self.pool_heads, k_pool_stream=put(self.pools.get("ks")), v_pool_stream=put(self.pools.get("vs")),
                       ring_table=put(self.ring) if self.two_way else None, kv_bits=self.bits)
        fill = lambda t: torch.cat([t, torch.full((pad,) + t.shape[1:], math.nan, dtype=t.dtype)]).to(dev)  # noqa: E731
        out = torch.full((total + pad, self.hq, D), 7.0, dtype=self.dtype, device=dev)
        lse_out = torch.full((total + pad, self.hq), 7.0, device=dev) if lse else None
        most = most or self.most
        bits = [r for see in self.see for r in pack_bits(see, self.words)] + [[-1] * self.words] * pad
        tree = {} if chain else {"tree_mask": torch.tensor(bits, dtype=torch.int64, device=dev), "positions": i32(self.pos + [0] * pad)}
        sel = {} if self.sel is None else {"sel_" + {"pages": "pages", "count": "count", "lens": "seq_len"}[k]: put(x) for k, x in self.sel.items()}
        if workspace is None:
            need = L.lserve_tree_workspace_bytes(desc, len(self.lens), total + pad, most, self.width,
                                                 0 if self.sel is None else self.sel["pages"].shape[2])
            workspace = torch.full((max(16, need),), 255, dtype=torch.uint8, device=dev)  # any contents
        cu = i32([0] + np.cumsum(self.counts).tolist())
        q, k, v = fill(self.q), fill(self.k), fill(self.v)

        def launch(stream=None):
            L.lserve_sparse_decode_tree(desc, kv, q, k, v, cu, most, out, lse_out, workspace=workspace, stream=stream, **tree, **sel)

        (run or (lambda f: f()))(launch)
        torch.cuda.synchronize()
        assert bool((out[total:] == 7.0).all()) and (lse_out is None or bool((lse_out[total:] == 7.0).all()))  # rows behind the last sequence
        return out[:total], None if lse_out is None else lse_out[:total]

    def check(self, got, lse=None, chain=False):
        """Output: weights are rounded to the type for the second product (half a step u each) and so are values of quantised pages;
        the result once more.  Scores are off by E at most (fp32 sums of 128 products), exponentials by 1e-5, so weights by 2 (E + 1e-5); below the
        smallest normal number of fp16 a weight is off by 2^-25 of the largest.  Log-sum-exp: the scores' error, exponentials and sums."""
        out, want, A, E = self.reference(chain)
        u = torch.finfo(self.dtype).eps / 2
        g = got.cpu().double()
        assert bool(torch.isfinite(g).all())
        soft = 2.0 ** -25 * 2 * (max(self.lens + [0]) + self.most) * 6 if self.dtype == torch.float16 else 0.0
        tol = u * out.abs() + (u * (1 if self.bits == 16 else 2) * (1 + u) + 4 * E[..., None] + 2e-5) * A + soft * 2.0 ** -2
        empty = want == -math.inf
        worst = ((g - out).abs() - tol).max()
        assert worst <= 0, f"output off by {float(worst):.3e} more than rounding explains"
        assert bool((g[empty] == 0).all())
        if lse is not None:
            x = lse.cpu().double()
            assert torch.equal(x == -math.inf, empty)
            off = ((x - want).abs() - (E + 1e-5 + want.abs() * 2.0 ** -22))[~empty]
            assert off.numel() == 0 or off.max() <= 0, f"log-sum-exp off by {float(off.max()):.3e} more than fp32 explains"
