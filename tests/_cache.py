"""Paged caches for the tests, and plain implementations in 64 bits (torch on the GPU, a
sequence at a time, from the definitions)."""
import math

import torch

DEV = "cuda"


def gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Cache:
    """A pool whose unused memory holds NaN, a page table in random order (unused entries -1)
    and the dense values of every sequence's first `lens` positions in 64 bits."""

    def __init__(self, lib, B, ctx, heads, D, page, dtype="bf16", layout="token", lens=None, seed=0, fill=True, spread=1.0):
        g = gen(seed)
        per = -(-ctx // page)
        n = B * per + 2
        self.page, self.dtype, self.layout, self.B, self.heads, self.D, self.ctx = page, dtype, layout, B, heads, D, per * page
        self.lens = lens if lens is not None else [ctx] * B
        shape = (n, page, heads, D) if layout == "token" else (n, heads, page, D)
        kind = torch.bfloat16 if dtype == "bf16" else torch.float8_e4m3fn
        self.pages = torch.randperm(n, generator=g, device=DEV)[: B * per].to(torch.int32).view(B, per).contiguous()
        self.pools, self.scales, self.dense = {}, {}, {}
        for name in "kv":
            x = torch.full(shape, float("nan"), device=DEV)
            s = torch.full((n, heads, page), float("nan"), device=DEV)
            if layout != "token":
                x = x.permute(0, 2, 1, 3)
            dense = []
            for b, L in enumerate(self.lens):
                y = torch.randn((L, heads, D), generator=g, device=DEV) * spread
                p = torch.arange(L, device=DEV)
                pg, slot = self.pages[b, p // page].long(), p % page
                if dtype == "e4m3":
                    amax = y.abs().amax(-1)
                    scale = amax / 448
                    y = (y / scale[..., None]).to(torch.float8_e4m3fn).float()
                    s[pg, :, slot] = scale
                    dense.append(y.double() * scale.double()[..., None])
                else:
                    y = y.bfloat16().float()
                    dense.append(y.double())
                if fill:
                    x[pg, slot] = y
            pool = (x if layout == "token" else x.permute(0, 2, 1, 3)).to(kind).contiguous()
            self.pools[name] = pool if layout == "token" else pool.permute(0, 2, 1, 3)
            self.scales[name] = s if dtype == "e4m3" else None
            self.dense[name] = dense
        for b, L in enumerate(self.lens):                       # what no position needs is no page
            self.pages[b, -(-L // page):] = -1
        if lib is not None:
            self.handle = lib.pldp_cache(self.pools["k"], self.pools["v"], self.pages, self.scales["k"], self.scales["v"])

    def at(self, name, b, positions):
        """The values held at positions of sequence b, 64 bits."""
        p = torch.as_tensor(positions, device=DEV)
        pg, slot = self.pages[b, p // self.page].long(), p % self.page
        pool = self.pools[name]
        if self.dtype == "bf16":
            return pool[pg, slot].double()
        x = pool.view(torch.uint8)[pg, slot].view(torch.float8_e4m3fn).double()
        return x * self.scales[name].permute(0, 2, 1)[pg, slot].double()[..., None]


def attend64(cache, q, seq_len, draft_len, scale, heads):
    """out, lse and sum_j p_j |v_j| (what a relative error of each p_j weighs) in 64 bits."""
    B, n, Hq, D = q.shape
    G = Hq // heads
    out = torch.zeros((B, n, Hq, D), dtype=torch.float64, device=DEV)
    size = torch.zeros_like(out)
    lse = torch.full((B, n, Hq), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(B):
        for i in range(n):
            if seq_len[b] < 1 or i > draft_len[b]:
                continue
            L = seq_len[b] + i
            k, v = (cache.dense[x][b][:L].repeat_interleave(G, 1) for x in "kv")
            s = torch.einsum("hd,jhd->hj", q[b, i].double(), k) * scale
            p = torch.softmax(s, -1)
            lse[b, i] = torch.logsumexp(s, -1)
            out[b, i] = torch.einsum("hj,jhd->hd", p, v)
            size[b, i] = torch.einsum("hj,jhd->hd", p, v.abs())
    return out, lse, size
