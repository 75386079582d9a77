"""What the prompt and page operators of the paged cache are measured on, each through the public entry
points of the Python binding, beside their plain form in elementary torch operations.

A request's life in the cache: its prompt's tokens, packed with those of other requests, are normed, rotated
and written (append), attend causally over the cache, behind a prefix that may be there already (attend); it
is forked into several samples that share the prompt's pages until they write (fork: the last generation's
pages freed, the table's rows forked, pages reserved for the next step's tokens, shared ones copied); and when
requests have ended, what is left moves to the front of the pool (compact).
Values, rotations and norms are N(0, 1)-like as behind a model's projections; sequences are ragged, some have
no tokens in a pass, and pages lie anywhere in their pool.
"""
import math

import torch

own = False

E4M3_MAX = 448.0


def listed():
    return [
        # one user, a short question: launches and latency
        dict(name="attend_b1_n47", op="attend", B=1, n=47, past=0, Hq=32, Hkv=8, D=128, page=16, cache="bf16", layout="token"),
        # a batch of short prompts, narrow heads, quantised
        dict(name="attend_b24_n900_e4m3", op="attend", B=24, n=900, past=0, Hq=32, Hkv=8, D=64, page=32, cache="e4m3", layout="token"),
        # the next questions to two books that are in the cache already, quantised: few rows, many keys
        dict(name="attend_b2_n512_past32k_e4m3", op="attend", B=2, n=512, past=32768, Hq=32, Hkv=8, D=128, page=128, cache="e4m3",
             layout="head"),
        # one document
        dict(name="attend_b1_n8k", op="attend", B=1, n=8192, past=0, Hq=32, Hkv=8, D=128, page=64, cache="bf16", layout="token"),
        # wide heads, each with keys of its own, chunks behind what earlier chunks left
        dict(name="attend_b3_n2000_past4k_d256", op="attend", B=3, n=2000, past=4096, Hq=8, Hkv=8, D=256, page=24, cache="bf16",
             layout="token"),
        # long documents packed in one pass, a wider model: the most work
        dict(name="attend_b4_n16k", op="attend", B=4, n=16384, past=0, Hq=40, Hkv=8, D=128, page=64, cache="bf16", layout="token"),
        # one user's short question from fp32 projections
        dict(name="append_b1_n47_f32", op="append", B=1, n=47, past=0, Hq=32, Hkv=8, D=128, page=16, inp="f32", cache="bf16",
             layout="token", rot=128, inter=False, norm=True),
        # ragged prompts of a batch, written quantised, pages with each head's positions side by side
        dict(name="append_b16_n2000_e4m3", op="append", B=16, n=2000, past=100, Hq=32, Hkv=8, D=128, page=64, inp="bf16",
             cache="e4m3", layout="head", rot=64, inter=True, norm=True),
        # four samples of one short prompt
        dict(name="fork_r1_s4_ctx500", op="fork", R=1, S=4, ctx=500, n=11, Hkv=8, D=128, page=16, cache="bf16", layout="token"),
        # a batch of 32 long prompts, seven samples each
        dict(name="fork_r32_s7_ctx16k", op="fork", R=32, S=7, ctx=16384, n=11, Hkv=8, D=128, page=64, cache="bf16", layout="head"),
        # a few short requests, some ended
        dict(name="compact_r8_ctx200_e4m3", op="compact", R=8, ctx=200, Hkv=8, D=128, page=16, cache="e4m3", layout="token"),
        # a pool of which half has ended or shrunk
        dict(name="compact_r64_ctx12k", op="compact", R=64, ctx=12288, Hkv=8, D=128, page=64, cache="bf16", layout="token"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "attend", "append", "fork", "compact"])
    Hkv = rng.choice([1, 2, 4, 8, 8])
    case = dict(op=op, Hkv=Hkv, D=rng.choice([64, 128, 128, 80, 256]), page=rng.choice([16, 16, 32, 64, 128, 24]),
                cache=rng.choice(["bf16", "bf16", "e4m3"]), layout=rng.choice(["token", "head"]))
    vec = Hkv * case["D"] * (1 if case["cache"] == "e4m3" else 2)
    if op in ("fork", "compact"):
        case["R"], case["ctx"] = _log(rng, 1, 64), _log(rng, 20, 16384)
        if op == "fork":
            case["S"], case["n"] = rng.randint(1, 8), rng.randint(1, 17)
        while case["R"] * (case["ctx"] + 2 * case["page"] * case.get("S", 0)) * vec > 1.6e9:
            if case["R"] > 1:
                case["R"] //= 2
            else:
                case["ctx"] //= 2
        return case
    case |= dict(B=_log(rng, 1, 64), n=_log(rng, 1, 16384), past=rng.choice([0, 0, _log(rng, 1, 65536)]),
                 Hq=Hkv * rng.choice([1, 3, 4, 5, 8]))
    if op == "append":
        case["inp"], case["rot"] = rng.choice(["bf16", "bf16", "f32"]), rng.choice([case["D"], case["D"] // 2, 0])
        case["inter"], case["norm"] = rng.random() < 0.5, rng.random() < 0.7
    def dear():
        if case["B"] * (case["n"] + case["past"]) * vec > 1.2e9:
            return True
        if op == "append":
            return case["B"] * case["n"] * (case["Hq"] + 2 * Hkv) * case["D"] > 19000 * 48 * 128
        return work(case)["flops"] > 6.1e12 or case["B"] * case["n"] * case["Hq"] * case["D"] > 48000 * 40 * 128
    while dear():
        if case["B"] > 1 and rng.random() < 0.7:
            case["B"] //= 2
        elif case["past"] > 2 * case["n"]:
            case["past"] //= 2
        else:
            case["n"] = max(1, case["n"] // 2)
    return case


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _counts(case):
    """Tokens of each sequence in this pass: from n down to a quarter of it, odd ones, some none; the same for every seed."""
    B, n = case["B"], case["n"]
    return [0 if b % 7 == 6 else max(1, n - n * 3 // 4 * b // B - b % 2) for b in range(B)]


def _starts(case):
    """Positions that each sequence has in the cache already: from past down to half of it."""
    return [max(0, case["past"] - case["past"] // 2 * b // case["B"] - b % 2) for b in range(case["B"])]


def _rows(case):
    rows = [0]
    for c in _counts(case):
        rows.append(rows[-1] + c)
    return rows


_BEHIND = 3                  # rows behind the last sequence, which belong to none


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[name]


def _codes(x):
    """Rounded to 8 bits with one scale for each last-axis vector: (e4m3 codes, scales)."""
    amax = x.abs().amax(-1)
    scale = torch.where(amax > 0, amax / E4M3_MAX, torch.ones_like(amax))
    return (x / scale[..., None]).to(torch.float8_e4m3fn), scale


def _pool(case, n, g, fill=True):
    """A pool of n pages holding N(0, 1)-like keys and values (or zeros)."""
    H, D, page = case["Hkv"], case["D"], case["page"]
    shape = (n, page, H, D) if case["layout"] == "token" else (n, H, page, D)
    s = {}
    for name in ("k", "v"):
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16) if fill else torch.zeros(shape, device="cuda", dtype=torch.bfloat16)
        if case["cache"] == "e4m3":
            x, scale = _codes(x.float())
            s[name + "_scale"] = scale.permute(0, 2, 1).contiguous() if case["layout"] == "token" else scale
        s[name + "_cache"] = x if case["layout"] == "token" else x.permute(0, 2, 1, 3)     # seen as [pages, page, H, D]
    return s


def _prepare_tokens(case, g):
    B, Hq, Hkv, D, page = case["B"], case["Hq"], case["Hkv"], case["D"], case["page"]
    counts, starts, rows = _counts(case), _starts(case), _rows(case)
    per = max(1, max(-(-(a + c) // page) for a, c in zip(starts, counts)))
    n = B * per + 3
    s = {"pages": torch.randperm(n, generator=g, device="cuda")[: B * per].to(torch.int32).view(B, per)}
    s |= _pool(case, n, g, fill=case["op"] == "attend")
    s["rows"], s["start"], s["count"] = _i32(rows), _i32(starts), _i32(counts)
    R = rows[-1] + _BEHIND
    if case["op"] == "attend":
        s["q"] = torch.randn((R, Hq, D), generator=g, device="cuda", dtype=torch.bfloat16)
        s["out"] = torch.zeros((R, Hq, D), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros((R, Hq), dtype=torch.float32, device="cuda")
        return s
    kind = _dtype(case["inp"])
    qkv = torch.randn((R, Hq + 2 * Hkv, D), generator=g, device="cuda", dtype=kind)       # one projection's output
    s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    s["q_norm"] = s["k_norm"] = s["cos"] = s["sin"] = None
    if case["norm"]:
        s["q_norm"], s["k_norm"] = (1 + 0.1 * torch.randn(D, generator=g, device="cuda").to(kind) for _ in "qk")
    if case["rot"]:
        r = case["rot"]
        angle = torch.arange(per * page, device="cuda", dtype=torch.float64)[:, None] * (
            10000.0 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r))
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    s["q_out"] = torch.zeros((R, Hq, D), dtype=torch.bfloat16, device="cuda")
    s["k_out"], s["v_out"] = (torch.zeros((B, max(counts), Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    return s


def _lens(case):
    """Contexts of the requests: ragged, odd."""
    return [max(1, case["ctx"] - case["ctx"] // 2 * b // case["R"] - (b * 7 + 1) % 5) for b in range(case["R"])]


def _keeps(case):
    """What compaction's requests keep: some nothing (they have ended), some a part, the rest everything (-1)."""
    return [0 if b % 3 == 0 and case["R"] > 1 else n // 2 if b % 3 == 1 else -1 for b, n in enumerate(_lens(case))]


def _prepare_pages(case, g):
    page, lens, R = case["page"], _lens(case), case["R"]
    held = [-(-n // page) for n in lens]
    if case["op"] == "fork":
        S, step = case["S"], case["n"]
        B = R * (S + 1)
        per = -(-(max(lens) + step) // page)
        n_pages = sum(held) + B * (-(-step // page) + 1)
    else:
        B, per, n_pages = R, max(held), sum(held) + 2
    order = torch.randperm(n_pages, generator=g, device="cuda")[: sum(held)].to(torch.int32)
    s = {"pages": torch.full((B, per), -1, dtype=torch.int32, device="cuda"), "refs": torch.zeros(n_pages, dtype=torch.int32, device="cuda")}
    at = 0
    for b, h in enumerate(held):
        s["pages"][b, :h] = order[at:at + h]
        at += h
    s["refs"][order.long()] = 1
    s |= _pool(case, n_pages, g)
    if case["op"] == "fork":
        # requests 0..R-1, then S samples of each; a sample's context is its request's but the last token, whose
        # place the next step writes first
        s["parent"] = _i32([-1] * R + [i // S for i in range(R * S)])
        s["len"] = _i32([n - 1 for n in lens] + [lens[i // S] - 1 for i in range(R * S)])
        s["keep"] = _i32([-1] * R + [0] * (R * S))
        s["count"] = _i32([0] * R + [step] * (R * S))
        s["copies"] = _i32([[-1, -1]] * B)
    else:
        s["keep"] = _i32(_keeps(case))
        s["pages_before"], s["refs_before"] = s["pages"].clone(), s["refs"].clone()
        s["copies"] = torch.full((max(1, n_pages // 2), 2), -1, dtype=torch.int32, device="cuda")
        s["n_copies"], s["used"] = _i32([0]), _i32([0])
    return s


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    s = {"case": case}
    s |= _prepare_tokens(case, g) if case["op"] in ("attend", "append") else _prepare_pages(case, g)
    if own:
        import paper_2412_01447_gb300 as pk
        s["cache"] = pk.pldp_cache(s["k_cache"], s["v_cache"], s["pages"], k_scale=s.get("k_scale"), v_scale=s.get("v_scale"))
        if case["op"] == "attend":
            s["workspace"] = torch.zeros(pk.pldp_attend_prompt_workspace_size(case["Hq"], case["Hkv"], case["D"]), dtype=torch.uint8, device="cuda")
        if case["op"] in ("fork", "compact"):
            s["table"] = pk.pldp_page_table(s["pages"], s["refs"], case["page"])
            s["workspace"] = torch.zeros(pk.pldp_pages_workspace_size(s["table"]), dtype=torch.uint8, device="cuda")
    return s


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def _kernels(s):
    import paper_2412_01447_gb300 as pk
    case, op = s["case"], s["case"]["op"]
    if op == "attend":
        pk.pldp_attend_prompt(s["cache"], s["q"], s["rows"], s["out"], s["workspace"], start=s["start"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "append":
        pk.pldp_cache_append_prompt(s["cache"], s["q"], s["k"], s["v"], s["rows"], s["q_out"], start=s["start"], q_norm=s["q_norm"],
                                    k_norm=s["k_norm"], eps=1e-6, cos=s["cos"], sin=s["sin"], interleaved=case["inter"])
        pk.pldp_cache_read(s["cache"], s["start"], s["count"], s["k_out"], s["v_out"])
        return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
    if op == "fork":
        pk.pldp_pages_free(s["table"], s["keep"])
        pk.pldp_pages_fork(s["table"], s["parent"], s["len"])
        pk.pldp_pages_reserve(s["table"], s["len"], s["copies"], s["workspace"], n=case["n"], count=s["count"])
        pk.pldp_cache_copy_pages(s["cache"], s["copies"])
        return _page_outputs(s)
    s["pages"].copy_(s["pages_before"])                       # (the table as it was, so that every pass finds the same)
    s["refs"].copy_(s["refs_before"])
    pk.pldp_pages_free(s["table"], s["keep"])
    pk.pldp_pages_compact(s["table"], s["copies"], s["n_copies"], s["workspace"], used=s["used"])
    pk.pldp_cache_copy_pages(s["cache"], s["copies"], s["n_copies"])
    return _page_outputs(s)


def _page_outputs(s):
    """The table, the counts and the pool, its 8 bits as they are: a copy's bytes are whole numbers."""
    out = {k: s[k] for k in ("pages", "refs", "used", "k_scale", "v_scale") if k in s}
    for name in ("k_cache", "v_cache"):
        x = s[name]
        out[name] = x.view(torch.int16) if x.dtype == torch.bfloat16 else x.view(torch.uint8)
    return out


def _sequence(s, name, b, n):
    """The first n positions of sequence b, fp32: [heads, n, D]."""
    table = s["pages"][b, : -(-n // s["case"]["page"])].long()
    x = s[name + "_cache"]
    if x.dtype == torch.float8_e4m3fn:
        y = x.view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * s[name + "_scale"][table].permute(0, 2, 1)[..., None]
    else:
        y = x[table].float()
    return y.flatten(0, 1)[:n].permute(1, 0, 2)


def _plain_attend(s):
    case = s["case"]
    R, Hq, D = s["q"].shape
    Hkv = case["Hkv"]
    out, lse = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    for b, (at, a, c) in enumerate(zip(_rows(case), _starts(case), _counts(case))):
        if c == 0:
            continue
        k, v = _sequence(s, "k", b, a + c), _sequence(s, "v", b, a + c)                 # [Hkv, a + c, D]
        # rows a block at a time, as many as keep the scores near 4 GB, against the keys that they see
        step = max(64, int(1e9 / (Hq * (a + c))))
        for i in range(0, c, step):
            j = min(c, i + step)
            q = s["q"][at + i:at + j].float().view(j - i, Hkv, -1, D).permute(1, 2, 0, 3)   # [Hkv, G, rows, D]
            x = torch.matmul(q.flatten(1, 2), k[:, : a + j].transpose(1, 2)).view(Hkv, -1, j - i, a + j)
            x *= 1 / math.sqrt(D)
            hidden = torch.arange(a + j, device="cuda") > a + torch.arange(i, j, device="cuda")[:, None]
            x.masked_fill_(hidden, -math.inf)
            m = x.amax(-1, keepdim=True)
            x -= m
            x.exp_()
            l = x.sum(-1, keepdim=True)
            o = torch.matmul(x.flatten(1, 2), v[:, : a + j]).view(Hkv, -1, j - i, D) / l
            out[at + i:at + j] = o.permute(2, 0, 1, 3).reshape(j - i, Hq, D).to(torch.bfloat16)
            lse[at + i:at + j] = (m + l.log())[..., 0].permute(2, 0, 1).reshape(j - i, Hq)
    return {"out": out, "lse": lse}


def _rotate(x, cos, sin, inter):
    r = 2 * cos.shape[-1]
    y, rest = x[..., :r], x[..., r:]
    cos, sin = cos[:, None], sin[:, None]
    a, b = (y[..., 0::2], y[..., 1::2]) if inter else (y[..., : r // 2], y[..., r // 2:])
    c, d = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((c, d), -1).flatten(-2) if inter else torch.cat((c, d), -1)
    return torch.cat((y, rest), -1)


def _plain_append(s):
    case = s["case"]
    R, B = s["q"].shape[0] - _BEHIND, case["B"]
    row = torch.arange(R, device="cuda")
    seq = (row[:, None] >= s["rows"][None, 1:].long()).sum(1)                           # the sequence of each row
    pos = row - s["rows"].long()[seq] + s["start"].long()[seq]
    q, k, v = s["q"][:R].float(), s["k"][:R].float(), s["v"][:R].float()
    if case["norm"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + 1e-6) * s["q_norm"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + 1e-6) * s["k_norm"].float()
    if case["rot"]:
        q, k = (_rotate(x, s["cos"][pos], s["sin"][pos], case["inter"]) for x in (q, k))
    pg, slot = s["pages"].long()[seq, pos // case["page"]], pos % case["page"]
    out = {"q": torch.cat((q.to(torch.bfloat16), s["q_out"][R:]))}
    for name, x in (("k", k), ("v", v)):
        cache = s[name + "_cache"]
        if case["cache"] == "e4m3":
            code, scale = _codes(x)
            cache.view(torch.uint8)[pg, slot] = code.view(torch.uint8)
            s[name + "_scale"].permute(0, 2, 1)[pg, slot] = scale
            back = cache.view(torch.uint8)[pg, slot].view(torch.float8_e4m3fn).float() * s[name + "_scale"].permute(0, 2, 1)[pg, slot][..., None]
        else:
            cache[pg, slot] = x.to(torch.bfloat16)
            back = cache[pg, slot].float()
        dense = torch.zeros_like(s[name + "_out"])
        dense[seq, row - s["rows"].long()[seq]] = back.to(torch.bfloat16)
        out[name] = dense
    return out


def _release(s, drop):
    """Entries of the table where drop says so are given back."""
    pages, refs = s["pages"], s["refs"]
    drop = drop & (pages >= 0)
    refs.index_add_(0, torch.where(drop, pages, 0).flatten(), -drop.int().flatten())
    pages.masked_fill_(drop, -1)


def _plain_free(s):
    keep, entry = s["keep"][:, None], torch.arange(s["pages"].shape[1], device="cuda")
    _release(s, (keep >= 0) & (entry * s["case"]["page"] >= keep))


def _copy(s, src, dst):
    for name in ("k_cache", "v_cache", "k_scale", "v_scale"):
        if name in s:
            x = s[name].view(torch.uint8) if s[name].dtype == torch.float8_e4m3fn else s[name]
            x[dst] = x[src]


def _plain_fork(s):
    pages, refs, page = s["pages"], s["refs"], s["case"]["page"]
    entry = torch.arange(pages.shape[1], device="cuda")
    _plain_free(s)
    forked = (s["parent"] >= 0)[:, None]
    _release(s, forked.expand_as(pages))
    theirs = torch.where(forked & (entry * page < s["len"][:, None]), pages[s["parent"].clamp(min=0).long()], -1)
    refs.index_add_(0, theirs.clamp(min=0).flatten(), (theirs >= 0).int().flatten())
    pages.copy_(torch.where(forked, theirs, pages))
    # pages for the next step's tokens
    first, last = s["len"][:, None], (s["len"] + s["count"])[:, None] - 1
    inside = (entry >= first // page) & (entry <= last // page) & (s["count"] > 0)[:, None]
    shared = (pages >= 0) & (refs[pages.clamp(min=0).long()] > 1)
    need = inside & ((pages < 0) | shared)
    free = torch.sort(refs != 0, stable=True).indices                                    # the free pages first, ascending
    number = (need.flatten().cumsum(0) - 1).view_as(need)
    new = torch.where(need, free[number.clamp(min=0)].int(), pages)
    moved = need & shared & (entry == first // page) & (first % page != 0)
    src, dst = pages[moved].long(), new[moved].long()
    _release(s, need)
    refs[new[need].long()] = 1
    pages.copy_(new)
    _copy(s, src, dst)
    return _page_outputs(s)


def _plain_compact(s):
    s["pages"].copy_(s["pages_before"])
    s["refs"].copy_(s["refs_before"])
    _plain_free(s)
    pages, refs = s["pages"], s["refs"]
    live = refs > 0
    used = int(live.sum())
    s["used"].fill_(used)
    dst = torch.nonzero(~live[:used])[:, 0]
    src = torch.nonzero(live[used:])[:, 0].flip(0) + used
    to = torch.arange(refs.numel(), device="cuda", dtype=torch.int32)
    to[src] = dst.int()
    refs[dst] = refs[src]
    refs[src] = 0
    pages.copy_(torch.where(pages >= 0, to[pages.clamp(min=0).long()], pages))
    _copy(s, src, dst)
    return _page_outputs(s)


def run(state):
    if own:
        return _kernels(state)
    return {"attend": _plain_attend, "append": _plain_append, "fork": _plain_fork, "compact": _plain_compact}[state["case"]["op"]](state)


# ----------------------------------------------------------------------------
# from the definitions, in 64 bits, a sequence at a time
# ----------------------------------------------------------------------------
def _dense64(s, name, b, n):
    """The first n positions of sequence b: [n, heads, D] in 64 bits."""
    page = s["case"]["page"]
    p = torch.arange(n, device="cuda")
    pg, slot = s["pages"][b].long()[p // page], p % page
    x = s[name + "_cache"]
    if x.dtype == torch.float8_e4m3fn:
        y = x.view(torch.uint8)[pg, slot].view(x.dtype).double()
        return y * s[name + "_scale"][pg, :, slot].double().unsqueeze(-1)
    return x[pg, slot].double()


def _exact_attend(case, s):
    R, Hq, D = s["q"].shape
    out = torch.zeros((R, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((R, Hq), dtype=torch.float64, device="cuda")
    rows, starts, counts = s["rows"].tolist(), s["start"].tolist(), s["count"].tolist()
    for b in range(case["B"]):
        if not counts[b]:
            continue
        T = starts[b] + counts[b]
        k, v = _dense64(s, "k", b, T), _dense64(s, "v", b, T)
        most = max(128, int(4e8 // (T * Hq // case["Hkv"])))
        for h in range(case["Hkv"]):
            heads = slice(h * Hq // case["Hkv"], (h + 1) * Hq // case["Hkv"])
            for i in range(0, counts[b], most):
                n = min(most, counts[b] - i)
                seen = starts[b] + i + n
                at = slice(rows[b] + i, rows[b] + i + n)
                w = torch.einsum("rgd,td->grt", s["q"][at, heads].double(), k[:seen, h]) / math.sqrt(D)
                w += torch.full((n, seen), -math.inf, dtype=torch.float64, device="cuda").triu(seen - n + 1)
                lse[at, heads] = torch.logsumexp(w, -1).T
                out[at, heads] = torch.einsum("grt,td->rgd", torch.softmax(w, -1), v[:seen, h])
    return {"out": out, "lse": lse}


def _exact_append(case, s):
    out = {"q": torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda")}
    out |= {x: torch.zeros(s[x + "_out"].shape, dtype=torch.float64, device="cuda") for x in "kv"}
    rows, starts = s["rows"].tolist(), s["start"].tolist()
    for b in range(case["B"]):
        c, first = rows[b + 1] - rows[b], starts[b]
        for name in "qkv":
            x = s[name][rows[b]:rows[b + 1]].double()
            if name != "v" and case["norm"]:
                x = x / (x.pow(2).sum(-1, keepdim=True) / case["D"] + 1e-6).sqrt() * s[name + "_norm"].double()
            if name != "v" and case["rot"]:
                z = torch.complex(s["cos"][first:first + c].double(), s["sin"][first:first + c].double())[:, None]
                r = case["rot"]
                even, odd = (slice(0, r, 2), slice(1, r, 2)) if case["inter"] else (slice(0, r // 2), slice(r // 2, r))
                w = torch.complex(x[..., even], x[..., odd]) * z
                x = x.clone()
                x[..., even], x[..., odd] = w.real, w.imag
            if name == "q":
                out["q"][rows[b]:rows[b + 1]] = x
                continue
            if case["cache"] == "e4m3":
                unit = x.abs().max(-1, keepdim=True).values / E4M3_MAX
                unit[unit == 0] = 1
                x = (x / unit).to(torch.float8_e4m3fn).double() * unit
            out[name][b, :c] = x
    return out


def _exact_pages(case, s):
    """One page after the other, as a program on the host would."""
    page, pages, refs = case["page"], s["pages"].tolist(), s["refs"].tolist()
    moves = []
    for b, keep in enumerate(s["keep"].tolist()):
        for e in range(len(pages[b])):
            if keep >= 0 and e * page >= keep and pages[b][e] >= 0:
                refs[pages[b][e]] -= 1
                pages[b][e] = -1
    if case["op"] == "fork":
        lens, counts = s["len"].tolist(), s["count"].tolist()
        for b, p in enumerate(s["parent"].tolist()):
            if p >= 0:
                pages[b] = [x if e * page < lens[b] else -1 for e, x in enumerate(pages[p])]
                for x in pages[b]:
                    if x >= 0:
                        refs[x] += 1
        held = list(refs)                                      # who holds what when the step's pages are asked for
        free = [x for x, r in enumerate(refs) if r == 0][::-1]
        for b in range(len(pages)):
            for e in range(lens[b] // page, (lens[b] + counts[b] - 1) // page + 1 if counts[b] else 0):
                old = pages[b][e]
                if old < 0 or held[old] > 1:
                    new = free.pop()
                    pages[b][e], refs[new] = new, 1
                    if old >= 0:
                        refs[old] -= 1
                        if e * page < lens[b]:
                            moves.append((old, new))
    else:
        live = [x for x, r in enumerate(refs) if r]
        holes = [x for x in range(len(live)) if refs[x] == 0]
        moves = list(zip(reversed(live), holes))
        to = dict(moves)
        for src, dst in moves:
            refs[dst], refs[src] = refs[src], 0
        pages = [[to.get(x, x) for x in row] for row in pages]
    out = {"pages": torch.tensor(pages), "refs": torch.tensor(refs)}
    if case["op"] == "compact":
        out["used"] = torch.tensor([len(live)])
    src, dst = (torch.tensor([m[i] for m in moves], dtype=torch.long, device="cuda") for i in (0, 1))
    for name in ("k_scale", "v_scale"):
        if name in s:
            x = s[name].double()
            x[dst] = x[src]
            out[name] = x
    return out | {"k_cache": None, "v_cache": None}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(case, s) if work(case)["flops"] < 1.5e13 else None
    return _exact_append(case, s) if case["op"] == "append" else _exact_pages(case, s)


def work(case):
    Hkv, D, page = case["Hkv"], case["D"], case["page"]
    vec = D * 2 if case["cache"] == "bf16" else D + 4                                  # one position's vector of one head
    if case["op"] in ("attend", "append"):
        Hq, counts, starts = case["Hq"], _counts(case), _starts(case)
        new = sum(counts)
        if case["op"] == "append":
            size = 4 if case["inp"] == "f32" else 2
            # the written vectors are read back
            return {"bytes": new * (Hq * D * (size + 2) + 2 * Hkv * (D * size + 2 * vec + D * 2) + 4 * case["rot"]), "flops": 8 * new * (Hq + Hkv) * D}
        return {"bytes": sum(a + c for a, c in zip(starts, counts) if c) * Hkv * 2 * vec + new * Hq * (4 * D + 4),
                "flops": sum(4 * D * Hq * (c * a + c * (c + 1) // 2) for a, c in zip(starts, counts))}
    lens = _lens(case)
    held = [-(-n // page) for n in lens]
    if case["op"] == "fork":
        S = case["S"]
        copied = S * sum((n - 1) % page != 0 for n in lens)
        entries = S * sum(held)                                # read once of each parent, written; counted
        return {"bytes": 2 * copied * page * Hkv * 2 * vec + 8 * entries + 4 * sum(held), "flops": 2 * entries}
    kept = [h if k < 0 else -(-k // page) for h, k in zip(held, _keeps(case))]
    moved = sum(kept) * (1 - sum(kept) / (sum(held) + 2))      # on average: those behind the first sum(kept) pages
    return {"bytes": int(2 * moved * page * Hkv * 2 * vec) + 8 * sum(held) + 8 * (sum(held) + 2), "flops": 2 * sum(held)}
