"""What the cache and attention operators around a PLD+ step are measured on, each through the
public entry points of the Python binding, beside their plain form in elementary torch operations.

One decode step of a target model under PLD+ feeds x_t and its draft (1 to K + 1 tokens a
sequence) through every layer: queries and keys are normed and rotated and the keys and values
written to a paged cache (append), the new tokens attend over it (attend), the candidates of the
next draft are ranked by that attention (rank, Eq. 2), and the logits are scored (logprobs).
Values, rotations and norms are N(0, 1)-like as behind a model's projections; contexts are ragged,
pages lie anywhere in their pool, and drafts have different lengths.
"""
import math

import torch

own = False

E4M3_MAX = 448.0


def listed():
    return [
        # one user, a short context, fp32 projections, x_t and ten draft tokens: launches and latency
        dict(name="append_b1_n11_f32", op="append", B=1, ctx=512, n=11, Hq=32, Hkv=8, D=128, page=16, inp="f32", cache="bf16",
             layout="token", rot=128, inter=False, norm=True),
        # a chunk of four prompts, written quantised, pages with each head's positions side by side
        dict(name="append_b4_n4095_e4m3", op="append", B=4, ctx=12288, n=4095, Hq=32, Hkv=8, D=128, page=64, inp="bf16",
             cache="e4m3", layout="head", rot=64, inter=True, norm=True),
        # quantised contexts of a small batch taken out of the cache whole
        dict(name="read_b8_ctx4k_e4m3", op="read", B=8, ctx=4096, Hkv=8, D=128, page=32, cache="e4m3", layout="token", out="bf16"),
        # one user, a short context, a full draft
        dict(name="attend_b1_ctx512_n11", op="attend", B=1, ctx=512, n=11, Hq=32, Hkv=8, D=128, page=16, cache="bf16",
             layout="token"),
        # a small batch without a draft (one new token each), quantised cache
        dict(name="attend_b8_ctx4k_n1_e4m3", op="attend", B=8, ctx=4096, n=1, Hq=32, Hkv=8, D=128, page=32, cache="e4m3",
             layout="token"),
        # two users with a whole book each: the cache's length is all there is to split
        dict(name="attend_b2_ctx128k_n1", op="attend", B=2, ctx=131072, n=1, Hq=32, Hkv=8, D=128, page=128, cache="bf16",
             layout="head"),
        # a serving batch with drafts of 10, narrow heads, quantised
        dict(name="attend_b32_ctx8k_n11_e4m3", op="attend", B=32, ctx=8192, n=11, Hq=32, Hkv=8, D=64, page=64, cache="e4m3",
             layout="token"),
        # a larger batch of a wider model with drafts of 16: the most work
        dict(name="attend_b64_ctx16k_n17", op="attend", B=64, ctx=16384, n=17, Hq=40, Hkv=8, D=128, page=64, cache="bf16",
             layout="token"),
        # candidates of a suffix match: a few a sequence, all heads
        dict(name="rank_b8_ctx4k", op="rank", B=8, ctx=4096, n=11, Hq=32, Hkv=8, D=128, page=16, cache="bf16", layout="token",
             C=16, R=32, agg="max"),
        # Eq. 1 as printed: hundreds of candidates a sequence, the eight induction heads, quantised
        dict(name="rank_b16_ctx32k_e4m3", op="rank", B=16, ctx=32768, n=11, Hq=32, Hkv=8, D=128, page=64, cache="e4m3",
             layout="token", C=512, R=8, agg="max"),
        # one user's step, fp32 logits
        dict(name="logprobs_b1_n11_v32000_f32", op="logprobs", B=1, n=11, V=32000, top=5, logits="f32", T=1.0),
        # the benchmark's step: 128 sequences of 13 rows
        dict(name="logprobs_b128_n13_v128256", op="logprobs", B=128, n=13, V=128256, top=20, logits="bf16", T=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend", "attend", "attend", "rank", "logprobs"])
    if op == "logprobs":
        B, n, V = _log(rng, 1, 128), rng.randint(1, 17), _log(rng, 2000, 160000)
        V = V if rng.random() < 0.4 else (V + 63) // 64 * 64
        kind = rng.choice(["bf16", "bf16", "f32"])
        while B * n * V * (4 if kind == "f32" else 2) > 426e6:
            B, n = (B // 2, n) if B > 1 else (1, max(1, n // 2))
        return dict(op=op, B=B, n=n, V=V, top=rng.choice([0, 1, 5, 8, 20]), logits=kind, T=rng.choice([1.0, 0.7]))
    Hkv = rng.choice([1, 2, 4, 8, 8])
    case = dict(op=op, B=_log(rng, 1, 128), ctx=_log(rng, 32, 65536), Hkv=Hkv, D=rng.choice([64, 128, 128, 80]),
                page=rng.choice([16, 16, 32, 64, 128, 24]), cache=rng.choice(["bf16", "e4m3"]), layout=rng.choice(["token", "head"]))
    size = 1 if case["cache"] == "e4m3" else 2
    if op != "read":
        case["Hq"] = Hkv * rng.choice([1, 3, 4, 5, 8])
        case["n"] = rng.choice([1, 1, rng.randint(2, 17), 11])
    if op == "append":
        if rng.random() < 0.5:
            case["n"] = _log(rng, 100, 4095)
            case["ctx"] = max(case["ctx"], case["n"] + 1)
        while case["B"] > 1 and case["B"] * case["n"] > 16000:
            case["B"] //= 2
        case["inp"], case["rot"] = rng.choice(["bf16", "bf16", "f32"]), rng.choice([case["D"], case["D"] // 2, 0])
        case["inter"], case["norm"] = rng.random() < 0.5, rng.random() < 0.7
    if op == "read":
        case["out"] = rng.choice(["bf16", "f32"])
    if op == "rank":
        case["C"], case["agg"] = _log(rng, 4, 512), rng.choice(["max", "max", "sum"])
        case["R"] = rng.choice([case["Hq"], max(1, case["Hq"] // 4)])
        case["ctx"] = max(case["ctx"], 2 * case["C"])
    most = {"append": 2e9, "read": 67e6, "attend": 2.1e9, "rank": 0.6e9}[op]       # elements of K: at most about the largest listed
    while case["B"] * case["ctx"] * Hkv * case["D"] * size > most:
        if case["B"] > 1:
            case["B"] //= 2
        elif case["ctx"] > 4096:
            case["ctx"] //= 2
        else:
            break
    if op == "attend":
        while case["B"] * case["ctx"] * case["Hq"] * case["n"] * case["D"] > 64 * 16384 * 40 * 17 * 128 // 2 and case["B"] > 1:
            case["B"] //= 2
    return case


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _lens(case):
    """Tokens in each context, x_t last: ragged from half of ctx up, all of them odd-sized; the same for every seed."""
    n = max(1, case.get("n", 1))
    top = max(1, case["ctx"] - (n - 1))                       # the step's tokens fit behind x_t
    if case["op"] == "append" and n > 64:
        top = max(1, case["ctx"] - n)                         # a chunk of a prompt
    return [max(1, top - (top // 2) * b // case["B"] - (1 if b % 2 else 0)) for b in range(case["B"])]


def _drafts(case):
    """Draft lengths: full, with some shorter and some empty ones."""
    n = case["n"]
    return [n - 1 if b % 4 != 3 else (n - 1) * (b % 5) // 5 for b in range(case["B"])]


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[name]


def _codes(x):
    """Rounded to 8 bits with one scale for each last-axis vector: (e4m3 codes, scales)."""
    amax = x.abs().amax(-1)
    scale = torch.where(amax > 0, amax / E4M3_MAX, torch.ones_like(amax))
    return (x / scale[..., None]).to(torch.float8_e4m3fn), scale


def _cache(case, g):
    """A pool of pages holding N(0, 1)-like keys and values, and each sequence's page table."""
    B, H, D, page = case["B"], case["Hkv"], case["D"], case["page"]
    per = -(-case["ctx"] // page)
    n = B * per + 3
    s = {"pages": torch.randperm(n, generator=g, device="cuda")[: B * per].to(torch.int32).view(B, per)}
    shape = (n, page, H, D) if case["layout"] == "token" else (n, H, page, D)
    for name in ("k", "v"):
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
        if case["cache"] == "e4m3":
            x, scale = _codes(x.float() if case["op"] != "append" else x.float() * 0)
            s[name + "_scale"] = scale.permute(0, 2, 1).contiguous() if case["layout"] == "token" else scale
        s[name + "_cache"] = x if case["layout"] == "token" else x.permute(0, 2, 1, 3)     # seen as [pages, page, H, D]
    return s


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    s = {"case": case}
    if case["op"] == "logprobs":
        B, n, V = case["B"], case["n"], case["V"]
        x = torch.randn((B, n, V), generator=g, device="cuda", dtype=torch.bfloat16 if case["logits"] == "bf16" else torch.float32)
        x *= 2
        s["tokens"] = torch.randint(0, V, (B, n), generator=g, device="cuda", dtype=torch.int32)
        x.scatter_add_(2, s["tokens"].long()[..., None], torch.full((B, n, 1), 9.0, device="cuda", dtype=x.dtype))
        s["logits"] = x
        f = dict(dtype=torch.float32, device="cuda")
        s["logprob"], s["entropy"] = torch.empty((B, n), **f), torch.empty((B, n), **f)
        if case["top"]:
            s["top_id"] = torch.empty((B, n, case["top"]), dtype=torch.int32, device="cuda")
            s["top_logprob"] = torch.empty((B, n, case["top"]), **f)
        if own:
            import paper_2412_01447_gb300 as pk
            s["workspace"] = torch.zeros(pk.pldp_token_logprobs_workspace_size(B * n, V), dtype=torch.uint8, device="cuda")
        return s
    s |= _cache(case, g)
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    lens = _lens(case)
    if case["op"] == "read":
        start = [1 if b % 2 else 0 for b in range(B)]
        s["start"], s["count"] = _i32(start), _i32([n - a for n, a in zip(lens, start)])
        s["k_out"], s["v_out"] = (torch.zeros((B, max(lens), Hkv, D), dtype=_dtype(case["out"]), device="cuda") for _ in "kv")
    else:
        n, Hq = case["n"], case["Hq"]
        s["seq_len"], s["draft_len"] = _i32(lens), _i32(_drafts(case))
    if case["op"] == "append":
        kind = _dtype(case["inp"])
        qkv = torch.randn((B, n, Hq + 2 * Hkv, D), generator=g, device="cuda", dtype=kind)       # one projection's output
        s["q"], s["k"], s["v"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
        s["q_norm"] = s["k_norm"] = s["cos"] = s["sin"] = None
        if case["norm"]:
            s["q_norm"], s["k_norm"] = (1 + 0.1 * torch.randn(D, generator=g, device="cuda").to(kind) for _ in "qk")
        if case["rot"]:
            r = case["rot"]
            angle = torch.arange(case["ctx"], device="cuda", dtype=torch.float64)[:, None] * (
                10000.0 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r))
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["q_out"] = torch.zeros((B, n, Hq, D), dtype=torch.bfloat16, device="cuda")
        s["start"], s["count"] = s["seq_len"] - 1, s["draft_len"] + 1
        s["k_out"], s["v_out"] = (torch.zeros((B, n, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    if case["op"] in ("attend", "rank"):
        s["q"] = torch.randn((B, n, Hq, D), generator=g, device="cuda", dtype=torch.bfloat16)
    if case["op"] == "attend":
        s["out"] = torch.zeros((B, n, Hq, D), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros((B, n, Hq), dtype=torch.float32, device="cuda")
    if case["op"] == "rank":
        # after verification: x_t' is one past what was accepted, query t'-1 is the accepted row
        C, R = case["C"], case["R"]
        s["row"] = _i32([d * (b % 3) // 2 for b, d in enumerate(_drafts(case))])
        s["kv_len"] = s["seq_len"] + s["row"]
        s["heads"] = torch.randperm(Hq, generator=g, device="cuda")[:R].sort().values.to(torch.int32)
        u = torch.rand((B, C), generator=g, device="cuda") + 0.01
        at = u.cumsum(1)
        at = at / (at[:, -1:] * 1.01) * (s["kv_len"][:, None] - C).clamp(min=0)
        s["cand_pos"] = (at.floor().int() + torch.arange(C, device="cuda", dtype=torch.int32)).clamp(max=case["ctx"] - 1)
        s["cand_count"] = torch.minimum(_i32([C if b % 3 else C // 2 for b in range(B)]), s["kv_len"])
        s["lse"] = math.log(case["ctx"]) + 0.5 + 0.2 * torch.rand((B, n, Hq), generator=g, device="cuda")
        # the copied token's source holds most of one head's attention
        b = torch.arange(B, device="cuda")
        src = s["cand_pos"][b, (s["cand_count"] // 2).long()]
        h = s["heads"][b % R].long()
        key = s["q"][b, s["row"].long(), h].float()
        key = key * ((6.0 + math.log(case["ctx"]) / 2) * math.sqrt(D) / key.square().sum(-1, keepdim=True))
        pg, slot, kv = s["pages"][b, (src // case["page"]).long()].long(), (src % case["page"]).long(), h // (Hq // Hkv)
        if case["cache"] == "e4m3":
            code, scale = _codes(key)
            s["k_cache"].view(torch.uint8)[pg, slot, kv] = code.view(torch.uint8)
            s["k_scale"][pg, kv, slot] = scale
        else:
            s["k_cache"][pg, slot, kv] = key.to(torch.bfloat16)
        s["scores"] = torch.zeros((B, C), dtype=torch.float32, device="cuda")
        s["best"], s["best_score"] = _i32([0] * B), torch.zeros(B, dtype=torch.float32, device="cuda")
    if own:
        import paper_2412_01447_gb300 as pk
        s["cache"] = pk.pldp_cache(s["k_cache"], s["v_cache"], s["pages"], k_scale=s.get("k_scale"), v_scale=s.get("v_scale"))
        if case["op"] == "attend":
            s["workspace"] = torch.zeros(pk.pldp_attend_workspace_size(B, n, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    return s


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def _kernels(s):
    import paper_2412_01447_gb300 as pk
    case, op = s["case"], s["case"]["op"]
    if op == "append":
        pk.pldp_cache_append(s["cache"], s["q"], s["k"], s["v"], s["seq_len"], s["q_out"], draft_len=s["draft_len"],
                             q_norm=s["q_norm"], k_norm=s["k_norm"], eps=1e-6, cos=s["cos"], sin=s["sin"],
                             interleaved=case["inter"])
        pk.pldp_cache_read(s["cache"], s["start"], s["count"], s["k_out"], s["v_out"])
        return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
    if op == "read":
        pk.pldp_cache_read(s["cache"], s["start"], s["count"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    if op == "attend":
        pk.pldp_attend_cache(s["cache"], s["q"], s["seq_len"], s["out"], s["workspace"], draft_len=s["draft_len"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "rank":
        pk.pldp_rank_cache(s["cache"], s["q"], s["row"], s["kv_len"], s["lse"], s["cand_pos"], s["cand_count"], s["best"],
                           heads=s["heads"], agg=case["agg"], scores=s["scores"], best_score=s["best_score"])
        return {"scores": s["scores"], "best": s["best"], "best_score": s["best_score"]}
    pk.pldp_token_logprobs(s["logits"], s["tokens"], s["logprob"], s["workspace"], entropy=s["entropy"], top_id=s.get("top_id"),
                           top_logprob=s.get("top_logprob"), temperature=case["T"])
    return {k: s[k] for k in ("logprob", "entropy", "top_id", "top_logprob") if k in s}


def _gather(s, name):
    """Every sequence's keys or values in order, fp32: [B, positions, heads, D]."""
    pages, x = s["pages"].long(), s[name + "_cache"]
    B = pages.shape[0]
    if x.dtype == torch.float8_e4m3fn:
        y = x.view(torch.uint8)[pages].view(torch.float8_e4m3fn).float()
        y *= s[name + "_scale"][pages].permute(0, 1, 3, 2)[..., None]
    else:
        y = x[pages].float()
    return y.reshape(B, -1, *x.shape[2:])


def _rotate(x, cos, sin, inter):
    r = 2 * cos.shape[-1]
    y, rest = x[..., :r], x[..., r:]
    cos, sin = cos[:, :, None], sin[:, :, None]
    a, b = (y[..., 0::2], y[..., 1::2]) if inter else (y[..., : r // 2], y[..., r // 2:])
    c, d = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((c, d), -1).flatten(-2) if inter else torch.cat((c, d), -1)
    return torch.cat((y, rest), -1)


def _plain_append(s):
    case, n = s["case"], s["case"]["n"]
    first, live = s["seq_len"].long() - 1, torch.arange(n, device="cuda") <= s["draft_len"].long()[:, None]
    pos = first[:, None] + torch.arange(n, device="cuda")
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    if case["norm"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + 1e-6) * s["q_norm"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + 1e-6) * s["k_norm"].float()
    if case["rot"]:
        at = pos.clamp(max=s["cos"].shape[0] - 1)
        q, k = (_rotate(x, s["cos"][at], s["sin"][at], case["inter"]) for x in (q, k))
    pg = torch.gather(s["pages"].long(), 1, (pos // case["page"]).clamp(max=s["pages"].shape[1] - 1))[live]
    slot = (pos % case["page"])[live]
    out = {"q": torch.where(live[..., None, None], q, 0).to(torch.bfloat16)}
    for name, x in (("k", k), ("v", v)):
        cache = s[name + "_cache"]
        if case["cache"] == "e4m3":
            code, scale = _codes(x[live])
            cache.view(torch.uint8)[pg, slot] = code.view(torch.uint8)
            s[name + "_scale"].permute(0, 2, 1)[pg, slot] = scale
            back = cache.view(torch.uint8)[pg, slot].view(torch.float8_e4m3fn).float() * s[name + "_scale"].permute(0, 2, 1)[pg, slot][..., None]
        else:
            cache[pg, slot] = x[live].to(torch.bfloat16)
            back = cache[pg, slot].float()
        dense = torch.zeros(x.shape, device="cuda")
        dense[live] = back
        out[name] = dense.to(torch.bfloat16)
    return out


def _plain_read(s):
    N = s["k_out"].shape[1]
    at = s["start"].long()[:, None] + torch.arange(N, device="cuda")
    live = (torch.arange(N, device="cuda") < s["count"].long()[:, None])[..., None, None]
    out = {}
    for name in ("k", "v"):
        x = _gather(s, name)
        x = torch.take_along_dim(x, at.clamp(max=x.shape[1] - 1)[..., None, None], 1)
        out[name] = torch.where(live, x, 0).to(s["k_out"].dtype)
    return out


def _plain_attend(s):
    case = s["case"]
    B, n, Hq, D = s["q"].shape
    Hkv = case["Hkv"]
    G = Hq // Hkv
    k, v = _gather(s, "k"), _gather(s, "v")
    q = s["q"].float().view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    x = torch.matmul(q, k.permute(0, 2, 3, 1)).view(B, Hkv, n, G, -1)
    del k
    x *= 1 / math.sqrt(D)
    i = torch.arange(n, device="cuda")
    live = i <= s["draft_len"][:, None]                                               # [B, n]
    last = s["seq_len"][:, None] - 1 + i
    seen = (torch.arange(x.shape[-1], device="cuda") <= last[..., None]) & live[..., None]
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    x -= torch.where(m > -math.inf, m, 0)
    x.exp_()
    l = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, Hkv, n * G, -1), v.permute(0, 2, 1, 3)).view(B, Hkv, n, G, D)
    o = torch.where(l > 0, o / l, 0).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    lse = (m + l.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(B, n, Hq)
    return {"out": o.to(torch.bfloat16), "lse": lse}


def _plain_rank(s):
    case, C = s["case"], s["case"]["C"]
    B, n, Hq, D = s["q"].shape
    b, heads = torch.arange(B, device="cuda")[:, None], s["heads"].long()
    at = s["cand_pos"].long()
    pg, slot = torch.gather(s["pages"].long(), 1, at // case["page"]), at % case["page"]
    if case["cache"] == "e4m3":
        k = s["k_cache"].view(torch.uint8)[pg, slot].view(torch.float8_e4m3fn).float()
        k = k * s["k_scale"].permute(0, 2, 1)[pg, slot][..., None]
    else:
        k = s["k_cache"][pg, slot].float()                                            # [B, C, Hkv, D]
    k = k[:, :, heads // (Hq // case["Hkv"])]
    row = s["row"].long()
    q = s["q"][b[:, 0], row][:, heads].float()
    p = torch.exp((k * q[:, None]).sum(-1) * (1 / math.sqrt(D)) - s["lse"][b[:, 0], row][:, None, heads])
    score = p.amax(-1) if case["agg"] == "max" else p.sum(-1)
    live = torch.arange(C, device="cuda") < s["cand_count"][:, None]
    score = torch.where(live, score, -math.inf)
    best = score.amax(-1, keepdim=True)
    first = torch.where(score == best, torch.arange(C, device="cuda"), C).amin(-1, keepdim=True)
    return {"scores": torch.where(live, score, 0), "best": torch.gather(s["cand_pos"], 1, first)[:, 0].int(), "best_score": best[:, 0]}


def _plain_logprobs(s):
    case, raw = s["case"], s["logits"].float()
    V = raw.shape[-1]
    x = raw / case["T"]
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    l = e.sum(-1, keepdim=True)
    lse = m + l.log()
    out = {"logprob": (torch.gather(x, 2, s["tokens"].long()[..., None]) - lse)[..., 0]}
    out["entropy"] = (l.log() - (e * (x - m)).sum(-1, keepdim=True) / l)[..., 0]
    if case["top"]:
        # one whole number for each value and index: the larger value first, then the lower index
        bits = (raw + 0.0).view(torch.int32).long()
        key = (torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) << 32) + (V - 1 - torch.arange(V, device="cuda"))
        ids = V - 1 - (torch.topk(key, case["top"], -1).values & 0xFFFFFFFF)
        out["top_id"], out["top_logprob"] = ids.int(), torch.gather(x, 2, ids) - lse
    return out


def run(state):
    if own:
        return _kernels(state)
    return {"append": _plain_append, "read": _plain_read, "attend": _plain_attend, "rank": _plain_rank,
            "logprobs": _plain_logprobs}[state["case"]["op"]](state)


# ----------------------------------------------------------------------------
# from the definitions, in 64 bits, a sequence at a time
# ----------------------------------------------------------------------------
def _dense64(s, name, b, n):
    """The first n positions of sequence b: [n, heads, D] in 64 bits."""
    page = s["case"]["page"]
    table = s["pages"][b, : -(-n // page)].long()
    x = s[name + "_cache"]
    rows = x.view(torch.uint8)[table].view(x.dtype) if x.dtype == torch.float8_e4m3fn else x[table]
    rows = rows.double()
    if x.dtype == torch.float8_e4m3fn:
        rows = rows * s[name + "_scale"][table].double().transpose(1, 2).unsqueeze(-1)
    return rows.flatten(0, 1)[:n]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "logprobs":
        parts = []
        for b in range(case["B"]):
            x = s["logits"][b].double()
            lp = torch.log_softmax(x / case["T"], -1)
            part = {"logprob": lp[torch.arange(case["n"], device="cuda"), s["tokens"][b].long()],
                    "entropy": -(lp.exp() * lp).sum(-1)}
            if case["top"]:
                ids = x.sort(dim=-1, descending=True, stable=True).indices[:, : case["top"]]
                part["top_id"], part["top_logprob"] = ids, lp.gather(1, ids)
            parts.append(part)
        return {k: torch.stack([p[k] for p in parts]) for k in parts[0]}
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    if case["op"] == "read":
        out = {k: torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda") for k in "kv"}
        for b in range(B):
            a, c = int(s["start"][b]), int(s["count"][b])
            for name in "kv":
                out[name][b, :c] = _dense64(s, name, b, a + c)[a:]
        return out
    n, Hq = case["n"], case["Hq"]
    if case["op"] == "append":
        out = {"q": torch.zeros((B, n, Hq, D), dtype=torch.float64, device="cuda")}
        out |= {x: torch.zeros((B, n, Hkv, D), dtype=torch.float64, device="cuda") for x in "kv"}
        for b in range(B):
            c, first = int(s["draft_len"][b]) + 1, int(s["seq_len"][b]) - 1
            for name in "qkv":
                x = s[name][b, :c].double()
                if name != "v" and case["norm"]:
                    x = x / (x.pow(2).sum(-1, keepdim=True) / D + 1e-6).sqrt() * s[name + "_norm"].double()
                if name != "v" and case["rot"]:
                    z = torch.complex(s["cos"][first:first + c].double(), s["sin"][first:first + c].double())[:, None]
                    r = case["rot"]
                    even, odd = (slice(0, r, 2), slice(1, r, 2)) if case["inter"] else (slice(0, r // 2), slice(r // 2, r))
                    w = torch.complex(x[..., even], x[..., odd]) * z
                    x = x.clone()
                    x[..., even], x[..., odd] = w.real, w.imag
                if name != "q" and case["cache"] == "e4m3":
                    unit = x.abs().max(-1, keepdim=True).values / E4M3_MAX
                    unit[unit == 0] = 1
                    x = (x / unit).to(torch.float8_e4m3fn).double() * unit
                out[name][b, :c] = x
        return out
    if case["op"] == "attend":
        out = torch.zeros((B, n, Hq, D), dtype=torch.float64, device="cuda")
        lse = torch.full((B, n, Hq), -math.inf, dtype=torch.float64, device="cuda")
        for b in range(B):
            c, first = int(s["draft_len"][b]) + 1, int(s["seq_len"][b]) - 1
            k, v = (_dense64(s, x, b, first + c).transpose(0, 1) for x in "kv")        # [Hkv, T, D]
            q = s["q"][b, :c].double().transpose(0, 1).reshape(Hkv, -1, D)               # rows (head of the group, token)
            w = (q @ k.transpose(1, 2)).view(Hq, c, -1) / math.sqrt(D)
            w += torch.full(w.shape[1:], -math.inf, dtype=torch.float64, device="cuda").triu(first + 1)
            lse[b, :c] = torch.logsumexp(w, -1).T
            out[b, :c] = (torch.softmax(w, -1).view(Hkv, -1, first + c) @ v).view(Hq, c, D).transpose(0, 1)
        return {"out": out, "lse": lse}
    scores = torch.zeros((B, case["C"]), dtype=torch.float64, device="cuda")
    best, best_score = [], []
    for b in range(B):
        c, row = int(s["cand_count"][b]), int(s["row"][b])
        at = s["cand_pos"][b, :c].long()
        k = _dense64(s, "k", b, int(s["kv_len"][b]))[at]
        p = [torch.exp(k[:, h * Hkv // Hq] @ s["q"][b, row, h].double() / math.sqrt(D) - s["lse"][b, row, h].double())
             for h in s["heads"].tolist()]
        p = torch.stack(p).max(0).values if case["agg"] == "max" else torch.stack(p).sum(0)
        scores[b, :c] = p
        best.append(int(at[int(p.cpu().numpy().argmax())]))
        best_score.append(p.max())
    return {"scores": scores, "best": torch.tensor(best), "best_score": torch.stack(best_score)}


def work(case):
    if case["op"] == "logprobs":
        rows = case["B"] * case["n"]
        return {"bytes": rows * (case["V"] * (4 if case["logits"] == "f32" else 2) + 12 + 8 * case["top"]), "flops": 5 * rows * case["V"]}
    lens, Hkv, D = _lens(case), case["Hkv"], case["D"]
    vec = D * 2 if case["cache"] == "bf16" else D + 4                                  # one position's vector of one head
    if case["op"] == "read":
        read = sum(n - b % 2 for b, n in enumerate(lens)) * Hkv * 2
        return {"bytes": read * (vec + D * (4 if case["out"] == "f32" else 2)), "flops": read * D}
    Hq, drafts = case["Hq"], _drafts(case)
    new = sum(d + 1 for d in drafts)
    if case["op"] == "append":
        size = 4 if case["inp"] == "f32" else 2
        move = new * (Hq * D * (size + 2) + 2 * Hkv * (D * size + 2 * vec + D * 2) + 4 * case["rot"])    # the written vectors are read back
        return {"bytes": move, "flops": 8 * new * (Hq + Hkv) * D}
    if case["op"] == "attend":
        return {"bytes": sum(n + d for n, d in zip(lens, drafts)) * Hkv * 2 * vec + new * Hq * (4 * D + 4),
                "flops": sum(4 * D * Hq * ((d + 1) * n + d * (d + 1) // 2) for n, d in zip(lens, drafts))}
    keys = sum(case["C"] if b % 3 else case["C"] // 2 for b in range(case["B"]))
    kv = min(Hkv, case["R"])
    return {"bytes": keys * (kv * vec + 8) + case["B"] * case["R"] * (2 * D + 4), "flops": 2 * keys * case["R"] * D}
