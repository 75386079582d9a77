"""pldp_cache_append_prompt against pldp_cache_append, a sequence at a time, whose arithmetic it has."""
import pytest
import torch

from tests._cache import DEV, Cache, gen, i32

pytestmark = pytest.mark.gpu


def _pool_bits(c):
    return [c.pools[x].view(torch.int16 if c.dtype == "bf16" else torch.uint8) for x in "kv"] + [c.scales[x].view(torch.int32) for x in "kv" if c.dtype != "bf16"]


# counts, starts, q heads, heads, D, page, rot, interleaved, norms
CASES = [
    ([1], [0], 4, 2, 64, 16, 64, False, True),
    ([47], [0], 32, 8, 128, 16, 128, False, True),
    ([0, 5, 1, 0, 130, 33, 0], [9, 0, 77, 3, 5, 100, 0], 8, 2, 128, 7, 64, True, True),
    ([900, 400, 1300], [0, 50, 1], 8, 8, 80, 24, 80, False, False),
    ([300, 2], [0, 30], 6, 3, 256, 1, 0, False, True),
    ([700] * 5, [0, 1, 2, 3, 4], 3, 1, 48, 32, 20, True, True),
]


@pytest.mark.parametrize("inp", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype,layout", [("bf16", "token"), ("e4m3", "head")])
@pytest.mark.parametrize("case", CASES)
def test_same_as_padded(lib, case, dtype, layout, inp):
    counts, starts, Hq, H, D, page, rot, inter, norms = case
    B, R = len(counts), sum(counts)
    lens = [a + b for a, b in zip(counts, starts)]
    packed, padded = (Cache(lib, B, max(lens), H, D, page, dtype, layout, lens=lens, seed=3) for _ in range(2))
    g = gen(11)
    qkv = torch.randn((R + 2, Hq + 2 * H, D), generator=g, device=DEV).to(inp)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    kw = {}
    if norms:
        kw["q_norm"], kw["k_norm"] = ((1 + 0.1 * torch.randn(D, generator=g, device=DEV)).to(inp) for _ in "qk")
    if rot:
        angle = torch.rand((max(lens), rot // 2), generator=g, device=DEV) * 6
        kw["cos"], kw["sin"], kw["interleaved"] = angle.cos(), angle.sin(), inter
    rows = [0]
    for n in counts:
        rows.append(rows[-1] + n)
    status = i32([0] * B)
    out = torch.full((R + 2, Hq, D), 7.0, device=DEV, dtype=torch.bfloat16)
    lib.pldp_cache_append_prompt(packed.handle, q, k, v, i32(rows), out, start=i32(starts), status=status, **kw)
    assert status.tolist() == [0] * B
    want = torch.full_like(out, 7.0)
    for b in range(B):
        if counts[b]:
            one = lib.pldp_cache(padded.pools["k"], padded.pools["v"], padded.pages[b:b + 1], padded.scales["k"], padded.scales["v"])
            s = slice(rows[b], rows[b + 1])
            lib.pldp_cache_append(one, q[s][None], k[s][None], v[s][None], i32([starts[b] + 1]), want[s][None], **kw)
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))
    assert all(torch.equal(a, b) for a, b in zip(_pool_bits(packed), _pool_bits(padded)))


def test_status(lib):
    """Starts and rows out of range, the capacity and the rotation's rows, a page that is none, queries in place."""
    c = Cache(lib, 6, 64, 1, 64, 16, lens=[64] * 6, seed=3, fill=False)
    c.pages[4, 1] = -1
    before = [x.clone() for x in _pool_bits(c)]
    qkv = torch.randn((40, 4, 64), generator=gen(2), device=DEV).bfloat16()
    q, k, v = qkv[:, :2], qkv[:, 2:3], qkv[:, 3:]
    old = q.clone()
    cos, sin = torch.ones((50, 32), device=DEV), torch.zeros((50, 32), device=DEV)
    status = i32([0] * 6)
    norm = torch.full((64,), 2.0, device=DEV, dtype=torch.bfloat16)
    rows = [1, 4, 8, 10, 20, 30, 33]
    lib.pldp_cache_append_prompt(c.handle, q, k, v, i32(rows), q, start=i32([0, -1, 51, 45, 14, 50]), q_norm=norm, cos=cos, sin=sin, status=status)
    S = lib
    assert status.tolist() == [0, S.PLDP_ST_SEQ_LEN, S.PLDP_ST_SEQ_LEN, S.PLDP_ST_CAPACITY, S.PLDP_ST_PAGE, S.PLDP_ST_CAPACITY]
    live = torch.zeros(40, dtype=torch.bool, device=DEV)
    live[1:4] = live[10:15] = live[20:30] = True
    assert torch.equal(q[~live], old[~live]) and not (q[live] == old[live]).all(-1).any()
    for x, was, name in zip(_pool_bits(c), before, "kv"):
        written = torch.zeros(x.shape[:2], dtype=torch.bool, device=DEV)
        for b, positions in ((0, range(3)), (3, range(45, 50)), (4, [14, 15])):
            for p in positions:
                written[c.pages[b, p // 16].long(), p % 16] = True
        assert torch.equal(x[~written], was[~written])
        assert torch.equal(x[c.pages[0, 0].long(), :3, 0], (k if name == "k" else v)[1:4, 0].contiguous().view(torch.int16))
    # rows that descend or pass the tensor; no rows at all
    status.zero_()
    lib.pldp_cache_append_prompt(c.handle, q, k, v, i32([0, 5, 3, 3, 3, 3, 41]), q.clone(), status=status)
    assert status.tolist() == [0, S.PLDP_ST_SEQ_LEN, 0, 0, 0, S.PLDP_ST_SEQ_LEN]
    status.zero_()
    lib.pldp_cache_append_prompt(c.handle, q[:0], k[:0], v[:0], i32([0, 0, 0, 1]), q[:0], status=status)
    assert status.tolist() == [0, 0, S.PLDP_ST_SEQ_LEN, 0, 0, 0]


def test_refusals(lib):
    c = Cache(lib, 2, 64, 2, 64, 16)
    q, k = torch.zeros((6, 4, 64), device=DEV), torch.zeros((6, 2, 64), device=DEV)
    ok = dict(cache=c.handle, q=q, k=k, v=k, rows=i32([0, 3, 6]), q_out=q.bfloat16())
    for bad, match in [(dict(q=q.half()), "float32"), (dict(k=k.bfloat16()), "k must be"), (dict(v=k[:2]), "shape"), (dict(q_out=q), "bfloat16"),
                       (dict(rows=i32([0, 1, 2, 3])), "page table"), (dict(start=i32([0])), "start"), (dict(cos=k[0]), "cos and sin"),
                       (dict(q=torch.zeros((6, 4, 32), device=DEV)), "head_dim"), (dict(cache=None), "pldp_cache")]:
        with pytest.raises(ValueError, match=match):
            lib.pldp_cache_append_prompt(**{**ok, **bad})
    for bad, match in [(dict(eps=-1.0), "eps"), (dict(cos=k[:, 0, :0], sin=k[:, 0, :0]), "rot"), (dict(cos=k[:, 0], sin=k[:, 0]), "contig|rot")]:
        with pytest.raises((lib.PldpError, ValueError), match=match):
            lib.pldp_cache_append_prompt(**{**ok, **bad})
