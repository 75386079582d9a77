"""pldp_token_logprobs against log softmax, entropy and a stable sort in 64 bits."""
import math

import pytest
import torch

from tests._cache import DEV, gen, i32

pytestmark = pytest.mark.gpu


def _run(lib, x, tokens, top, T=1.0, **kw):
    shape, f = x.shape[:-1], dict(dtype=torch.float32, device=DEV)
    rows = x.numel() // x.shape[-1]
    o = dict(logprob=torch.full(shape, -7.0, **f), entropy=torch.full(shape, -7.0, **f))
    if top:
        o |= dict(top_id=torch.full((*shape, top), -7, dtype=torch.int32, device=DEV), top_logprob=torch.full((*shape, top), -7.0, **f))
    ws = torch.full((lib.pldp_token_logprobs_workspace_size(rows, x.shape[-1]),), 77, dtype=torch.uint8, device=DEV)
    lib.pldp_token_logprobs(x, tokens, o["logprob"], ws, entropy=o["entropy"], top_id=o.get("top_id"),
                            top_logprob=o.get("top_logprob"), temperature=T, **kw)
    return o


def _check(o, x, tokens, top, T=1.0):
    x64 = x.double()
    lp = torch.log_softmax(x64 / T, -1)
    # fp32: x / T rounded (2^-24 of it, twice), sums of positive terms, a logarithm
    tol = 1e-6 * (4 + 2 * x64.masked_fill(x64 == -math.inf, 0).abs().amax(-1) / T)
    want = lp.gather(-1, tokens.long()[..., None])[..., 0]
    live = torch.isfinite(want)
    assert torch.equal(o["logprob"] == -math.inf, ~live)
    assert ((o["logprob"].double() - want).abs()[live] <= tol[live]).all()
    ent = -(lp.exp() * lp.masked_fill(lp == -math.inf, 0)).sum(-1)
    assert ((o["entropy"].double() - ent).abs() <= 2 * tol).all(), ((o["entropy"].double() - ent).abs() - 2 * tol).max()
    if top:
        ids = (x64 + 0.0).sort(dim=-1, descending=True, stable=True).indices[..., :top]
        assert torch.equal(o["top_id"].long(), ids)
        want = lp.gather(-1, ids)
        live = torch.isfinite(want)
        assert torch.equal(o["top_logprob"] == -math.inf, ~live)
        assert ((o["top_logprob"].double() - want).abs()[live] <= tol[..., None].expand_as(want)[live]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,V", [((1,), 1), ((1,), 2), ((3,), 31), ((2, 3), 33), ((5,), 255), ((5,), 256), ((5,), 257),
                                    ((4,), 1000), ((7,), 2048), ((3,), 4099), ((2, 11), 32000), ((3, 5), 32001), ((2,), 128256),
                                    ((2,), 128255), ((1,), 300001)])
def test_rows(lib, dtype, rows, V):
    x = (torch.randn((*rows, V), generator=gen(V), device=DEV) * 3).to(dtype)
    tokens = torch.randint(0, V, rows, generator=gen(V + 1), device=DEV, dtype=torch.int32)
    for top, T in ((min(V, 5), 1.0), (min(V, 32), 0.7), (0, 1.3), (1, 2.0)):
        _check(_run(lib, x, tokens, top, T), x, tokens, top, T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_and_masks(lib, dtype):
    """Equal logits, few values, infinities and the type's lowest value as masks, signed
    zeros, large offsets, one token left, one token that holds everything."""
    V, low = 5000, torch.finfo(dtype).min
    g = gen(3)
    x = torch.zeros((12, V), device=DEV)
    x[1] = torch.randint(0, 3, (V,), generator=g, device=DEV).float()
    x[2] = -0.0
    x[2, ::7] = 0.0
    x[3] = torch.randn(V, generator=g, device=DEV)
    x[3, torch.rand(V, generator=g, device=DEV) < 0.9] = -math.inf
    x[4] = -math.inf
    x[4, 4321] = 2.5
    x[5] = low
    x[5, 100:140] = torch.randn(40, generator=g, device=DEV)
    x[6] = -1e4
    x[6, 77] = 50.0
    x[7] = torch.randn(V, generator=g, device=DEV) + 3000
    x[8] = -math.inf
    x[8, 10:13] = 1.0
    x[9] = low
    x[10] = torch.arange(V, device=DEV) // 250
    x[11] = -(torch.arange(V, device=DEV) // 250)
    x = x.to(dtype)
    tokens = i32([0, V - 1, 3, 5, 4321, 120, 77, 4, 11, 9, 4999, 0])
    for top in (0, 3, 32):
        o = _run(lib, x, tokens, top)
        _check(o, x, tokens, top)


def test_all_masked_and_tokens_outside(lib):
    x = torch.full((3, 300), -math.inf, device=DEV)
    x[1:] = torch.randn((2, 300), generator=gen(1), device=DEV)
    o = _run(lib, x, i32([5, -1, 300]), 4)
    assert (o["logprob"] == -math.inf).all() and o["entropy"][0] == 0 and torch.isfinite(o["entropy"][1:]).all()
    assert o["top_id"][0].tolist() == [0, 1, 2, 3] and (o["top_logprob"][0] == -math.inf).all()
    assert torch.equal(o["top_id"][1], x[1].topk(4).indices.int())


def test_parts_left_out(lib):
    """Each output by itself, unaligned rows, another stream."""
    base = torch.randn(4 * 501 + 1, generator=gen(1), device=DEV)
    x = base[1:].view(4, 501)
    tokens = i32([1, 2, 3, 4])
    full = _run(lib, x, tokens, 6)
    _check(full, x, tokens, 6)
    ws = torch.empty(lib.pldp_token_logprobs_workspace_size(4, 501), dtype=torch.uint8, device=DEV)
    ent, ids, lps = torch.zeros(4, device=DEV), i32([[0] * 6] * 4), torch.zeros((4, 6), device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    lib.pldp_token_logprobs(x, None, None, ws, entropy=ent, stream=s)
    lib.pldp_token_logprobs(x, None, None, ws, top_id=ids, stream=s)
    lib.pldp_token_logprobs(x, None, None, ws, top_logprob=lps, stream=s)
    s.synchronize()
    assert torch.equal(ent, full["entropy"]) and torch.equal(ids, full["top_id"]) and torch.equal(lps, full["top_logprob"])


def test_many_rows(lib):
    """Offsets past 2^32 bytes of logits."""
    x = torch.zeros((17000, 128256), device=DEV, dtype=torch.bfloat16)          # 4.4 GB
    x[16990:, 5] = 4
    x[16995, 100000] = 9
    tokens = torch.full((17000,), 5, dtype=torch.int32, device=DEV)
    o = _run(lib, x, tokens, 2)
    _check({k: v[16980:] for k, v in o.items()}, x[16980:], tokens[16980:], 2)
    assert (o["top_id"][:16990] == i32([0, 1])).all()


def test_refusals(lib):
    x = torch.zeros((2, 10), device=DEV)
    ws = torch.zeros(lib.pldp_token_logprobs_workspace_size(2, 10), dtype=torch.uint8, device=DEV)
    ok = dict(logits=x, tokens=i32([0, 0]), logprob=torch.zeros(2, device=DEV), workspace=ws)
    for bad, match in [(dict(logits=x[:, ::2]), "contiguous"), (dict(logits=x.half()), "dtype"), (dict(tokens=i32([0])), "tokens"),
                       (dict(top_id=i32([[0, 0]])), "top_id"), (dict(top_id=i32([[0, 0]] * 2), top_logprob=torch.zeros((2, 3), device=DEV)),
                                                              "same last")]:
        with pytest.raises(ValueError, match=match):
            lib.pldp_token_logprobs(**{**ok, **bad})
    for bad, match in [(dict(temperature=0.0), "temperature"), (dict(top_id=i32([[0] * 11] * 2)), "top"), (dict(logprob=None), "together"),
                       (dict(workspace=ws[:8]), "workspace")]:
        with pytest.raises(lib.PldpError, match=match):
            lib.pldp_token_logprobs(**{**ok, **bad})
