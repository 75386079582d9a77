"""pldp_rank_cache (Eq. 2 from the cache) against the attention probabilities in 64 bits, and
against pldp_rank_attention on the written-out rows."""
import math

import pytest
import torch

from tests._cache import DEV, Cache, attend64, gen, i32

pytestmark = pytest.mark.gpu


def _setup(lib, L, n, Hq, H, D, page, dtype, seed=5):
    c = Cache(lib, len(L), max(L) + n, H, D, page, dtype, lens=[a + n - 1 for a in L], seed=seed)
    q = torch.randn((len(L), n, Hq, D), generator=gen(seed + 1), device=DEV, dtype=torch.bfloat16)
    lse = attend64(c, q, L, [n - 1] * len(L), D ** -0.5, H)[1]
    return c, q, lse


def _scores64(c, q, lse, row, cand, heads, G, scale, agg):
    """Probabilities of one row at the candidates: [candidates]."""
    k = c.dense["k"]
    out = []
    for b, js in enumerate(cand):
        i = row[b]
        p = torch.stack([torch.exp(k[b][js, h // G] @ q[b, i, h].double() * scale - lse[b, i, h]) for h in heads])
        out.append(p.amax(0) if agg == "max" else p.sum(0))
    return out


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("agg", ["max", "sum"])
@pytest.mark.parametrize("Hq,H,D,page,sel,C", [(32, 8, 128, 16, None, 40), (32, 8, 128, 24, 8, 600), (6, 2, 80, 7, 3, 5),
                                               (4, 4, 256, 64, None, 70), (8, 1, 64, 1, 5, 33), (5, 1, 16, 32, 1, 1),
                                               (40, 8, 128, 64, None, 130)])
def test_scores(lib, dtype, agg, Hq, H, D, page, sel, C):
    L, n = [700, 130, 1, 2000], 5
    c, q, lse64 = _setup(lib, L, n, Hq, H, D, page, dtype)
    row = [0, 4, 2, 3]
    kv = [a + r for a, r in zip(L, row)]
    g = gen(11)
    heads = list(range(Hq)) if sel is None else torch.randperm(Hq, generator=g, device=DEV)[:sel].tolist()
    cand = [torch.randperm(kv[b], generator=g, device=DEV)[: max(1, C - 3 * b)].sort().values for b in range(4)]
    pos = torch.full((4, C), -1, dtype=torch.int32, device=DEV)
    for b, js in enumerate(cand):
        pos[b, : len(js)] = js
    scores = torch.full((4, C), -7.0, device=DEV)
    best, best_score, status = i32([0] * 4), torch.zeros(4, device=DEV), i32([0] * 4)
    args = (c.handle, q, i32(row), i32(kv), lse64.float(), pos, i32([len(x) for x in cand]), best)
    kw = dict(heads=None if sel is None else i32(heads), agg=agg, status=status)
    lib.pldp_rank_cache(*args, scores=scores, best_score=best_score, **kw)
    assert status.tolist() == [0] * 4
    want = _scores64(c, q, lse64, row, cand, heads, Hq // H, D ** -0.5, agg)
    for b, w in enumerate(want):
        m = len(w)
        # 32-bit scores of up to some tens: their rounding is the exponential's relative error
        assert ((scores[b, :m].double() - w).abs() <= 3e-5 * w).all()
        assert (scores[b, m:] == -7).all()
        top = int(scores[b, :m].argmax())
        assert int(best[b]) == int(cand[b][top]) and float(best_score[b]) == float(scores[b, top])
    # another layer's scores: the larger of both, or their sum
    other = torch.rand((4, C), generator=g, device=DEV) * 0.01
    both = other.clone()
    lib.pldp_rank_cache(*args, scores=both, accumulate=True, **kw)
    for b, w in enumerate(want):
        m = len(w)
        now = torch.maximum(scores[b, :m], other[b, :m]) if agg == "max" else scores[b, :m] + other[b, :m]
        assert torch.equal(both[b, :m], now) and torch.equal(both[b, m:], other[b, m:])
        assert int(best[b]) == int(cand[b][int(now.argmax())])


def test_against_the_written_rows(lib):
    """The ranking of pldp_rank_attention on the same row's probabilities."""
    L, n, Hq, H, D = [900, 300], 3, 8, 2, 64
    c, q, lse = _setup(lib, L, n, Hq, H, D, 16, "bf16")
    kv, row = [901, 302], [1, 2]
    A = torch.zeros((2, Hq, 1024), device=DEV)
    for b in range(2):
        k = c.dense["k"][b][: kv[b]].repeat_interleave(4, 1)
        A[b, :, : kv[b]] = torch.exp(torch.einsum("hd,jhd->hj", q[b, row[b]].double(), k) / 8 - lse[b, row[b], :, None]).float()
    pos = torch.stack([torch.arange(3, 300, 9, device=DEV), torch.arange(0, 297, 9, device=DEV)]).int()
    cnt = i32([33, 33])
    a, b, s = i32([0, 0]), i32([0, 0]), torch.zeros(2, device=DEV)
    lib.pldp_rank_attention(A, i32([x + 1 for x in kv]), pos, cnt, a, best_score=s)
    s2 = torch.zeros(2, device=DEV)
    lib.pldp_rank_cache(c.handle, q, i32(row), i32(kv), lse.float(), pos, cnt, b, best_score=s2)
    assert a.tolist() == b.tolist() and ((s - s2).abs() <= 3e-5 * s).all()


def test_edges(lib):
    """No candidates, ones outside the context, rows, lengths, heads and pages that are none, ties,
    and rows without attention."""
    B, n, D = 8, 2, 32
    c, q, lse = _setup(lib, [50] * B, n, 2, 1, D, 16, "bf16")
    lse = lse.float()
    lse[6] = -math.inf
    c.pages[7, 1] = -1
    c.pools["k"][c.pages[5, 1].long(), 3] = c.pools["k"][c.pages[5, 0].long(), 9]
    c.pools["k"][c.pages[5, 1].long(), 7] = c.pools["k"][c.pages[5, 0].long(), 9]
    pos = i32([[3, 60, -1, 20]] * B)
    pos[5] = i32([9, 19, 23, 9])
    row, kv = [0, 2, -1, 0, 0, 0, 0, 0], [50, 50, 50, 1000, -1, 50, 50, 50]
    cnt = i32([0, 4, 4, 4, 4, 3, 4, 99])
    scores, best, bs, st = torch.full((B, 4), -7.0, device=DEV), i32([9] * B), torch.zeros(B, device=DEV), i32([0] * B)
    lib.pldp_rank_cache(c.handle, q, i32(row), i32(kv), lse, pos, cnt, best, scores=scores, best_score=bs, status=st)
    S = lib
    assert st.tolist() == [0, S.PLDP_ST_ROW_INDEX, S.PLDP_ST_ROW_INDEX, S.PLDP_ST_SEQ_LEN, S.PLDP_ST_SEQ_LEN, 0, 0, S.PLDP_ST_PAGE]
    assert best.tolist()[:5] == [-1] * 5 and (bs[:5] == -math.inf).all()
    assert (scores[0] == -7).all() and (scores[1:5] == -math.inf).all()
    assert int(best[5]) == 9 and scores[5, 0] == scores[5, 1] == scores[5, 2] and scores[5, 3] == -7
    assert scores[6].tolist() == [0, -math.inf, -math.inf, 0] and int(best[6]) == 3
    assert scores[7, 0] > 0 and (scores[7, 1:] == -math.inf).all() and int(best[7]) == 3
    st.zero_()
    lib.pldp_rank_cache(c.handle, q, None, i32([50] * B), lse, pos, cnt, best, heads=i32([2, 1, -1]), scores=scores, status=st)
    assert st.tolist()[:7] == [S.PLDP_ST_ROW_INDEX] * 7
    one = scores.clone()
    lib.pldp_rank_cache(c.handle, q, None, i32([50] * B), lse, pos, cnt, best, heads=i32([1]), scores=one)
    assert torch.equal(one, scores)


def test_refusals(lib):
    c = Cache(lib, 2, 64, 2, 64, 16)
    q = torch.zeros((2, 3, 4, 64), device=DEV, dtype=torch.bfloat16)
    ok = dict(cache=c.handle, q=q, row=None, kv_len=i32([1, 1]), lse=torch.zeros((2, 3, 4), device=DEV),
              cand_pos=i32([[0, 1]] * 2), cand_count=i32([1, 1]), best_pos=i32([0, 0]))
    for bad, match in [(dict(lse=torch.zeros((2, 3, 3), device=DEV)), "lse"), (dict(cand_pos=i32([[0]])), "cand_pos"),
                       (dict(scores=torch.zeros((2, 1), device=DEV)), "scores"), (dict(kv_len=None), "kv_len"),
                       (dict(heads=torch.zeros(2, device=DEV)), "heads"), (dict(best_pos=i32([0])), "best_pos")]:
        with pytest.raises(ValueError, match=match):
            lib.pldp_rank_cache(**{**ok, **bad})
    for bad, match in [(dict(accumulate=True), "accumulate"), (dict(agg=3), "agg"), (dict(heads=i32([])), "n_sel"),
                       (dict(scale=float("inf")), "scale"), (dict(heads=i32([0] * 769)), "n_sel")]:
        with pytest.raises(lib.PldpError, match=match):
            lib.pldp_rank_cache(**{**ok, **bad})


@pytest.mark.parametrize("dtype,D,H,Hq,sel", [("bf16", 16, 1024, 1024, None), ("e4m3", 16, 64, 128, 3072), ("bf16", 256, 4, 48, 192),
                                             ("e4m3", 48, 5, 10, 1024)])
def test_many_heads(lib, dtype, D, H, Hq, sel):
    """As many key/value heads, and as many selected entries, as there may be; repeated ones among them."""
    L = [90, 33]
    c = Cache(lib, 2, 96, H, D, 16, dtype, lens=L, seed=3)
    g = gen(4)
    q = torch.randn((2, 1, Hq, D), generator=g, device=DEV, dtype=torch.bfloat16)
    lse = torch.full((2, 1, Hq), 3.0, device=DEV)
    heads = None if sel is None else torch.randint(0, Hq, (sel,), generator=g, device=DEV, dtype=torch.int32)
    cand = [torch.randperm(n, generator=g, device=DEV)[:20].sort().values for n in L]
    pos, best = torch.stack(cand).int(), i32([0, 0])
    for agg in ("max", "sum"):
        scores = torch.zeros((2, 20), device=DEV)
        lib.pldp_rank_cache(c.handle, q, None, i32(L), lse, pos, i32([20, 20]), best, heads=heads, agg=agg, scores=scores)
        for b in range(2):
            k = c.dense["k"][b][cand[b]].repeat_interleave(Hq // H, 1)
            p = torch.exp(torch.einsum("hd,jhd->hj", q[b, 0].double(), k) * D ** -0.5 - 3.0)
            p = p if heads is None else p[heads.long()]
            want = p.amax(0) if agg == "max" else p.sum(0)
            # sums of up to 3072 positive terms in 32 bits, in a fixed order: 2^-24 each of what has been added up
            assert ((scores[b].double() - want).abs() <= 2e-4 * want).all()
