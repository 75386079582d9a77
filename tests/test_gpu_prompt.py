"""pldp_attend_prompt against causal softmax attention in 64 bits."""
import math

import pytest
import torch

from tests._cache import DEV, Cache, gen, i32

pytestmark = pytest.mark.gpu


def _rows(counts):
    rows = [0]
    for c in counts:
        rows.append(rows[-1] + c)
    return rows


def _queries(R, Hq, D, seed=7):
    return torch.randn((R, Hq, D), generator=gen(seed), device=DEV, dtype=torch.bfloat16)


def prompt64(c, q, rows, starts, scale, live=None):
    """out, lse, sum_j p_j |v_j|, the number of keys and the largest |v| of every row in 64 bits; `live`: by sequence, the
    positions that there are."""
    R, Hq, D = q.shape
    G = Hq // c.heads
    out = torch.zeros((R, Hq, D), dtype=torch.float64, device=DEV)
    size, most, lse = torch.zeros_like(out), torch.zeros((2, R, 1, 1), dtype=torch.float64, device=DEV), torch.full((R, Hq), -math.inf, dtype=torch.float64, device=DEV)
    for b, p in enumerate(starts):
        r0, r1 = rows[b], rows[b + 1]
        n = min(r1 - r0, c.ctx - p)
        if n <= 0:
            continue
        k, v = (c.dense[x][b][: p + n] for x in "kv")
        s = torch.einsum("rhgd,jhd->hgrj", q[r0:r0 + n].double().view(n, c.heads, G, D), k) * scale
        hidden = torch.arange(p + n, device=DEV) > p + torch.arange(n, device=DEV)[:, None]
        if live is not None and live[b] is not None:
            hidden = hidden | ~live[b][: p + n]
        s.masked_fill_(hidden, -math.inf)
        l = torch.logsumexp(s, -1)
        w = torch.exp(s - torch.where(l > -math.inf, l, 0)[..., None])
        lse[r0:r0 + n] = l.permute(2, 0, 1).reshape(n, Hq)
        out[r0:r0 + n] = torch.einsum("hgrj,jhd->rhgd", w, v).reshape(n, Hq, D)
        size[r0:r0 + n] = torch.einsum("hgrj,jhd->rhgd", w, v.abs()).reshape(n, Hq, D)
        most[0, r0:r0 + n], most[1, r0:r0 + n] = p + n, v.abs().max()
    return out, lse, size, most


def _run(lib, c, q, rows, starts, scale=None, ws=None, **kw):
    R, Hq, D = q.shape
    B = len(rows) - 1
    out = torch.full((R, Hq, D), 7.0, device=DEV, dtype=torch.bfloat16)
    lse = torch.full((R, Hq), 7.0, device=DEV)
    status = i32([0] * B)
    if ws is None:
        ws = torch.full((lib.pldp_attend_prompt_workspace_size(Hq, c.heads, D),), 255, dtype=torch.uint8, device=DEV)
    lib.pldp_attend_prompt(c.handle, q, i32(rows), out, ws, start=None if starts is None else i32(starts), lse=lse, scale=scale,
                           status=status, **kw)
    return out, lse, status.tolist()


def _check(out, lse, want, dtype="bf16"):
    """One rounding of the result to bf16 (half a step, 2^-8 of it), the rest but what follows in 32 bits: scores up to some
    tens, their sums of head_dim products.

    bf16: each weight is rounded to bf16, 2^-8 of what it weighs.
    e4m3: weights, the values' scales and the values are each rounded to f16, three times 2^-11.  Small ones are off by half
    of f16's smallest step instead, 2^-25: of weights w_j = 2^(x_j - m + 7), whose sum l is 2^7 at least (the key that m was
    set by), together by sum_j 2^-25 |v_j| / l <= n 2^-32 max |v|; scales and values are held in a unit of at most 8
    times the largest scale, which is max |v| / 448 at most: by 448 * 2^-25 * 8 / 448 max |v| = 2^-22 max |v|, and by 2^-30 max |v|."""
    o, l, size, most = want
    assert torch.equal(torch.isinf(lse), torch.isinf(l))
    live = torch.isfinite(l)
    assert ((lse.double() - l).abs()[live] <= 2e-5 * (1 + l.abs()[live])).all(), (lse.double() - l).abs()[live].max()
    err = (out.double() - o).abs()
    bound = 2 ** -8 * o.abs() + ((2 ** -8 if dtype == "bf16" else 3 * 2 ** -11) + 1e-5) * size
    if dtype == "e4m3":
        bound = bound + (2 ** -32 * most[0] + 2 ** -21) * most[1]
    assert (err <= bound).all(), (err - bound).max()
    assert (out[~live] == 0).all()


def _some(want, rows):
    return *(x[rows] for x in want[:3]), want[3][:, rows]


# counts, starts, q heads, heads, D, page
CASES = [
    ([1], [0], 1, 1, 64, 16),
    ([1], [0], 32, 8, 128, 16),
    ([47], [0], 32, 8, 128, 16),
    ([0, 1, 2, 127, 128, 129, 0, 255, 256, 257, 0], [0] * 11, 1, 1, 128, 16),
    ([0, 1, 2, 31, 33, 63, 65, 0], [5, 127, 126, 128, 100, 1, 0, 9], 8, 2, 64, 32),
    ([700, 3, 513], [0, 1000, 77], 5, 1, 128, 24),
    ([300, 90], [0, 31], 6, 2, 80, 7),
    ([130, 20], [3, 200], 16, 1, 112, 1),
    ([200, 90], [0, 60], 3, 3, 16, 100),
    ([300, 1, 129], [0, 500, 128], 8, 2, 256, 64),
    ([150, 33], [10, 0], 6, 2, 192, 16),
    ([9, 70], [100, 0], 131, 1, 48, 200),
    ([40], [4096], 8, 1, 128, 128),
]


@pytest.mark.parametrize("dtype,layout", [("bf16", "token"), ("e4m3", "token"), ("bf16", "head"), ("e4m3", "head")])
@pytest.mark.parametrize("case", CASES)
def test_attend_prompt(lib, case, dtype, layout):
    counts, starts, Hq, H, D, page = case
    lens = [a + b for a, b in zip(counts, starts)]
    c = Cache(lib, len(counts), max(lens), H, D, page, dtype, layout, lens=lens, seed=5)
    rows = _rows(counts)
    q = _queries(rows[-1], Hq, D)
    out, lse, status = _run(lib, c, q, rows, starts)
    assert status == [0] * len(counts)
    _check(out, lse, prompt64(c, q, rows, starts, D ** -0.5), dtype)
    again, _, _ = _run(lib, c, q, rows, starts)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,Hq,H", [(64, 8, 8), (128, 8, 2), (256, 4, 2)])
def test_many_tiles_a_cta(lib, D, Hq, H, dtype):
    """Far more tiles than the GPU has SMs: several units a CTA, every ring comes round several times."""
    counts, starts = [3300, 1, 2777, 1500, 64], [0, 700, 111, 2049, 6000]
    c = Cache(lib, 5, 6064, H, D, 64, dtype, lens=[a + b for a, b in zip(counts, starts)], seed=8)
    rows = _rows(counts)
    q = _queries(rows[-1], Hq, D)
    out, lse, status = _run(lib, c, q, rows, starts)
    assert status == [0] * 5
    _check(out, lse, prompt64(c, q, rows, starts, D ** -0.5), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_many_short_sequences(lib, dtype):
    B = 400
    counts, starts = [(37 * b) % 90 for b in range(B)], [(53 * b) % 200 for b in range(B)]
    c = Cache(lib, B, 290, 2, 64, 16, dtype, lens=[a + b for a, b in zip(counts, starts)], seed=2)
    rows = _rows(counts)
    q = _queries(rows[-1], 4, 64)
    out, lse, status = _run(lib, c, q, rows, starts)
    assert status == [0] * B
    _check(out, lse, prompt64(c, q, rows, starts, 0.125), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,Hq,H", [(64, 32, 16), (128, 32, 16), (256, 16, 16)])
def test_units_in_turn(lib, D, Hq, H, dtype):
    """Several units a CTA, of few tiles each, over and over: what a role finds of another one, which may be a tile ahead or not,
    is different every time, and the result is not."""
    counts, starts = [300] * 24, [7] * 24
    c, rows = Cache(lib, 24, 307, H, D, 16, dtype, seed=8), _rows(counts)
    q = _queries(rows[-1], Hq, D)
    first, lse, status = _run(lib, c, q, rows, starts)
    _check(first, lse, prompt64(c, q, rows, starts, D ** -0.5), dtype)
    for _ in range(30):
        out, again, status = _run(lib, c, q, rows, starts)
        assert status == [0] * 24 and torch.equal(out, first) and torch.equal(again, lse)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_peaked_and_growing_scores(lib, dtype):
    """Scores that grow along the context (each tile's maximum above the last, in the end by more than any lazy
    maximum may leave), a few that hold all the weight, large negative ones, and a scale of zero."""
    counts, starts, H, D = [700, 300], [0, 900], 2, 128
    c = Cache(lib, 2, 1200, H, D, 16, dtype, lens=[700, 1200], seed=9)
    rows = _rows(counts)
    q = _queries(1000, 4, D)
    for scale in (0.0, 0.5, 3.0, -3.0):
        out, lse, _ = _run(lib, c, q, rows, starts, scale=scale)
        _check(out, lse, prompt64(c, q, rows, starts, scale), dtype)
    if dtype == "bf16":
        pos = torch.arange(1200, device=DEV)
        base = q[800, 0].double()
        q[700:] = q[800, 0]
        for sign in (1, -1):
            k = (sign * base * (pos[:, None] / 1200 * 400 / base.square().sum())).bfloat16()[:, None].expand(-1, H, -1)
            c.dense["k"][1] = k.double()
            pg, slot = c.pages[1, pos // 16].long(), pos % 16
            c.pools["k"][pg, slot] = k
            out, lse, _ = _run(lib, c, q, rows, starts, scale=1.0)
            _check(out, lse, prompt64(c, q, rows, starts, 1.0), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_strides_and_streams(lib, dtype):
    """Queries and results as slices of larger tensors, on another stream, without lse and start."""
    counts, Hq, H, D = [150, 400], 8, 2, 64
    rows = _rows(counts)
    c = Cache(lib, 2, 410, H, D, 16, dtype, lens=counts, seed=5)
    big = _queries(rows[-1] + 3, Hq + 4, D)
    q = big[3:, 2:2 + Hq]
    want = prompt64(c, q, rows, [0, 0], D ** -0.5)
    room = torch.full((Hq + 1, rows[-1] + 2, D), -7.0, device=DEV, dtype=torch.bfloat16)
    out = room.transpose(0, 1)[1:1 + rows[-1], :Hq]
    ws = torch.zeros(lib.pldp_attend_prompt_workspace_size(Hq, H, D), dtype=torch.uint8, device=DEV)
    r = i32(rows)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        lib.pldp_attend_prompt(c.handle, q, r, out, ws)
    s.synchronize()
    _check(out, want[1].float(), want, dtype)
    assert (room[Hq] == -7).all() and (room[:, 0] == -7).all() and (room[:, rows[-1] + 1:] == -7).all()


# how a pool [pages, positions, heads, D] lies in memory: keys and values of a position side by side, of a head, and heads' positions
# with room behind them
def _side_by_side(k, v):
    both = torch.cat((k, v), 2)
    return both[:, :, : k.shape[2]], both[:, :, k.shape[2]:]


def _in_heads(k, v):
    both = torch.stack((k, v), 3)
    return both[:, :, :, 0], both[:, :, :, 1]


def _with_room(k, v):
    n, page, H, D = k.shape
    out = []
    for x in (k, v):
        room = torch.full((n, H, page + 8, D), float("nan"), device=DEV, dtype=torch.float32).to(x.dtype)
        room[:, :, :page] = x.permute(0, 2, 1, 3)
        out.append(room[:, :, :page].permute(0, 2, 1, 3))
    return out


@pytest.mark.parametrize("lie", [_side_by_side, _in_heads, _with_room])
@pytest.mark.parametrize("D,H,page", [(256, 2, 24), (256, 1, 8), (256, 2, 4), (256, 3, 64), (128, 2, 8), (256, 1, 512)])
def test_pools(lib, D, H, page, lie):
    """Keys and values in pools of other strides, and a page that is none."""
    counts, starts, Hq = [150, 33, 290], [10, 0, 200], 2 * H
    lens, rows = [a + b for a, b in zip(counts, starts)], _rows(counts)
    c = Cache(lib, 3, 512, H, D, page, lens=lens, seed=5)
    c.pools = dict(zip("kv", lie(c.pools["k"], c.pools["v"])))
    c.handle = lib.pldp_cache(c.pools["k"], c.pools["v"], c.pages)
    q = _queries(rows[-1], Hq, D)
    out, lse, status = _run(lib, c, q, rows, starts)
    assert status == [0] * 3
    _check(out, lse, prompt64(c, q, rows, starts, D ** -0.5))
    c.pages[2, 100 // page] = -1
    live = torch.arange(lens[2], device=DEV) // page != 100 // page
    out, lse, status = _run(lib, c, q, rows, starts)
    assert status == [0, 0, lib.PLDP_ST_PAGE]
    _check(out, lse, prompt64(c, q, rows, starts, D ** -0.5, live=[None, None, live]))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_status(lib, dtype):
    """Starts and rows out of range, the capacity, pages that are none, rows of no sequence."""
    D, S = 64, lib
    c = Cache(lib, 6, 192, 1, D, 16, dtype, lens=[192] * 6, seed=4)
    c.pages[4, 1] = -1
    c.pages[4, 5] = 99999
    c.pages[5] = -1
    starts, counts = [0, -1, 193, 185, 80, 3], [5, 4, 6, 20, 60, 4]
    rows = [2 + r for r in _rows(counts)]                          # rows 0, 1 and the last three are nobody's
    q = _queries(rows[-1] + 3, 2, D)
    out, lse, status = _run(lib, c, q, rows, starts)
    assert status == [0, S.PLDP_ST_SEQ_LEN, S.PLDP_ST_SEQ_LEN, S.PLDP_ST_CAPACITY, S.PLDP_ST_PAGE, S.PLDP_ST_PAGE]
    live = torch.ones(192, dtype=torch.bool, device=DEV)
    live[16:32] = live[80:96] = False
    eff = [0, 192, 192, 185, 80, 3]                                # (from the capacity on: nothing)
    want = prompt64(c, q, rows, eff, 0.125, [None] * 4 + [live, torch.zeros_like(live)])
    mine = slice(2, rows[-1])
    _check(out[mine], lse[mine], _some(want, mine), dtype)
    assert (out[:2] == 7).all() and (out[rows[-1]:] == 7).all() and (lse[rows[-1]:] == 7).all()
    # rows that descend, or pass the tensor
    out, lse, status = _run(lib, c, q, [0, 5, 3, 3, 3, 3, rows[-1] + 4], [0] * 6)
    assert status == [0, S.PLDP_ST_SEQ_LEN, 0, 0, 0, S.PLDP_ST_SEQ_LEN]
    want = prompt64(c, q, [0, 5], [0], 0.125)
    _check(out[:5], lse[:5], _some(want, slice(0, 5)), dtype)
    assert (out[5:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_memory_past_the_end_is_not_used(lib, dtype):
    """NaN and infinity in unwritten positions of the last page (these tests' pools hold NaN in all unused memory),
    at sequence ends in every place of a tile."""
    for L in (1, 15, 17, 127, 130, 200):
        c = Cache(lib, 1, 256, 1, 64, 64, dtype, lens=[L])
        if dtype == "bf16":
            c = Cache(lib, 1, 256, 1, 64, 64, dtype, lens=[256], seed=3)
            p = torch.arange(L, 256, device=DEV)
            pg, slot = c.pages[0, p // 64].long(), p % 64
            c.pools["k"][pg, slot], c.pools["v"][pg, slot] = math.inf, -math.inf
        q = _queries(L, 2, 64)
        out, lse, _ = _run(lib, c, q, [0, L], None)
        _check(out, lse, prompt64(c, q, [0, L], [0], 0.125), dtype)


def test_long_offsets(lib):
    """Pages beyond 2^32 bytes into the pool."""
    n, page, H, D = 9000, 128, 8, 256
    pool = torch.zeros((n, page, H, D), device=DEV, dtype=torch.bfloat16)
    x = torch.randn((2, page, H, D), generator=gen(1), device=DEV, dtype=torch.bfloat16)
    pool[n - 1], pool[n - 2] = x[0], x[1]
    small = Cache(None, 1, 2 * page, H, D, page)
    small.dense = {"k": [x.reshape(-1, H, D).double()], "v": [x.reshape(-1, H, D).double()]}
    small.handle = lib.pldp_cache(pool, pool, i32([[n - 1, n - 2]]))
    q = _queries(200, H, D)
    out, lse, _ = _run(lib, small, q, [0, 200], None)
    _check(out, lse, prompt64(small, q, [0, 200], [0], D ** -0.5))


def test_two_at_once(lib):
    """Calls on two streams, each with a workspace of its own, while the other's run."""
    calls = []
    for seed, (counts, starts, Hq, H, D, dtype) in enumerate([([900, 40, 1300], [0, 700, 5], 8, 2, 128, "bf16"), ([700] * 9, [3] * 9, 4, 4, 64, "e4m3")]):
        rows = _rows(counts)
        c = Cache(lib, len(counts), max(a + b for a, b in zip(counts, starts)), H, D, 16, dtype, lens=[a + b for a, b in zip(counts, starts)], seed=seed)
        q, r, st = _queries(rows[-1], Hq, D, seed), i32(rows), i32(starts)
        ws = torch.empty(lib.pldp_attend_prompt_workspace_size(Hq, H, D), dtype=torch.uint8, device=DEV)
        outs = [torch.zeros_like(q) for _ in range(12)]
        _check(*_run(lib, c, q, rows, starts)[:2], prompt64(c, q, rows, starts, D ** -0.5), dtype)
        calls.append((c, q, r, st, ws, outs, _run(lib, c, q, rows, starts)[0], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for i in range(12):
        for c, q, r, st, ws, outs, _, stream in calls:
            with torch.cuda.stream(stream):
                lib.pldp_attend_prompt(c.handle, q, r, outs[i], ws, start=st)
    torch.cuda.synchronize()
    for *_, outs, want, _ in calls:
        assert all(torch.equal(x, want) for x in outs)


def test_graph_replay_and_one_workspace(lib):
    """Captured once, replayed on other rows and starts; calls of other shapes on the same workspace between."""
    H, D, R = 2, 64, 700
    c = Cache(lib, 2, 900, H, D, 16, lens=[900, 900], seed=6)
    other = Cache(lib, 1, 3000, 1, 128, 16, "e4m3", lens=[3000], seed=6)
    q, q2 = _queries(R, 4, D), _queries(2500, 4, 128)
    out, lse = torch.empty((R, 4, D), device=DEV, dtype=torch.bfloat16), torch.empty((R, 4), device=DEV)
    ws = torch.zeros(lib.pldp_attend_prompt_workspace_size(4, 1, 128), dtype=torch.uint8, device=DEV)
    rows, start = i32([0, 100, 400]), i32([0, 0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        lib.pldp_attend_prompt(c.handle, q, rows, out, ws, start=start, lse=lse)
    for r, p in (([0, 100, 400], [0, 0]), ([0, 0, 700], [5, 200]), ([300, 301, 302], [899, 0])):
        rows.copy_(i32(r))
        start.copy_(i32(p))
        _run(lib, other, q2, [0, 2500], [500], ws=ws)
        g.replay()
        torch.cuda.synchronize()
        live = slice(r[0], r[-1])
        _check(out[live], lse[live], _some(prompt64(c, q, r, p, D ** -0.5), live))


def test_a_step_is_the_same_as_a_prompt(lib):
    """The rows of a step by pldp_attend_cache, and the same positions as a chunk of a prompt."""
    L, n, Hq, H, D = [300, 40], 7, 8, 2, 128
    c = Cache(lib, 2, 310, H, D, 16, lens=[a + n - 1 for a in L], seed=6)
    q = _queries(2 * n, Hq, D)
    out, lse, _ = _run(lib, c, q, [0, n, 2 * n], [a - 1 for a in L])
    step, step_lse = torch.empty((2, n, Hq, D), device=DEV, dtype=torch.bfloat16), torch.empty((2, n, Hq), device=DEV)
    ws = torch.zeros(lib.pldp_attend_workspace_size(2, n, Hq, H, D), dtype=torch.uint8, device=DEV)
    lib.pldp_attend_cache(c.handle, q.view(2, n, Hq, D), i32(L), step, ws, lse=step_lse)
    want = prompt64(c, q, [0, n, 2 * n], [a - 1 for a in L], D ** -0.5)
    _check(out, lse, want)
    _check(step.view(2 * n, Hq, D), step_lse.view(2 * n, Hq), want)


def test_refusals(lib):
    c = Cache(lib, 2, 64, 2, 64, 16)
    q = torch.zeros((6, 4, 64), device=DEV, dtype=torch.bfloat16)
    ws = torch.zeros(lib.pldp_attend_prompt_workspace_size(4, 2, 64) + 256, dtype=torch.uint8, device=DEV)
    ok = dict(cache=c.handle, q=q, rows=i32([0, 3, 6]), out=torch.empty_like(q), workspace=ws)
    for bad, match in [(dict(q=q.float()), "bfloat16"), (dict(out=q[:2]), "shape"), (dict(rows=i32([0, 1, 2, 3])), "page table"),
                       (dict(rows=i32([[0, 6]])), "rows"), (dict(lse=torch.zeros(23, device=DEV)), "lse"), (dict(q=q[..., ::2]), "unit inner"),
                       (dict(start=i32([0])), "start"), (dict(cache=None), "pldp_cache"), (dict(status=i32([0])), "status")]:
        with pytest.raises(ValueError, match=match):
            lib.pldp_attend_prompt(**{**ok, **bad})
    three = torch.zeros((6, 3, 64), device=DEV, dtype=torch.bfloat16)
    odd = torch.zeros((6, 4, 68), device=DEV, dtype=torch.bfloat16)[..., 4:]
    for bad, match in [(dict(q=three, out=three), "multiple"), (dict(q=odd), "16"), (dict(scale=float("nan")), "scale"),
                       (dict(workspace=ws[:16]), "workspace"), (dict(workspace=ws[16:]), "aligned")]:
        with pytest.raises(lib.PldpError, match=match):
            lib.pldp_attend_prompt(**{**ok, **bad})
    assert lib.pldp_attend_prompt_workspace_size(5, 2, 64) == 0
    lib.pldp_attend_prompt(**{**ok, "rows": i32([0])})             # no sequences
    lib.pldp_attend_prompt(**{**ok, "rows": i32([0, 0, 0]), "q": q[:0], "out": q[:0]})
