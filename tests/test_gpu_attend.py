"""pldp_attend_cache against softmax attention in 64 bits."""
import math

import pytest
import torch

from tests._cache import DEV, Cache, attend64, gen, i32

pytestmark = pytest.mark.gpu


def _run(lib, c, q, L, d, scale=None, ws=None, **kw):
    B, n, Hq, D = q.shape
    out = torch.full((B, n, Hq, D), float("nan"), device=DEV, dtype=torch.bfloat16)
    lse = torch.full((B, n, Hq), float("nan"), device=DEV)
    status = i32([0] * B)
    if ws is None:
        ws = torch.zeros(lib.pldp_attend_workspace_size(B, n, Hq, c.heads, D), dtype=torch.uint8, device=DEV)
    lib.pldp_attend_cache(c.handle, q, i32(L), out, ws, draft_len=None if d is None else i32(d), lse=lse, scale=scale,
                          status=status, **kw)
    return out, lse, status.tolist()


def _check(out, lse, want):
    """One rounding of the result to bf16 (2^-9), each weight rounded to 16 bits (at worst 2^-9 of
    what it weighs), the rest in 32 bits: scores up to some tens, their sums of head_dim products."""
    o, l, size = want
    assert torch.equal(torch.isinf(lse), torch.isinf(l))
    live = torch.isfinite(l)
    assert ((lse.double() - l).abs()[live] <= 2e-5 * (1 + l.abs()[live])).all(), (lse.double() - l).abs()[live].max()
    err = (out.double() - o).abs()
    bound = 2 ** -9 * 1.01 * (o.abs() + size) + 1e-5 * size
    assert (err <= bound).all(), (err - bound).max()
    assert (out[~live] == 0).all()


def _queries(B, n, Hq, D, seed=7):
    return torch.randn((B, n, Hq, D), generator=gen(seed), device=DEV, dtype=torch.bfloat16)


# lengths (with x_t), n, q heads, heads, D, page
CASES = [
    ([1], 1, 1, 1, 64, 16),
    ([1, 2, 127, 128, 129, 255, 256, 257], 1, 8, 2, 128, 16),
    ([1, 2, 127, 128, 129, 255, 256, 257], 4, 8, 2, 64, 16),
    ([700, 3, 1500], 11, 32, 8, 128, 32),
    ([530, 121, 1999], 17, 40, 8, 128, 24),
    ([300, 5000], 13, 6, 2, 80, 7),
    ([64, 4097], 2, 16, 1, 112, 1),
    ([333, 90], 5, 3, 3, 16, 100),
    ([700, 1], 3, 8, 2, 256, 64),
    ([200, 77], 33, 8, 1, 128, 128),
    ([40000], 1, 8, 1, 128, 64),
    ([9000, 128, 30], 12, 4, 4, 192, 16),
]


@pytest.mark.parametrize("dtype,layout", [("bf16", "token"), ("e4m3", "token"), ("bf16", "head"), ("e4m3", "head")])
@pytest.mark.parametrize("case", CASES)
def test_attend(lib, case, dtype, layout):
    L, n, Hq, H, D, page = case
    d = [n - 1 if b % 3 != 1 else (n - 1) // 2 for b in range(len(L))]
    c = Cache(lib, len(L), max(L) + n, H, D, page, dtype, layout, lens=[a + b for a, b in zip(L, d)], seed=5)
    q = _queries(len(L), n, Hq, D)
    out, lse, status = _run(lib, c, q, L, d)
    assert status == [0] * len(L)
    _check(out, lse, attend64(c, q, L, d, D ** -0.5, H))


# n, q heads a key/value head: 16, 32, 52, 85 and 99 query rows
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,n,G", [(D, n, G) for D in (64, 128, 256) for n, G in ((4, 4), (8, 4), (13, 4), (17, 5), (33, 3))
                                   if D < 256 or n < 33])
def test_many_tiles_a_cta(lib, D, n, G, dtype):
    """Far more tiles of keys than the GPU has SMs: every ring comes round several times."""
    L, H = [3300, 3171, 2900, 3500], 16
    c = Cache(lib, 4, 3600, H, D, 64, dtype, lens=[a + n - 1 for a in L], seed=8)
    q = _queries(4, n, H * G, D)
    out, lse, status = _run(lib, c, q, L, None)
    assert status == [0] * 4
    _check(out, lse, attend64(c, q, L, [n - 1] * 4, D ** -0.5, H))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_many_short_sequences(lib, dtype):
    """More units of work than the GPU has SMs, empty sequences among them; twice on one workspace."""
    B = 300
    L = [(37 * b) % 300 for b in range(B)]
    c = Cache(lib, B, 304, 2, 64, 16, dtype, lens=[a + 2 if a else 0 for a in L], seed=2)
    q = _queries(B, 3, 4, 64)
    ws = torch.zeros(lib.pldp_attend_workspace_size(B, 3, 4, 2, 64), dtype=torch.uint8, device=DEV)
    want = attend64(c, q, L, [2] * B, 0.125, 2)
    first = None
    for _ in range(2):
        out, lse, status = _run(lib, c, q, L, None, ws=ws)
        assert status == [0] * B
        _check(out, lse, want)
        assert first is None or torch.equal(first, out)          # the same inputs, the same bits
        first = out


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_peaked_and_growing_scores(lib, dtype):
    """Scores that grow along the context (each tile's maximum above the last), a few that
    hold all the weight, large negative ones, and a scale of zero."""
    L, H, D = [2000, 700], 2, 128
    c = Cache(lib, 2, 2010, H, D, 16, dtype, lens=[2004, 704], seed=9, spread=1.0)
    q = _queries(2, 5, 4, D)
    for scale in (0.0, 0.5, 3.0, -3.0):
        out, lse, _ = _run(lib, c, q, L, None, scale=scale)
        _check(out, lse, attend64(c, q, L, [4, 4], scale, H))
    if dtype == "bf16":
        pos = torch.arange(2004, device=DEV)
        base = q[0, 0, 0].double()
        for sign in (1, -1):
            k = (sign * base * (pos[:, None] / 2004 * 60 / base.square().sum())).bfloat16()[:, None].expand(-1, H, -1)
            c.dense["k"][0] = k.double()
            pg, slot = c.pages[0, pos // 16].long(), pos % 16
            c.pools["k"][pg, slot] = k
            out, lse, _ = _run(lib, c, q, L, None, scale=1.0)
            _check(out, lse, attend64(c, q, L, [4, 4], 1.0, H))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_strides_and_streams(lib, dtype):
    """Queries and results as slices of larger tensors, on another stream, without lse."""
    L, n, Hq, H, D = [150, 400], 3, 8, 2, 64
    c = Cache(lib, 2, 410, H, D, 16, dtype, lens=[152, 402], seed=5)
    big = _queries(2, n + 1, Hq + 4, D)
    q = big[:, 1:, 2:2 + Hq]
    want = attend64(c, q, L, [2, 2], D ** -0.5, H)
    room = torch.full((2, Hq + 1, n + 2, D), -7.0, device=DEV, dtype=torch.bfloat16)
    out = room.transpose(1, 2)[:, 1:1 + n, :Hq]
    s = torch.cuda.Stream()
    ws = torch.zeros(lib.pldp_attend_workspace_size(2, n, Hq, H, D), dtype=torch.uint8, device=DEV)
    Lt = i32(L)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        lib.pldp_attend_cache(c.handle, q, Lt, out, ws)
    s.synchronize()
    _check(out, want[1].float(), want)
    assert (room[:, Hq] == -7).all() and (room[:, :, 0] == -7).all() and (room[:, :, n + 1:] == -7).all()


def test_status(lib):
    """Rows with nothing to attend to, lengths, drafts, capacity, and pages that are none."""
    B, n, D = 7, 4, 64
    c = Cache(lib, B, 192, 1, D, 16, lens=[192] * B, seed=4)
    L, d = [0, -1, 193, 190, 10, 100, 40], [3, 3, 3, 3, 9, -1, 0]
    c.pages[6, 1] = -1
    q = _queries(B, n, 2, D)
    out, lse, status = _run(lib, c, q, L, d)
    S = lib
    assert status == [0, S.PLDP_ST_SEQ_LEN, S.PLDP_ST_SEQ_LEN, S.PLDP_ST_CAPACITY, S.PLDP_ST_DRAFT_LEN, S.PLDP_ST_DRAFT_LEN,
                      S.PLDP_ST_PAGE]
    eff_L, eff_d = [0, 0, 0, 190, 10, 100, 24], [0, 0, 0, 2, 3, 0, 0]
    for x in "kv":                                                # sequence 6 without its second page
        c.dense[x][6] = torch.cat([c.dense[x][6][:16], c.dense[x][6][32:40]])
    _check(out, lse, attend64(c, q, eff_L, eff_d, 0.125, 1))
    c.pages[6] = -1                                               # and without any
    out, lse, status = _run(lib, c, q, L, d)
    assert status[6] == S.PLDP_ST_PAGE and (out[6] == 0).all() and (lse[6] == -math.inf).all()


def test_memory_past_the_end_is_not_used(lib):
    """NaN and infinity in unwritten positions of the last page and in other pages' memory
    (the pools of these tests hold NaN there), and a whole pool of them beyond one token."""
    c = Cache(lib, 1, 64, 1, 64, 64, lens=[1])
    c.pools["k"][c.pages[0, 0].long(), 1:] = math.inf
    c.pools["v"][c.pages[0, 0].long(), 1:] = -math.inf
    q = _queries(1, 1, 2, 64)
    out, lse, _ = _run(lib, c, q, [1], None)
    assert torch.equal(out[0, 0, 0].double(), c.dense["v"][0][0, 0]) and torch.equal(out[0, 0, 1], out[0, 0, 0])


def test_long_offsets(lib):
    """Pages beyond 2^32 bytes into the pool."""
    n, page, H, D = 9000, 128, 8, 256
    pool = torch.zeros((n, page, H, D), device=DEV, dtype=torch.bfloat16)
    x = torch.randn((2, page, H, D), generator=gen(1), device=DEV, dtype=torch.bfloat16)
    pool[n - 1], pool[n - 2] = x[0], x[1]
    small = Cache(None, 1, 2 * page, H, D, page)
    small.dense = {"k": [x.reshape(-1, H, D).double()], "v": [x.reshape(-1, H, D).double()]}
    small.handle = lib.pldp_cache(pool, pool, i32([[n - 1, n - 2]]))
    q = _queries(1, 2, H, D)
    out, lse, _ = _run(lib, small, q, [200], None)
    _check(out, lse, attend64(small, q, [200], [1], D ** -0.5, H))


def test_graph_replay(lib):
    """Captured once, replayed on other lengths."""
    L, n, H, D = [300, 40], 2, 2, 64
    c = Cache(lib, 2, 600, H, D, 16, lens=[600, 600], seed=6)
    q = _queries(2, n, 4, D)
    out, lse = torch.empty((2, n, 4, D), device=DEV, dtype=torch.bfloat16), torch.empty((2, n, 4), device=DEV)
    ws = torch.zeros(lib.pldp_attend_workspace_size(2, n, 4, H, D), dtype=torch.uint8, device=DEV)
    Lt = i32(L)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        lib.pldp_attend_cache(c.handle, q, Lt, out, ws, lse=lse)
    for now in (L, [599, 1], [128, 0]):
        Lt.copy_(i32(now))
        g.replay()
        torch.cuda.synchronize()
        _check(out, lse, attend64(c, q, now, [1, 1], D ** -0.5, H))


def test_refusals(lib):
    c = Cache(lib, 2, 64, 2, 64, 16)
    q = torch.zeros((2, 3, 4, 64), device=DEV, dtype=torch.bfloat16)
    ws = torch.zeros(lib.pldp_attend_workspace_size(2, 3, 4, 2, 64), dtype=torch.uint8, device=DEV)
    ok = dict(cache=c.handle, q=q, seq_len=i32([1, 1]), out=torch.empty_like(q), workspace=ws)
    for bad, match in [(dict(q=q.float()), "bfloat16"), (dict(out=q[:, :2]), "shape"), (dict(seq_len=i32([1])), "seq_len"),
                       (dict(lse=torch.zeros(23, device=DEV)), "lse"), (dict(q=q[..., ::2]), "unit inner"),
                       (dict(draft_len=i32([0])), "draft_len"), (dict(cache=None), "pldp_cache")]:
        with pytest.raises(ValueError, match=match):
            lib.pldp_attend_cache(**{**ok, **bad})
    three = torch.zeros((2, 3, 3, 64), device=DEV, dtype=torch.bfloat16)
    odd = torch.zeros((2, 3, 4, 68), device=DEV, dtype=torch.bfloat16)[..., 4:]
    for bad, match in [(dict(q=three, out=three), "multiple"), (dict(q=odd), "16"), (dict(scale=float("nan")), "scale"),
                       (dict(workspace=ws[:16]), "workspace"), (dict(workspace=torch.zeros(ws.numel() + 16, dtype=torch.uint8,
                                                                                          device=DEV)[16:]), "aligned")]:
        with pytest.raises(lib.PldpError, match=match):
            lib.pldp_attend_cache(**{**ok, **bad})
    assert lib.pldp_attend_workspace_size(2, 3, 5, 2, 64) == 0
