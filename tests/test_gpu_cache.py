"""pldp_cache_append and pldp_cache_read against the definitions in 64 bits."""
import pytest
import torch

from tests._cache import DEV, Cache, gen, i32

pytestmark = pytest.mark.gpu


def _rotate64(x, cos, sin, rot, inter):
    even, odd = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
    y = x.clone()
    y[..., even] = x[..., even] * cos - x[..., odd] * sin
    y[..., odd] = x[..., odd] * cos + x[..., even] * sin
    return y


def _table(rows, rot, seed):
    a = torch.rand((rows, rot // 2), generator=gen(seed), device=DEV, dtype=torch.float64) * 6.28
    return a.cos().float(), a.sin().float()


# B, n, q heads, heads, D, page, input, cache, layout, rot, interleaved, norms
CASES = [
    (1, 1, 1, 1, 16, 1, "f32", "bf16", "token", 0, False, False),
    (3, 11, 32, 8, 128, 16, "bf16", "bf16", "token", 128, False, True),
    (3, 11, 32, 8, 128, 16, "bf16", "e4m3", "head", 128, True, True),
    (4, 5, 6, 2, 80, 24, "f32", "e4m3", "token", 40, False, True),
    (4, 5, 6, 2, 80, 24, "f32", "bf16", "head", 80, True, False),
    (2, 3, 3, 3, 64, 7, "bf16", "e4m3", "token", 64, False, False),
    (2, 3, 5, 1, 256, 32, "f32", "e4m3", "head", 34, False, True),
    (2, 300, 8, 8, 48, 64, "bf16", "bf16", "token", 2, True, True),
    (5, 2, 16, 16, 112, 128, "bf16", "e4m3", "head", 112, False, True),
]


@pytest.mark.parametrize("case", CASES)
def test_append(lib, case):
    B, n, Hq, H, D, page, inp, dtype, layout, rot, inter, norms = case
    ctx = n + 40
    L = [1 + (7 * b) % 37 for b in range(B)]
    d = [n - 1 if b % 2 == 0 else n // 3 for b in range(B)]
    c = Cache(lib, B, ctx, H, D, page, dtype, layout, lens=[a + m for a, m in zip(L, d)], seed=1, fill=False)
    kind = torch.float32 if inp == "f32" else torch.bfloat16
    qkv = torch.randn((B, n, Hq + 2 * H, D), generator=gen(2), device=DEV, dtype=kind) * 3
    qkv[0, 0, Hq] = 0                                             # a key of zeros
    qkv[0, 0, Hq + H] = 0
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
    w = [(1 + 0.2 * torch.randn(D, generator=gen(3 + i), device=DEV)).to(kind) if norms else None for i in range(2)]
    cos, sin = _table(ctx, rot, 5) if rot else (None, None)
    q_out = torch.full((B, n, Hq, D), -7.0, device=DEV, dtype=torch.bfloat16)
    before = {x: c.pools[x].clone() for x in "kv"}
    status = i32([0] * B)
    lib.pldp_cache_append(c.handle, q, k, v, i32(L), q_out, draft_len=i32(d), q_norm=w[0], k_norm=w[1], eps=1e-5, cos=cos,
                          sin=sin, interleaved=inter, status=status)
    assert status.tolist() == [0] * B
    written = torch.zeros(c.pools["k"].shape[:2], dtype=torch.bool, device=DEV)
    for b in range(B):
        m, p0 = d[b] + 1, L[b] - 1
        assert (q_out[b, m:] == -7).all()
        pos = torch.arange(p0, p0 + m, device=DEV)
        written[c.pages[b, pos // page].long(), pos % page] = True
        for name, x, wt in (("q", q, w[0]), ("k", k, w[1]), ("v", v, None)):
            y = x[b, :m].double()
            if wt is not None:
                y = y / (y.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * wt.double()
            if rot and name != "v":
                y = _rotate64(y, cos[pos, None].double(), sin[pos, None].double(), rot, inter)
            got = q_out[b, :m].double() if name == "q" else c.at(name, b, pos)
            # 32-bit arithmetic on values up to the vector's largest, then one rounding: to
            # bf16 (8 significant bits) half of 2^-7, to e4m3 half of 2^-3 or, below its normal numbers, 2^-10 of the scale
            top = y.abs().amax(-1, keepdim=True)
            if name == "q" or dtype == "bf16":
                bound = y.abs() * 2 ** -8 * 1.001 + top * 4e-6
            else:
                bound = torch.maximum(y.abs() * 2 ** -4, top / 448 * 2 ** -10) * 1.001 + top * 4e-6
                assert torch.isfinite(c.scales[name][c.pages[b, pos // page].long(), :, pos % page]).all()
            assert ((got - y).abs() <= bound).all(), (name, b, ((got - y).abs() - bound).max())
    for x in "kv":                                                 # nothing else is written
        same = c.pools[x].view(torch.uint8)[~written] == before[x].view(torch.uint8)[~written]
        assert same.all()


# more tokens than the GPU takes at once
MANY = [
    (3, 701, 5, 3, 128, 16, "bf16", "e4m3", "head", 64, True, True),
    (3, 701, 5, 3, 80, 24, "f32", "bf16", "token", 80, False, True),
    (5, 600, 9, 3, 64, 64, "bf16", "e4m3", "token", 64, False, True),
    (5, 600, 2, 1, 64, 64, "f32", "e4m3", "token", 64, False, False),
    (3, 450, 3, 1, 256, 7, "bf16", "bf16", "head", 34, True, True),
    (40, 17, 33, 11, 112, 128, "f32", "e4m3", "head", 112, False, True),
    (900, 3, 7, 1, 16, 1, "bf16", "e4m3", "token", 16, True, False),
]


@pytest.mark.parametrize("case", MANY)
def test_append_many_tokens(lib, case):
    test_append(lib, case)


def test_append_in_place_and_default_drafts(lib):
    """q_out may be q; without draft_len every sequence has n tokens."""
    c = Cache(lib, 2, 32, 2, 64, 16, lens=[9, 20], fill=False)
    qkv = torch.randn((2, 4, 8, 64), generator=gen(1), device=DEV, dtype=torch.bfloat16)
    w = torch.ones(64, device=DEV, dtype=torch.bfloat16) * 2
    a, out = qkv.clone(), torch.empty((2, 4, 4, 64), device=DEV, dtype=torch.bfloat16)
    for x, o in ((qkv, out), (a, a[:, :, :4])):
        lib.pldp_cache_append(c.handle, x[:, :, :4], x[:, :, 4:6], x[:, :, 6:], i32([6, 17]), o, q_norm=w)
    assert torch.equal(out, a[:, :, :4]) and torch.equal(a[:, :, 4:], qkv[:, :, 4:])
    assert torch.equal(c.at("v", 1, range(16, 20)), qkv[1, :, 6:].double())


def test_append_status(lib):
    """Lengths, drafts, capacity, the rotation's rows and pages that are none."""
    B, n, D = 7, 4, 32
    c = Cache(lib, B, 32, 1, D, 8, lens=[32] * B, fill=False)
    c.pages[5, 1] = -1
    c.pages[6, 0] = 1 << 30
    x = torch.randn((B, n, 3, D), generator=gen(1), device=DEV, dtype=torch.bfloat16)
    q_out = torch.full((B, n, 1, D), -7.0, device=DEV, dtype=torch.bfloat16)
    cos, sin = _table(31, D, 5)
    status = i32([0] * B)
    L, d = [0, -1, 33, 30, 1, 8, 1], [3, 3, 3, 3, 9, 1, -2]
    before = {s: c.pools[s].clone() for s in "kv"}
    lib.pldp_cache_append(c.handle, x[:, :, :1], x[:, :, 1:2], x[:, :, 2:], i32(L), q_out, draft_len=i32(d), cos=cos, sin=sin,
                          status=status)
    assert status.tolist() == [0, lib.PLDP_ST_SEQ_LEN, lib.PLDP_ST_SEQ_LEN, lib.PLDP_ST_CAPACITY, lib.PLDP_ST_DRAFT_LEN,
                               lib.PLDP_ST_PAGE, lib.PLDP_ST_DRAFT_LEN | lib.PLDP_ST_PAGE]
    counts = [0, 0, 0, 2, 4, 2, 1]
    for b in range(B):
        assert (q_out[b, counts[b]:] == -7).all() and (q_out[b, :counts[b]] != -7).any(-1).all()
    changed = (c.pools["v"].view(torch.uint8) != before["v"].view(torch.uint8)).view(*c.pools["v"].shape[:2], -1).any(-1)
    assert int(changed.sum()) == 2 + 4 + 1
    assert torch.equal(c.at("v", 5, [7]), x[5, :1, 2:].double())


@pytest.mark.parametrize("dtype,layout,D,H,page,out", [
    ("bf16", "token", 128, 8, 16, "bf16"), ("e4m3", "head", 80, 3, 24, "f32"), ("e4m3", "token", 64, 1, 1, "bf16"),
    ("bf16", "head", 256, 2, 100, "f32"), ("e4m3", "token", 16, 5, 64, "f32")])
def test_read(lib, dtype, layout, D, H, page, out):
    lens = [0, 1, 77, 300, 129]
    c = Cache(lib, 5, 300, H, D, page, dtype, layout, lens=lens, seed=3)
    start = [0, 0, 5, 0, 128]
    count = [L - s for L, s in zip(lens, start)]
    kind = torch.float32 if out == "f32" else torch.bfloat16
    ko, vo = (torch.full((5, 303, H + 1, D), -7.0, device=DEV, dtype=kind)[:, :301, :H] for _ in "kv")
    status = i32([0] * 5)
    lib.pldp_cache_read(c.handle, i32(start), i32(count), ko, vo, status=status)
    assert status.tolist() == [0] * 5
    for x, name in ((ko, "k"), (vo, "v")):
        for b in range(5):
            want = c.dense[name][b][start[b]:]
            assert (x[b, count[b]:] == -7).all()
            bound = want.abs() * (2 ** -8 if out == "bf16" else 2 ** -23) * 1.001
            assert ((x[b, :count[b]].double() - want).abs() <= bound).all()
    only = torch.empty_like(vo)
    lib.pldp_cache_read(c.handle, None, i32(lens), None, only)
    assert torch.equal(only[3, :300], vo[3, :300])


def test_read_status(lib):
    c = Cache(lib, 5, 32, 1, 32, 8, lens=[32] * 5)
    c.pages[4, 0] = -3
    ko, vo = (torch.full((5, 20, 1, 32), -7.0, device=DEV) for _ in "kv")
    status = i32([0] * 5)
    lib.pldp_cache_read(c.handle, i32([0, 0, 30, 33, 4]), i32([-1, 21, 5, 1, 6]), ko, vo, status=status)
    assert status.tolist() == [lib.PLDP_ST_SEQ_LEN, lib.PLDP_ST_SEQ_LEN, lib.PLDP_ST_CAPACITY, lib.PLDP_ST_CAPACITY,
                               lib.PLDP_ST_PAGE]
    for b, m in enumerate([0, 20, 2, 0, 6]):
        assert (ko[b, m:] == -7).all() and (ko[b, :m] != -7).any(-1).all()
    assert (vo[4, :4] == 0).all() and torch.equal(vo[4, 4:6].double(), c.dense["v"][4][8:10])


def test_long_offsets(lib):
    """Pages beyond 2^32 bytes into the pool, and beyond 2^31 elements."""
    n, page, H, D = 9000, 128, 8, 256                             # 4.7 GB a pool
    pool = torch.empty((n, page, H, D), device=DEV, dtype=torch.bfloat16)
    pages = i32([[n - 1, 0], [1, n - 2]])
    h = lib.pldp_cache(pool, pool, pages)
    x = torch.randn((2, 2, 3 * H, D), generator=gen(1), device=DEV, dtype=torch.bfloat16)
    q_out = torch.empty((2, 2, H, D), device=DEV, dtype=torch.bfloat16)
    lib.pldp_cache_append(h, x[:, :, :H], x[:, :, H:2 * H], x[:, :, H:2 * H], i32([5, 200]), q_out)
    assert torch.equal(pool[n - 1, 4:6], x[0, :, H:2 * H]) and torch.equal(pool[n - 2, 71:73], x[1, :, H:2 * H])
    ko, vo = (torch.empty((2, 2, H, D), device=DEV, dtype=torch.bfloat16) for _ in "kv")
    lib.pldp_cache_read(h, i32([4, 199]), i32([2, 2]), ko, vo)
    assert torch.equal(ko, x[:, :, H:2 * H]) and torch.equal(vo, ko)


def test_on_another_stream(lib):
    c = Cache(lib, 2, 64, 2, 64, 16, lens=[40, 64])
    ko, vo = (torch.zeros((2, 64, 2, 64), device=DEV) for _ in "kv")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    lib.pldp_cache_read(c.handle, None, i32([40, 64]), ko, vo, stream=s)
    s.synchronize()
    assert torch.equal(ko[0, :40].double(), c.dense["k"][0]) and torch.equal(vo[1].double(), c.dense["v"][1])


def test_refusals(lib):
    c = Cache(lib, 2, 64, 2, 64, 16)
    x = torch.zeros((2, 3, 8, 64), device=DEV, dtype=torch.bfloat16)
    q, k, v, L, out = x[:, :, :4], x[:, :, 4:6], x[:, :, 6:], i32([1, 1]), torch.zeros_like(x[:, :, :4])
    call = lib.pldp_cache_append
    for bad, match in [
        (dict(k=k.float()), "k must be"), (dict(k=x[:, :, 4:7]), "shape"), (dict(q_out=out.float()), "q_out"),
        (dict(q=torch.zeros((2, 3, 4, 32), device=DEV, dtype=torch.bfloat16)), "head_dim"), (dict(seq_len=L[:1]), "seq_len"),
        (dict(q_norm=torch.ones(32, device=DEV, dtype=torch.bfloat16)), "q_norm"), (dict(cos=torch.ones((4, 8), device=DEV)), "cos"),
        (dict(cache=c.pools["k"]), "pldp_cache"), (dict(q=q.cpu()), "CUDA"), (dict(status=torch.zeros(2, device=DEV)), "status"),
    ]:
        with pytest.raises(ValueError, match=match):
            call(**{**dict(cache=c.handle, q=q, k=k, v=v, seq_len=L, q_out=out), **bad})
    odd = torch.zeros((2, 3, 4, 68), device=DEV, dtype=torch.bfloat16)[..., 4:]
    with pytest.raises(lib.PldpError, match="16"):
        call(c.handle, odd, k, v, L, out)
    with pytest.raises(lib.PldpError, match="rot"):
        call(c.handle, q, k, v, L, out, cos=torch.ones((64, 40), device=DEV), sin=torch.ones((64, 40), device=DEV))
    with pytest.raises(lib.PldpError, match="eps"):
        call(c.handle, q, k, v, L, out, eps=-1.0)
    p = c.pools["k"]
    for bad, match in [(dict(k_cache=p.float()), "bfloat16"), (dict(v_cache=p[1:]), "same shape"), (dict(pages=c.pages.long()), "int32"),
                       (dict(k_scale=torch.ones(1, device=DEV)), "float8"), (dict(k_cache=p.to(torch.float8_e4m3fn),
                        v_cache=p.to(torch.float8_e4m3fn)), "k_scale")]:
        with pytest.raises(ValueError, match=match):
            lib.pldp_cache(**{**dict(k_cache=p, v_cache=p, pages=c.pages), **bad})
    few = lib.pldp_cache(p, p, c.pages[:1])
    with pytest.raises(ValueError, match="rows"):
        call(few, q, k, v, L, out)
    narrow = torch.zeros((2, 16, 2, 24), device=DEV, dtype=torch.bfloat16)
    with pytest.raises(lib.PldpError, match="multiple of 16"):
        lib.pldp_cache_read(lib.pldp_cache(narrow, narrow, c.pages), None, L, *(torch.zeros((2, 3, 2, 24), device=DEV),) * 2)
    with pytest.raises(ValueError, match="strides"):
        lib.pldp_cache_read(c.handle, None, L, torch.zeros((2, 3, 2, 64), device=DEV), torch.zeros((2, 3, 3, 64), device=DEV)[:, :, :2])
