"""An e4m3 cache with vectors of zeros: a key that holds most of the attention and whose value is zero."""
import pytest
import torch

from tests._cache import DEV, Cache, attend64, gen, i32

pytestmark = pytest.mark.gpu


def _append(lib, c, k, v):
    """Writes k, v [1, n, H, D] at positions 0.. and takes what the cache then holds into c.dense."""
    n, H, D = k.shape[1:]
    q = torch.zeros((1, n, H, D), device=DEV)
    lib.pldp_cache_append(c.handle, q, k, v, i32([1]), q.bfloat16())
    for x in "kv":
        c.dense[x] = [c.at(x, 0, range(n))]


@pytest.mark.parametrize("D,n", [(64, 1), (128, 11)])
@pytest.mark.parametrize("size", [0.02, 1.0, 300.0])
@pytest.mark.parametrize("nats", [10.0, 12.5, 15.0])
def test_sink_of_zeros(lib, D, n, size, nats):
    """A first key some nats above all others, which are alike, its value zeros; the others' values are of one size.
    Each weight rounds to f16 (2^-11), the result to bf16 (2^-8), and the rest is in 32 bits."""
    L, H = 32768, 2
    c = Cache(lib, 1, L, H, D, 64, "e4m3", lens=[L], fill=False)
    g = gen(1)
    q = torch.randn((1, n, H, D), generator=g, device=DEV).bfloat16()
    q[:] = q[:, :1].clone()
    k = torch.zeros((1, L, H, D), device=DEV)
    k[0, 0] = q[0, 0].float() * (nats * D ** 0.5 / q[0, 0].float().square().sum(-1, keepdim=True))
    v = (0.5 + 0.5 * torch.rand((1, L, H, D), generator=g, device=DEV)) * size
    v[..., 3] = size
    v[0, 0] = 0
    _append(lib, c, k, v)
    start = [L - n + 1]
    o, l, mass = attend64(c, q, start, [n - 1], D ** -0.5, H)
    out, lse, st = torch.zeros_like(q), torch.zeros((1, n, H), device=DEV), i32([0])
    ws = torch.zeros(lib.pldp_attend_workspace_size(1, n, H, H, D), dtype=torch.uint8, device=DEV)
    lib.pldp_attend_cache(c.handle, q, i32(start), out, ws, lse=lse, status=st)
    assert st.tolist() == [0]
    assert ((lse.double() - l).abs() <= 2e-5 * (1 + l.abs())).all()
    assert ((out.double() - o).abs() <= 2 ** -8 * o.abs() + 2 ** -11 * mass + 1e-5 * mass).all()


def test_all_zeros(lib):
    """Nothing but zeros, in more keys than a small scale's inverse leaves room for in 32 bits: results of zero, and the
    log of the number of keys."""
    L, H, D = 1 << 19, 1, 16
    c = Cache(lib, 1, L, H, D, 4096, "e4m3", lens=[1], fill=False)
    c.pages[0] = torch.arange(c.pages.shape[1], device=DEV, dtype=torch.int32)
    x = torch.zeros((1, L, H, D), device=DEV, dtype=torch.bfloat16)
    k = x.clone()
    k[0, :, 0, 0] = 5.0 * torch.arange(L, device=DEV) / L         # scores that grow to 5 nats
    q = torch.zeros((1, 1, H, D), device=DEV, dtype=torch.bfloat16)
    q[..., 0] = 1
    lib.pldp_cache_append(c.handle, x, k, x, i32([1]), torch.empty_like(x))
    out, lse = torch.ones_like(q), torch.zeros((1, 1, H), device=DEV)
    ws = torch.zeros(lib.pldp_attend_workspace_size(1, 1, H, H, D), dtype=torch.uint8, device=DEV)
    lib.pldp_attend_cache(c.handle, q, i32([L]), out, ws, lse=lse, scale=1.0)
    want = torch.logsumexp(c.at("k", 0, range(L))[:, 0, 0], 0)
    assert (out == 0).all() and abs(float(lse) - float(want)) <= 2e-5 * (1 + float(want))
