"""How far pldp_attend_cache rounds the weights: values that cancel, so that the result's own rounding hides nothing."""
import pytest
import torch

from tests._cache import DEV, Cache, attend64, i32
from tests.test_gpu_attend import _queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,layout", [("bf16", "token"), ("e4m3", "token"), ("bf16", "head"), ("e4m3", "head")])
@pytest.mark.parametrize("D,H,L", [(64, 8, 50), (128, 8, 100), (128, 2, 3000), (64, 64, 1300), (256, 4, 70), (80, 3, 129)])
def test_cancelling_values(lib, D, H, L, dtype, layout):
    """Every head's values less their own weighted mean: what is left of the result is some 2^-8 of the values, and the
    rounding of each weight shows.  In a bf16 cache a weight is a sum of two bf16 (2^-17), in an e4m3 cache an f16
    (2^-11); the result rounds to bf16 (2^-8 of itself); scores of up to 20 and sums are in 32 bits (2e-5)."""
    c = Cache(lib, 2, L, H, D, 16, dtype, layout, lens=[L, L - 1], seed=D)
    q = _queries(2, 1, H, D)
    lens, scale = [L, L - 1], 3 * D ** -0.5
    mean = attend64(c, q, lens, [0, 0], scale, H)[0]              # [2, 1, H, D]
    for b in range(2):
        v = (c.dense["v"][b] - mean[b]).float()
        pos = torch.arange(lens[b], device=DEV)
        pg, slot = c.pages[b, pos // 16].long(), pos % 16
        if dtype == "bf16":
            c.pools["v"][pg, slot] = v.bfloat16()
        else:
            s = v.abs().amax(-1) / 448
            c.pools["v"].view(torch.uint8)[pg, slot] = (v / s[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
            c.scales["v"].permute(0, 2, 1)[pg, slot] = s
        c.dense["v"][b] = c.at("v", b, pos)
    o, l, size = attend64(c, q, lens, [0, 0], scale, H)
    assert (o.abs() < 0.1 * size).double().mean() > 0.9           # they do cancel
    out, lse, st = torch.zeros_like(q), torch.zeros((2, 1, H), device=DEV), i32([0, 0])
    ws = torch.zeros(lib.pldp_attend_workspace_size(2, 1, H, H, D), dtype=torch.uint8, device=DEV)
    lib.pldp_attend_cache(c.handle, q, i32(lens), out, ws, lse=lse, scale=scale, status=st)
    assert st.tolist() == [0, 0]
    assert ((lse.double() - l).abs() <= 2e-5 * (1 + l.abs())).all()
    weight = 2 ** -17 if dtype == "bf16" else 2 ** -11
    assert ((out.double() - o).abs() <= 2 ** -8 * o.abs() + (weight + 2e-5) * size).all()
