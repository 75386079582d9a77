"""The codes and scales that pldp_cache_append writes are those of its formula in 32 bits."""
import pytest
import torch

from tests._cache import DEV, Cache, gen, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,spread", [(64, 1.0), (128, 3e-5), (16, 1e18), (256, 700.0)])
def test_codes_are_quotients(lib, kind, D, spread):
    """scale = max|x| (1/448) and code = x / scale, a product and a quotient in 32 bits: every code and scale is the
    same (ties between codes, which a product with the scale's inverse would miss by one step, among them)."""
    B, n, H = 2, 3000, 3
    c = Cache(lib, B, n, H, D, 64, "e4m3", lens=[n] * B, fill=False)
    x = (torch.randn((B, n, 4 * H, D), generator=gen(D), device=DEV) * spread).to(kind)
    few = torch.randint(-30, 31, (B, n // 2, 4 * H, D), generator=gen(D + 1), device=DEV).to(kind)
    x[:, : n // 2] = few * (spread / 16)                          # few distinct values: many ties
    q, k, v = x[:, :, : 2 * H], x[:, :, 2 * H: 3 * H], x[:, :, 3 * H:]
    lib.pldp_cache_append(c.handle, q, k, v, i32([1] * B), torch.empty(q.shape, dtype=torch.bfloat16, device=DEV))
    pos = torch.arange(n, device=DEV)
    for b in range(B):
        pg, slot = c.pages[b, pos // 64].long(), pos % 64
        for name, y in (("k", k), ("v", v)):
            y = y[b].float()
            top = y.abs().amax(-1)
            scale = top * torch.tensor(1 / 448, dtype=torch.float32, device=DEV)
            live = top > 0
            code = (y / scale[..., None]).to(torch.float8_e4m3fn).float()
            got = c.pools[name].view(torch.uint8)[pg, slot].view(torch.float8_e4m3fn).float()
            assert torch.equal(c.scales[name][pg, :, slot][live], scale[live])
            assert torch.equal(got[live], code[live])
            assert (got[~live] == 0).all()
