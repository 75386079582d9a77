"""pldp_token_logprobs at the smallest temperatures: all of the probability on the largest logits."""
import math

import pytest
import torch

from tests._cache import DEV, gen, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1e-30, 1e-38, 1e-40, 1.5e-45])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [300, 32000])
def test_cold(lib, V, dtype, T):
    x = torch.randn((4, V), generator=gen(V), device=DEV).to(dtype)
    x[:, [7, 150]] = 9.0
    x[1, 150] = -math.inf
    x[2] = 0.0
    x[3] = -math.inf
    x[3, 20:24] = -3.0
    want = [2, 1, V, 4]                                           # how many share the largest value
    first = [7, 7, 0, 20]
    out = dict(dtype=torch.float32, device=DEV)
    lp, ent, ids, top = torch.ones(4, **out), torch.ones(4, **out), i32([[0] * 5] * 4), torch.ones((4, 5), **out)
    ws = torch.zeros(lib.pldp_token_logprobs_workspace_size(4, V), dtype=torch.uint8, device=DEV)
    lib.pldp_token_logprobs(x, i32(first), lp, ws, entropy=ent, top_id=ids, top_logprob=top, temperature=T)
    for r in range(4):
        l = math.log(want[r])
        # (a sum of whole numbers of equal weights of 1, its logarithm in 32 bits)
        assert abs(float(lp[r]) + l) <= 1e-6 * (1 + l) and abs(float(ent[r]) - l) <= 1e-6 * (1 + l)
        assert int(ids[r, 0]) == first[r]
        live = min(want[r], 5)
        assert ((top[r, :live] + l).abs() <= 1e-6 * (1 + l)).all() and (top[r, live:] < -1e25).all()
