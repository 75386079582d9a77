"""pldp_token_logprobs on rows that a model spoiled: alternatives are always tokens, all of them written."""
import math

import pytest
import torch

from tests._cache import DEV, gen, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 257, 5000, 32001])
def test_alternatives_are_tokens(lib, V, dtype):
    x = torch.randn((9, V), generator=gen(V), device=DEV)
    x[0] = math.nan
    x[1, 3:] = math.nan
    x[2, torch.rand(V, generator=gen(1), device=DEV) < 0.5] = math.nan
    x[3, : V // 2] = math.nan
    x[4] = -math.nan
    x[5] = math.nan
    x[5, V - 1] = -math.inf
    x[6] = math.inf
    x[7, 11] = math.inf
    x = x.to(dtype)
    for top in (1, 20, 32):
        ids, lps = torch.full((9, top), -7, dtype=torch.int32, device=DEV), torch.full((9, top), -7.0, device=DEV)
        lp, ent = torch.full((9,), -7.0, device=DEV), torch.full((9,), -7.0, device=DEV)
        ws = torch.zeros(lib.pldp_token_logprobs_workspace_size(9, V), dtype=torch.uint8, device=DEV)
        lib.pldp_token_logprobs(x, i32([5] * 9), lp, ws, entropy=ent, top_id=ids, top_logprob=lps)
        assert ((ids >= 0) & (ids < V)).all() and (lps != -7).all() and (lp != -7).all() and (ent != -7).all()
        for r in range(9):
            assert len(set(ids[r].tolist())) == top
        assert int(ids[7, 0]) == 11 and torch.equal(ids[8].long(), x[8].double().sort(descending=True, stable=True).indices[:top])
