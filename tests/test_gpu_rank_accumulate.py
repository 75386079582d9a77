"""pldp_rank_cache: what is refused, or has no attention, beside scores of other layers."""
import math

import pytest
import torch

from tests._cache import DEV, Cache, attend64, gen, i32

pytestmark = pytest.mark.gpu


def _setup(lib, B):
    c = Cache(lib, B, 52, 1, 32, 16, "bf16", lens=[51] * B, seed=5)
    q = torch.randn((B, 2, 2, 32), generator=gen(6), device=DEV, dtype=torch.bfloat16)
    lse = attend64(c, q, [50] * B, [1] * B, 32 ** -0.5, 1)[1].float()
    return c, q, lse


@pytest.mark.parametrize("agg", ["max", "sum"])
def test_refused_beside_other_layers(lib, agg):
    """Rows and lengths that are none, and candidates outside [0, kv_len): -INFINITY, never chosen, whatever the
    other layers' scores are; beyond the count nothing is touched."""
    B = 6
    c, q, lse = _setup(lib, B)
    row, kv = [0, 2, -1, 0, 0, 0], [50, 50, 50, 1000, -1, 10]
    pos = i32([[60, 3, -1, 20, 7]] * B)
    count = i32([4] * B)
    before = torch.tensor([[9.0, 0.25, 9.0, 0.5, 9.0]] * B, device=DEV)
    alone, both = torch.full((B, 5), -7.0, device=DEV), before.clone()
    args = (c.handle, q, i32(row), i32(kv), lse, pos, count)
    best, bs, st = i32([9] * B), torch.zeros(B, device=DEV), i32([0] * B)
    lib.pldp_rank_cache(*args, i32([9] * B), agg=agg, scores=alone)
    lib.pldp_rank_cache(*args, best, agg=agg, scores=both, best_score=bs, accumulate=True, status=st)
    S = lib
    assert st.tolist() == [0, S.PLDP_ST_ROW_INDEX, S.PLDP_ST_ROW_INDEX, S.PLDP_ST_SEQ_LEN, S.PLDP_ST_SEQ_LEN, 0]
    assert (both[:, 4] == 9).all()
    assert best.tolist()[1:5] == [-1] * 4 and (bs[1:5] == -math.inf).all() and (both[1:5, :4] == -math.inf).all()
    for b, live in ((0, [1, 3]), (5, [1])):
        for i in range(4):
            if i in live:
                x, y = float(before[b, i]), float(alone[b, i])
                assert float(both[b, i]) == (max(x, y) if agg == "max" else float(before[b, i] + alone[b, i]))
            else:
                assert float(both[b, i]) == -math.inf
        top = max(live, key=lambda i: float(both[b, i]))
        assert int(best[b]) == int(pos[b, top]) and float(bs[b]) == float(both[b, top])


@pytest.mark.parametrize("agg", ["max", "sum"])
def test_layer_without_scores(lib, agg):
    """No selected head that is one, or no page: no score of this layer, so -INFINITY by itself and the other
    layers' score beside them."""
    c, q, lse = _setup(lib, 2)
    pos, count = i32([[3, 20, 40]] * 2), i32([3] * 2)
    before = torch.tensor([[0.25, 0.75, 0.5]] * 2, device=DEV)
    for heads in ([-1], [2, 7, -1]):
        scores, best, bs, st = torch.zeros((2, 3), device=DEV), i32([9, 9]), torch.zeros(2, device=DEV), i32([0, 0])
        args = (c.handle, q, None, i32([50, 50]), lse, pos, count, best)
        lib.pldp_rank_cache(*args, heads=i32(heads), agg=agg, scores=scores, best_score=bs, status=st)
        assert st.tolist() == [lib.PLDP_ST_ROW_INDEX] * 2
        assert (scores == -math.inf).all() and best.tolist() == [-1, -1] and (bs == -math.inf).all()
        both = before.clone()
        lib.pldp_rank_cache(*args, heads=i32(heads), agg=agg, scores=both, best_score=bs, accumulate=True)
        assert torch.equal(both, before) and best.tolist() == [20, 20] and bs.tolist() == [0.75, 0.75]
    c.pages[0, 1] = -1                                            # positions 16..31
    alone, both, st = torch.zeros((2, 3), device=DEV), before.clone(), i32([0, 0])
    args = (c.handle, q, None, i32([50, 50]), lse, pos, count)
    lib.pldp_rank_cache(*args, best, agg=agg, scores=alone, status=st)
    assert st.tolist() == [lib.PLDP_ST_PAGE, 0] and float(alone[0, 1]) == -math.inf and int(best[0]) != 20
    lib.pldp_rank_cache(*args, best, agg=agg, scores=both, accumulate=True)
    assert float(both[0, 1]) == 0.75
