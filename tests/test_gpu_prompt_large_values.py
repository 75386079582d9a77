"""pldp_attend_prompt over an e4m3 cache of values near fp32's largest: rows whose keys several CTAs share give what rows
of one CTA give."""
import pytest
import torch

from tests._cache import Cache
from tests.test_gpu_prompt import _check, _queries, _rows, _run, prompt64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("counts,starts", [([30], [9000]), ([200, 3], [0, 4000])])
def test_values_near_the_largest(lib, counts, starts, D):
    Hq, H = 4, 2
    lens, rows = [a + b for a, b in zip(counts, starts)], _rows(counts)
    c = Cache(lib, len(counts), max(lens), H, D, 64, "e4m3", lens=lens, seed=5)
    # positive ones, so that sums of weights times values are as large as they get; the results are averages of them
    c.pools["v"].view(torch.uint8).bitwise_and_(127)
    c.scales["v"] *= 2.0 ** 122
    c.dense["v"] = [x.abs() * 2.0 ** 122 for x in c.dense["v"]]
    q = _queries(rows[-1], Hq, D)
    out, lse, status = _run(lib, c, q, rows, starts)
    assert status == [0] * len(counts) and torch.isfinite(out).all()
    _check(out, lse, prompt64(c, q, rows, starts, D ** -0.5), "e4m3")
