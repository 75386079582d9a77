"""pldp_attend_prompt with a scale of zero (every key that a row sees weighs the same) and queries of any size."""
import pytest
import torch

from tests._cache import Cache
from tests.test_gpu_prompt import _check, _queries, _rows, _run, prompt64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-38, -1e-38])
def test_small_queries(lib, D, scale, dtype):
    counts, starts, Hq, H = [150, 33], [0, 300], 4, 2
    lens, rows = [a + b for a, b in zip(counts, starts)], _rows(counts)
    c = Cache(lib, 2, max(lens), H, D, 16, dtype, lens=lens, seed=5)
    q = _queries(rows[-1], Hq, D)
    for power, some in ((-12, slice(20, 60)), (-60, slice(60, 90)), (-120, slice(90, 120))):
        q[some] *= 2.0 ** power
    q[10:20] = 0
    q[150:155] = 0
    q[155:170] *= 2.0 ** -30
    out, lse, status = _run(lib, c, q, rows, starts, scale=scale)
    assert status == [0, 0]
    _check(out, lse, prompt64(c, q, rows, starts, scale), dtype)
