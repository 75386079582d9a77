"""pldp_attend_prompt with queries that hold NaN or infinity: NaN for these rows, as pldp_attend_cache gives, and not the zeros of
a row that sees nothing; other rows are not touched by it."""
import math

import pytest
import torch

from tests._cache import DEV, Cache, i32
from tests.test_gpu_prompt import _queries, _rows, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("counts,starts", [([100, 7], [0, 30]), ([3, 40], [9000, 2000])])       # units of one CTA, and of many
def test_rows_of_nan(lib, counts, starts, D, dtype):
    Hq, H = 4, 2
    lens, rows = [a + b for a, b in zip(counts, starts)], _rows(counts)
    c = Cache(lib, 2, max(lens), H, D, 16, dtype, lens=lens, seed=5)
    c.pages[1, 0] = -1                                             # (rows of the second see none of their first page)
    q = _queries(rows[-1], Hq, D)
    want, want_lse, _ = _run(lib, c, q, rows, starts)
    bad = torch.zeros((rows[-1], Hq), dtype=torch.bool, device=DEV)
    for (row, head, e), x in {(0, 1, 3): math.nan, (rows[1] - 1, 3, D - 1): math.inf, (rows[1] + 1, 0, 0): -math.inf, (rows[1] + 2, 2, 17): math.nan,
                              (rows[-1] - 1, 3, 8): math.nan}.items():
        q[row, head, e], bad[row, head] = x, True
    out, lse, _ = _run(lib, c, q, rows, starts)
    assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all()
    assert torch.equal(out[~bad], want[~bad]) and torch.equal(lse[~bad], want_lse[~bad])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_rows_that_see_nothing(lib, dtype):
    """Zeros, whatever the queries hold."""
    c = Cache(lib, 1, 64, 1, 64, 16, dtype, lens=[64], seed=5)
    c.pages[:] = -1
    q = _queries(40, 2, 64)
    q[3], q[7, 1, 2] = math.nan, math.inf
    out, lse, status = _run(lib, c, q, [0, 40], [0])
    assert status == [lib.PLDP_ST_PAGE] and (out == 0).all() and (lse == -math.inf).all()


def test_the_same_as_a_step(lib):
    n, L, D = 5, 70, 64
    c = Cache(lib, 1, L + n, 1, D, 16, lens=[L + n - 1], seed=6)
    q = _queries(n, 2, D)
    q[2, 1, 5] = math.nan
    out, lse, _ = _run(lib, c, q, [0, n], [L - 1])
    step, step_lse = torch.empty((1, n, 2, D), device=DEV, dtype=torch.bfloat16), torch.empty((1, n, 2), device=DEV)
    ws = torch.zeros(lib.pldp_attend_workspace_size(1, n, 2, 1, D), dtype=torch.uint8, device=DEV)
    lib.pldp_attend_cache(c.handle, q[None], i32([L]), step, ws, lse=step_lse)
    assert torch.equal(torch.isnan(out), torch.isnan(step[0])) and torch.equal(torch.isnan(lse), torch.isnan(step_lse[0]))
