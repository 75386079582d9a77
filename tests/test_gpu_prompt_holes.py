"""pldp_attend_prompt where whole tiles of keys have no page: the flags that say so are worked out beside the copies of a
tile (which read nothing there and are done at once), and have to be those of this tile and not of an earlier one."""
import pytest
import torch

from tests._cache import DEV, Cache
from tests.test_gpu_prompt import _check, _queries, _rows, _run, prompt64

pytestmark = pytest.mark.gpu

TILE = 128


# which tiles of the prefix have no page at all
GONE = {"first": lambda t: t == 0, "all": lambda t: True, "every_other": lambda t: t % 2 == 0, "after_eight": lambda t: t >= 8,
        "odd_runs": lambda t: t % 11 in (1, 2, 7)}


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 128), (128, 1), (128, 6), (256, 64), (256, 32)])
@pytest.mark.parametrize("gone", GONE)
def test_tiles_without_pages(lib, gone, D, page, dtype):
    counts, starts, Hq, H = [70, 200, 33], [23 * TILE, 15 * TILE + 50, 9 * TILE + 127], 4, 2
    lens, rows = [a + b for a, b in zip(counts, starts)], _rows(counts)
    c = Cache(lib, 3, max(lens), H, D, page, dtype, lens=lens, seed=5)
    live = []
    for b, L in enumerate(lens):
        pos = torch.arange(L, device=DEV)
        there = ~torch.tensor([GONE[gone](t) and (t + 1) * TILE <= starts[b] for t in range(-(-L // TILE))], device=DEV)[pos // TILE]
        first = pos[::page]                                       # (a page that reaches into a tile that is there stays)
        keep = torch.stack([there[p:p + page].any() for p in first.tolist()])
        c.pages[b, : len(first)][~keep] = -1
        live.append(keep[pos // page])
    q = _queries(rows[-1], Hq, D)
    want = prompt64(c, q, rows, starts, D ** -0.5, live=live)
    out, lse, status = _run(lib, c, q, rows, starts)
    assert status == [0 if l.all() else lib.PLDP_ST_PAGE for l in live]
    _check(out, lse, want, dtype)
    for _ in range(20):
        again, again_lse, _ = _run(lib, c, q, rows, starts)
        assert torch.equal(again, out) and torch.equal(again_lse, lse)
