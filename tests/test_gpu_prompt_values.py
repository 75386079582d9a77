"""pldp_attend_prompt over an e4m3 cache whose values differ in size by far more than f16 holds: what later tokens hold must
not show in earlier rows, wherever the tiles, the units and the CTAs' parts end."""
import pytest
import torch

from tests._cache import DEV, Cache
from tests.test_gpu_prompt import _check, _queries, _rows, _run, prompt64

pytestmark = pytest.mark.gpu


def _scale_values(c, b, positions, factor):
    """Multiplies the values at `positions` of sequence b by a power of two (0: they become zeros, of the smallest scale)."""
    pg, slot = c.pages[b, positions // c.page].long(), positions % c.page
    if factor == 0:
        c.pools["v"].view(torch.uint8)[pg, slot] = 0
        c.scales["v"][pg, :, slot] = 2.0 ** -80
    else:
        c.scales["v"][pg, :, slot] *= factor
    c.dense["v"][b][positions] *= factor


def _causal(c, want, rows, starts, Hq):
    """`want` with the largest |v| of each row's own head and keys in place of that of the whole sequence.

    The bounds of `_check` then hold a row to what it sees.  Where scales are held in a unit 2^unit for all of a tile, of at most 8
    times the largest scale that the row sees, small scales are off by 2^-25 of it, 2^-22 of the largest |v|, and values by 2^-30
    of that.  In tiles that hide much larger values from some rows, codes are exact and a weight w_j = 2^(x_j - m + 7) is multiplied by
    4 scale / 2^unit before it is rounded, once (2^-11) in place of three times, 2^unit at most 8 times the largest scale that the
    row sees; a small one by 2^-25, of which l >= 2^7 leaves 448 / 4 * 2^unit 2^-32, so 2^-31 of the largest |v| a key.  Of such keys
    there are at most 3 tiles (256 tokens of a unit and the tile that they begin in), 384 * 2^-31 < 2^-22; with the 2^-22 above
    below 2^-21.  (The exponents are sums of two then: 2^-23 of some tens more, which two roundings of 2^-11 fewer cover.)"""
    G = Hq // c.heads
    most = want[3].expand(2, -1, Hq, 1).clone()
    for b, p in enumerate(starts):
        n = rows[b + 1] - rows[b]
        top = c.dense["v"][b][: p + n].abs().amax(-1).cummax(0).values[p:]            # [n, heads]
        most[1, rows[b]:rows[b + 1], :, 0] = top.repeat_interleave(G, 1)
    return *want[:3], most


# counts, starts, q heads, heads, D, page
SHAPES = [
    ([300, 77], [0, 0], 4, 2, 64, 16),
    ([400], [0], 8, 8, 128, 32),                # one query head a head: a unit spans tiles that its first rows do not see
    ([130, 300], [513, 60], 6, 2, 128, 7),
    ([250], [2000], 32, 8, 128, 64),
    ([300, 90], [31, 127], 4, 2, 256, 16),
    ([5, 1, 200], [123, 127, 255], 16, 1, 80, 24),
]


@pytest.mark.parametrize("power", [1, 2, 3, 8, 24, 60, 120, -24, -60])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_step_in_size(lib, shape, power):
    """From a position in a tile on, all values are 2^power times as large as before."""
    counts, starts, Hq, H, D, page = shape
    lens, rows = [a + b for a, b in zip(counts, starts)], _rows(counts)
    for at in (1, 40, 127):
        c = Cache(lib, len(counts), max(lens), H, D, page, "e4m3", lens=lens, seed=5)
        for b, L in enumerate(lens):
            if power > 60:                                        # (within fp32)
                _scale_values(c, b, torch.arange(L, device=DEV), 2.0 ** (60 - power))
            first = min(starts[b] // 128 * 128 + at, L)
            _scale_values(c, b, torch.arange(first, L, device=DEV), 2.0 ** power)
        q = _queries(rows[-1], Hq, D)
        out, lse, status = _run(lib, c, q, rows, starts)
        assert status == [0] * len(counts)
        _check(out, lse, _causal(c, prompt64(c, q, rows, starts, D ** -0.5), rows, starts, Hq), "e4m3")


@pytest.mark.parametrize("shape", SHAPES)
def test_values_of_any_size(lib, shape):
    """Each position's values of a size of its own, ever larger at their largest; some are zeros, the first ones too."""
    counts, starts, Hq, H, D, page = shape
    lens, rows = [a + b for a, b in zip(counts, starts)], _rows(counts)
    c = Cache(lib, len(counts), max(lens), H, D, page, "e4m3", lens=lens, seed=6)
    for b, L in enumerate(lens):
        for p in range(L):
            power = 0 if p < 3 or p % 29 == 5 else 2.0 ** (p * 37 % min(p // 8 + 2, 100) - 20)
            _scale_values(c, b, torch.tensor([p], device=DEV), power)
    q = _queries(rows[-1], Hq, D)
    out, lse, _ = _run(lib, c, q, rows, starts)
    _check(out, lse, _causal(c, prompt64(c, q, rows, starts, D ** -0.5), rows, starts, Hq), "e4m3")
    again, _, _ = _run(lib, c, q, rows, starts)
    assert torch.equal(out, again)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_in_chunks(lib, D):
    """A prompt in one call, and cut before a token of large values: the rows before it, which do not see it."""
    n, cut, Hq, H = 500, 307, 8, 2
    c = Cache(lib, 1, n, H, D, 16, "e4m3", lens=[n], seed=5)
    _scale_values(c, 0, torch.tensor([cut], device=DEV), 2.0 ** 30)
    q = _queries(n, Hq, D)
    whole = _run(lib, c, q, [0, n], [0])
    first = _run(lib, c, q[:cut], [0, cut], [0])
    want = _causal(c, prompt64(c, q, [0, n], [0], D ** -0.5), [0, n], [0], Hq)
    before = *(x[:cut] for x in want[:3]), want[3][:, :cut]
    _check(whole[0], whole[1], want, "e4m3")
    _check(whole[0][:cut], whole[1][:cut], before, "e4m3")
    _check(*first[:2], before, "e4m3")


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("gone", [0, 1, 200])
def test_with_missing_pages(lib, D, gone):
    """The same where a page of the tile is none."""
    n, Hq, H, page = 400, 4, 2, 8
    c = Cache(lib, 1, n, H, D, page, "e4m3", lens=[n], seed=5)
    _scale_values(c, 0, torch.arange(220, n, device=DEV), 2.0 ** 40)
    c.pages[0, gone // page] = -1
    live = torch.arange(n, device=DEV) // page != gone // page
    q = _queries(n, Hq, D)
    out, lse, status = _run(lib, c, q, [0, n], [0])
    assert status == [lib.PLDP_ST_PAGE]
    _check(out, lse, _causal(c, prompt64(c, q, [0, n], [0], D ** -0.5, live=[live]), [0, n], [0], Hq), "e4m3")
