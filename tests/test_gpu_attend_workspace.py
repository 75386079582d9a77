"""One workspace of pldp_attend_cache, zeroed once, for calls of different shapes."""
import pytest
import torch

from tests._cache import DEV, Cache, attend64, i32
from tests.test_gpu_attend import _check, _queries

pytestmark = pytest.mark.gpu


def _call(lib, c, q, L, ws):
    out = torch.full(q.shape, float("nan"), device=DEV, dtype=torch.bfloat16)
    lse = torch.full(q.shape[:3], float("nan"), device=DEV)
    status = i32([0] * len(L))
    lib.pldp_attend_cache(c.handle, q, i32(L), out, ws, lse=lse, status=status)
    assert status.tolist() == [0] * len(L)
    return out, lse


# One long sequence, whose parts fill the workspace, and then many units of work, most of them cut between CTAs:
# sequences, tokens, heads, length of either call
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,few,many", [(64, (1, 1, 32, 5000), (64, 1, 32, 420)), (128, (1, 1, 32, 5000), (40, 1, 64, 420)),
                                       (128, (4, 1, 8, 1500), (4, 1100, 8, 400)), (256, (1, 2, 8, 3000), (68, 2, 64, 300))])
def test_shapes_in_turn(lib, D, few, many, dtype):
    calls = []
    for seed, (B, n, H, L) in enumerate((few, many)):
        lens = [L - 3 * b for b in range(B)]
        c = Cache(lib, B, L + n, H, D, 64, dtype, lens=[x + n - 1 for x in lens], seed=seed)
        q = _queries(B, n, H, D, seed=seed + 10)
        if n <= 2:
            want = attend64(c, q, lens, [n - 1] * B, D ** -0.5, H)
        else:
            # of a chunk every token's row against a workspace of its own: the same bits
            want = _call(lib, c, q, lens, torch.zeros(lib.pldp_attend_workspace_size(B, n, H, H, D), dtype=torch.uint8, device=DEV))
        calls.append((c, q, lens, want))
    size = max(lib.pldp_attend_workspace_size(B, n, H, H, D) for B, n, H, _ in (few, many))
    ws = torch.zeros(size, dtype=torch.uint8, device=DEV)
    for c, q, lens, want in (*calls, *calls, calls[0]):
        out, lse = _call(lib, c, q, lens, ws)
        if len(want) == 3:
            _check(out, lse, want)
        else:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
