"""pldp_cache_append_prompt with rows that do not ascend: a sequence whose pair is bad is skipped, and no other one; the same
sequences take part in pldp_attend_prompt."""
import pytest
import torch

from tests._cache import DEV, Cache, gen, i32

pytestmark = pytest.mark.gpu

R = 50
# rows, whether each pair is within [0, R] and does not descend
LISTS = [
    ([0, 10, 60, 20, 40], [True, False, False, True]),
    ([0, 30, 5, 8, 9], [True, False, True, True]),
    ([-5, 10, 3, 50], [False, False, True]),
    ([40, 60, 0, 25, 24, 50], [False, False, True, False, True]),
    ([50, 0, 20, -1, 20, 45], [False, True, False, False, True]),
    ([7, 7, 20, 20, 31], [True] * 4),                              # (well formed: rows before and behind are nobody's)
    ([0, 2**31 - 1, 20, 50], [False, False, True]),
]


def _vectors(c, b, n):
    return [x for name in "kv" for x in (c.at(name, b, torch.arange(n, device=DEV)),)]


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("e4m3", 128), ("bf16", 256)])
@pytest.mark.parametrize("rows,good", LISTS)
def test_good_sequences_of_a_bad_list(lib, rows, good, dtype, D):
    B, Hq, H = len(good), 4, 2
    c, alone = (Cache(lib, B, R, H, D, 16, dtype, seed=3, lens=[R] * B, fill=False) for _ in range(2))
    qkv = torch.randn((R, Hq + 2 * H, D), generator=gen(2), device=DEV).bfloat16()
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    norm = (1 + 0.1 * torch.randn(D, generator=gen(4), device=DEV)).bfloat16()
    out, status = torch.full((R, Hq, D), 7.0, device=DEV, dtype=torch.bfloat16), i32([0] * B)
    lib.pldp_cache_append_prompt(c.handle, q, k, v, i32(rows), out, q_norm=norm, k_norm=norm, status=status)
    assert status.tolist() == [0 if g else lib.PLDP_ST_SEQ_LEN for g in good]
    claims = [0] * R
    for b, g in enumerate(good):
        for r in range(rows[b], rows[b + 1]) if g else ():
            claims[r] += 1
    want = torch.full_like(out, 7.0)
    for b, g in enumerate(good):
        n = rows[b + 1] - rows[b] if g else 0
        if n:
            s = slice(rows[b], rows[b + 1])
            handle = lib.pldp_cache(alone.pools["k"], alone.pools["v"], alone.pages[b:b + 1], alone.scales["k"], alone.scales["v"])
            lib.pldp_cache_append(handle, q[s][None], k[s][None], v[s][None], i32([1]), want[s][None], q_norm=norm, k_norm=norm)
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))
    for b, g in enumerate(good):
        n = rows[b + 1] - rows[b] if g else 0
        mine = torch.tensor([claims[r] == 1 for r in range(rows[b], rows[b] + n)], dtype=torch.bool, device=DEV)
        for x, y in zip(_vectors(c, b, n), _vectors(alone, b, n)):
            assert torch.equal(x[mine], y[mine])
    # attention over what was written takes the same sequences
    again, st = torch.full_like(out, 7.0), i32([0] * B)
    ws = torch.empty(lib.pldp_attend_prompt_workspace_size(Hq, H, D), dtype=torch.uint8, device=DEV)
    lib.pldp_attend_prompt(c.handle, out, i32(rows), again, ws, status=st)
    assert st.tolist() == status.tolist()
    claimed = torch.tensor([n > 0 for n in claims], dtype=torch.bool, device=DEV)
    assert (again[~claimed] == 7).all()


def test_many_sequences_and_rows_of_none(lib):
    """A padded batch: hundreds of sequences, and as many rows behind the last one."""
    B, H, D = 600, 1, 64
    c = Cache(lib, B, 16, H, D, 16, lens=[1] * B, seed=3, fill=False)
    before = c.pools["k"].view(torch.int16).clone()
    qkv = torch.randn((3 * B, 3, D), generator=gen(2), device=DEV).bfloat16()
    out, status = torch.full((3 * B, 1, D), 7.0, device=DEV, dtype=torch.bfloat16), i32([0] * B)
    lib.pldp_cache_append_prompt(c.handle, qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], i32(list(range(B + 1))), out, status=status)
    assert not status.any() and torch.equal(out[:B], qkv[:B, :1]) and (out[B:] == 7).all()
    after = c.pools["k"].view(torch.int16)
    first = c.pages[:, 0].long()
    assert torch.equal(after[first, 0, 0], qkv[:B, 1].contiguous().view(torch.int16))
    after = after.clone()
    after[first, 0] = before[first, 0]
    assert torch.equal(after, before)
