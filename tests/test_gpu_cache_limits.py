"""The cache calls at the ends of their ranges."""
import pytest
import torch

from tests._cache import DEV, Cache, gen, i32

pytestmark = pytest.mark.gpu


def _large_read(lib, n):
    """A read into n rows that all lie in the same place, of which one is written."""
    c = Cache(lib, 1, 64, 1, 16, 16, lens=[64])
    room = torch.zeros((1, 1, 1, 16), device=DEV, dtype=torch.bfloat16)
    lib.pldp_cache_read(c.handle, i32([3]), i32([1]), room.expand(1, n, 1, 16), None)
    return room[0, 0].double(), c.dense["k"][0][3]


@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31 - 512, 1 << 30])
def test_room_for_many_rows(lib, n):
    """As many rows as 32 bits count, of which the first is read."""
    got, want = _large_read(lib, n)
    assert torch.equal(got, want)


def test_the_last_of_many_rows(lib):
    """2^31 - 2 positions of one vector each (69 GB), their last page alone another."""
    page, per = 42966, 49981
    n = page * per
    assert n == 2 ** 31 - 2
    pool = torch.zeros((2, page, 1, 16), device=DEV, dtype=torch.bfloat16)
    pool[1] = torch.randn((page, 1, 16), generator=gen(1), device=DEV, dtype=torch.bfloat16)
    pages = torch.zeros((1, per), dtype=torch.int32, device=DEV)
    pages[0, -1] = 1
    c = lib.pldp_cache(pool, pool, pages)
    room, status = torch.empty((1, n, 1, 16), device=DEV, dtype=torch.bfloat16), i32([0])
    room[0, -2 * page:] = 7
    lib.pldp_cache_read(c, None, i32([n]), None, room, status=status)
    same = torch.equal(room[0, -page:], pool[1]) and bool((room[0, -2 * page:-page] == 0).all())
    del room
    torch.cuda.empty_cache()
    assert same and status.tolist() == [0]


@pytest.mark.parametrize("n", [2 ** 31 - 1, 5])
def test_a_call_answers_for_itself(lib, n):
    """Whatever one call answers, the next one's status is its own."""
    try:
        _large_read(lib, n)
    except lib.PldpError:
        pass
    c = Cache(lib, 1, 32, 2, 64, 16, lens=[9], fill=False)
    x = torch.randn((1, 4, 6, 64), generator=gen(1), device=DEV, dtype=torch.bfloat16)
    q = torch.empty((1, 4, 2, 64), device=DEV, dtype=torch.bfloat16)
    lib.pldp_cache_append(c.handle, x[:, :, :2], x[:, :, 2:4], x[:, :, 4:], i32([6]), q)
    assert torch.equal(q, x[:, :, :2]) and torch.equal(c.at("v", 0, range(5, 9)), x[0, :, 4:].double())
