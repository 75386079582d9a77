"""pldp_cache_copy_pages with a list of 2^30 pairs and more, nearly all of them none."""
import pytest
import torch

from tests._cache import DEV, Cache, i32

pytestmark = pytest.mark.gpu


def test_pairs_past_two_to_the_30(lib):
    n = 2 ** 30 + 3
    if torch.cuda.mem_get_info()[0] < 12 * 2 ** 30:
        pytest.skip("needs 12 GiB")
    c = Cache(lib, 4, 16, 1, 16, 16, lens=[16] * 4, seed=1)
    a, b, x, y = c.pages[:, 0].tolist()
    copies = torch.full((n, 2), -1, dtype=torch.int32, device=DEV)
    copies[5], copies[n - 1] = i32([a, b]), i32([x, y])
    lib.pldp_cache_copy_pages(c.handle, copies)
    for name in "kv":
        assert torch.equal(c.at(name, 1, [0, 7, 15]), c.dense[name][0][[0, 7, 15]])
        assert torch.equal(c.at(name, 3, [0, 7, 15]), c.dense[name][2][[0, 7, 15]])
