"""The rotation's staging in pldp_cache_append from one token to the next: many tokens a group of lanes, an odd number
of rotated vectors in each, and nothing between them (no norms, no scales) that would keep a group's lanes together."""
import pytest

from tests.test_gpu_cache import test_append as append

pytestmark = pytest.mark.gpu

# B, n, q heads, heads, D, page, input, cache, layout, rot, interleaved, norms
CASES = [
    (3, 1400, 32, 8, 64, 16, "bf16", "bf16", "token", 64, False, False),     # five a group
    (2, 2100, 12, 2, 128, 64, "f32", "bf16", "head", 128, False, False),     # four or three
    (2, 2100, 12, 4, 128, 64, "bf16", "bf16", "token", 64, False, False),    # four, values between
    (2, 1200, 5, 1, 256, 32, "bf16", "bf16", "token", 256, False, False),    # three
    (2, 1500, 6, 2, 80, 24, "bf16", "bf16", "token", 40, False, False),      # pairs that cross the lanes' pieces
    (700, 5, 3, 1, 112, 16, "f32", "bf16", "head", 112, False, False),       # one a group
]


@pytest.mark.parametrize("case", CASES)
def test_rotation_without_norms(lib, case):
    append(lib, case)
