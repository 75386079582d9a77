"""Checks of the cache calls at the ends of their ranges, without a GPU."""
import ctypes

import pytest

import paper_2412_01447_gb300 as pk
from tests.test_cache_abi import P, _cache, _three, so  # noqa: F401  (a fixture)


@pytest.mark.parametrize("page_size,max_pages", [(2 ** 31 - 1, 1), (2 ** 31 - 4095, 1), (1 << 20, 2047), (1, 2 ** 31 - 4096)])
def test_attention_needs_room_above_the_last_position(so, page_size, max_pages):  # noqa: F811
    """Positions are counted in tiles beyond the last one, in 32 bits: a cache of up to 2^31 - 4096 of them is attended to,
    a larger one refused before anything is launched (B = 0 launches nothing either)."""
    cache = _cache(page_size=page_size, max_pages=max_pages, pages_stride=max_pages, page_stride=1 << 40)
    a = pk.pldp_attend_args(cache=cache, q=P(256), B=0, n=3, q_heads=4, q_strides=_three(768, 256, 64), seq_len=P(256), scale=0.1,
                            out=P(256), out_strides=_three(768, 256, 64), workspace=P(256),
                            workspace_bytes=pk.pldp_attend_workspace_size(2, 3, 4, 2, 64))
    most = page_size * max_pages <= 2 ** 31 - 4096
    assert so.pldp_attend_cache(ctypes.byref(a), None) == (0 if most else 2)
    assert most or "positions" in pk.pldp_last_error()
