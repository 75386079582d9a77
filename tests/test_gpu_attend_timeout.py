"""The bounded waits of pldp_attend_cache and their status bit, without a fault.

A test build of the attention (PLDP_TEST_STUCK_SCORES) has the softmax warps wait, tile by tile, on a barrier that nothing
arrives on, with a short bound on every wait; the copies and products of the tiles are all made.  After the first wait has
run out the roles of a CTA no longer wait for one another: the call still has to return, with TIMEOUT on every sequence,
and the context has to stay usable."""
import ctypes

import pytest
import torch

from paper_2412_01447_gb300 import _build
from tests._cache import DEV, Cache, attend64, i32
from tests.test_gpu_attend import _check, _queries, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def stuck(lib):
    path = _build.build_variant("stuck_scores", ["attend.cu", "attend_bf16.cu", "attend_e4m3.cu", "cache.cu", "abi.cu"],
                                extra_flags=["-DPLDP_TEST_STUCK_SCORES"])
    so = ctypes.CDLL(path)
    so.pldp_attend_cache.argtypes = [ctypes.POINTER(lib.pldp_attend_args), ctypes.c_void_p]
    so.pldp_attend_cache.restype = ctypes.c_int
    return so


# tiles a CTA: one; some; many, in rings of keys and values of an even and (heads of 256) an odd number of places
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("L,n,Hq,H,D,page", [([100, 1], 1, 4, 2, 64, 16), ([900, 1500, 40], 11, 8, 2, 128, 32),
                                            ([3300, 3171, 2900, 3500], 4, 32, 16, 64, 64),
                                            ([3300, 3171, 2900, 3500], 17, 80, 16, 128, 7),
                                            ([3300, 3171, 2900, 3500], 2, 16, 16, 256, 64)])
def test_waits_run_out(lib, stuck, L, n, Hq, H, D, page, dtype):
    B = len(L)
    c = Cache(lib, B, max(L) + n, H, D, page, dtype, lens=[a + n - 1 for a in L], seed=8)
    q = _queries(B, n, Hq, D)
    out, status, Lt = torch.zeros_like(q), i32([0] * B), i32(L)
    ws = torch.zeros(lib.pldp_attend_workspace_size(B, n, Hq, H, D), dtype=torch.uint8, device=DEV)
    a = lib.pldp_attend_args(cache=c.handle.args, q=q.data_ptr(), B=B, n=n, q_heads=Hq, q_strides=(ctypes.c_int64 * 3)(*q.stride()[:3]),
                             seq_len=Lt.data_ptr(), scale=D ** -0.5, out=out.data_ptr(),
                             out_strides=(ctypes.c_int64 * 3)(*out.stride()[:3]), status=status.data_ptr(), workspace=ws.data_ptr(),
                             workspace_bytes=ws.numel())
    assert stuck.pldp_attend_cache(ctypes.byref(a), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()                                      # the call returned and completed
    assert status.tolist() == [lib.PLDP_ST_TIMEOUT] * B
    # the context is still usable, and the product build takes the same inputs normally
    out, lse, status = _run(lib, c, q, L, None, ws=ws.zero_())
    assert status == [0] * B
    _check(out, lse, attend64(c, q, L, [n - 1] * B, D ** -0.5, H))
