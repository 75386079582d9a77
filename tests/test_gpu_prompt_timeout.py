"""The bounded waits of pldp_attend_prompt and their status bit, without a fault: as for pldp_attend_cache, a test build
(PLDP_TEST_STUCK_SCORES) has the softmax warps wait, tile by tile, on a barrier that nothing arrives on, with a short bound
on every wait.  After the first wait has run out the roles of a CTA no longer wait for one another: the call still has to
return, with TIMEOUT on every sequence and no row written that is none of a sequence, and the context has to stay usable."""
import ctypes

import pytest
import torch

from paper_2412_01447_gb300 import _build
from tests._cache import DEV, Cache, i32
from tests.test_gpu_prompt import _check, _queries, _rows, _run, prompt64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def stuck(lib):
    path = _build.build_variant("stuck_prompt", ["prompt.cu", "prompt_bf16.cu", "prompt_e4m3.cu", "attend.cu", "attend_bf16.cu",
                                                 "attend_e4m3.cu", "cache.cu", "abi.cu"], extra_flags=["-DPLDP_TEST_STUCK_SCORES"])
    so = ctypes.CDLL(path)
    so.pldp_attend_prompt.argtypes = [ctypes.POINTER(lib.pldp_attend_prompt_args), ctypes.c_void_p]
    so.pldp_attend_prompt.restype = ctypes.c_int
    return so


# units a CTA: one; parts of one; many, of one tile of rows and of two, with queries by boxes and (of 3 heads) without
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("counts,starts,Hq,H,D,page", [([100, 1], [0, 900], 4, 2, 64, 16), ([700], [2000], 8, 2, 128, 32),
                                                       ([300] * 24, [7] * 24, 32, 16, 64, 16), ([130] * 40, [0] * 40, 48, 16, 128, 7),
                                                       ([200] * 30, [100] * 30, 32, 16, 256, 64)])
def test_waits_run_out(lib, stuck, counts, starts, Hq, H, D, page, dtype):
    B, rows = len(counts), _rows(counts)
    c = Cache(lib, B, max(n + s for n, s in zip(counts, starts)), H, D, page, dtype, lens=[n + s for n, s in zip(counts, starts)], seed=8)
    q = _queries(rows[-1], Hq, D)
    room = torch.full((rows[-1] + 64, Hq, D), 7.0, device=DEV, dtype=torch.bfloat16)
    out, status, rt, st = room[32:-32], i32([0] * B), i32(rows), i32(starts)
    ws = torch.full((lib.pldp_attend_prompt_workspace_size(Hq, H, D),), 255, dtype=torch.uint8, device=DEV)
    a = lib.pldp_attend_prompt_args(cache=c.handle.args, q=q.data_ptr(), R=rows[-1], B=B, q_heads=Hq,
                                    q_strides=(ctypes.c_int64 * 2)(*q.stride()[:2]), rows=rt.data_ptr(), start=st.data_ptr(), scale=D ** -0.5,
                                    out=out.data_ptr(), out_strides=(ctypes.c_int64 * 2)(*out.stride()[:2]), status=status.data_ptr(),
                                    workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    assert stuck.pldp_attend_prompt(ctypes.byref(a), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()                                      # the call returned and completed
    assert status.tolist() == [lib.PLDP_ST_TIMEOUT] * B
    assert (room[:32] == 7).all() and (room[-32:] == 7).all()
    # the context is still usable, and the product build takes the same inputs normally
    out, lse, status = _run(lib, c, q, rows, starts, ws=ws)
    assert status == [0] * B
    _check(out, lse, prompt64(c, q, rows, starts, D ** -0.5), dtype)
