"""The prompt and page calls without a GPU: argument blocks as the header lays them out, the host's checks before
anything is launched, and the arithmetic of the list of tiles."""
import ctypes
import os
import random
import subprocess

import pytest

import paper_2412_01447_gb300 as pk
from tests.test_cache_abi import BAD_CACHES, HEADER, P, _cache, so  # noqa: F401  (a fixture)


@pytest.mark.parametrize("struct,cls", [("pldp_cache_append_prompt_args", pk.pldp_cache_append_prompt_args),
                                        ("pldp_attend_prompt_args", pk.pldp_attend_prompt_args),
                                        ("pldp_page_table", pk.pldp_page_table_args)])
def test_blocks_match_the_header(tmp_path, struct, cls):
    names = [f for f, _ in cls._fields_]
    src = ["#include <stdio.h>", "#include <stddef.h>", f'#include "{HEADER}"', "int main(void) {", f'printf("%zu\\n", sizeof({struct}));']
    src += [f'printf("%zu\\n", offsetof({struct}, {n}));' for n in names] + ["return 0; }"]
    (tmp_path / "layout.c").write_text("\n".join(src))
    subprocess.check_call(["gcc", str(tmp_path / "layout.c"), "-o", str(tmp_path / "layout")])
    out = [int(x) for x in subprocess.check_output([str(tmp_path / "layout")]).split()]
    assert out == [ctypes.sizeof(cls)] + [getattr(cls, n).offset for n in names]


def _two(*x):
    return (ctypes.c_int64 * 2)(*x)


def _append(**kw):
    a = pk.pldp_cache_append_prompt_args(cache=_cache(**kw.pop("cache", {})), q=P(256), k=P(256), v=P(256), dtype=1, B=2, R=5, q_heads=4,
                                         q_strides=_two(256, 64), k_strides=_two(256, 64), v_strides=_two(256, 64), eps=1e-6,
                                         rows=P(256), q_out=P(256), q_out_strides=_two(256, 64))
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _attend(**kw):
    a = pk.pldp_attend_prompt_args(cache=_cache(**kw.pop("cache", {})), q=P(256), B=2, R=5, q_heads=4, q_strides=_two(256, 64), rows=P(256),
                                   scale=0.1, out=P(256), out_strides=_two(256, 64), workspace=P(256), workspace_bytes=1 << 30)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _table(**kw):
    t = pk.pldp_page_table_args(pages=P(256), pages_stride=4, B=2, max_pages=3, page_size=16, refs=P(256), n_pages=10)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


BAD_ROWS = [(dict(B=-1), 1, "B < 0"), (dict(R=-1), 1, "R < 0"), (dict(q_heads=0), 1, "q_heads < 1"), (dict(R=2**31 - 100), 2, "rows|R must"),
            (dict(rows=None), 1, "null"), (dict(q=None), 1, "null"), (dict(q=P(264)), 1, "q is not 16-byte"),
            (dict(q_strides=_two(252, 64)), 1, "q strides"), (dict(q_strides=_two(-256, 64)), 1, "q strides")]


@pytest.mark.parametrize("bad,rc,why", BAD_ROWS + [
    (dict(dtype=2), 2, "dtype"), (dict(q_heads=65537), 2, "65536"), (dict(eps=-1.0), 1, "eps"), (dict(eps=float("nan")), 1, "eps"),
    (dict(cos=P(256)), 1, "go together"), (dict(cos=P(256), sin=P(256), rot=3, rot_rows=9), 1, "rot"),
    (dict(cos=P(256), sin=P(256), rot=4, rot_rows=0), 1, "rot"), (dict(cos=P(264), sin=P(256), rot=4, rot_rows=9), 1, "aligned"),
    (dict(k=None), 1, "null"), (dict(q_out=None), 1, "null"), (dict(q_out=P(260)), 1, "q_out"), (dict(q_norm=P(258)), 1, "norms")]
    + [(dict(cache=c), rc, why) for c, rc, why in BAD_CACHES])
def test_append_refusals(so, bad, rc, why):  # noqa: F811
    assert so.pldp_cache_append_prompt(ctypes.byref(_append(**dict(bad))), None) == rc
    import re
    assert re.search(why, pk.pldp_last_error()), pk.pldp_last_error()


@pytest.mark.parametrize("bad,rc,why", BAD_ROWS + [
    (dict(q_heads=3), 1, "multiple"), (dict(scale=float("inf")), 1, "scale"), (dict(workspace=None), 1, "null"),
    (dict(workspace=P(128)), 1, "aligned"), (dict(workspace_bytes=1000), 1, "workspace needs"), (dict(out=None), 1, "null"),
    (dict(out_strides=_two(256, 60)), 1, "out strides"), (dict(R=2**30, q_heads=8), 2, "too many rows"),
    (dict(cache=dict(page_size=2**30 - 1, max_pages=2, pages_stride=2)), 2, "positions a sequence")]
    + [(dict(cache=c), rc, why) for c, rc, why in BAD_CACHES])
def test_attend_refusals(so, bad, rc, why):  # noqa: F811
    assert so.pldp_attend_prompt(ctypes.byref(_attend(**dict(bad))), None) == rc
    import re
    assert re.search(why, pk.pldp_last_error()), pk.pldp_last_error()


def test_null_blocks_and_nothing_to_do(so):  # noqa: F811
    assert so.pldp_cache_append_prompt(None, None) == 1 and so.pldp_attend_prompt(None, None) == 1
    assert so.pldp_cache_append_prompt(ctypes.byref(_append(B=0, rows=None)), None) == 0
    assert so.pldp_attend_prompt(ctypes.byref(_attend(B=0, rows=None)), None) == 0
    assert so.pldp_attend_prompt_workspace_size(5, 2, 64) == 0 and so.pldp_attend_prompt_workspace_size(4, 2, 300) == 0
    small, large = (so.pldp_attend_prompt_workspace_size(4, 2, d) for d in (64, 128))
    assert 0 < small < large


BAD_TABLES = [(None, 1, "null table"), (dict(B=-1), 1, "B < 0"), (dict(max_pages=0), 1, "max_pages"), (dict(page_size=0), 1, "page_size"),
              (dict(n_pages=0), 1, "n_pages"), (dict(pages_stride=2), 1, "pages_stride"), (dict(page_size=2**30), 1, "2\\^31"),
              (dict(B=65536), 2, "65535"), (dict(n_pages=2**31 - 1), 2, "2\\^31 - 4096"), (dict(pages=None), 1, "null"), (dict(refs=None), 1, "null")]


@pytest.mark.parametrize("bad,rc,why", BAD_TABLES)
def test_table_refusals(so, bad, rc, why):  # noqa: F811
    import re
    t = None if bad is None else ctypes.byref(_table(**bad))
    calls = [lambda: so.pldp_pages_free(t, P(256), None), lambda: so.pldp_pages_fork(t, P(256), P(256), None, None),
             lambda: so.pldp_pages_reserve(t, P(256), None, 5, P(256), None, P(256), 1 << 40, None),
             lambda: so.pldp_pages_compact(t, P(256), 2**31 - 1, P(256), None, P(256), 1 << 40, None)]
    for call in calls:
        assert call() == rc and re.search(why, pk.pldp_last_error()), pk.pldp_last_error()


def test_page_refusals(so):  # noqa: F811
    t, none = ctypes.byref(_table()), ctypes.byref(_table(B=0, pages=None, refs=None))
    need = so.pldp_pages_workspace_size(2, 3, 10)
    for rc, why, got in [
            (1, "null", lambda: so.pldp_pages_free(t, None, None)), (1, "null", lambda: so.pldp_pages_fork(t, None, P(256), None, None)),
            (1, "null", lambda: so.pldp_pages_fork(t, P(256), None, None, None)),
            (1, "n < 0", lambda: so.pldp_pages_reserve(t, P(256), None, -1, P(256), None, P(256), need, None)),
            (1, "null", lambda: so.pldp_pages_reserve(t, None, None, 1, P(256), None, P(256), need, None)),
            (1, "null", lambda: so.pldp_pages_reserve(t, P(256), None, 1, None, None, P(256), need, None)),
            (1, "8-byte", lambda: so.pldp_pages_reserve(t, P(256), None, 1, P(260), None, P(256), need, None)),
            (1, "null", lambda: so.pldp_pages_reserve(t, P(256), None, 1, P(256), None, None, need, None)),
            (1, "workspace needs", lambda: so.pldp_pages_reserve(t, P(256), None, 1, P(256), None, P(256), need - 1, None)),
            (1, "aligned", lambda: so.pldp_pages_reserve(t, P(256), None, 1, P(256), None, P(264), need, None)),
            (1, "room for 4", lambda: so.pldp_pages_compact(t, P(256), 4, P(256), None, P(256), need, None)),
            (1, "null", lambda: so.pldp_pages_compact(t, None, 5, P(256), None, P(256), need, None)),
            (1, "null", lambda: so.pldp_pages_compact(t, P(256), 5, None, None, P(256), need, None)),
            (1, "8-byte", lambda: so.pldp_pages_compact(t, P(260), 5, P(256), None, P(256), need, None)),
            (1, "workspace needs", lambda: so.pldp_pages_compact(t, P(256), 5, P(256), None, P(256), 16, None)),
            (1, "null cache", lambda: so.pldp_cache_copy_pages(None, P(256), 1, None, None)),
            (1, "n < 0", lambda: so.pldp_cache_copy_pages(ctypes.byref(_cache()), P(256), -1, None, None)),
            (1, "null", lambda: so.pldp_cache_copy_pages(ctypes.byref(_cache()), None, 1, None, None))]:
        assert got() == rc and why in pk.pldp_last_error(), (why, pk.pldp_last_error())
    assert so.pldp_pages_free(none, None, None) == 0 and so.pldp_pages_fork(none, None, None, None, None) == 0
    assert so.pldp_pages_reserve(none, None, None, 1, None, None, None, 0, None) == 0
    assert so.pldp_cache_copy_pages(ctypes.byref(_cache()), None, 0, None, None) == 0
    assert so.pldp_pages_workspace_size(-1, 3, 10) == so.pldp_pages_workspace_size(2, 0, 10) == so.pldp_pages_workspace_size(2, 3, 0) == 0
    assert need >= 4 * 2 * 10 and so.pldp_pages_workspace_size(65535, 2**20, 2**20) > 65535 * 2**17


@pytest.mark.parametrize("bad,rc,why", [b for b in BAD_CACHES])
def test_copy_refusals(so, bad, rc, why):  # noqa: F811
    import re
    assert so.pldp_cache_copy_pages(ctypes.byref(_cache(**bad)), P(256), 1, None, None) == rc
    assert re.search(why, pk.pldp_last_error()), pk.pldp_last_error()


def test_sums_of_tiles(tmp_path):
    """The closed form of the list's sums (host code of the kernel's header) against adding up."""
    src = open(os.path.join(os.path.dirname(HEADER), "..", "paper_2412_01447_gb300", "csrc", "pldp_prompt.cuh")).read()
    body = src[src.index("__host__ __device__ inline uint64_t quotient"):src.index("// The rows of a sequence and kv head")]
    (tmp_path / "sum.c").write_text("#include <stdint.h>\n#include <stdbool.h>\n#include <stdio.h>\n#define __host__\n#define __device__\n#define PLDP_ONE_COPY\n" + body +
                                    'int main(void) { unsigned long long n, m, a, b; while (scanf("%llu %llu %llu %llu", &n, &m, &a, &b) == 4) '
                                    'printf("%llu\\n", (unsigned long long)floor_sum(n, m, a, b)); return 0; }')
    subprocess.check_call(["gcc", "-std=c99", "-Dinline=static", str(tmp_path / "sum.c"), "-o", str(tmp_path / "sum")])
    r = random.Random(5)
    rows = [(r.randint(0, 3000), 128 * r.choice([1, 2, 3, 5, 8, 40, 131]), r.choice([128, 256]), r.randint(0, 10**9)) for _ in range(300)]
    out = subprocess.run([str(tmp_path / "sum")], input="\n".join(" ".join(map(str, x)) for x in rows), capture_output=True, text=True, check=True)
    assert [int(x) for x in out.stdout.split()] == [sum((a * i + b) // m for i in range(n)) for n, m, a, b in rows]
