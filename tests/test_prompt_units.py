"""How pldp_attend_prompt's work is cut: the tiles before a unit in closed form, and the unit that holds a place of the list, against
a count unit by unit.  The host's copy of the functions that the kernel uses."""
import bisect
import ctypes
import itertools
import random
import subprocess

import pytest

from paper_2412_01447_gb300 import _build

SOURCE = """
#include "pldp_prompt.cuh"
using namespace pldp;
template <int UR>
static int at(int group, int start, int count, long long x, long long* before) {
    const Units s = {static_cast<int64_t>(count) * group, group, start, count};
    int64_t b;
    const int u = unit_at<UR>(s, unit_count<UR>(s), x, &b);
    *before = b;
    return u;
}
extern "C" __attribute__((visibility("default"))) long long cost(int rows, int group, int start, int count, int u) {
    const Units s = {static_cast<int64_t>(count) * group, group, start, count};
    return rows == 128 ? cost_before<128>(s, u) : cost_before<256>(s, u);
}
extern "C" __attribute__((visibility("default"))) int unit(int rows, int group, int start, int count, long long x, long long* before) {
    return rows == 128 ? at<128>(group, start, count, x, before) : at<256>(group, start, count, x, before);
}
"""
COST, TILE = 2, 128                          # what a unit costs beside its tiles, and a tile's keys


@pytest.fixture(scope="module")
def units(tmp_path_factory):
    d = tmp_path_factory.mktemp("units")
    (d / "units.cu").write_text(SOURCE)
    out = str(d / "libunits.so")
    r = subprocess.run([_build.nvcc(), *_build.ARCH, *_build.NVCC_FLAGS, "-shared", str(d / "units.cu"), "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    so = ctypes.CDLL(out)
    i, x = ctypes.c_int, ctypes.c_longlong
    so.cost.argtypes, so.cost.restype = [i] * 5, x
    so.unit.argtypes, so.unit.restype = [i] * 4 + [x, ctypes.POINTER(x)], i
    return so


def _costs(rows, group, start, count, most=None):
    """cost[u]: what the units before u cost, for all units (or the first `most`)."""
    n = -(-count * group // rows)
    cost = [0]
    for u in range(n if most is None else min(n, most)):
        last = (min(count * group, (u + 1) * rows) - 1) // group
        cost.append(cost[-1] + COST + (start + last) // TILE + 1)
    return cost


@pytest.mark.parametrize("rows", [128, 256])
def test_small(units, rows):
    for group, start, count in itertools.product([1, 2, 3, 4, 5, 7, 8, 127, 128, 131, 300], [0, 1, 63, 127, 128, 129, 1000], [1, 2, 63, 64, 129, 700]):
        cost = _costs(rows, group, start, count)
        assert [units.cost(rows, group, start, count, u) for u in range(len(cost))] == cost, (group, start, count)


@pytest.mark.parametrize("rows", [128, 256])
def test_places(units, rows):
    rng = random.Random(5)
    before = ctypes.c_longlong()
    for _ in range(300):
        group, start, count = rng.choice([1, 3, 4, 5, 8, 40, 131]), rng.choice([0, 5, 4096, rng.randrange(10 ** 6)]), rng.randrange(1, 3000)
        cost = _costs(rows, group, start, count)
        for x in {0, cost[-1] - 1, *(rng.randrange(cost[-1]) for _ in range(20))}:
            u = units.unit(rows, group, start, count, x, ctypes.byref(before))
            assert u == bisect.bisect_right(cost, x) - 1 and before.value == cost[u], (group, start, count, x)


@pytest.mark.parametrize("rows", [128, 256])
@pytest.mark.parametrize("group,start,count", [(1, 2 ** 31 - 4096 - 1000, 1000), (65536, 2 ** 31 - 4096 - 300, 300), (1, 0, 2 ** 31 - 4096),
                                               (7, 10 ** 9 + 7, 300_000_000), (2 ** 20 + 1, 12345, 2000)])
def test_far(units, rows, group, start, count):
    cost = _costs(rows, group, start, count, 2000)
    assert [units.cost(rows, group, start, count, u) for u in range(len(cost))] == cost
    # and one unit's step, far on
    n = -(-count * group // rows)
    for u in (n // 2, n - 2, n - 1):
        if u >= 0:
            last = (min(count * group, (u + 1) * rows) - 1) // group
            assert units.cost(rows, group, start, count, u + 1) - units.cost(rows, group, start, count, u) == COST + (start + last) // TILE + 1
