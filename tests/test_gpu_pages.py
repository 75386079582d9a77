"""The page calls against a plain page table on the host, and pldp_cache_copy_pages."""
import random

import pytest
import torch

from tests._cache import DEV, i32

pytestmark = pytest.mark.gpu


class Host:
    """One page after the other, as the header words it."""

    def __init__(self, B, max_pages, n_pages, page):
        self.pages, self.refs, self.page, self.n = [[-1] * max_pages for _ in range(B)], [0] * n_pages, page, n_pages

    def reserve(self, start, count):
        held = list(self.refs)
        free, given, spent = [x for x, r in enumerate(held) if r == 0], 0, 0
        copies, status = [], []
        for b, row in enumerate(self.pages):
            copies.append([-1, -1])
            status.append(0)
            if start[b] < 0 or count[b] < 0:
                status[b] = 8
                continue
            if count[b] == 0:
                continue
            if start[b] + count[b] > len(row) * self.page:
                status[b] = 4
                continue
            first = start[b] // self.page
            need = [e for e in range(first, (start[b] + count[b] - 1) // self.page + 1) if not 0 <= row[e] < self.n or held[row[e]] > 1]
            spent += len(need)
            if need and spent > len(free):
                status[b] = 4
                continue
            for e in need:
                old, row[e] = row[e], free[given]
                self.refs[free[given]] = 1
                given += 1
                if 0 <= old < self.n:
                    self.refs[old] -= 1
                    if e == first and start[b] % self.page:
                        copies[b] = [old, row[e]]
        return copies, status

    def fork(self, parent, lens):
        before = [list(r) for r in self.pages]
        status = [0] * len(parent)
        for b, p in enumerate(parent):
            if p == -1 or p == b:
                continue
            if not 0 <= p < len(parent) or (0 <= parent[p] < len(parent) and parent[p] != p):
                status[b] |= 32
            if 0 <= p < len(parent) and not 0 <= lens[b] <= len(before[b]) * self.page:
                status[b] |= 8
            if status[b]:
                continue
            for e, old in enumerate(before[b]):
                now = before[p][e] if e * self.page < lens[b] else -1
                if not 0 <= now < self.n:
                    now = -1
                if now >= 0:
                    self.refs[now] += 1
                if 0 <= old < self.n:
                    self.refs[old] -= 1
                self.pages[b][e] = now
        return status

    def free(self, keep):
        for b, k in enumerate(keep):
            for e, old in enumerate(self.pages[b]):
                if k >= 0 and e * self.page >= k:
                    if 0 <= old < self.n:
                        self.refs[old] -= 1
                    self.pages[b][e] = -1

    def compact(self):
        live = [x for x, r in enumerate(self.refs) if r > 0]
        holes = [x for x in range(len(live)) if self.refs[x] == 0]
        moves = list(zip(reversed(live), holes))
        to = dict(moves)
        for a, b in moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.pages = [[to.get(x, x) for x in r] for r in self.pages]
        return moves, len(live)


class Device:
    def __init__(self, lib, B, max_pages, n_pages, page, offset=0):
        self.lib = lib
        self.room = torch.full((B, max_pages + 3), -5, dtype=torch.int32, device=DEV)
        self.pages = self.room[:, :max_pages]
        self.pages.fill_(-1)
        self.refs = torch.zeros(n_pages + offset, dtype=torch.int32, device=DEV)[offset:]
        self.table = lib.pldp_page_table(self.pages, self.refs, page)
        self.ws = torch.full((lib.pldp_pages_workspace_size(self.table),), 255, dtype=torch.uint8, device=DEV)
        self.B, self.n_pages = B, n_pages

    def same(self, h):
        assert self.pages.tolist() == h.pages
        assert self.refs.tolist() == h.refs
        assert (self.room[:, self.pages.shape[1]:] == -5).all()

    def reserve(self, start, count, n=None):
        copies, status = torch.full((self.B, 2), 77, dtype=torch.int32, device=DEV), i32([0] * self.B)
        self.lib.pldp_pages_reserve(self.table, i32(start), copies, self.ws, n=max([0, *count]) if n is None else n, count=i32(count),
                                    status=status)
        return copies.tolist(), status.tolist()

    def fork(self, parent, lens):
        status = i32([0] * self.B)
        self.lib.pldp_pages_fork(self.table, i32(parent), i32(lens), status=status)
        return status.tolist()

    def compact(self):
        copies, n, used = torch.full((max(1, self.n_pages // 2), 2), 77, dtype=torch.int32, device=DEV), i32([-3]), i32([-3])
        self.lib.pldp_pages_compact(self.table, copies, n, self.ws, used=used)
        return [tuple(x) for x in copies.tolist()[: int(n)]], int(used)


# sequences, entries a row, pages, page size, longest reservation, the refs' place against 16 bytes
SIZES = [(1, 1, 1, 1, 1, 0), (3, 4, 9, 16, 20, 0), (8, 40, 200, 16, 100, 1), (20, 7, 60, 7, 30, 2), (5, 300, 700, 1, 120, 3),
         (300, 12, 2500, 64, 90, 0), (2, 3000, 5000, 16, 40000, 1), (33, 20, 100001, 32, 300, 0)]


@pytest.mark.parametrize("size", SIZES)
def test_a_pools_life(lib, size):
    """Random calls one after the other: the table, the counts, copies, moves and statuses after each."""
    B, per, n_pages, page, most, offset = size
    rng = random.Random(B * 1000 + per)
    h, d = Host(B, per, n_pages, page), Device(lib, B, per, n_pages, page, offset)
    lens = [0] * B
    for step in range(24):
        what = rng.choice(["reserve", "reserve", "reserve", "fork", "free", "compact"])
        if what == "reserve":
            start = [max(0, n - rng.choice([0, 0, 1, page])) for n in lens]
            count = [rng.choice([0, 1, rng.randint(0, most), -1 if rng.random() < 0.1 else 2]) for _ in range(B)]
            count = [min(c, most) for c in count]
            if rng.random() < 0.2:
                start[rng.randrange(B)] = -4
            want = h.reserve(start, count)
            assert d.reserve(start, count, n=most) == want
            for b in range(B):
                if want[1][b] == 0 and count[b] > 0:
                    lens[b] = max(lens[b], start[b] + count[b])
        elif what == "fork":
            parent = [rng.choice([-1, -1, b, rng.randrange(B)]) if rng.random() < 0.95 else rng.choice([-2, B]) for b in range(B)]
            kept = [lens[p] if 0 <= p < B else 0 for p in parent]
            kept = [k if rng.random() < 0.8 else rng.choice([k // 2, -1, per * page + 1]) for k in kept]
            want = h.fork(parent, kept)
            assert d.fork(parent, kept) == want
            old = list(lens)
            for b, p in enumerate(parent):
                if 0 <= p < B and p != b and want[b] == 0:
                    lens[b] = min(kept[b], old[p])
        elif what == "free":
            keep = [rng.choice([-1, -1, 0, lens[b] // 2, lens[b], 2 ** 31 - 1]) for b in range(B)]
            h.free(keep)
            lib.pldp_pages_free(d.table, i32(keep))
            lens = [n if k < 0 else min(n, k) for n, k in zip(lens, keep)]
        else:
            assert d.compact() == h.compact()
        d.same(h)


def test_samples_of_a_prompt(lib):
    """A fork shares everything; the samples' first step gives each its own last page, and the prompt's row keeps its."""
    h, d = Host(5, 8, 30, 16), Device(lib, 5, 8, 30, 16)
    for x in (h.reserve, d.reserve):
        x([0] * 5, [40, 0, 0, 0, 0])
    parent, lens = [-1, 0, 0, 0, 0], [40] * 5
    assert d.fork(parent, lens) == h.fork(parent, lens) == [0] * 5
    assert d.refs.tolist()[:3] == [5, 5, 5]
    copies, status = d.reserve([39] * 5, [0, 5, 5, 5, 20])
    assert (copies, status) == h.reserve([39] * 5, [0, 5, 5, 5, 20])
    assert copies == [[-1, -1], [2, 3], [2, 4], [2, 5], [2, 6]] and status == [0] * 5
    d.same(h)
    assert d.refs.tolist()[:8] == [5, 5, 1, 1, 1, 1, 1, 1]
    # all of a page written anew: none to copy
    d.fork([-1, 0, -1, -1, -1], [32] * 5), h.fork([-1, 0, -1, -1, -1], [32] * 5)
    assert d.reserve([0, 16, 0, 0, 0], [0, 20, 0, 0, 0]) == h.reserve([0, 16, 0, 0, 0], [0, 20, 0, 0, 0])
    d.same(h)


def test_too_few_pages(lib):
    """A sequence gets all of its pages or none, and what is left goes to those before it."""
    h, d = Host(4, 8, 6, 16), Device(lib, 4, 8, 6, 16)
    for start, count in (([0] * 4, [40, 60, 1, 0]), ([40, 0, 0, 0], [8, 0, 0, 16]), ([48, 0, 0, 0], [100, 0, 0, 0])):
        got = d.reserve(start, count)
        assert got == h.reserve(start, count)
        d.same(h)
    assert d.reserve([0] * 4, [1 << 30, 1, 1, 1])[1] == [4, 0, 0, 0]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("shape", [(9, 16, 2, 64, "token"), (9, 16, 2, 64, "head"), (40, 7, 3, 80, "token"), (5, 1, 8, 256, "token"),
                                   (6, 200, 1, 16, "head"), (7, 64, 8, 128, "wide"), (33, 4, 2, 32, "apart")])
def test_copy_pages(lib, shape, dtype):
    n, page, H, D, layout = shape
    if layout == "head":
        bits = [torch.randint(0, 120, (n, H, page, D), device=DEV, dtype=torch.uint8).permute(0, 2, 1, 3) for _ in "kv"]
    elif layout == "wide":                                        # a larger stride from head to head, and from page to page
        bits = [torch.randint(0, 120, (n + 1, page, H + 1, D + 32), device=DEV, dtype=torch.uint8)[1:, :, 1:, :D] for _ in "kv"]
    elif layout == "apart":                                       # pages are the inner dimension
        bits = [torch.randint(0, 120, (page, n, H, D), device=DEV, dtype=torch.uint8).transpose(0, 1) for _ in "kv"]
    else:
        bits = [torch.randint(0, 120, (n, page, H, D), device=DEV, dtype=torch.uint8) for _ in "kv"]
    if dtype == torch.bfloat16:
        bits = [b.to(torch.bfloat16) for b in bits]
    pools = [b if dtype == torch.bfloat16 else b.view(dtype) for b in bits]
    scales = [None, None] if dtype == torch.bfloat16 else [torch.rand((n, H, page), device=DEV) for _ in "kv"]
    cache = lib.pldp_cache(*pools, i32([[0]]), *scales)
    pairs = [[0, n - 1], [2, 1], [-1, -1], [3, n], [-1, 3], [3, 3]]
    want, want_scales = [b.clone() for b in bits], [None if s is None else s.clone() for s in scales]
    for x in want + [s for s in want_scales if s is not None]:
        x[n - 1], x[1] = x[0].clone(), x[2].clone()
    for n_copies in (i32([0]), i32([-9]), None, i32([100]), i32([2])):
        lib.pldp_cache_copy_pages(cache, i32(pairs), n_copies)
        if n_copies is not None and int(n_copies) <= 0:
            assert not all(torch.equal(a, b) for a, b in zip(bits, want))
            continue
        assert all(torch.equal(a, b) for a, b in zip(bits, want))
        assert all(a is None or torch.equal(a, b) for a, b in zip(scales, want_scales))
    lib.pldp_cache_copy_pages(cache, torch.zeros((0, 2), dtype=torch.int32, device=DEV))


def test_many_large_pages(lib):
    """More pieces than CTAs, beyond 2^32 bytes."""
    n, page, H, D = 9000, 128, 8, 256
    pool = torch.zeros((n, page, H, D), device=DEV, dtype=torch.bfloat16)
    pool[:400] = torch.randn((400, page, H, D), device=DEV, dtype=torch.bfloat16)
    cache = lib.pldp_cache(pool, pool, i32([[0]]))
    pairs = torch.stack((torch.arange(400), n - 1 - torch.arange(400)), 1).to(torch.int32).to(DEV)
    lib.pldp_cache_copy_pages(cache, pairs)
    assert torch.equal(pool[:400], pool[n - 400:].flip(0))
    assert (pool[400:n - 400] == 0).all()


def test_graph_replay(lib):
    """A step's reservation, captured once, on lengths that move."""
    h, d = Host(3, 20, 50, 16), Device(lib, 3, 20, 50, 16)
    start, copies = i32([0, 0, 0]), torch.zeros((3, 2), dtype=torch.int32, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        lib.pldp_pages_reserve(d.table, start, copies, d.ws, n=11)
    for now in ([0, 5, 9], [7, 16, 20], [18, 27, 31], [29, 38, 42]):
        start.copy_(i32(now))
        g.replay()
        torch.cuda.synchronize()
        h.reserve(now, [11] * 3)
        d.same(h)


def test_refusals(lib):
    d = Device(lib, 2, 4, 10, 16)
    pairs, one = torch.zeros((5, 2), dtype=torch.int32, device=DEV), i32([0])
    two = i32([0, 0])
    for call, match in [(lambda: lib.pldp_pages_reserve(d.table, two, pairs, d.ws, n=1), "copies"),
                        (lambda: lib.pldp_pages_reserve(d.table, one, pairs[:2], d.ws, n=1), "start"),
                        (lambda: lib.pldp_pages_reserve(None, two, pairs[:2], d.ws, n=1), "pldp_page_table"),
                        (lambda: lib.pldp_pages_fork(d.table, one, two), "parent"),
                        (lambda: lib.pldp_pages_fork(d.table, two, one), "len"),
                        (lambda: lib.pldp_pages_free(d.table, one), "keep_len"),
                        (lambda: lib.pldp_pages_compact(d.table, pairs.view(-1), one, d.ws), "copies"),
                        (lambda: lib.pldp_cache_copy_pages(None, pairs), "pldp_cache"),
                        (lambda: lib.pldp_page_table(d.pages, d.refs.float(), 16), "refs"),
                        (lambda: lib.pldp_page_table(d.pages.long(), d.refs, 16), "pages")]:
        with pytest.raises(ValueError, match=match):
            call()
    for call, match in [(lambda: lib.pldp_pages_reserve(d.table, two, pairs[:2], d.ws, n=-1), "n < 0"),
                        (lambda: lib.pldp_pages_reserve(d.table, two, pairs[:2], d.ws[:16], n=1), "workspace"),
                        (lambda: lib.pldp_pages_compact(d.table, pairs[:4], one, d.ws), "room"),
                        (lambda: lib.pldp_pages_free(lib.pldp_page_table(d.pages, d.refs, 0), two), "page_size"),
                        (lambda: lib.pldp_pages_free(lib.pldp_page_table(d.pages, d.refs, 1 << 30), two), "2\\^31")]:
        with pytest.raises(lib.PldpError, match=match):
            call()
