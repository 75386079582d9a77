"""The packed calls, the pages and a step's calls together, as a server of samples uses them: prompts, copies of their pages'
entries, steps of each copy, sequences that end, pages that move, and prompts behind what is held already."""
import pytest
import torch

from tests._cache import DEV, attend64, gen, i32
from tests.test_gpu_prompt import _check as check_prompt, _rows, prompt64

pytestmark = pytest.mark.gpu


class Layer:
    """A layer's cache, and what was appended of every sequence in 64 bits: read from its pages at once, whatever happens
    to them later."""

    def __init__(self, lib, B, pages, n_pages, page, heads, D, dtype, seed):
        self.lib, self.pages, self.page, self.heads, self.D, self.dtype, self.B = lib, pages, page, heads, D, dtype, B
        self.ctx, self.g = pages.shape[1] * page, gen(seed)
        kind = torch.bfloat16 if dtype == "bf16" else torch.float8_e4m3fn
        self.pools = [torch.full((n_pages, page, heads, D), float("nan"), device=DEV).to(kind) for _ in "kv"]
        self.scales = [torch.full((n_pages, heads, page), float("nan"), device=DEV) if dtype == "e4m3" else None for _ in "kv"]
        self.handle = lib.pldp_cache(*self.pools, pages, *self.scales)
        self.dense = {x: [torch.zeros((0, heads, D), dtype=torch.float64, device=DEV) for _ in range(B)] for x in "kv"}

    def draw(self, *size):
        return torch.randn((*size, self.D), generator=self.g, device=DEV, dtype=torch.bfloat16)

    def record(self, b, start, given):
        """Sequence b's positions from `start` now hold `given` (k and v [count, heads, D])."""
        p = start + torch.arange(given[0].shape[0], device=DEV)
        pg, slot = self.pages[b, p // self.page].long(), p % self.page
        for name, pool, scale, want in zip("kv", self.pools, self.scales, given):
            x = pool.view(torch.int16 if scale is None else torch.uint8)[pg, slot].view(pool.dtype).double()
            if scale is not None:
                x = x * scale.permute(0, 2, 1)[pg, slot].double()[..., None]
                # half a step of the code, and of the smallest codes 2^-10 of a scale of 1/448 of the largest element
                bound = 2 ** -4 * want.double().abs() + 2 ** -10 / 448 * want.double().abs().amax(-1, keepdim=True)
                assert ((x - want.double()).abs() <= bound * (1 + 1e-6)).all()
            else:
                assert torch.equal(x, want.double())
            self.dense[name][b] = torch.cat((self.dense[name][b][:start], x))

    def prompt(self, counts, starts, Hq):
        """Appends packed tokens and attends for them."""
        rows = _rows(counts)
        q, k, v = (self.draw(rows[-1], h) for h in (Hq, self.heads, self.heads))
        status, r, at = i32([0] * self.B), i32(rows), i32(starts)
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
        ws = torch.empty(self.lib.pldp_attend_prompt_workspace_size(Hq, self.heads, self.D), dtype=torch.uint8, device=DEV)
        raw = q.clone()
        self.lib.pldp_cache_append_prompt(self.handle, raw, k, v, r, q, start=at, status=status)
        self.lib.pldp_attend_prompt(self.handle, q, r, out, ws, start=at, lse=lse, status=status)
        assert status.tolist() == [0] * self.B and torch.equal(q, raw)
        for b, n in enumerate(counts):
            if n:
                self.record(b, starts[b], [x[rows[b]:rows[b + 1]] for x in (k, v)])
        check_prompt(out, lse, prompt64(self, q, rows, starts, self.D ** -0.5), self.dtype)

    def step(self, lens, drafts, Hq):
        """One token and its draft of every sequence behind the `lens` positions that it holds (None: it does not exist)."""
        n = max(drafts) + 1
        q, k, v = (self.draw(self.B, n, h) for h in (Hq, self.heads, self.heads))
        L = [0 if x is None else x + 1 for x in lens]
        status, Lt, dt = i32([0] * self.B), i32(L), i32(drafts)
        out, lse = torch.zeros_like(q), torch.full(q.shape[:3], -float("inf"), device=DEV)
        ws = torch.zeros(self.lib.pldp_attend_workspace_size(self.B, n, Hq, self.heads, self.D), dtype=torch.uint8, device=DEV)
        self.lib.pldp_cache_append(self.handle, q.clone(), k, v, Lt, q, draft_len=dt, status=status)
        self.lib.pldp_attend_cache(self.handle, q, Lt, out, ws, draft_len=dt, lse=lse, status=status)
        assert all(s == 0 for s, x in zip(status.tolist(), lens) if x is not None)
        for b, x in enumerate(lens):
            if x is not None:
                self.record(b, x, [y[b, : drafts[b] + 1] for y in (k, v)])
        # the result is rounded to bf16 (half a step, 2^-8 of it), each weight to 16 bits (2^-8 of what it weighs at most)
        o, l, size = attend64(self, q, L, drafts, self.D ** -0.5, self.heads)
        assert torch.equal(torch.isinf(lse), torch.isinf(l))
        live = torch.isfinite(l)
        assert ((lse.double() - l).abs()[live] <= 2e-5 * (1 + l.abs()[live])).all()
        assert ((out.double() - o).abs() <= 2 ** -8 * (o.abs() + size) + 1e-5 * size).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,D,Hq,H", [(16, 64, 4, 2), (7, 128, 6, 2), (64, 256, 3, 1)])
def test_samples(lib, page, D, Hq, H, dtype):
    B, per = 7, -(-300 // page)
    n_pages = 4 * per
    pages, refs = torch.full((B, per), -1, dtype=torch.int32, device=DEV), i32([0] * n_pages)
    table = lib.pldp_page_table(pages, refs, page)
    ws = torch.empty(lib.pldp_pages_workspace_size(table), dtype=torch.uint8, device=DEV)
    copies, status = i32([[-1, -1]] * B), i32([0] * B)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layers = [Layer(lib, B, pages, n_pages, page, H, D, dtype, seed) for seed in (1, 2)]

        def reserve(starts, counts):
            lib.pldp_pages_reserve(table, i32(starts), copies, ws, n=max(counts), count=i32(counts), status=status)
            for layer in layers:
                lib.pldp_cache_copy_pages(layer.handle, copies)

        def held_once_an_entry():
            flat = pages[pages >= 0].long()
            assert torch.equal(torch.bincount(flat, minlength=n_pages).int(), refs)

        # two prompts
        counts = [37, 0, 0, 0, 130, 0, 0]
        reserve([0] * B, counts)
        for layer in layers:
            layer.prompt(counts, [0] * B, Hq)
        # three samples of the first (one of a part of it), one of the second
        lens = [37, 37, 37, 30, 130, 130, None]
        lib.pldp_pages_fork(table, i32([-1, 0, 0, 0, -1, 4, -1]), i32([0, 37, 37, 30, 0, 130, 0]), status=status)
        for layer in layers:
            for x in layer.dense.values():
                x[1], x[2], x[3], x[5] = x[0], x[0], x[0][:30], x[4]
        held_once_an_entry()
        for drafts in ([0] * B, [2, 0, 3, 1, 3, 0, 0], [0, 3, 0, 0, 1, 2, 0]):
            reserve([x or 0 for x in lens], [0 if x is None else d + 1 for x, d in zip(lens, drafts)])
            for layer in layers:
                layer.step(lens, drafts, Hq)
            lens = [None if x is None else x + d + 1 for x, d in zip(lens, drafts)]
        held_once_an_entry()
        # one ends, one goes back to its first 20 positions, and the pages move together
        lib.pldp_pages_free(table, i32([-1, 0, -1, 20, -1, -1, -1]))
        moves, n_moves, used = i32([[-1, -1]] * (n_pages // 2)), i32([0]), i32([0])
        lib.pldp_pages_compact(table, moves, n_moves, ws, used=used)
        for layer in layers:
            lib.pldp_cache_copy_pages(layer.handle, moves, n_copies=n_moves)
        held_once_an_entry()
        assert int(used) == int((refs > 0).sum()) and (refs[: int(used)] > 0).all()
        for layer in layers:
            for x in layer.dense.values():
                x[1] = x[1][:0]
                x[3] = x[3][:20]
        # a new prompt, more of an old one and single tokens, packed, behind what each holds
        starts, counts = [lens[0], 0, lens[2], 20, lens[4], lens[5], 0], [1, 50, 1, 70, 100, 1, 0]
        reserve(starts, counts)
        for layer in layers:
            layer.prompt(counts, starts, Hq)
        assert status.tolist() == [0] * B
        held_once_an_entry()
        lib.pldp_pages_free(table, i32([0] * B))
        assert (pages == -1).all() and (refs == 0).all()
    torch.cuda.current_stream().wait_stream(stream)
