"""Pages of a cache: fork, reserve, free, compact and copy against a plain state machine."""
import numpy as np
import pytest
import torch

import paper_2609_18063_b200 as edg
from _latent_ref import Pages

pytestmark = pytest.mark.gpu


class Both:
    """The pool on the device and the state machine beside it.  A row's value is its own number; the machine keeps numbers."""

    def __init__(self, n_pages, page, n_seqs, max_pages, layers=2, row=8, seed=0):
        self.ref = Pages(n_pages, page, n_seqs, max_pages, layers)
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        self.table = torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(n_seqs, dtype=torch.int32, device="cuda")
        self.cache = torch.arange(layers * n_pages * page, dtype=torch.int32, device="cuda").view(layers, n_pages, page, 1).repeat(1, 1, 1, row).contiguous()
        for l in range(layers):
            for p in range(n_pages):
                for r in range(page):
                    self.ref.rows[l][p][r] = (l * n_pages + p) * page + r
        self.pool = edg.make_page_pool(self.refs, self.table, self.lens, page=page)
        self.pc = edg.make_page_cache(self.cache)
        self.ws = torch.zeros(edg.pages_workspace_bytes(self.pool), dtype=torch.uint8, device="cuda")

    def t(self, v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    def fork(self, a, c):
        edg.pages_fork(self.pool, len(a), self.t(a), self.t(c), self.ws)
        return self.ref.fork(a, c)

    def reserve(self, s, n):
        edg.pages_reserve(self.pool, self.pc, len(s), self.t(s), self.t(n), self.ws)
        return self.ref.reserve(s, n)

    def free(self, s):
        edg.pages_free(self.pool, len(s), self.t(s), self.ws)
        return self.ref.free(s)

    def compact(self):
        edg.pages_compact(self.pool, self.pc, self.ws)
        self.ref.compact()

    def check(self, status=0):
        assert edg.workspace_status(self.ws) == status
        assert self.refs.cpu().tolist() == self.ref.refs.tolist()
        assert self.lens.cpu().tolist() == self.ref.lens.tolist()
        tab = self.table.cpu().numpy()
        for s, ps in enumerate(self.ref.pages):
            assert tab[s, :len(ps)].tolist() == ps
        got = self.cache.cpu().numpy()
        assert (got == got[..., :1]).all()
        assert np.array_equal(got[..., 0], np.array(self.ref.rows))


def test_fork_grow_and_free():
    b = Both(64, 16, 12, 8)
    b.reserve([0, 1], [40, 16])
    b.check()
    b.fork([0, 0, 1, 0], [2, 3, 4, 5])
    b.check()
    b.reserve([2, 4, 3, 5, 0], [1, 1, 30, 0, 8])       # 2 and 3 copy, 4 takes a page of its own, 5 stays, 0 copies (5 still holds it)
    b.check()
    b.reserve([5], [3])                                 # nobody else holds the page any more
    b.check()
    b.free([0, 3])
    b.check()
    b.reserve([0, 6], [100, 5])                         # the lowest free pages again
    b.check()
    b.compact()
    b.check()


def test_all_holders_grow_at_once():
    b = Both(64, 16, 12, 8)
    b.reserve([0], [20])
    b.fork([0] * 4, [1, 2, 3, 4])
    b.reserve([4, 2, 0, 1, 3], [1, 1, 1, 1, 1])         # the last in the list keeps the page
    b.check()
    assert b.ref.pages[3][-1] == 1


def test_too_few_pages_change_nothing():
    b = Both(8, 16, 6, 8)
    b.reserve([0, 1], [60, 30])
    b.check()
    before = (b.refs.clone(), b.table.clone(), b.lens.clone(), b.cache.clone())
    assert b.reserve([2, 1, 3], [16, 16, 20])[1]
    for x, y in zip(before, (b.refs, b.table, b.lens, b.cache)):
        assert torch.equal(x, y)
    b.check(-3)


def test_mistakes_are_skipped_and_raised():
    b = Both(64, 16, 8, 4)
    b.reserve([0], [20])
    for op, a in [(b.fork, ([0, 0, 9, 0, 3], [1, 1, 2, -1, 3])), (b.fork, ([0, 1], [4, 0])), (b.reserve, ([1, 1, 8, 2, 3], [2, 2, 1, -1, 65])),
                  (b.free, ([1, 1, -2, 70],))]:
        b.ws[:4096].zero_()
        bad = op(*a)
        assert (bad[0] if isinstance(bad, tuple) else bad)
        b.check(-4)


def test_freeing_twice_in_one_list_is_once():
    b = Both(16, 16, 4, 4)
    b.reserve([0], [20])
    b.fork([0], [1])
    b.free([0, 0])
    b.check()


@pytest.mark.parametrize("seed", range(6))
def test_a_long_run(seed):
    rng = np.random.default_rng(seed)
    page = int(rng.choice([16, 32]))
    b = Both(int(rng.integers(30, 120)), page, 20, 12, layers=int(rng.integers(1, 4)))
    short = False
    for _ in range(40):
        k = rng.integers(0, 8)
        live = [s for s in range(20) if b.ref.lens[s] > 0]
        empty = [s for s in range(20) if b.ref.lens[s] == 0]
        if k < 4:
            s = [int(x) for x in rng.permutation(20)[:rng.integers(1, 8)]]
            n = [int(min(rng.integers(0, 2 * page), 12 * page - b.ref.lens[x])) for x in s]
            short |= b.reserve(s, n)[1]
        elif k < 6 and live and empty:
            c = empty[:int(rng.integers(1, 4))]
            b.fork([int(x) for x in rng.choice(live, len(c))], c)
        elif k == 6 and live:
            b.free([int(x) for x in rng.choice(live, min(3, len(live)), replace=False)])
        else:
            b.compact()
        b.check(-3 if short else 0)


@pytest.mark.parametrize("n_pages", [1, 7, 1023, 1024, 8192, 8193, 20000])
def test_pools_of_many_pages(n_pages):
    b = Both(n_pages, 1, 3, n_pages, layers=1, row=4)
    rng = np.random.default_rng(n_pages)
    b.reserve([0, 1], [n_pages // 2, n_pages - n_pages // 2])
    b.check()
    b.free([0])
    b.compact()
    b.check()
    b.reserve([2], [int(rng.integers(0, n_pages // 2 + 1))])
    b.check()


def test_the_longest_lists():
    b = Both(4096, 16, 1025, 4, layers=1, row=4)
    b.reserve([0], [17])
    b.fork([0] * 1023, list(range(1, 1024)))
    b.check()
    b.reserve(list(range(1024)), [16] * 1024)
    b.check()
    b.free(list(range(0, 1024)))
    b.check()


def test_copy_between_and_within_caches():
    src = torch.randn(3, 10, 16, 8, device="cuda")
    dst = torch.zeros(3, 20, 16, 8, device="cuda")
    s, d = edg.make_page_cache(src), edg.make_page_cache(dst)
    ws = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    t = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")      # noqa: E731
    edg.pages_copy(d, s, 4, t([19, 3, 3, 0]), t([0, 1, 2, 9]), ws)        # 3 is named twice: the last one counts
    torch.cuda.synchronize()
    want = torch.zeros_like(dst)
    want[:, 19], want[:, 3], want[:, 0] = src[:, 0], src[:, 2], src[:, 9]
    assert torch.equal(dst, want) and edg.workspace_status(ws) == 0
    edg.pages_copy(d, d, 3, t([5, 6, 7]), t([19, 19, 7]), ws)
    want[:, 5], want[:, 6] = want[:, 19], want[:, 19]
    assert torch.equal(dst, want) and edg.workspace_status(ws) == 0
    edg.pages_copy(d, d, 2, t([19, 8]), t([3, 19]), ws)                   # 19 is read and written in one call
    want[:, 8] = want[:, 19]
    torch.cuda.synchronize()
    assert torch.equal(dst, want) and edg.workspace_status(ws) == -4
    ws.zero_()
    edg.pages_copy(d, s, 3, t([20, 1, -1]), t([0, 10, 0]), ws)
    torch.cuda.synchronize()
    assert torch.equal(dst, want) and edg.workspace_status(ws) == -4


def test_replayed_and_on_another_stream():
    b = Both(64, 16, 8, 16)
    b.reserve([0], [50])
    s, n = b.t([0, 1]), b.t([5, 9])
    a, c = b.t([0]), b.t([1])
    f = b.t([1])
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
        edg.pages_fork(b.pool, 1, a, c, b.ws)
        edg.pages_reserve(b.pool, b.pc, 2, s, n, b.ws)
        edg.pages_free(b.pool, 1, f, b.ws)
    for _ in range(4):
        g.replay()
        b.ref.fork([0], [1])
        b.ref.reserve([0, 1], [5, 9])
        b.ref.free([1])
        b.check()
