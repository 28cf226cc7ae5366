"""Page operators on the GPU, bit for bit against the host model."""
import numpy as np
import pytest
import torch

from paper_2605_21603_amd import binding as B
from pages_model import DONE, NONE_LEFT, REFUSED, Model

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Case:
    """A pool on the GPU beside the model of it."""

    def __init__(self, *, layers=3, pages=50, kv=2, ps=16, hd=16, dtype=torch.bfloat16, rows=8, width=10, max_requests=16, placed=False, seed=0):
        gen = torch.Generator().manual_seed(seed)
        k = torch.randn((layers, pages, kv, ps, hd), generator=gen).to(dtype)
        v = torch.randn((layers, pages, kv, hd, ps), generator=gen).to(dtype)
        bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
        self.bits = bits
        table, lens, ref = np.full((rows, width), 7, np.int32), np.zeros(rows, np.int32), np.zeros(pages, np.int32)
        self.model = Model(k.view(bits).numpy(), v.view(bits).numpy(), table, lens, ref, ps)
        # a guard on both sides of every cache layer
        self.held = [[torch.zeros(t[0].numel() + 2 * 64, dtype=dtype, device=DEV) for _ in range(layers)] for t in (k, v)]
        if placed:
            self.k = [h[64:-64].view(k[0].shape).copy_(t) for h, t in zip(self.held[0], k)]
            self.v = [h[64:-64].view(v[0].shape).copy_(t) for h, t in zip(self.held[1], v)]
        else:
            self.k, self.v = k.to(DEV), v.to(DEV)
        self.table, self.lens, self.ref = (torch.from_numpy(a.copy()).to(DEV) for a in (table, lens, ref))
        self.pool = B.PagePool(self.k, self.v, self.table, self.lens, self.ref, max_requests)

    def ints(self, a):
        return torch.tensor(list(a), dtype=torch.int32, device=DEV)

    def check(self):
        torch.cuda.synchronize()
        m = self.model
        assert np.array_equal(self.lens.cpu().numpy(), m.lens)
        assert np.array_equal(self.ref.cpu().numpy(), m.ref)
        assert np.array_equal(self.table.cpu().numpy(), m.table)
        for mine, want in ((self.k, m.k), (self.v, m.v)):
            for layer, t in enumerate(mine):
                assert np.array_equal(t.view(self.bits).cpu().numpy(), want[layer]), layer
        for h in self.held[0] + self.held[1]:
            assert not h[:64].any() and not h[-64:].any()

    def fork(self, parents, children):
        got = self.pool.fork(self.ints(parents), self.ints(children))
        want = self.model.fork(list(parents), list(children))
        assert got.tolist() == want
        self.check()
        return want

    def resize(self, rows, lengths):
        got = self.pool.resize(self.ints(rows), self.ints(lengths))
        want = self.model.resize(list(rows), list(lengths))
        assert got.tolist() == want
        self.check()
        return want

    def compact(self):
        new_page, n_live = self.pool.compact()
        want, live = self.model.compact()
        assert np.array_equal(new_page.cpu().numpy(), want) and n_live.item() == live
        self.check()


def test_a_row_grows_is_forked_cut_back_and_freed():
    c = Case()
    assert c.resize([2, 5], [37, 16]) == [DONE, DONE]              # three pages, one exactly full
    assert c.fork([2, 5, 2, 1], [0, 1, 3, 4]) == [DONE] * 4         # a full last page is shared; an empty row has nothing to share
    assert c.resize([0], [90]) == [DONE]                            # the fork goes on, on its own pages
    assert c.resize([3], [20]) == [DONE]                            # back into a page the others still name: a copy
    assert c.resize([2], [32]) == [DONE]                            # back to the end of a shared page: none
    assert c.resize([0, 2, 3], [0, 0, 0]) == [DONE] * 3
    c.compact()
    assert c.resize([1, 5], [0, 0]) == [DONE] * 2
    assert (c.model.ref == 0).all()
    c.compact()                                                     # nothing is left to move


def test_requests_are_served_in_order_until_the_pages_run_out():
    c = Case(pages=10, rows=6, width=10)
    assert c.resize([0, 1, 2, 3], [70, 40, 60, 0]) == [DONE, DONE, NONE_LEFT, DONE]     # 5 + 3 of 10, 4 more do not fit
    assert c.fork([0, 0, 1, 0], [2, 3, 4, 5]) == [DONE, DONE, NONE_LEFT, NONE_LEFT]     # two free pages, each fork needs one
    assert c.resize([0, 2, 2], [0, 0, 5]) == [DONE, DONE, REFUSED]
    assert c.resize([4, 5], [80, 1]) == [NONE_LEFT, NONE_LEFT]                           # what lies behind one that does not fit does not either
    assert c.resize([5], [1]) == [DONE]


def test_requests_that_name_nothing_or_the_same_are_refused():
    c = Case()
    c.resize([0, 1], [20, 20])
    assert c.resize([-1, 8, 0, 0, 1, 1], [5, 5, -1, 21, 161, 3]) == [REFUSED, REFUSED, REFUSED, REFUSED, REFUSED, REFUSED]
    assert c.fork([0, 0, -1, 9, 2, 0, 0], [1, 0, 3, 4, 2, 5, 5]) == [REFUSED, REFUSED, REFUSED, REFUSED, REFUSED, DONE, REFUSED]
    assert c.resize([5, 5, 0], [0, 10, 0]) == [DONE, REFUSED, DONE]


def test_numbers_that_no_pool_holds_are_never_followed():
    """A row whose entries and length are nonsense: refused or skipped, everything else served."""
    c = Case()
    c.resize([0, 1, 2], [40, 40, 33])
    for row, entry in ((1, -1), (2, 1 << 30)):
        c.table[row, 2] = entry                       # the partly filled last page
    c.lens[3] = 1 << 20
    got = c.pool.fork(c.ints([1, 2, 3, 0]), c.ints([4, 5, 6, 7]))
    assert got.tolist() == [REFUSED, REFUSED, REFUSED, DONE]
    assert c.pool.resize(c.ints([3, 1, 2]), c.ints([0, 35, 0])).tolist() == [REFUSED, REFUSED, DONE]
    c.pool.copy(c.ints([0, -1, 50, 3]), c.ints([49, 48, 47, 99]))
    torch.cuda.synchronize()
    assert torch.equal(c.k[:, 49], c.k[:, 0])
    assert np.array_equal(c.k[:, 47:49].view(torch.int16).cpu().numpy(), c.model.k[:, 47:49])
    c.pool.compact()
    torch.cuda.synchronize()


@pytest.mark.parametrize("placed,layers,kv,ps,hd,dtype", [(False, 1, 1, 1, 8, torch.bfloat16), (True, 3, 8, 16, 128, torch.bfloat16), (False, 2, 3, 48, 64, torch.float32),
                                                         (True, 130, 1, 16, 8, torch.float32), (False, 65, 2, 5, 8, torch.bfloat16)])
def test_copies_of_every_size_and_number_of_layers(placed, layers, kv, ps, hd, dtype):
    c = Case(layers=layers, kv=kv, ps=ps, hd=hd, dtype=dtype, placed=placed, pages=30)
    c.pool.copy(c.ints([3, 3, 7, 0]), c.ints([29, 5, 11, 0]))
    c.model.copy([3, 3, 7], [29, 5, 11])
    c.check()
    c.resize([0, 1, 2], [4 * ps, 3 * ps - (ps > 1), 2 * ps])
    c.fork([1, 1], [3, 4])
    c.resize([0], [0])
    c.compact()


@pytest.mark.parametrize("seed", range(4))
def test_a_long_run_of_calls(seed):
    rs = np.random.RandomState(seed)
    c = Case(pages=150, rows=40, width=16, layers=2, hd=8, max_requests=64, seed=seed)
    seen = set()
    for _ in range(40):
        n = rs.randint(1, 40)
        rows = rs.randint(-1, 41, n)
        what = rs.randint(5)
        if what < 2:
            seen.update(c.resize(rows, rs.choice([0, 16, 100, 255, 256, 257], n)))
        elif what < 4:
            seen.update(c.fork(rs.randint(-1, 41, n), rows))
        else:
            c.compact()
    assert seen == {DONE, NONE_LEFT, REFUSED}


def test_more_requests_and_pages_than_a_workgroup_looks_at_in_one_round():
    """2500 rows, 40000 pages: searches of several rounds, requests of several batches, sums carried between them."""
    rs = np.random.RandomState(1)
    c = Case(pages=40000, rows=3000, width=20, layers=1, kv=1, hd=8, max_requests=3000)
    rows = rs.permutation(3000)[:2500]
    c.resize(rows, rs.randint(0, 300, 2500))
    gone = rs.permutation(rows)[:1300]
    c.resize(gone, np.zeros(1300, np.int64))
    empty = np.flatnonzero(c.model.lens == 0)
    c.fork(rs.choice(rows, 1200), empty[:1200])
    c.resize(rs.permutation(3000), rs.randint(0, 321, 3000))
    c.compact()
    # a pool whose only free pages are its last ones
    full = Case(pages=40000, rows=2, width=2, layers=1, kv=1, hd=8)
    full.ref[:39998] = 1
    full.model.ref[:39998] = 1
    assert full.resize([0, 1], [17, 16]) == [DONE, NONE_LEFT] and full.model.table[0, 0] == 39998
    # more asked for than 32 bits count, in one call
    cache = torch.zeros((1, 20, 1, 16, 8), dtype=torch.bfloat16, device=DEV)
    table = torch.zeros((2100, 1 << 20), dtype=torch.int32, device=DEV)
    pool = B.PagePool(cache, cache.view(1, 20, 1, 8, 16), table, full.ints([0] * 2100), full.ints([0] * 20), 2100)
    got = pool.resize(full.ints(range(2100)), full.ints([1] + [16 << 20] * 2098 + [0]))
    assert got.tolist() == [DONE] + [NONE_LEFT] * 2098 + [DONE] and table.sum().item() == 0 and pool.seq_len.sum().item() == 1


def test_captured_calls_replay_on_what_the_tables_hold_then():
    """Fork, grow, free and compact in one graph, replayed with the program's own work and waits between."""
    c = Case(pages=80, rows=12)
    c.resize([0, 1], [40, 23])
    parents, children = c.ints([0, 1, 0]), c.ints([4, 5, 6])
    lengths, status = c.ints([50, 24, 41]), torch.empty((3, 3), dtype=torch.int32, device=DEV)
    nothing, new_page, n_live = c.ints([0, 0, 0]), torch.empty(80, dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)

    def calls():
        c.pool.fork(parents, children, status[0])
        c.pool.resize(children, lengths, status[1])
        c.pool.resize(children, nothing, status[2])
        c.pool.compact(new_page, n_live)

    def model():
        out = [c.model.fork([0, 1, 0], [4, 5, 6]), c.model.resize([4, 5, 6], lengths.tolist()), c.model.resize([4, 5, 6], [0, 0, 0])]
        return out, c.model.compact()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
        model()
    torch.cuda.current_stream().wait_stream(side)
    c.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for step in range(4):
        c.resize([2, 3], [step * 30, 90 - step * 30])
        lengths.copy_(c.ints([50 + step, 24 + 9 * step, 41]))
        graph.replay()
        want, (pages, live) = model()
        c.check()
        assert status.tolist() == want and n_live.item() == live and np.array_equal(new_page.cpu().numpy(), pages)


def test_two_streams_and_two_pools():
    """Calls on a stream that is not the current one, beside another pool's on another."""
    a, b = Case(seed=1), Case(seed=2)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for c, s in ((a, sa), (b, sb)):
        rows, lens, kids = c.ints([0, 1]), c.ints([40, 100]), c.ints([4, 5])
        torch.cuda.synchronize()
        c.pool.resize(rows, lens, stream=s)
        c.pool.fork(rows, kids, stream=s)
        c.model.resize([0, 1], [40, 100])
        c.model.fork([0, 1], [4, 5])
    a.check()
    b.check()


def test_pools_beyond_32_bit_offsets():
    """Pages whose bytes lie beyond 2^32 are copied, forked from and moved to the front."""
    n, ps = 140000, 16
    k, v = (torch.zeros((1, n, 8, a, b), dtype=torch.bfloat16, device=DEV) for a, b in ((ps, 128), (128, ps)))
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    last = list(range(n - 5, n))
    k[0, n - 5:], v[0, n - 5:] = torch.randn((5, 8, ps, 128), device=DEV).bfloat16(), torch.randn((5, 8, 128, ps), device=DEV).bfloat16()
    want_k, want_v = k[0, n - 5:].clone(), v[0, n - 5:].clone()
    table, lens, ref = torch.zeros((3, 6), dtype=torch.int32, device=DEV), ints([5 * ps - 3, 0, 0]), torch.zeros(n, dtype=torch.int32, device=DEV)
    table[0, :5] = ints(last)
    ref[n - 5:] = 1
    ref[:n - 5] = 1                                                   # nothing is free below
    ref[n - 7:n - 5] = 0
    pool = B.PagePool(k, v, table, lens, ref, 2)
    assert pool.fork(ints([0, 0]), ints([1, 2])).tolist() == [B.DYN_PAGES_DONE] * 2
    assert table[1, :5].tolist() == last[:4] + [n - 7] and table[2, :5].tolist() == last[:4] + [n - 6]
    for p in (n - 7, n - 6):
        assert torch.equal(k[0, p], want_k[4]) and torch.equal(v[0, p], want_v[4])
    pool.copy(ints([n - 3, n - 1]), ints([7, n - 2]))
    assert torch.equal(k[0, 7], want_k[2]) and torch.equal(v[0, 7], want_v[2]) and torch.equal(k[0, n - 2], want_k[4])
    ref[:n - 7] = 0                                                   # all but the rows' pages are free
    want = [(k[0, p].clone(), v[0, p].clone()) for p in range(n - 7, n)]
    new_page, n_live = pool.compact()
    assert n_live.tolist() == [7] and new_page[n - 7:].tolist() == list(range(7)) and (new_page[:n - 7] == -1).all()
    for p, (a, b) in enumerate(want):
        assert torch.equal(k[0, p], a) and torch.equal(v[0, p], b)
    assert table[1, :5].tolist() == [2, 3, 4, 5, 0] and ref[:7].tolist() == [1, 1, 3, 3, 3, 3, 1] and not ref[7:].any()
