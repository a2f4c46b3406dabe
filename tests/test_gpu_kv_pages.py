"""The pages' bookkeeping against the same operations on Python lists, page
by page, and the copied pages' content."""
import numpy as np
import pytest
import torch

import paper_2607_16973_amd as tq
from tests.reader import HostPages

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Both:
    """Device and host state side by side."""

    def __init__(self, rows, width, pages, layers=2, heads=1, d=64, kind="int8"):
        self.cache = tq.KVCache(layers, pages, heads, d, kind)
        self.dev, self.host = tq.KVPages(rows, width, pages), HostPages(rows, width, pages)
        for t in (self.cache.k, self.cache.v):
            t.view(torch.int8).random_(-100, 100)
        for t in (self.cache.k_scale, self.cache.v_scale):
            t.uniform_()

    def _state(self):
        return [t.view(torch.int8) if t.element_size() == 1 else t
                for t in (self.cache.k, self.cache.v, self.cache.k_scale, self.cache.v_scale)]

    def _done(self, before, copies):
        assert self.dev.tables.tolist() == self.host.tables
        assert self.dev.lens.tolist() == self.host.lens
        assert self.dev.refs.tolist() == self.host.refs
        for was, now in zip(before, self._state()):
            want = was.clone()
            for a, b in copies:
                want[:, b] = was[:, a]
            assert torch.equal(now, want)
        if self.host.full:
            with pytest.raises(RuntimeError, match="did not get the pages"):
                self.cache.check()
            self.host.full = False
        else:
            self.cache.check()

    def resize(self, goals):
        before = [t.clone() for t in self._state()]
        copies = self.host.resize(goals)
        self.dev.resize(ints(goals), self.cache)
        self._done(before, copies)

    def fork(self, src, dst):
        before = [t.clone() for t in self._state()]
        copies = self.host.fork(src, dst)
        self.dev.fork(ints(src), ints(dst), self.cache)
        self._done(before, copies)

    def compact(self):
        before = [t.clone() for t in self._state()]
        live, moves = self.host.compact()
        got = self.dev.compact(self.cache)
        assert got.item() == live
        self._done(before, moves)


def test_by_hand():
    b = Both(4, 3, 6)
    b.resize([100, 1, 0, -1])             # pages 0, 1 and 2
    assert b.dev.tables.tolist()[:2] == [[0, 1, -1], [2, -1, -1]]
    b.fork([0, 0], [2, 3])                # page 0 shared, copies of page 1 in 3 and 4
    assert b.dev.tables.tolist() == [[0, 1, -1], [2, -1, -1], [0, 3, -1], [0, 4, -1]]
    b.resize([-1, 0, 64, 130])            # 2 and 3 free; row 3 takes page 2
    b.resize([60, -1, 50, -1])            # back into the shared page
    b.resize([61, -1, 51, -1])            # and out of it: each takes a copy
    b.resize([-1, 500, -1, -1])           # wider than the table
    b.resize([-1, 192, -1, -1])           # more pages than are left
    b.compact()
    b.resize([0, 0, 0, 0])
    b.compact()


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("rows,width,pages", [(1, 1, 1), (7, 5, 30), (40, 9, 200), (33, 3, 3)])
def test_random_steps(rows, width, pages, seed):
    r = np.random.RandomState(seed)
    b = Both(rows, width, pages, layers=1 + seed % 2, heads=1 + seed % 3, kind=["int8", "fp8"][seed % 2])
    for _ in range(25):
        what = r.randint(0, 5)
        if what < 3:
            near = r.rand() < 0.5
            b.resize([int(np.clip(n + r.randint(-70, 90), 0, width * 64)) if near else int(r.randint(-30, width * 64 + 3))
                      for n in b.host.lens])
        elif what == 3 and rows > 1:
            n = r.randint(1, rows + 1)
            b.fork(r.randint(0, rows, n).tolist(), r.permutation(rows)[:n].tolist())
        else:
            b.compact()


def test_many_rows_and_pages():
    # more than one tile of the plan's 1,024 rows and 4,096 pages
    r = np.random.RandomState(3)
    b = Both(3001, 6, 14000, layers=1)
    b.resize(r.randint(0, 380, 3001).tolist())
    b.resize([int(n) if r.rand() < 0.7 else 0 for n in r.randint(-5, 380, 3001)])
    b.fork(r.randint(0, 3001, 2100).tolist(), r.permutation(3001)[:2100].tolist())
    b.compact()


def test_tables_that_grids_change():
    # over 4,096 rows and 32,768 entries, rows of one to eight pages
    r = np.random.RandomState(5)
    b = Both(5003, 8, 24000, layers=1)
    b.resize(r.randint(0, 500, 5003).tolist())
    b.resize([int(n) if r.rand() < 0.6 else 3 for n in r.randint(-90, 512, 5003)])
    b.fork(r.randint(0, 5003, 4200).tolist(), r.permutation(5003)[:4200].tolist())
    b.resize([max(0, n - int(r.randint(0, 70))) for n in b.host.lens])
    b.resize([n + int(r.randint(0, 9)) for n in b.host.lens])
    b.compact()


@pytest.mark.parametrize("rows,width", [(1100, 1), (60, 34), (61, 34), (300, 9)])
def test_forks_around_the_limits_of_one_workgroup(rows, width):
    # 1,024 pairs and 2,048 cells
    r = np.random.RandomState(rows)
    b = Both(rows, width, rows * width + 50, layers=1)
    b.resize(r.randint(0, width * 64 // 2 + 1, rows).tolist())
    for n in (rows, rows - 1, min(rows, 1024)):
        b.fork(r.randint(0, rows, n).tolist(), r.permutation(rows)[:n].tolist())


def test_long_rows():
    # many columns at once: the ranges that the whole workgroup takes
    b = Both(5, 300, 1100, layers=1)
    b.resize([19200, 5, 9000, 0, 700])
    b.fork([0, 2], [3, 1])
    b.resize([0, 12000, 64, 100, -1])
    b.resize([10000, 0, 19200, 101, 0])
    b.compact()


def test_empty_calls():
    b = Both(2, 2, 4)
    b.fork([], [])
    b.fork([1], [1])
    b.resize([-1, -1])
    none = tq.KVPages.over(torch.empty(0, 3, dtype=torch.int32, device="cuda"), ints([]).int(), torch.zeros(4, dtype=torch.int32, device="cuda"))
    none.resize(ints([]).int(), b.cache)
    assert none.compact(b.cache).item() == 0


def test_pairs_that_name_no_row_change_nothing():
    b = Both(2, 2, 4)
    b.resize([70, 0])
    before = b.dev.tables.clone()
    b.dev.fork(ints([0, 5, -1]), ints([9, 1, 1]), b.cache)
    assert torch.equal(b.dev.tables, before) and b.dev.refs.tolist() == [1, 1, 0, 0]


def test_graph_of_a_resize():
    b = Both(3, 2, 8)
    b.resize([10, 20, 30])
    up, down = ints([70, 80, 30]), ints([10, 20, 0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.dev.resize(up, b.cache)
        b.dev.resize(down, b.cache)
    b.host.resize([70, 80, 30])
    b.host.resize([10, 20, 0])
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert b.dev.tables.tolist() == b.host.tables and b.dev.refs.tolist() == b.host.refs
        b.host.resize([70, 80, 30])
        b.host.resize([10, 20, 0])


def test_workspaces_of_streams_and_graphs():
    # a workspace that work of another stream or a graph may still use is not given away
    b = Both(6, 4, 30)
    b.resize([100, 70, 0, 0, 0, 0])
    main, side = b.dev._ws, torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.resize([130, 70, 10, 0, 0, 0])
        assert b.dev._ws is not main and b.dev._ws_stream == side.cuda_stream
    torch.cuda.current_stream().wait_stream(side)
    b.resize([130, 80, 10, 0, 0, 0])
    kept, goals = b.dev._ws, ints([0] * 6)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.dev.resize(goals, b.cache)
    assert b.dev._ws is kept
    b.fork([0, 1], [3, 4])
    b.fork([0, 1, 0], [3, 4, 5])                 # a larger one: the kept one goes
    junk = torch.full((1 << 20,), -1, dtype=torch.int32, device="cuda")
    for step in ([200, 80, 10, 130, 80, 130], [64, 0, 10, 1, 80, 256], [7, 7, 7, 7, 7, 7]):
        before = [t.clone() for t in b._state()]
        copies = b.host.resize(step)
        goals.copy_(ints(step))
        graph.replay()
        b._done(before, copies)
    assert bool((junk == -1).all())
