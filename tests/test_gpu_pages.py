"""GPU tests of pages that sequences share against a plain simulation: every table
entry, count, pair and state exact, contents byte for byte."""
import numpy as np
import pytest
import torch

import draft_ref as plain
import paper_2607_24593_amd as pv
from gpu_util import dev, host, say

pytestmark = pytest.mark.gpu


class Pages:
    """The library's pool beside the plain one."""

    def __init__(self, slots, max_pages, page, n_pages, rng, widths=()):
        self.plain = plain.Pool(slots, max_pages, page, n_pages)
        self.table, self.refs = dev(self.plain.table), dev(self.plain.refs)
        self.pages = pv.make_pages(self.table, self.refs, page)
        self.arrays = [torch.from_numpy(rng.integers(0, 256, (n_pages * page, w), dtype=np.uint8)).cuda() for w in widths]
        self.rows = [x.cpu().clone() for x in self.arrays]

    def same(self):
        assert np.array_equal(host(self.table), self.plain.table)
        assert np.array_equal(host(self.refs), self.plain.refs)
        for x, y in zip(self.arrays, self.rows):
            assert torch.equal(x.cpu(), y)

    def fork(self, src, dst, tokens):
        pv.pivot_pages_fork(self.pages, src, dst, tokens)
        self.plain.fork(src, dst, tokens)
        self.same()

    def free(self, slots, tokens, keep):
        pv.pivot_pages_free(self.pages, slots, tokens, keep)
        self.plain.free(slots, tokens, keep)
        self.same()

    def copy(self, pairs, want):
        if not self.arrays:
            return
        pv.pivot_pages_copy(self.pages, pairs, self.arrays)
        p = self.plain.page
        for old, new in want:
            if old >= 0:
                for y in self.rows:
                    y[new * p:new * p + p] = y[old * p:old * p + p].clone()

    def grow(self, slots, tokens, new):
        pairs, state = pv.pivot_pages_grow(self.pages, slots, tokens, new)
        want, st = self.plain.grow(slots, tokens, new)
        assert np.array_equal(host(pairs), want) and tuple(host(state)) == st
        self.copy(pairs, want)
        self.same()
        return st

    def compact(self, most):
        moves, state = pv.pivot_pages_compact(self.pages, most)
        want, st = self.plain.compact(most)
        assert np.array_equal(host(moves), want) and tuple(host(state)) == st
        self.copy(moves, want)
        self.same()
        return st


def test_a_shared_last_page():
    """Three forks of a partly filled page and their source grow in one call: three
    get copies, the last keeps it; with a fifth holder outside all four get one."""
    rng = np.random.default_rng(1)
    p = Pages(8, 6, 16, 40, rng, (4, 132))
    say("pages shared")
    p.grow([5], [0], [50])
    p.fork([5, 5, 5], [1, 3, 0], [50, 50, 50])
    p.grow([3, 1, 5, 0], [50] * 4, [51, 50, 70, 60])   # slot 1 does not grow: it holds the page on
    p.free([3, 1, 5, 0], [51, 50, 70, 60], [0, 0, 50, 0])
    p.fork([5, 5, 5], [1, 3, 0], [50, 50, 50])
    p.grow([3, 1, 0, 5], [50] * 4, [64, 51, 96, 52])
    p.free([3, 1, 0, 5], [64, 51, 96, 52], [0, 0, 0, 50])
    p.fork([5, 5, 5, 5], [1, 3, 0, 7], [50, 49, 33, 50])
    p.grow([1, 3, 0, 5], [50, 49, 33, 50], [51, 51, 51, 51])


def test_growing_back_into_a_full_page():
    """A fork that goes back into a full, shared page gets its own when it grows."""
    rng = np.random.default_rng(2)
    p = Pages(4, 8, 32, 30, rng, (16,))
    say("pages back")
    p.grow([0], [0], [128])
    p.fork([0], [1], [128])
    p.free([1], [128], [70])
    p.grow([1], [70], [71])
    p.free([0], [128], [0])
    p.grow([1], [71], [96])
    p.grow([2], [0], [0])   # nothing grows


def test_too_few_pages():
    rng = np.random.default_rng(3)
    p = Pages(4, 10, 16, 9, rng, (4,))
    say("pages missing")
    assert p.grow([0, 1], [0, 0], [80, 60]) == (0, 0)
    assert p.grow([2], [0], [1]) == (1, 0)
    p.fork([0], [2], [77])
    assert p.grow([2, 0], [77, 77], [78, 78]) == (1, 0)   # a copy is wanted
    p.free([1], [60], [20])
    assert p.grow([2, 0], [77, 77], [100, 96]) == (2, 2)
    assert p.grow([2, 0], [77, 77], [78, 78]) == (0, 1)
    assert p.grow([0], [78], [96]) == (0, 0)


@pytest.mark.parametrize("slots,max_pages,page,n_pages,widths", [
    (1, 1, 16, 1, (4,)), (3, 5, 16, 7, (4, 48)), (20, 30, 16, 300, (8,)), (40, 40, 64, 700, ()), (16, 400, 16, 4096, ()),
    (16, 600, 16, 4097, ()), (64, 700, 16, 20000, ()), (200, 300, 16, 9000, ()), (6, 12, 4096, 40, (4,)),
])
def test_many_steps(slots, max_pages, page, n_pages, widths):
    """Requests come, fork, grow, go back and end at random; now and then the pool is
    compacted."""
    rng = np.random.default_rng(slots + n_pages)
    p = Pages(slots, max_pages, page, n_pages, rng, widths)
    length = {}
    say("pages steps", slots, max_pages, page, n_pages)
    most = max_pages * page
    for step in range(30):
        kind = rng.integers(0, 6)
        empty = [s for s in range(slots) if s not in length]
        held = list(length)
        rng.shuffle(empty)
        rng.shuffle(held)
        if (kind == 0 or not held) and empty:
            new = [int(s) for s in empty[:rng.integers(1, len(empty) + 1)]]
            to = [int(rng.integers(0, most + 1)) for _ in new]
            if p.grow(new, [0] * len(new), to)[0] == 0:
                length.update(zip(new, to))
        elif kind == 1 and empty and held:
            k = min(len(empty), 5)
            src = [int(rng.choice(held[:3])) for _ in range(k)]
            n = [int(rng.integers(0, length[s] + 1)) for s in src]
            dst = [int(s) for s in empty[:k]]
            p.fork(src, dst, n)
            length.update(zip(dst, n))
        elif kind == 2 and held:
            out = [int(s) for s in held[:rng.integers(1, len(held) + 1)]]
            keep = [int(rng.integers(0, length[s] + 1)) if rng.random() < 0.5 else 0 for s in out]
            p.free(out, [length[s] for s in out], keep)
            for s, k in zip(out, keep):
                length[s] = k
                if k == 0:
                    del length[s]
        elif kind == 3:
            p.compact(int(rng.integers(0, n_pages + 1)))
        elif held:
            to = [min(most, length[s] + int(rng.integers(0, 3 * page))) for s in held]
            held = [int(s) for s in held]
            if p.grow(held, [length[s] for s in held], to)[0] == 0:
                length.update(zip(held, to))
    p.compact(n_pages)


def test_compacting_by_parts():
    rng = np.random.default_rng(5)
    p = Pages(12, 2000, 16, 17000, rng, (4,))
    say("pages compact")
    p.grow(list(range(12)), [0] * 12, [16 * int(n) for n in rng.integers(900, 1400, 12)])
    length = [int((p.plain.table[s] >= 0).sum()) * 16 for s in range(12)]
    p.free([0, 3, 4, 8], [length[s] for s in (0, 3, 4, 8)], [0, 16 * 100, 0, 160])
    p.fork([1, 2], [0, 4], [length[1] // 2, 5000])
    assert p.compact(0)[0] == 0
    assert p.compact(7)[0] == 7
    assert p.compact(1000)[0] == 1000
    n, live = p.compact(17000)
    assert n > 0 and p.plain.refs[:live].all() and not p.plain.refs[live:].any()
    assert p.compact(50) == (0, live)


def test_a_pool_of_many_pages():
    """2^20 pages and more: blocks past the first thousand."""
    rng = np.random.default_rng(6)
    n_pages = (1 << 20) + 77
    p = Pages(3, 400000, 16, n_pages, rng)
    say("pages many")
    p.grow([0, 1, 2], [0, 0, 0], [16 * 300000, 16 * 300001, 16 * 333333])
    p.free([1], [16 * 300001], [16 * 100000])
    p.grow([0, 2], [16 * 300000, 16 * 333333], [16 * 300000 + 5, 16 * 399999])
    p.free([0], [16 * 300000 + 5], [3])
    p.compact(1000)
    p.compact(n_pages)


def test_entries_that_are_no_pages():
    """Entries outside the pool are left alone, pairs outside it left out."""
    table = torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
    table[0] = torch.tensor([2, 99, -5, 1], dtype=torch.int32)
    refs = torch.tensor([0, 1, 1, 0], dtype=torch.int32, device="cuda")
    pages = pv.make_pages(table, refs, 16)
    say("pages outside")
    pv.pivot_pages_fork(pages, [0], [1], [64])
    assert host(table)[1].tolist() == [2, -1, -1, 1] and host(refs).tolist() == [0, 2, 2, 0]
    pv.pivot_pages_free(pages, [0], [64], [16])
    assert host(table)[0].tolist() == [2, 99, -5, -1] and host(refs).tolist() == [0, 1, 2, 0]
    pairs, state = pv.pivot_pages_grow(pages, [0], [20], [30])   # its partly filled page is none
    assert host(pairs).tolist() == [[-1, -1]] and host(state).tolist() == [0, 2]
    moves, state = pv.pivot_pages_compact(pages, 4)
    assert host(state).tolist() == [1, 2] and host(moves)[0].tolist() == [2, 0]
    assert host(table).tolist() == [[0, 99, -5, -1], [0, -1, -1, 1], [-1] * 4]
    x = torch.arange(64 * 4, dtype=torch.int32, device="cuda").view(64, 4)
    want = x.clone()
    want[48:64] = want[16:32]
    pairs = torch.tensor([[1, 3], [-1, 0], [0, 4], [9, 2], [2, 2], [2, -1]], dtype=torch.int32, device="cuda")
    pv.pivot_pages_copy(pages, pairs, [x])
    assert torch.equal(x, want)


def test_copies_of_rows_that_are_aligned_to_four_bytes():
    rng = np.random.default_rng(8)
    backing = torch.from_numpy(rng.integers(0, 256, 5 * 16 * 12 + 4, dtype=np.uint8)).cuda()
    x = backing[4:].view(80, 12)
    refs, table = torch.ones(5, dtype=torch.int32, device="cuda"), torch.zeros((1, 5), dtype=torch.int32, device="cuda")
    want = x.clone()
    want[0:16], want[64:80] = want[16:32].clone(), want[48:64].clone()
    say("pages of odd rows")
    pairs = torch.tensor([[1, 0], [3, 4]], dtype=torch.int32, device="cuda")
    pv.pivot_pages_copy(pv.make_pages(table, refs, 16), pairs, [x])
    assert torch.equal(x, want) and torch.equal(backing[:4], backing[:4].clone())


def test_pages_in_a_graph():
    """Free, fork, grow and copy captured once, replayed with eager work between."""
    rng = np.random.default_rng(9)
    p = Pages(4, 20, 16, 64, rng, (32,))
    p.grow([0, 2], [0, 0], [100, 37])
    start = p.table.clone(), p.refs.clone()
    pairs = torch.empty((4, 2), dtype=torch.int32, device="cuda")
    state = torch.empty(2, dtype=torch.int32, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")

    def step():
        pv.pivot_pages_free(p.pages, [1, 3, 0, 2], [120, 57, 120, 57], [0, 0, 100, 37])
        pv.pivot_pages_fork(p.pages, [0, 2], [1, 3], [100, 37])
        pv.pivot_pages_grow(p.pages, [1, 3, 0, 2], [100, 37, 100, 37], [120, 57, 120, 57], copies=pairs, state=state, ws=ws)
        pv.pivot_pages_copy(p.pages, pairs, p.arrays)

    say("pages graph")
    graph = torch.cuda.CUDAGraph()
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (p.table, p.refs, pairs, state, p.arrays[0])]
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        if i % 2:
            p.table.copy_(start[0])
            p.refs.copy_(start[1])
        pairs.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((p.table, p.refs, pairs, state, p.arrays[0]), want):
            assert torch.equal(x, y)
