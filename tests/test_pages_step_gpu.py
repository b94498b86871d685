"""A step's page tables on the GPU, against the same on lists (q4_ref.step):
whole numbers, equal to the last entry."""
import random

import pytest
import torch

import q4_ref as ref
from test_paged_gpu import I32, _ints, st  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


class _Server:
    """Sessions on the GPU and the same on lists."""

    def __init__(self, st, S, page, M, n_pages, places, seed, lens=None):
        r = self.r = random.Random(seed)
        self.st, self.S, self.page, self.M, self.n_pages, self.places = st, S, page, M, n_pages, places
        self.lens = list(lens or [0] * S)
        order = r.sample(range(n_pages), n_pages)
        self.table = [[r.choice([-3, 7, n_pages + 1]) for _ in range(M)] for _ in range(S)]
        for s, n in enumerate(self.lens):
            for i in range(-(-max(0, min(n, M * page)) // page)):
                self.table[s][i] = order.pop()
        self.n_free = len(order)
        self.free = order + [-9] * (n_pages - len(order))
        self.d = [_ints(x) for x in (self.table, self.lens, [5] * (S + 1), self.free, [self.n_free], [8] * places)]
        self.pt = st.make_pages(n_pages, page, *self.d[:3])

    def step(self, keep, fresh, run=None):
        if run is None:
            self.st.stlite_pages_step(self.pt, None if keep is None else _ints(keep), _ints(fresh), self.d[3], self.d[4], self.d[5])
        else:
            run()
        cu, self.n_free, slot = ref.step(self.table, self.lens, keep, fresh, self.free, self.n_free, self.n_pages, self.page, self.places)
        for got, want in zip(self.d, (self.table, self.lens, cu, self.free, [self.n_free], slot)):
            assert got.tolist() == want
        return cu, slot


@pytest.mark.parametrize("S,page,M,n_pages,places", [
    (1, 16, 5, 5, 40), (1, 1, 9, 7, 9), (7, 16, 6, 30, 60), (33, 7, 12, 100, 90), (200, 16, 40, 3000, 4000), (512, 64, 9, 2000, 700),
    (513, 16, 5, 1500, 3000), (1300, 3, 7, 4000, 6000), (3, 100, 2, 4, 0), (5, 128, 700, 2500, 200000)])
def test_sessions_come_and_go(st, S, page, M, n_pages, places):
    """Growth, refused drafts, ends, requests that do not fit the table, the pool or the step, wild numbers."""
    s = _Server(st, S, page, M, n_pages, places, S + page)
    r = s.r
    for turn in range(6):
        keep = [r.choice([n, n, n, n - r.randint(0, 5), 0, n + 3, -2]) for n in s.lens]
        fresh = [r.choice([0, 1, 1, 5, r.randint(0, M * page), r.randint(0, page), -4, 2 ** 31 - 1 if r.random() < 0.1 else 2]) for _ in range(S)]
        if turn == 2:
            keep = None
        if turn == 4:
            keep, fresh = [0] * S, [0] * S  # all end
        s.step(keep, fresh)


def test_wild_lengths_and_tables(st):
    """Lengths outside the table, pages named twice and pages outside the pool are moved as they are; slots say -1."""
    s = _Server(st, 4, 8, 6, 40, 64, 1, lens=[20, 48, 3, 0])
    s.lens[1], s.lens[3] = 1000, -5
    s.table[0][2] = 77
    s.d[0].copy_(torch.tensor(s.table))
    s.d[1].copy_(torch.tensor(s.lens))
    cu, slot = s.step([20, 9, 3, 0], [4, 7, 60, 1])
    assert cu == [0, 4, 11, 11, 12] and slot[:4] == [-1] * 4
    s.step([0, 0, 0, 0], [9, 9, 9, 9])  # the page outside the pool comes back into use


def test_more_free_pages_than_the_pool(st):
    """A count past the pool counts as the pool; pages that have no room are dropped."""
    s = _Server(st, 2, 4, 4, 6, 16, 2, lens=[8, 4])
    s.n_free = 900
    s.d[4].fill_(900)
    s.step([0, 4], [0, 9])
    assert s.n_free == 3


def test_without_slots_and_in_a_graph(st):
    """slot NULL with its number of places; one capture follows whatever the arrays hold at replay."""
    s = _Server(st, 9, 16, 8, 60, 50, 3)
    keep, fresh = _ints([0] * 9), _ints([7] * 9)
    graph = torch.cuda.CUDAGraph()
    s.st.stlite_pages_step(s.pt, keep, fresh, s.d[3], s.d[4], s.d[5])
    cu, s.n_free, _ = ref.step(s.table, s.lens, [0] * 9, [7] * 9, s.free, s.n_free, 60, 16, 50)
    with torch.cuda.graph(graph):
        s.st.stlite_pages_step(s.pt, keep, fresh, s.d[3], s.d[4], s.d[5])
    for turn in range(4):
        k, f = [s.r.randint(0, 9) + n - 5 for n in s.lens], [s.r.randint(0, 40) for _ in range(9)]
        keep.copy_(torch.tensor(k))
        fresh.copy_(torch.tensor(f))
        s.step(k, f, graph.replay)
    before = s.d[5].clone()
    s.st.stlite_pages_step(s.pt, None, fresh.fill_(3), s.d[3], s.d[4], 20)
    cu, s.n_free, _ = ref.step(s.table, s.lens, None, [3] * 9, s.free, s.n_free, 60, 16, 20)
    assert s.d[2].tolist() == cu and torch.equal(before, s.d[5]) and s.d[0].tolist() == s.table
