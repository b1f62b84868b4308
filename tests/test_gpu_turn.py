"""Pages handed out and taken back against their rules, one sequence after the other: few sequences (one launch) and many,
requests that do not fit the table, the rows or the list, lists and lengths out of their ranges, graphs, streams."""
import random

import pytest
import torch

from step_reference import Turn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dcl():
    import paper_2607_20467_amd as m
    m.load_library()
    return m


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class OnDevice:
    """The same state on the device."""

    def __init__(self, dcl, ref, T):
        self.dcl, self.B, self.T = dcl, len(ref.len), T
        self.pool = dcl.KVPages(ref.n_pages, ref.page, 1, 64, dcl.DCL_DTYPE_E2M1)
        self.table, self.len, self.free, self.n_free = ints(ref.table), ints(ref.len), ints(ref.free), ints([ref.n_free])
        self.cu, self.pos = ints([7] * (self.B + 1)), ints([7] * T)
        self.slot = torch.full((T,), 7, dtype=torch.int64, device="cuda")
        self.need = dcl.dcl_pages_turn_workspace_bytes(self.B)
        self.ws = torch.full((self.need,), 0xFF, dtype=torch.uint8, device="cuda")

    def extend(self, count, stream=None, rows=True):
        self.dcl.dcl_pages_extend(self.pool, self.table, self.len, count, self.B, self.T, self.free, self.n_free, self.cu,
                                  self.pos if rows else None, self.slot if rows else None, self.ws, self.need, stream)

    def shrink(self, keep, stream=None):
        self.dcl.dcl_pages_shrink(self.pool, self.table, self.len, keep, self.B, self.free, self.n_free, self.ws, self.need,
                                  stream)

    def check(self, ref, rows=None):
        assert self.n_free.tolist() == [ref.n_free]
        assert self.len.tolist() == ref.len
        assert self.table.tolist() == ref.table
        assert self.free.tolist() == ref.free
        if rows:
            assert self.cu.tolist() == rows[0]
            assert self.pos.tolist() == rows[1]
            assert self.slot.tolist() == rows[2]


def state(r, B, page, width, lo, hi, spare):
    """Sequences of lo .. hi positions with their pages dealt in no order, and `spare` pages on the list."""
    lens = [r.randint(lo, hi) for _ in range(B)]
    need = [-(-n // page) for n in lens]
    pool = sum(need) + spare + 1
    order = list(range(pool))
    r.shuffle(order)
    table = [[-1] * width for _ in range(B)]
    at = 0
    for b, c in enumerate(need):
        table[b][:c] = order[at:at + c]
        at += c
    free = order[at:at + spare] + [-3] * (pool - spare)
    return Turn(table, lens, free, spare, page, pool)


@pytest.mark.parametrize("B,page,width,hi,most,T,spare", [
    (1, 16, 4, 60, 70, 70, 5),
    (5, 16, 6, 40, 30, 100, 12),
    (64, 64, 8, 400, 1, 64, 40),
    (200, 16, 5, 60, 20, 5000, 150),        # too few pages for the last ones
    (300, 32, 4, 100, 25, 2000, 4000),      # too few rows, and rows of the table that are full
    (256, 16, 8, 100, 5, 1024, 300),        # a small workgroup's most
    (257, 16, 8, 100, 5, 1024, 300),
    (1024, 16, 16, 200, 3, 4000, 1000),     # one launch's most
    (1025, 16, 6, 60, 3, 4000, 1000),       # and one more
    (700, 16, 40, 500, 60, 30000, 1700),    # more rows than one launch has
    (3000, 16, 3, 40, 5, 9000, 900),
    (4097, 16, 3, 40, 2, 9000, 3000),       # more than one window
    (65536, 16, 2, 30, 2, 60000, 20000),
])
def test_many_turns_match_the_rules(dcl, B, page, width, hi, most, T, spare):
    r = random.Random(B)
    ref = state(r, B, page, width, 0, min(hi, width * page), spare)
    dev = OnDevice(dcl, ref, T)
    for step in range(4):
        count = [r.choice([0, 1, 1, r.randint(0, most)]) for _ in range(B)]
        if step == 2:
            count = None
        rows = ref.extend(count, T)
        dev.extend(None if count is None else ints(count))
        dev.check(ref, rows)
        # some sequences end, some lose their newest tokens, some keep all or ask for what they do not have
        keep = [r.choice([n, -1, n + 3, 0, max(0, n - r.randint(0, 5)), r.randint(0, max(0, n))]) for n in ref.len]
        ref.shrink(keep)
        dev.shrink(ints(keep))
        dev.check(ref)


def test_many_pages_come_back_at_once(dcl):
    """Every page of 40 long sequences: more than one window of the list a workgroup, over several launches and in one."""
    for B, width in ((40, 3000), (5, 3000)):
        r = random.Random(B)
        ref = state(r, B, 16, width, width * 14, width * 16, 10)
        dev = OnDevice(dcl, ref, 8)
        for b in range(0, B, 2):
            ref.table[b][width // 2] = (-1, ref.n_pages, 2 ** 31 - 1, -2 ** 31)[b // 2 % 4]
        dev.table.copy_(ints(ref.table))
        keep = [0] * B
        ref.shrink(keep)
        dev.shrink(ints(keep))
        dev.check(ref)


@pytest.mark.parametrize("B,page,width,hi,cut", [
    (64, 16, 600, 300, 40),                 # a few pages of what the tables could name
    (300, 16, 100, 110, 200),               # some 1000 of them
    (700, 16, 40, 150, 200),                # more than the first launch takes by itself
    (4096, 16, 8, 40, 17),                  # sequences that its tables in shared memory hold
    (4097, 16, 8, 40, 17),
])
def test_pages_come_back_from_wide_tables(dcl, B, page, width, hi, cut):
    r = random.Random(B)
    ref = state(r, B, page, width, 0, hi, 3)
    dev = OnDevice(dcl, ref, 1)
    for b in range(0, B, 7):                # entries that name no page, which come back from nowhere
        ref.table[b][0] = r.choice([-1, ref.n_pages, 2 ** 31 - 1])
    dev.table = ints(ref.table)
    for turn in range(3):
        keep = [max(-1, n - r.randint(0, cut)) if r.random() < 0.5 else n for n in ref.len]
        ref.shrink(keep)
        dev.shrink(ints(keep))
        dev.check(ref)


def test_what_was_taken_goes_back_where_it_came_from(dcl):
    r = random.Random(3)
    ref = state(r, 50, 16, 20, 1, 200, 300)
    dev = OnDevice(dcl, ref, 3000)
    before = [x.clone() for x in (dev.table, dev.len, dev.free, dev.n_free)]
    keep = dev.len.clone()
    for _ in range(3):
        dev.extend(ints([r.randint(0, 60) for _ in range(50)]))
        assert int(dev.n_free) < 300
        dev.shrink(keep)
        assert all(torch.equal(x, y) for x, y in zip(before, (dev.table, dev.len, dev.free, dev.n_free)))


def test_requests_that_do_not_fit(dcl):
    """The list runs out in the middle: who comes later and needs a page gets none, who needs none gets its tokens. Requests past
    the table or below zero, lengths out of range, rows that run out."""
    ref = Turn([[0, 1, -1], [2, -1, -1], [3, -1, -1], [4, -1, -1], [5, 6, 7]], [20, 10, 16, 3, 48], [8, 9, 10, 11, -1, -1, -1, -1, -1,
                                                                                                  -1, -1, -1], 2, 16, 12)
    for count, T in (([4, 25, 1, 5, 1], 40), ([1, 2, 3, 4, 0], 5), ([-1, 39, 2 ** 31 - 1, 46, -2 ** 31], 60), ([0] * 5, 0),
                     ([1, 1, 1, 1, 1], 3)):
        dev = OnDevice(dcl, ref, T)
        rows = ref.extend(count, T)
        dev.extend(ints(count))
        dev.check(ref, rows)
    ref.len = [-1, 49, 2 ** 31 - 1, -2 ** 31, 48]
    for call in ("extend", "shrink"):
        dev = OnDevice(dcl, ref, 9)
        if call == "extend":
            rows = ref.extend([1, 0, 1, 1, 0], 9)
            dev.extend(ints([1, 0, 1, 1, 0]))
            dev.check(ref, rows)
        else:
            ref.shrink([0, 0, 0, 0, 17])
            dev.shrink(ints([0, 0, 0, 0, 17]))
            dev.check(ref)


@pytest.mark.parametrize("B", [6, 1500])
def test_lists_and_tables_out_of_range(dcl, B):
    """Lengths of the list outside [0, n_pages], entries of the list and of the table that name no page, a list that is full."""
    r = random.Random(8)
    for n_free in (-5, 0, 2 ** 31 - 1, -2 ** 31):
        ref = state(r, B, 16, 4, 0, 60, 20)
        ref.n_free = n_free
        for i in range(0, ref.n_pages, 3):
            ref.free[i] = (-1, ref.n_pages, 2 ** 31 - 1, -2 ** 31)[i % 4]
        for b in range(B):
            ref.table[b][b % 4] = (-1, ref.n_pages + 7, 2 ** 31 - 1, 3)[b // 4 % 4]
        dev = OnDevice(dcl, ref, 2 * B)
        count = [r.randint(0, 3) for _ in range(B)]
        rows = ref.extend(count, 2 * B)
        dev.extend(ints(count))
        dev.check(ref, rows)
        keep = [r.randint(0, 20) for _ in range(B)]
        ref.shrink(keep)
        dev.shrink(ints(keep))
        dev.check(ref)


def test_rows_may_be_left_out(dcl):
    for B, T in ((4, 10), (2000, 4000)):
        ref = state(random.Random(1), B, 16, 3, 0, 30, 500)
        dev = OnDevice(dcl, ref, T)
        cu, _, _ = ref.extend(None, T)
        dev.extend(None, rows=False)
        dev.check(ref)
        assert dev.cu.tolist() == cu and bool((dev.pos == 7).all())


@pytest.mark.parametrize("B,T", [(40, 90), (1200, 3000)])
def test_replayed_graphs(dcl, B, T):
    """A captured iteration (extend, then cut to the lengths asked for) replayed in turn with another state's graph and eager
    calls between, each against the rules."""
    r = random.Random(B)
    refs = [state(r, B, 16, 6, 0, 80, 2 * B) for _ in range(2)]
    devs = [OnDevice(dcl, ref, T) for ref in refs]
    asks = [[ints([1] * B), ints([0] * B)] for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for dev, (count, keep) in zip(devs, asks):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            dev.extend(count)
            dev.shrink(keep)
        graphs.append(graph)
    for step, i in enumerate((0, 1, 1, 0, 0, 1)):
        count = [r.randint(0, 4) for _ in range(B)]
        keep = [r.choice([-1, -1, 0, r.randint(0, 90)]) for _ in range(B)]
        asks[i][0].copy_(ints(count))
        asks[i][1].copy_(ints(keep))
        torch.cuda.synchronize()
        rows = refs[i].extend(count, T)
        refs[i].shrink(keep)
        if step == 3:
            devs[i].extend(asks[i][0])
            devs[i].shrink(asks[i][1])
        else:
            graphs[i].replay()
        torch.cuda.synchronize()
        devs[i].check(refs[i], rows)


def test_two_streams(dcl):
    r = random.Random(2)
    refs = [state(r, 1100, 16, 6, 0, 80, 900) for _ in range(2)]
    devs = [OnDevice(dcl, ref, 2000) for ref in refs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for dev, s in zip(devs, streams):
        for _ in range(3):
            dev.extend(None, s)
    torch.cuda.synchronize()
    for dev, ref in zip(devs, refs):
        for _ in range(3):
            rows = ref.extend(None, 2000)
        dev.check(ref, rows)
