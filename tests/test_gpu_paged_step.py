"""A paged decode loop as a service runs it, every step on the device: pages for the new tokens, heads normalised and rotated at the
positions that the lengths give, keys and values into pages of 4 bits, attention over them, rejected tokens and ended sequences
taken back. Eager against plain forms, and replayed from a graph against eager."""
import pytest
import torch

from step_reference import E2M1, Turn, attention_rows4, e2m1_rows, norm_rope, scale_of

pytestmark = pytest.mark.gpu

B, H, HKV, DH, PAGE, WIDTH, POOL, NEW = 4, 6, 2, 128, 16, 6, 14, 9
T, EPS, BASE, SCALE = 30, 1e-6, 1e4, 0.088


@pytest.fixture(scope="module")
def dcl():
    import paper_2607_20467_amd as m
    m.load_library()
    return m


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Service:
    """The loop's buffers. rot: rotated dimensions."""

    def __init__(self, dcl, rot, e2m1=True):
        g = torch.Generator().manual_seed(rot)
        self.dcl, self.rot = dcl, rot
        self.pool = dcl.KVPages(POOL, PAGE, HKV, DH, dcl.DCL_DTYPE_E2M1 if e2m1 else dcl.DCL_DTYPE_BF16)
        self.table, self.len, self.count, self.keep = ints([[-1] * WIDTH] * B), ints([0] * B), ints([0] * B), ints([-1] * B)
        self.free, self.n_free = ints(list(range(POOL))), ints([POOL])
        self.cu, self.pos = ints([0] * (B + 1)), ints([0] * T)
        self.slot = torch.zeros(T, dtype=torch.int64, device="cuda")
        self.rows = torch.zeros(T, H + 2 * HKV, DH, dtype=torch.bfloat16, device="cuda")
        self.gq, self.gk = ((1 + 0.2 * torch.randn(DH, generator=g)).cuda() for _ in range(2))
        self.out = torch.zeros(T, H, DH, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.zeros(T, H, device="cuda")
        self.nt = dcl.dcl_pages_turn_workspace_bytes(B)
        self.na = dcl.dcl_pages_attention_workspace_bytes(self.pool, H, B, T, NEW, WIDTH)
        self.wt, self.wa = (torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in (self.nt, self.na))

    def step(self):
        d, q, k, v = self.dcl, self.rows[:, :H], self.rows[:, H:H + HKV], self.rows[:, H + HKV:]
        d.dcl_pages_extend(self.pool, self.table, self.len, self.count, B, T, self.free, self.n_free, self.cu, self.pos,
                           self.slot, self.wt, self.nt)
        d.dcl_heads_norm_rope(q, k, self.pos, T, H, HKV, DH, self.gq, self.gk, EPS, BASE, self.rot, q, k)
        at = (self.pool, self.table, self.len, self.cu, B, T, NEW)
        d.dcl_pages_write(*at, k, v)
        d.dcl_pages_attention(*at, q, H, SCALE, True, self.out, self.lse, self.wa, self.na)
        d.dcl_pages_shrink(self.pool, self.table, self.len, self.keep, B, self.free, self.n_free, self.wt, self.nt)

    def state(self):
        return [x.clone() for x in (self.table, self.len, self.n_free, self.free, self.cu, self.pos, self.slot, self.rows, self.out,
                                    self.lse, self.pool.k, self.pool.v, self.pool.k_scale, self.pool.v_scale)]


# new tokens asked for and lengths kept, step by step: prompts, tokens, a block of drafts most of which are rejected, an ended
# sequence whose pages the others need, more than the list holds, more than the rows
STEPS = [
    ([9, 5, 1, 0], [-1, -1, -1, -1]),
    ([9, 9, 9, 1], [-1, 12, -1, -1]),
    ([1, 1, 1, 1], [-1, -1, -1, -1]),
    ([9, 9, 3, 9], [20, -1, 0, -1]),
    ([9, 9, 9, 9], [-1, -1, -1, -1]),
    ([9, 9, 9, 9], [-1, 0, -1, -1]),
    ([1, 9, 1, 1], [-1, -1, -1, 3]),
    ([0, 0, 0, 0], [0, 0, 0, 0]),
]


def inputs(step):
    g = torch.Generator().manual_seed(100 + step)
    return torch.randn(T, H + 2 * HKV, DH, generator=g).to(torch.bfloat16)


@pytest.mark.parametrize("rot", [128, 64])
def test_every_step_against_the_plain_forms(dcl, rot):
    s = Service(dcl, rot)
    ref = Turn([[-1] * WIDTH] * B, [0] * B, list(range(POOL)), POOL, PAGE, POOL)
    K, V = [[] for _ in range(B)], [[] for _ in range(B)]           # what each sequence's positions hold
    refused = 0
    for i, (count, keep) in enumerate(STEPS):
        row = inputs(i)
        s.rows.copy_(row), s.out.fill_(7), s.lse.fill_(7)
        s.count.copy_(ints(count)), s.keep.copy_(ints(keep))
        s.step()
        torch.cuda.synchronize()
        cu, pos, slot = ref.extend(count, T)
        refused += cu[B] < sum(count)
        assert s.cu.tolist() == cu and s.pos.tolist() == pos and s.slot.tolist() == slot
        got = s.rows.cpu()
        at = torch.tensor(pos, dtype=torch.int32)
        for part, gain in ((slice(0, H), s.gq), (slice(H, H + HKV), s.gk)):
            want, err = norm_rope(row[:, part].double(), at, gain.cpu(), EPS, BASE, rot)
            live = at >= 0
            assert bool(((got[:, part].double() - want).abs() <= err)[live].all())
        assert torch.equal(got[at < 0], row[at < 0]) and torch.equal(got[:, H + HKV:], row[:, H + HKV:])
        out, lse = s.out.double().cpu(), s.lse.double().cpu()
        for b in range(B):
            lo, hi = cu[b], cu[b + 1]
            for what, part in ((K, slice(H, H + HKV)), (V, slice(H + HKV, None))):
                code, e = e2m1_rows(got[lo:hi, part].double())
                what[b] += list(E2M1[code] * scale_of(e).repeat_interleave(32, -1))
            if lo == hi:
                continue
            n, k, v = len(K[b]), torch.stack(K[b]), torch.stack(V[b])
            sees = torch.arange(n)[None] <= n - (hi - lo) + torch.arange(hi - lo)[:, None]
            for h in range(H):
                o, want, eo, el = attention_rows4(got[lo:hi, h].double(), k[:, h // 3], v[:, h // 3], SCALE, sees)
                assert bool(((out[lo:hi, h] - o).abs() <= eo).all()), (i, b, h)
                assert bool(((lse[lo:hi, h] - want).abs() <= el).all()), (i, b, h)
        assert bool((out[cu[B]:] == 7).all()) and bool((lse[cu[B]:] == 7).all())
        ref.shrink(keep)
        for b in range(B):
            if 0 <= keep[b] < len(K[b]):
                del K[b][keep[b]:], V[b][keep[b]:]
        assert s.len.tolist() == ref.len == [len(x) for x in K]
        assert s.table.tolist() == ref.table and s.free.tolist() == ref.free and s.n_free.tolist() == [ref.n_free]
    assert refused >= 2 and s.n_free.tolist() == [POOL]


def test_replayed_steps_are_the_eager_ones(dcl):
    """Two services, one of them as a graph, through the same steps; the eager one runs between the other's replays."""
    eager, played = Service(dcl, 128), Service(dcl, 128)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        played.step()
    torch.cuda.synchronize()
    for i, (count, keep) in enumerate(STEPS + STEPS):
        for s in (eager, played):
            s.rows.copy_(inputs(i % len(STEPS)))
            s.count.copy_(ints(count)), s.keep.copy_(ints(keep))
        eager.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(eager.state(), played.state()):
            assert torch.equal(x, y), i


def test_bfloat16_pages_take_the_same_steps(dcl):
    """The turnover and the heads serve pages of every type: the first steps over bfloat16 pages."""
    s = Service(dcl, 128, e2m1=False)
    K, V = [[] for _ in range(B)], [[] for _ in range(B)]
    for i, (count, keep) in enumerate(STEPS[:3]):
        s.rows.copy_(inputs(i))
        s.count.copy_(ints(count)), s.keep.copy_(ints(keep))
        s.step()
        torch.cuda.synchronize()
        cu, got, out = s.cu.tolist(), s.rows.double().cpu(), s.out.double().cpu()
        for b in range(B):
            lo, hi = cu[b], cu[b + 1]
            K[b] += list(got[lo:hi, H:H + HKV])
            V[b] += list(got[lo:hi, H + HKV:])
            if lo < hi:
                n, k, v = len(K[b]), torch.stack(K[b]), torch.stack(V[b])
                sees = torch.arange(n)[None] <= n - (hi - lo) + torch.arange(hi - lo)[:, None]
                for h in range(H):
                    o, _, eo, _ = attention_rows4(got[lo:hi, h], k[:, h // 3], v[:, h // 3], SCALE, sees)
                    assert bool(((out[lo:hi, h] - o).abs() <= eo).all()), (i, b, h)
            if 0 <= keep[b] < len(K[b]):
                del K[b][keep[b]:], V[b][keep[b]:]
