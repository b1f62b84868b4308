"""Drawn tokens against a sorted float64 row: every filter alone and together, vocabularies from one id to 152064, ties,
many nearly equal values, masked, infinite and NaN logits, settings at and past their ends, rows apart, graphs."""
import math

import numpy as np
import pytest
import torch

from serving_reference import sample_row

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dcl():
    import paper_2607_20467_amd as m
    m.load_library()
    return m


def draw(dcl, x, u, temperature=None, top_k=None, top_p=None, min_p=None, n=None, V=None, stream=None):
    """x: device logits [n, V]; settings: numbers or arrays. Returns token, conf, kept (numpy)."""
    n, V = x.shape[0] if n is None else n, x.shape[1] if V is None else V

    def dev(v, dt):
        return None if v is None else torch.tensor(np.broadcast_to(np.asarray(v), (n,)).copy(), dtype=dt).cuda()
    token = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    conf = torch.full((n,), -9.0, device="cuda")
    kept = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    need = dcl.dcl_sample_workspace_bytes(n, V)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    f = torch.float32
    dcl.dcl_sample_tokens(x, n, V, dev(temperature, f), dev(top_k, torch.int32), dev(top_p, f), dev(min_p, f), dev(u, f),
                          token, conf, kept, ws, need, stream)
    torch.cuda.synchronize()
    return token.cpu().numpy(), conf.cpu().numpy(), kept.cpu().numpy()


def check(x, got, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The settings as the call took them (float32). Weights are whole numbers of one unit, 2^-45 of the largest or, so that
    V of them stay below 2^62, 2^-(62 - bits): each is off by half a unit (and 2^-42 of itself: the series and its
    table), a sum of V of them by V halves, the sum is at least 1, and conf is rounded to float32 (2^-24 of itself)."""
    x = x.double().cpu().numpy()
    n, V = x.shape
    bits = math.ceil(math.log2(V)) if V > 1 else 0

    def at(v, r, dt=np.float32):
        return float(np.broadcast_to(np.asarray(v, dtype=dt), (n,))[r])
    for r in range(n):
        k = int(np.broadcast_to(np.asarray(top_k), (n,))[r])
        t, c, kept = sample_row(x[r], at(temperature, r), k, at(top_p, r), at(min_p, r), at(u, r))
        assert (got[0][r], got[2][r]) == (t, kept), (r, got[0][r], t, got[2][r], kept)
        half = 2.0 ** -(min(45, 62 - bits) + 1)
        assert abs(float(got[1][r]) - c) <= c * (2.0 ** -24 + 2.0 ** -41 + V * half) + half, (r, got[1][r], c)


def logits(n, V, seed, std=2.0, peaks=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, V, generator=g) * std
    if peaks and V > 20:
        x.scatter_add_(1, torch.randint(0, V, (n, 8), generator=g), torch.rand(n, 8, generator=g) * 9)
    return x, g


SETTINGS = [
    {}, {"temperature": 0.7}, {"top_k": 5}, {"top_p": 0.9}, {"min_p": 0.05}, {"temperature": 1.7, "top_k": 40, "top_p": 0.8},
    {"temperature": 0.3, "top_p": 0.95, "min_p": 0.01}, {"top_k": 300, "min_p": 0.02, "top_p": 0.5}, {"temperature": 0.0},
    {"temperature": 3.0, "top_k": 3000, "top_p": 0.99},
]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("V", [1, 2, 3, 17, 433, 1024, 1025, 2048, 2049, 4096, 40010])
def test_matches_sorted_rows(dcl, V, bf16):
    n = 8 if V < 5000 else 4
    for i, how in enumerate(SETTINGS):
        x, g = logits(n, V, 31 * i + V)
        x = (x.to(torch.bfloat16) if bf16 else x).cuda()
        u = torch.rand(n, generator=g).numpy()
        check(x, draw(dcl, x, u, **how), u, **how)


@pytest.mark.parametrize("bf16", [False, True])
def test_every_row_its_own_settings_at_the_full_vocabulary(dcl, bf16):
    n, V = 24, 152064
    x, g = logits(n, V, 5, std=1.5)
    x[:, V - 1] = -math.inf
    x[3, :1000] = math.nan
    x = (x.to(torch.bfloat16) if bf16 else x).cuda()
    r = np.random.default_rng(1)
    how = dict(temperature=r.choice([0.0, 0.2, 0.6, 1.0, 1.4], n), top_k=r.choice([0, 0, 1, 20, 50, 1000, 5000, 200000], n),
               top_p=r.choice([1.0, 0.5, 0.9, 0.999], n), min_p=r.choice([0.0, 0.0, 0.05, 1e-4], n))
    u = torch.rand(n, generator=g).numpy()
    check(x, draw(dcl, x, u, **how), u, **how)


@pytest.mark.parametrize("V", [5, 2048, 2049, 30000, 152064])
def test_equal_logits(dcl, V):
    """All ids alike: kept ids are the lowest ones, the draw is the id at u of them; borders are exact."""
    x = torch.full((6, V), 3.25)
    u = np.array([0.0, 0.25, 0.5, 0.999, 0.75, 1.0 - 2.0 ** -24], dtype=np.float32)
    for how in ({}, {"top_k": 3}, {"top_p": 0.5}, {"top_k": 4, "top_p": 0.25}, {"min_p": 1.0}, {"top_k": V - 1, "top_p": 0.75}):
        xd = x.cuda()
        got = draw(dcl, xd, u, **how)
        check(xd, got, u, **how)


@pytest.mark.parametrize("bf16", [False, True])
def test_few_values(dcl, bf16):
    """Two to five distinct values over a large vocabulary, -0 and +0 among them."""
    g = torch.Generator().manual_seed(7)
    vals = torch.tensor([1.0, 0.0, -0.0, -1.5, 0.0078125])
    x = vals[torch.randint(0, 5, (6, 50000), generator=g)]
    x = (x.to(torch.bfloat16) if bf16 else x).cuda()
    u = torch.rand(6, generator=g).numpy()
    for how in ({}, {"top_k": 12000}, {"top_k": 20001, "top_p": 0.9}, {"top_p": 0.3}, {"temperature": 0.5, "min_p": 0.2}):
        check(x, draw(dcl, x, u, **how), u, **how)


def test_many_nearly_equal_values_in_one_bin(dcl):
    """40000 distinct values within 1 / 100 of each other, ids in no order; and with ties among them."""
    g = torch.Generator().manual_seed(8)
    base = 1.0 + torch.arange(40000).float() * 2.0 ** -22
    rows = []
    for i in range(4):
        x = base[torch.randperm(40000, generator=g)].clone()
        if i > 1:
            x[:15000] = base[20000]
        rows.append(x)
    x = torch.stack(rows).cuda()
    u = np.array([0.1, 0.77, 0.5, 0.3], dtype=np.float32)
    for how in ({}, {"top_k": 17}, {"top_k": 25000, "top_p": 0.7}, {"top_p": 0.123}, {"min_p": 0.995}, {"top_k": 30000}):
        check(x, draw(dcl, x, u, **how), u, **how)


@pytest.mark.parametrize("V", [3001, 1801, 1000])
def test_masked_infinite_and_nan_logits(dcl, V):
    x, g = logits(8, V, 9)
    x[0] = -math.inf
    x[1] = math.nan
    x[2] = -math.inf
    x[2, V - 2] = -5e30
    x[3, [7, V - 1]] = math.inf
    x[4] = torch.finfo(torch.float32).min
    x[4, 5:9] = 0.0
    x[5, ::2] = math.nan
    x[6, 1:] = torch.finfo(torch.float32).min
    x[7] = 3e38
    x[7, 12] = -3e38
    for bf16 in (False, True):
        xd = (x.to(torch.bfloat16) if bf16 else x).cuda()
        u = torch.rand(8, generator=g).numpy()
        for how in ({}, {"top_k": 4}, {"top_p": 0.6}, {"min_p": 0.1}, {"top_k": V - 500}):
            got = draw(dcl, xd, u, **how)
            check(xd, got, u, **how)
            assert got[0][0] == got[0][1] == -1 and got[1][0] == 0 and got[2][1] == 0
            assert got[0][2] == V - 2 and got[0][3] in (7, V - 1)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("V", [1000, 5000, 24000])
def test_settings_at_and_past_their_ends(dcl, V, bf16):
    x, _ = logits(12, V, 10)
    x = (x.to(torch.bfloat16) if bf16 else x).cuda()
    nan, inf = math.nan, math.inf
    u = np.array([0, 0, 0.5, 1.0, 2.0, nan, -1.0, 0.9, 0.3, 0.99, 0.4, 0.6], dtype=np.float32)
    for how in ({}, {"temperature": [nan, -1, 0, inf, 1e-40, 1e30, 1e-6, 1, 5, 0.01, -inf, 2]},
                {"top_k": [0, -1, V, V + 1, 2 ** 31 - 1, 1, 2, -2 ** 31, 3, 999, 500, 7]},
                {"top_p": [0, -1, nan, 1, 2, inf, -inf, 1e-30, 0.5, 1 - 2.0 ** -24, 0.1, 0.2]},
                {"min_p": [0, -1, nan, 1, 2, inf, -inf, 1e-30, 0.5, 1 - 2.0 ** -24, 0.1, 0.2]}):
        got = draw(dcl, x, u, **how)
        ref = {k: np.asarray(v, dtype=np.float32 if k != "top_k" else np.int64) for k, v in how.items()}
        check(x, got, u, **ref)


@pytest.mark.parametrize("V", [6001, 2000])
def test_bfloat16_values_of_every_size(dcl, V):
    """Magnitudes from the least to the largest in one row, both zeros, few and many counts of a value; temperatures under
    which little or all of the type's range counts."""
    n = 6
    g = torch.Generator().manual_seed(77)
    x = torch.zeros(n, V)
    x[0] = torch.randn(V, generator=g) * 2.0 ** torch.randint(-130, 127, (V,), generator=g)
    x[1] = torch.randint(-2, 3, (V,), generator=g).float() * 0.5
    x[1][x[1] == 0] = -0.0
    x[1][::3] = 0.0
    x[2] = torch.randn(V, generator=g) * 1e30
    x[3, ::2] = -0.0
    x[4] = -torch.rand(V, generator=g) * 2.0 ** -120
    x[5] = torch.randn(V, generator=g) * 1e5
    x[5, V // 3 * 2:] = -math.inf
    x = x.to(torch.bfloat16)
    assert bool(torch.isfinite(x[:5]).all())
    x = x.cuda()
    for T in (0.01, 1.0, 1e4, 1e30, 3e38):
        for how in ({}, {"top_p": 0.7}, {"top_k": 700}, {"top_k": 5000, "top_p": 0.9}, {"min_p": 0.6}):
            u = torch.rand(n, generator=g).numpy()
            check(x, draw(dcl, x, u, temperature=T, **how), u, temperature=T, **how)


def test_rows_apart_and_not_aligned(dcl):
    for dt in (torch.float32, torch.bfloat16):
        for V, extra, first in ((1001, 3, 1), (64, 7, 3), (4097, 1, 1), (4099, 13, 6), (20011, 5, 3)):
            wide = torch.full((5, V + extra), 99.0, dtype=dt, device="cuda")
            x, g = logits(5, V, V)
            view = wide[:, first:first + V] if first + V <= V + extra else wide[:, :V]
            view.copy_(x)
            u = torch.rand(5, generator=g).numpy()
            for how in ({}, {"top_k": 9, "top_p": 0.9}):
                check(view, draw(dcl, view, u, **how), u, **how)


def test_draws_follow_the_distribution(dcl):
    """Evenly spaced u over one row: each id is drawn its share of the time, to within one draw per border."""
    V, n = 50, 20000
    x, _ = logits(1, V, 12)
    p = torch.softmax(x[0].double(), 0).numpy()
    u = (np.arange(n) + 0.5) / n
    t, c, k = draw(dcl, x.cuda().expand(n, V).contiguous(), u)
    freq = np.bincount(t, minlength=V) / n
    assert np.abs(freq - p).max() <= 1.5 / n + 2.0 ** -23 and (k == V).all()
    assert np.abs(c - p[t]).max() <= 2.0 ** -22


def test_optional_outputs_and_no_rows(dcl):
    x, _ = logits(3, 100, 2)
    x = x.cuda()
    u = torch.tensor([0.2, 0.4, 0.9], device="cuda")
    ws = torch.empty(dcl.dcl_sample_workspace_bytes(3, 100), dtype=torch.uint8, device="cuda")
    tok = torch.empty(3, dtype=torch.int32, device="cuda")
    dcl.dcl_sample_tokens(x, 3, 100, None, None, None, None, u, tok, None, None, ws, ws.numel())
    assert (tok.cpu().numpy() == draw(dcl, x, [0.2, 0.4, 0.9])[0]).all()
    dcl.dcl_sample_tokens(x, 0, 100, None, None, None, None, u, tok, None, None, ws, ws.numel())


def test_replays_and_streams(dcl):
    x, g = logits(6, 40010, 3)
    x = x.cuda()
    u = torch.rand(6, generator=g).cuda()
    k = torch.full((6,), 40, dtype=torch.int32, device="cuda")
    p = torch.full((6,), 0.9, device="cuda")
    need = dcl.dcl_sample_workspace_bytes(6, 40010)
    bufs = [(torch.empty(6, dtype=torch.int32, device="cuda"), torch.empty(6, device="cuda"),
             torch.empty(6, dtype=torch.int32, device="cuda"), torch.empty(need, dtype=torch.uint8, device="cuda"))
            for _ in range(2)]

    def go(i, stream=None):
        dcl.dcl_sample_tokens(x, 6, 40010, None, k, p, None, u, *bufs[i], need, stream)
    go(0)
    torch.cuda.synchronize()
    ref = [b.clone() for b in bufs[0][:3]]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        go(0, side)
    for _ in range(4):
        for b in bufs[0]:
            b.fill_(77)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bufs[0], ref))
    with torch.cuda.stream(side):
        go(1)
    go(0)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(c, b) for a, b, c in zip(bufs[0], ref, bufs[1]))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("V", [16384 + 5, 20000, 70001])
def test_few_rows_are_drawn_as_many_are(dcl, V, bf16):
    """Workgroups share the rows of small calls: the same rows, special ones among them, in calls of 300 and of 1 to 90."""
    n = 300
    x, g = logits(n, V, V)
    x[1] = -math.inf
    x[2] = math.nan
    x[3, [7, 100, V - 1]] = math.inf
    x[4] = 3.25
    x[5] = torch.finfo(torch.float32).min
    x[5, V - 1] = 0
    x[6, V // 2:] = -math.inf
    x[7] = 20 + torch.arange(V) * 2.0 ** -19                      # one bin, and in bfloat16 few values
    x[8, :V - 600] = math.nan
    x[9] *= 0.01
    x[10, :] = -40
    x[10, 3] = 0
    x[11] = torch.arange(V).float() * -1e-3
    x[12, :] = -math.inf
    x[12, V - 3:] = -2.5
    x = (x.to(torch.bfloat16) if bf16 else x).cuda()
    r = np.random.default_rng(V)
    how = dict(temperature=r.choice([0.0, 0.2, 0.6, 1.0, 1.0, 1.4], n), top_k=r.choice([0, 0, 0, 1, 20, 512, 513, 1500, 5000], n),
               top_p=r.choice([1.0, 0.5, 0.9, 0.999], n), min_p=r.choice([0.0, 0.0, 0.05, 1e-4], n))
    u = torch.rand(n, generator=g).numpy()
    for settings in (how, {}, {"top_k": 40}, {"top_p": 0.9}):
        def part(rows):
            return {k: (v[rows] if isinstance(v, np.ndarray) else v) for k, v in settings.items()}
        whole = draw(dcl, x, u, **settings)
        check(x[:16], [w[:16] for w in whole], u[:16], **part(slice(0, 16)))
        first = 0
        for m in (1, 2, 5, 14, 33, 90):
            rows = slice(first, first + m)
            got = draw(dcl, x[rows], u[rows], **part(rows))
            for a, b in zip(got, whole):
                assert np.array_equal(a, b[rows], equal_nan=True), (m, np.nonzero(a != b[rows])[0][:5] + first)
            first += m


def test_more_rows_than_a_launch_has(dcl):
    n, V = (1 << 21) + 3, 2
    x = torch.zeros(n, V, device="cuda")
    x[::3, 1] = 1.0
    u = torch.zeros(n, device="cuda")
    u[5::7] = 0.999
    need = dcl.dcl_sample_workspace_bytes(n, V)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    token, kept = (torch.full((n,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    top_k = torch.zeros(n, dtype=torch.int32, device="cuda")
    top_k[n - 1] = 1
    dcl.dcl_sample_tokens(x, n, V, None, top_k, None, None, u, token, None, kept, ws, need)
    best = (x[:, 1] > 0).int()
    want = torch.where(u > 0.5, 1 - best, best)                   # the less likely id has a quarter or a half
    want[n - 1] = best[n - 1]
    assert torch.equal(token, want) and int(kept[n - 1]) == 1 and bool((kept[:n - 1] == 2).all())


@pytest.mark.parametrize("bf16", [False, True])
def test_more_rows_than_a_window_of_workgroups_and_replays(dcl, bf16):
    """1500 rows, open and answered ones mixed; then the same call captured and replayed with other numbers."""
    n, V = 1500, 300
    x, g = logits(n, V, 41)
    x[::7] = -math.inf
    x = (x.to(torch.bfloat16) if bf16 else x).cuda()
    r = np.random.default_rng(5)
    how = dict(temperature=r.choice([0.0, 0.7, 1.0], n), top_k=r.choice([0, 0, 1, 5], n), top_p=r.choice([1.0, 0.9], n))
    u = torch.rand(n, generator=g)
    check(x, draw(dcl, x, u.numpy(), **how), u.numpy(), **how)

    T, k, p = (torch.tensor(how[name], dtype=dt).cuda() for name, dt in
               (("temperature", torch.float32), ("top_k", torch.int32), ("top_p", torch.float32)))
    ud = u.cuda()
    token, kept = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
    conf = torch.empty(n, device="cuda")
    need = dcl.dcl_sample_workspace_bytes(n, V)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def go():
        dcl.dcl_sample_tokens(x, n, V, T, k, p, None, ud, token, conf, kept, ws, need)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        go()
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        u = torch.rand(n, generator=g)
        ud.copy_(u)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        want = draw(dcl, x, u.numpy(), **how)
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip((token, conf, kept), want))


def beside(V, groups, rest, g):
    """Row of V float32 logits: groups of (count, value), the rest below, ids in no order."""
    x = torch.full((V,), rest)
    at = 0
    for count, value in groups:
        x[at:at + count] = value
        at += count
    return x[torch.randperm(V, generator=g)]


@pytest.mark.parametrize("n", [2, 140])
@pytest.mark.parametrize("V", [9001, 30000])
def test_top_k_among_neighbouring_floats_far_apart_in_weight(dcl, V, n):
    """The next float below a logit is many bins of the histogram away: what is looked at for the border's bin is more than the
    list holds though the bins up to it are few. Few rows are shared, many are not."""
    g = torch.Generator().manual_seed(V + n)
    f = [12.0]
    for _ in range(2):
        f.append(float(np.nextafter(np.float32(f[-1]), np.float32(0))))
    few = [(10, f[0]), (30, f[1]), (5000, f[2])]            # the border below the first ones, all others past the list
    many = [(1500, f[0]), (200, f[1]), (400, f[2])]         # the border's bin alone fits it
    for groups, ks in ((few, (20, 40, 600)), (many, (1501, 1600, 1700))):
        x = torch.stack([beside(V, groups, -5.0, g) for _ in range(2)]).repeat(n // 2, 1).cuda()
        u = torch.rand(n, generator=g).numpy()
        for k in ks:
            for T in (1e-6, 3e-6, 1e-5):
                for how in ({}, {"top_p": 0.6}, {"min_p": 0.5}, {"top_p": 0.9, "min_p": 1e-3}):
                    got = draw(dcl, x, u, temperature=T, top_k=k, **how)
                    check(x[:4], [a[:4] for a in got], u[:4], temperature=T, top_k=k, **how)


@pytest.mark.parametrize("V,n", [(152064, 2), (9001, 3), (152064, 130)])
def test_top_k_of_logits_with_a_large_offset(dcl, V, n):
    """Steps of a sixteenth (of 1 and 2) between the logits, temperature 1: a bin is a third of a step or less."""
    g = torch.Generator().manual_seed(V)
    x = (1e6 + 2 * torch.randn(2, V, generator=g)).repeat((n + 1) // 2, 1)[:n]
    big = torch.stack([beside(V, [(600, 12582912.0), (600, 12582911.0), (V // 2, 12582910.0)], 12582000.0, g)] * n)
    for x, ks in ((x, (300, 1850, 1900, 1945, 2040)), (big, (1000, 1200, 1201))):
        x = x.cuda()
        u = torch.rand(n, generator=g).numpy()
        for k in ks:
            for how in ({}, {"top_p": 0.7}, {"top_p": 0.95, "min_p": 0.02}):
                got = draw(dcl, x, u, top_k=k, **how)
                check(x[:3], [a[:3] for a in got], u[:3], top_k=k, **how)


@pytest.mark.parametrize("bf16", [False, True])
def test_more_rows_than_a_window_of_the_kernels_by_rows(dcl, bf16):
    """1500 rows too long for one list: open and answered rows mixed over two windows of 1024 workgroups, windows without an open
    row and full of them; then captured and replayed over a workspace of other bits."""
    n, V = 1500, 2500
    x, g = logits(n, V, 43)
    x[::7] = -math.inf
    x[5::11, ::3] = math.nan
    x = (x.to(torch.bfloat16) if bf16 else x).cuda()
    r = np.random.default_rng(6)
    how = dict(temperature=r.choice([0.0, 0.7, 1.0], n), top_k=r.choice([0, 0, 1, 5, 700], n), top_p=r.choice([1.0, 0.9], n))
    u = torch.rand(n, generator=g)
    check(x, draw(dcl, x, u.numpy(), **how), u.numpy(), **how)
    answered = np.arange(n) < 1024
    for rows in (answered, ~answered, answered | True):
        some = dict(temperature=np.where(rows, 0.0, 0.9))
        check(x, draw(dcl, x, u.numpy(), **some), u.numpy(), **some)
    check(x, draw(dcl, x, u.numpy()), u.numpy())

    T, k, p = (torch.tensor(how[name], dtype=dt).cuda() for name, dt in
               (("temperature", torch.float32), ("top_k", torch.int32), ("top_p", torch.float32)))
    ud = u.cuda()
    token, kept = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
    conf = torch.empty(n, device="cuda")
    need = dcl.dcl_sample_workspace_bytes(n, V)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def go():
        dcl.dcl_sample_tokens(x, n, V, T, k, p, None, ud, token, conf, kept, ws, need)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        go()
    torch.cuda.current_stream().wait_stream(side)
    for fill in (0xFF, 0, 0x7F):
        u = torch.rand(n, generator=g)
        ud.copy_(u)
        ws.fill_(fill)
        graph.replay()
        torch.cuda.synchronize()
        got = [a.cpu().numpy() for a in (token, conf, kept)]
        check(x, got, u.numpy(), **how)
        assert all(np.array_equal(a, b) for a, b in zip(got, draw(dcl, x, u.numpy(), **how)))
