"""Pages of 4 bits against a plain float64 form: writing and reading, and attention over page sizes from 16 to 256, lengths from
nothing to more than one part, tokens that see nothing, pages that are missing, NaN scales behind the last key and in keys that only
some rows see, graphs, streams."""
import math

import pytest
import torch

from serving_reference import starts
from step_reference import E2M1, Pool4, attention_rows4, check4, e2m1_rows, key_bytes, key_codes, scale_of, value_bytes, value_codes
from test_gpu_pages import attend, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dcl():
    import paper_2607_20467_amd as m
    m.load_library()
    return m


@pytest.mark.parametrize("dh,hkv,page,lens,counts", [
    (128, 2, 16, [1, 16, 17, 33, 0], [1, 3, 17, 20, 0]),
    (64, 3, 64, [200, 64, 130], [200, 1, 66]),
    (128, 1, 128, [129, 5], [129, 9]),
    (64, 1, 32, [1000], [777]),
    (128, 5, 1024, [1100, 2], [60, 1]),
])
def test_write_and_read(dcl, dh, hkv, page, lens, counts):
    """Pages after a write: the tokens' places hold the rounded values, every other byte is as it was; reading gives the
    values back. Tokens before position 0 (more tokens than positions) are skipped and read as zeros."""
    pool = Pool4(dcl, lens, page, hkv, dh, seed=11)
    g = torch.Generator().manual_seed(4)
    cu = starts(counts)
    T = int(cu[-1]) + 2
    k = (torch.randn(T, hkv, dh, generator=g) * torch.exp(3 * torch.randn(T, hkv, dh, generator=g))).to(torch.bfloat16)
    v = torch.randn(T, hkv, dh, generator=g).to(torch.bfloat16)
    k[0, 0] = 0
    v[0, hkv - 1, dh - 1] = math.nan
    k[0, hkv - 1, 33] = -math.inf
    dev = pool.device()
    a = (dev, pool.table.cuda(), pool.len.cuda(), cu.cuda(), len(lens), T, max(counts))
    dcl.dcl_pages_write(*a, strided(k.cuda(), 8)[0], v.cuda())
    want = [x.clone() for x in (pool.k, pool.v, pool.ks, pool.vs)]
    back_k, back_v = torch.full((T, hkv, dh), 9.0).double(), torch.full((T, hkv, dh), 9.0).double()
    (ck, ek), (cv, ev) = e2m1_rows(k.double()), e2m1_rows(v.double())
    for b, n in enumerate(counts):
        for i in range(n):
            x, t = lens[b] - n + i, int(cu[b]) + i
            if x < 0:
                back_k[t] = back_v[t] = 0
                continue
            pg, off = int(pool.table[b, x // page]), x % page
            want[0][pg, :, off], want[1][pg, :, :, off] = key_bytes(ck[t]), value_bytes(cv[t])
            want[2][pg, :, :, off], want[3][pg, :, :, off] = ek[t].to(torch.uint8), ev[t].to(torch.uint8)
            back_k[t] = E2M1[ck[t]] * scale_of(ek[t]).repeat_interleave(32, -1)
            back_v[t] = E2M1[cv[t]] * scale_of(ev[t]).repeat_interleave(32, -1)
    for name, x, y in zip(("k", "v", "k_scale", "v_scale"), (dev.k, dev.v, dev.k_scale, dev.v_scale), want):
        assert torch.equal(x.cpu(), y), name
    rk, wide = strided(torch.full((T, hkv, dh), 9.0, dtype=torch.bfloat16, device="cuda"), 16)
    rv = torch.full((T, hkv, dh), 9.0, dtype=torch.bfloat16, device="cuda")
    dcl.dcl_pages_read(*a, rk, rv)
    for got, back in ((rk, back_k), (rv, back_v)):
        got = got.double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(back)) and torch.equal(got.nan_to_num(0), back.nan_to_num(0))
    assert bool((wide[:, hkv * dh:] == 99).all())


def test_every_bfloat16_is_rounded_to_the_nearest_e2m1(dcl):
    """All 65536 bit patterns, each in a row whose largest magnitude fixes the scale: infinities, NaN, subnormals, the
    largest numbers, ties."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    rows = []
    for top in (6.0, 2.0 ** -100, 3e38, 1.9 * 2.0 ** -126, 5.0, 0.0):
        x = bits.reshape(-1, 1, 64).clone()
        x[:, :, 31] = x[:, :, 63] = top
        big = (x.double().abs() > top) & torch.isfinite(x.double()) & (top > 0)
        rows.append(torch.where(big, torch.zeros_like(x), x))
    k = torch.cat(rows)
    T = len(k)
    pool = Pool4(dcl, [T], 64, 1, 64)
    dev = pool.device()
    a = (dev, pool.table.cuda(), pool.len.cuda(), starts([T]).cuda(), 1, T, T)
    dcl.dcl_pages_write(*a, k.cuda(), k.cuda())
    pool.k, pool.v, pool.ks, pool.vs = (x.cpu() for x in (dev.k, dev.v, dev.k_scale, dev.v_scale))
    code, e = e2m1_rows(k.double())
    pg, off = pool.places(0)
    for got in (key_codes(pool.k.permute(0, 2, 1, 3)[pg, off]), value_codes(pool.v.permute(0, 3, 1, 2)[pg, off])):
        assert torch.equal(got, code)
    for got in (pool.ks, pool.vs):
        assert torch.equal(got.permute(0, 3, 1, 2)[pg, off].long(), e)
    rk = torch.empty_like(k, device="cuda")
    rv = torch.empty_like(rk)
    dcl.dcl_pages_read(*a, rk, rv)
    # read back they are those values, each a bfloat16 number
    want = E2M1[code] * scale_of(e).repeat_interleave(32, -1)
    assert float(want.nan_to_num(0).abs().max()) == 3 * 2.0 ** 126
    got = rk.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(0, 1, -1), want.nan_to_num(0, 1, -1))
    assert torch.equal(rk.view(torch.int16), rv.view(torch.int16))


@pytest.mark.parametrize("dh,heads,hkv", [(128, 4, 2), (64, 8, 8)])
def test_largest_numbers_stay_out_of_rows_that_do_not_see_them(dcl, dh, heads, hkv):
    """Tokens of bfloat16's largest numbers behind a row's own position: as if they were anything else."""
    n, new = 70, 6
    g = torch.Generator().manual_seed(71)
    k, v = (torch.randn(n, hkv, dh, generator=g).bfloat16() for _ in range(2))
    q = torch.randn(new, heads, dh, generator=g).bfloat16().cuda()
    top = torch.finfo(torch.bfloat16).max
    outs = []
    for values in ([0.0, 0.0, 0.0], [top, -top, 3.2e38]):
        pool = Pool4(dcl, [n], 16, hkv, dh)
        dev = pool.device()
        v[n - 3:, :, 1] = v[n - 3:, :, dh - 1] = torch.tensor(values).bfloat16()[:, None]
        table, length = pool.table.cuda(), pool.len.cuda()
        dcl.dcl_pages_write(dev, table, length, starts([n]).cuda(), 1, n, n, k.cuda(), v.cuda())
        nb = dcl.dcl_pages_attention_workspace_bytes(dev, heads, 1, new, new, table.shape[1])
        out = torch.empty(new, heads, dh, dtype=torch.bfloat16, device="cuda")
        dcl.dcl_pages_attention(dev, table, length, starts([new]).cuda(), 1, new, new, q, heads, 0.1, True, out, None,
                                torch.empty(nb, dtype=torch.uint8, device="cuda"), nb)
        outs.append(out.float().cpu())
    a, b = outs
    assert torch.equal(a[:new - 3], b[:new - 3])
    assert bool(torch.isfinite(b).all()) and float(b[new - 3:].abs().max()) > 1e34


@pytest.mark.parametrize("dh,heads,hkv,page,lens,counts,causal", [
    (64, 1, 1, 16, [1], [1], True),
    (128, 4, 4, 16, [1, 15, 16, 17, 0], [1, 1, 1, 1, 1], True),
    (128, 28, 4, 64, [63, 64, 65, 300], [1, 2, 3, 5], True),
    (128, 8, 1, 32, [257, 40], [9, 3], True),
    (64, 14, 2, 128, [1000, 129, 5], [1, 1, 1], False),
    (64, 6, 6, 32, [70, 33], [17, 33], True),
    (128, 4, 2, 64, [200, 64], [64, 31], False),
    (64, 16, 2, 16, [90, 20], [9, 20], True),
    (128, 2, 2, 256, [2100], [1], False),
    (64, 7, 1, 1024, [1500, 900], [3, 1], True),
])
def test_attention_matches_float64(dcl, dh, heads, hkv, page, lens, counts, causal):
    pool = Pool4(dcl, lens, page, hkv, dh, seed=5, fill=0x7F)
    scale = 1 / math.sqrt(dh)
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, causal, scale, pad=2)
    check4(pool, out, lse, q, cu, counts, heads, causal, scale)
    assert bool((out[int(cu[-1]):] == 7).all()) and bool((lse[int(cu[-1]):] == 7).all())


@pytest.mark.parametrize("dh", [64, 128])
def test_many_rows(dcl, dh):
    """Partial last tiles of rows and keys, NaN behind every end, a group of NaN that only the last token sees, a missing
    page, sequences without new tokens."""
    lens = [70, 33, 20, 64, 65, 21, 40, 100, 1, 300, 24]
    counts = [20, 20, 20, 7, 20, 20, 3, 20, 0, 20, 19]
    pool = Pool4(dcl, lens, 16, 4, dh, seed=12, fill=0x7F)
    pg, off = pool.places(0)
    pool.vs[pg[69], 1, dh // 32 - 1, off[69]] = 255
    gone = pool.table[7, 2].clone()
    pool.table[7, 2] = -1
    heads = 28
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, True, 0.11)
    pool.table[7, 2] = gone

    def seen(b, n):
        return torch.arange(n) // 16 != 2 if b == 7 else torch.ones(n, dtype=torch.bool)
    check4(pool, out, lse, q, cu, counts, heads, True, 0.11, seen=seen)
    assert torch.isnan(out[19, 7:14, dh - 32:]).all() and torch.isfinite(out[:19]).all()
    assert torch.isfinite(out[19, 7:14, :dh - 32]).all()


def test_many_parts(dcl):
    """More parts than one group of lanes joins, most of them empty for the short sequence, and a page missing from each."""
    pool = Pool4(dcl, [12000, 300, 0], 32, 1, 128, seed=13)
    missing = pool.table[:2, 3].clone()
    pool.table[:2, 3] = -1
    out, lse, q, cu, _ = attend(dcl, pool, [2, 1, 1], 3, True, 0.09)
    pool.table[:2, 3] = missing
    check4(pool, out, lse, q, cu, [2, 1, 1], 3, True, 0.09, seen=lambda b, n: torch.arange(n) // 32 != 3)
    again = attend(dcl, pool, [2, 1, 1], 3, True, 0.09)[0]
    assert torch.equal(attend(dcl, pool, [2, 1, 1], 3, True, 0.09)[0], again)


def test_tokens_that_see_nothing(dcl):
    """No key at all; fewer keys than new tokens (the first ones precede the sequence's start)."""
    pool = Pool4(dcl, [0, 3, 20], 16, 2, 64, fill=0xFF)
    counts = [2, 6, 0]
    out, lse, q, cu, _ = attend(dcl, pool, counts, 4, True, 0.125)
    assert bool((out[:5] == 0).all()) and bool((lse[:5] == -math.inf).all())
    check4(pool, out, lse, q, cu, counts, 4, True, 0.125)


def test_missing_pages_take_no_part(dcl):
    """Entries outside [0, n_pages) inside a sequence, all of them in another, and a table shorter than the length."""
    pool = Pool4(dcl, [200, 90, 400], 32, 2, 128, seed=2)
    for bad, (b, c) in zip((-1, pool.n_pages, 2 ** 31 - 1, -2 ** 31, -5), ((0, 1), (0, 3), (1, 0), (1, 1), (1, 2))):
        pool.table[b, c] = bad
    keep = pool.table.clone()
    out, lse, q, cu, _ = attend(dcl, pool, [2, 3, 1], 4, True, 0.09)
    pool.table = torch.where((keep < 0) | (keep >= pool.n_pages), torch.zeros_like(keep), keep)

    def seen(b, n):
        page = keep[b].long()[torch.arange(n) // 32]
        return (page >= 0) & (page < pool.n_pages)
    check4(pool, out, lse, q, cu, [2, 3, 1], 4, True, 0.09, seen=seen)
    assert bool((out[2:5] == 0).all())
    pool.width = 3                                       # 96 of the positions
    pool.table = pool.table[:, :3].contiguous()
    pool.table[1] = torch.tensor([5, 6, 7])
    out, lse, q, cu, _ = attend(dcl, pool, [1, 1, 2], 4, True, 0.09)
    check4(pool, out, lse, q, cu, [1, 1, 2], 4, True, 0.09)


@pytest.mark.parametrize("dh,heads", [(64, 2), (128, 8)])
def test_nan_groups_reach_only_rows_that_see_them(dcl, dh, heads):
    """NaN in groups of the values and keys of positions that only later tokens see, and in a query."""
    pool = Pool4(dcl, [150, 40, 200], 32, 2, dh, seed=9)

    def put(scales, b, x, h, g):
        scales[pool.table[b, x // 32].long(), h, g, x % 32] = 255
    put(pool.vs, 0, 146, 0, 0)
    put(pool.vs, 0, 148, 1, 1)
    put(pool.vs, 2, 70, 1, dh // 32 - 1)                 # in a tile that every row sees
    put(pool.ks, 1, 38, 1, 1)
    counts = [7, 5, 2]
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, True, 0.125)
    check4(pool, out, lse, q, cu, counts, heads, True, 0.125)
    assert torch.isfinite(out[:1]).all() and not torch.isfinite(out[6]).all()
    q[12, 1, 40] = math.nan
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, True, 0.125, q=q)
    assert torch.isnan(out[12, 1]).all() and torch.isfinite(out[12, 0]).all() and torch.isfinite(out[13, 0]).all()


@pytest.mark.parametrize("dh,heads", [(64, 2), (128, 8)])
def test_infinite_values_reach_only_rows_that_see_them(dcl, dh, heads):
    """Scale bytes a caller may put into its pages, under which some codes stand for 2^128 and more: nothing to the rows that do
    not see them, NaN to those that do, in the dimensions of these codes; what is finite under them counts as it is."""
    pool = Pool4(dcl, [150, 40], 32, 2, dh, seed=31)
    counts, last = [9, 6], dh // 32 - 1
    for b, x, h, g, byte in ((0, 145, 0, 0, 254), (0, 148, 1, last, 253), (1, 37, 0, last, 253), (1, 38, 1, 0, 255)):
        pool.vs[pool.table[b, x // 32].long(), h, g, x % 32] = byte
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, True, 0.125)
    group, odd = heads // 2, 0
    for b, n in enumerate(counts):
        k, v = pool.rows(b)
        v = torch.where(v.abs() >= 2.0 ** 128, math.nan, v)
        sees = torch.arange(pool.lens[b])[None, :] <= (pool.lens[b] - n + torch.arange(n))[:, None]
        for h in range(heads):
            rows = slice(int(cu[b]), int(cu[b]) + n)
            want, _, tol, _ = attention_rows4(q[rows, h].double(), k[:, h // group], v[:, h // group], 0.125, sees)
            got, ok = out[rows, h], ~torch.isnan(want)
            assert torch.equal(torch.isnan(got), ~ok), (b, h)
            assert bool(((got - want).abs()[ok] <= tol[ok]).all()), (b, h)
            odd += int((~ok).sum())
    assert odd > 100 and torch.isfinite(out[:4]).all()


def test_large_scores_and_rescaling(dcl):
    """Scores whose maximum keeps growing along the sequence, and a scale of either sign."""
    for scale in (1.0, -0.7, 0.0):
        pool = Pool4(dcl, [700, 64], 64, 1, 128, seed=1)
        pool.ks[pool.table[0].long()[:11]] += (torch.arange(11) // 4).to(torch.uint8)[:, None, None, None]
        out, lse, q, cu, _ = attend(dcl, pool, [1, 1], 4, True, scale)
        check4(pool, out, lse, q, cu, [1, 1], 4, True, scale)


@pytest.mark.parametrize("dh", [64, 128])
def test_queries_of_unlike_sizes(dcl, dh):
    """A few dimensions of a query far larger than the others, met by keys that are zero there or not."""
    pool = Pool4(dcl, [90, 300], 32, 2, dh, seed=21)
    g = torch.Generator().manual_seed(6)
    counts, heads = [2, 1], 4
    q = torch.randn(3, heads, dh, generator=g)
    q[:, :2, 5] *= 300
    q[:, 2, 40] = 60000.0
    q[1, 3] *= 1e-3
    pool.k[:, :, :, 20] &= 0xF0                          # dimension 40: no key has it
    q = q.to(torch.bfloat16)
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, False, 0.1, q=q)
    check4(pool, out, lse, q, cu, counts, heads, False, 0.1)


def test_rows_past_max_new_are_left(dcl):
    pool = Pool4(dcl, [100, 80], 32, 2, 64)
    out, lse, q, cu, _ = attend(dcl, pool, [5, 2], 2, True, 0.1, max_new=3)
    assert bool((out[3:5] == 7).all())
    check4(pool, out, lse, q, cu, [5, 2], 2, True, 0.1, max_new=3)


def test_borders_and_lengths_out_of_range(dcl):
    """Borders that fall, leave [0, T] or are negative, and lengths below 0 or past the table, stay inside the buffers."""
    pool = Pool4(dcl, [64, 64, 64, 64], 32, 1, 64)
    dev = pool.device()
    q = torch.randn(8, 2, 64).to(torch.bfloat16).cuda()
    k = torch.randn(8, 1, 64).to(torch.bfloat16).cuda()
    for cu in ([0, 2, 1, 4, 8], [-5, 2, 4, 6, 100], [8, 9, 10, 11, 12], [3, 2, 1, 0, -1]):
        for ln in ([64, -1, 2 ** 31 - 1, 5], [-2 ** 31, 0, 70, 1 << 20]):
            cu_d, ln_d = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (cu, ln))
            out = torch.zeros(8, 2, 64, dtype=torch.bfloat16, device="cuda")
            need = dcl.dcl_pages_attention_workspace_bytes(dev, 2, 4, 8, 8, pool.width)
            ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
            a = (dev, pool.table.cuda(), ln_d, cu_d, 4, 8, 8)
            dcl.dcl_pages_attention(*a, q, 2, 0.1, True, out, None, ws, need)
            dcl.dcl_pages_write(*a, k, k)
            dcl.dcl_pages_read(*a, k, k)
            torch.cuda.synchronize()


def test_nothing_to_do(dcl):
    pool = Pool4(dcl, [4], 16, 1, 64)
    dev = pool.device()
    e = torch.empty(0, 1, 64, dtype=torch.bfloat16, device="cuda")
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    a = (dev, pool.table.cuda(), pool.len.cuda(), zero, 1, 0, 0)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    before = dev.k.clone()
    dcl.dcl_pages_write(*a, e, e)
    dcl.dcl_pages_read(*a, e, e)
    dcl.dcl_pages_attention(*a, e, 1, 0.1, False, e, None, ws, 256)
    torch.cuda.synchronize()
    assert torch.equal(before, dev.k)


def test_replayed_graph_and_second_stream(dcl):
    """Captured calls replay bit for bit with eager work between them; two streams with a workspace each."""
    pool = Pool4(dcl, [900, 300], 64, 2, 128, seed=8)
    out, lse, q, cu, args = attend(dcl, pool, [1, 3], 8, True, 0.09)
    dev, table, ln, cu_d, B, T, most, q_d, heads, scale, causal, o, l, ws, need = args
    k = torch.randn(T, 2, 128).to(torch.bfloat16).cuda()
    dcl.dcl_pages_write(dev, table, ln, cu_d, B, T, most, k, k)
    dcl.dcl_pages_attention(*args)
    torch.cuda.synchronize()
    ref, ref_l = o.clone(), l.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        dcl.dcl_pages_write(dev, table, ln, cu_d, B, T, most, k, k, side)
        dcl.dcl_pages_attention(*args, side)
    for _ in range(4):
        o.fill_(5), l.fill_(5), ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, ref) and torch.equal(l, ref_l)
    ws2, o2 = torch.empty_like(ws), torch.empty_like(o)
    with torch.cuda.stream(side):
        dcl.dcl_pages_attention(*args[:11], o2, None, ws2, need)
    dcl.dcl_pages_attention(*args)
    torch.cuda.synchronize()
    assert torch.equal(o, ref) and torch.equal(o2, ref)


def test_offsets_past_32_bits(dcl):
    """The last page of a pool of more than 2^32 bytes per array."""
    pages = 2 ** 32 // (8 * 64 * 64) + 9
    kp = torch.zeros((pages, 8, 64, 64), dtype=torch.uint8, device="cuda")
    vp = torch.zeros((pages, 8, 64, 64), dtype=torch.uint8, device="cuda")
    dev = dcl.KVPages(pages, 64, 8, 128, dcl.DCL_DTYPE_E2M1, k=kp, v=vp)
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32, device="cuda")
    ln, cu = torch.tensor([150], dtype=torch.int32, device="cuda"), starts([150]).cuda()
    g = torch.Generator().manual_seed(0)
    k, v = (torch.randn(150, 8, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    a = (dev, table, ln, cu, 1, 150, 150)
    dcl.dcl_pages_write(*a, k.cuda(), v.cuda())
    rk, rv = torch.empty_like(k, device="cuda"), torch.empty_like(v, device="cuda")
    dcl.dcl_pages_read(*a, rk, rv)
    want = []
    for x, got in ((k, rk), (v, rv)):
        code, e = e2m1_rows(x.double())
        want.append(E2M1[code] * scale_of(e).repeat_interleave(32, -1))
        assert torch.equal(got.double().cpu(), want[-1])
    assert torch.equal(kp[pages - 1].cpu(), key_bytes(e2m1_rows(k[:64].double())[0]).transpose(0, 1))
    q = torch.randn(1, 8, 128, generator=g).to(torch.bfloat16)
    need = dcl.dcl_pages_attention_workspace_bytes(dev, 8, 1, 1, 1, 3)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = torch.empty(1, 8, 128, dtype=torch.bfloat16, device="cuda")
    dcl.dcl_pages_attention(dev, table, ln, starts([1]).cuda(), 1, 1, 1, q.cuda(), 8, 0.09, True, out, None, ws, need)
    for h in range(8):
        o, _, eo, _ = attention_rows4(q[0, h].double()[None], want[0][:, h], want[1][:, h], 0.09,
                                     torch.ones(1, 150, dtype=torch.bool))
        assert bool(((out[0, h].double().cpu() - o[0]).abs() <= eo[0]).all())


@pytest.mark.parametrize("dh,heads,hkv,page,lens,counts,causal", [
    (128, 4, 4, 64, [1280, 700], [64, 64], False),
    (128, 28, 4, 16, [130, 64, 1], [11, 64, 1], True),
    (64, 8, 2, 32, [40, 64, 65, 200], [40, 20, 9, 33], True),
    (64, 3, 1, 128, [129, 900], [12, 100], False),
    (128, 8, 1, 1024, [1100, 0, 63], [5, 0, 63], True),
])
def test_blocks_of_more_than_32_rows(dcl, dh, heads, hkv, page, lens, counts, causal):
    pool = Pool4(dcl, lens, page, hkv, dh, seed=31, fill=0xA7)
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, causal, 0.1, pad=1)
    check4(pool, out, lse, q, cu, counts, heads, causal, 0.1)
    assert bool((out[int(cu[-1]):] == 7).all())


@pytest.mark.parametrize("dh", [64, 128])
def test_blocks_with_odd_groups_and_missing_pages(dcl, dh):
    """In several tiles, seen by all rows, by some and by none."""
    lens, counts, heads = [400, 190], [60, 64], 4
    pool = Pool4(dcl, lens, 16, 2, dh, seed=32, fill=0x7F)

    def put(scales, b, x, h, g):
        scales[pool.table[b, x // 16].long(), h, g, x % 16] = 255
    for x in (345, 370, 399):
        put(pool.vs, 0, x, 0, x % (dh // 32))
    put(pool.vs, 1, 10, 1, 1)
    put(pool.ks, 1, 150, 0, 0)
    gone = pool.table[:, 4].clone()
    pool.table[:, 4] = torch.tensor([-1, pool.n_pages])
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, True, 0.1)
    pool.table[:, 4] = gone
    check4(pool, out, lse, q, cu, counts, heads, True, 0.1, seen=lambda b, n: torch.arange(n) // 16 != 4)
    assert torch.isfinite(out[:5]).all() and torch.isnan(out[59, 0]).any() and torch.isfinite(out[59, 2:]).all()
    again = attend(dcl, pool, counts, heads, True, 0.1)[0]
    assert torch.equal(attend(dcl, pool, counts, heads, True, 0.1)[0].nan_to_num(3), again.nan_to_num(3))


def test_blocks_in_parts(dcl):
    """Few rows' tiles over a long cache: parts, the last of them short, and a sequence that ends in the first."""
    pool = Pool4(dcl, [5000, 100], 32, 1, 128, seed=33)
    out, lse, q, cu, args = attend(dcl, pool, [40, 10], 1, True, 0.09)
    assert args[-1] > 256                                # the workspace of parts
    rows = [0, 7, 39, 40, 49]
    for t in rows:
        b, i = (0, t) if t < 40 else (1, t - 40)
        k, v = pool.rows(b)
        sees = (torch.arange(pool.lens[b]) <= pool.lens[b] - (40, 10)[b] + i)[None]
        o, s, eo, es = attention_rows4(q[t, 0].double()[None], k[:, 0], v[:, 0], 0.09, sees)
        assert bool(((out[t, 0] - o[0]).abs() <= eo[0]).all()) and abs(float(lse[t, 0] - s[0])) <= float(es[0]), t


@pytest.mark.parametrize("dh,heads,hkv,lens,new", [(64, 4, 4, [64, 900], 1), (128, 8, 2, [64, 1500], 1), (128, 4, 4, [640], 20),
                                                  (64, 8, 4, [512], 30), (128, 16, 4, [256] * 3, 32)])
def test_probabilities_keep_sixteen_bits(dcl, dh, heads, hkv, lens, new):
    """Half of the keys have a probability 1 + 0.69 * 2^-7 times that of the other half, with values 1 and -1: o is their difference
    over the sum of all, some 2^-9. In bfloat16 the two are a whole number of steps apart, 2^-7 or 0 of them, and o is off by a
    third or more; two parts keep each probability to 2^-16, the scores to 2^-20 (four roundings of sums below 2), and the sums of
    m terms to m * 2^-23."""
    pool = Pool4(dcl, lens, 64, hkv, dh, seed=11)
    slot = torch.arange(64) % 16
    kind = torch.where(slot < 2, 0, 1 + slot % 2)
    code = torch.zeros(64, dh, dtype=torch.int64)
    code[kind > 0, 0] = 8 + 2                            # -1 in the first 32 dimensions
    code[kind == 1, 32] = 2                              # 1 under a scale of 2^-7 in the next
    pool.k[:] = key_bytes(code)
    pool.ks.fill_(127)
    pool.ks[:, :, 1] = 120
    val = torch.zeros(64, dh, dtype=torch.int64)
    val[kind == 1], val[kind == 2] = 2, 10
    pool.v[:] = value_bytes(val).T
    pool.vs.fill_(127)
    counts = [new] * len(lens)
    q = torch.zeros(sum(counts), heads, dh, dtype=torch.bfloat16)
    q[:, :, 0] = q[:, :, 32] = 1
    out, lse, *_ = attend(dcl, pool, counts, heads, False, math.log(2.0), q=q)
    for b, n in enumerate(lens):
        k, v = pool.rows(b)
        p = torch.exp2(k[:, 0, 0] + k[:, 0, 32])
        want = float((p * v[:, 0, 0]).sum() / p.sum())
        assert 2.0 ** -11 < want < 2.0 ** -8
        got = out[b * new:(b + 1) * new]
        assert float((got - want).abs().max()) <= want * 2.0 ** -8 + 2.0 ** -16 + 2.0 ** -20 + n * 2.0 ** -23, (b, want)
        assert float((lse[b * new:(b + 1) * new] - math.log(float(p.sum()))).abs().max()) <= (n + 64) * 2.0 ** -23


@pytest.mark.parametrize("dh,heads,hkv,page,n,lo,hi,new,causal", [
    (128, 8, 8, 16, 40, 0, 150, 1, True), (64, 16, 8, 32, 40, 0, 120, 1, True), (128, 4, 4, 16, 24, 20, 120, 110, True),
    (64, 4, 4, 16, 24, 60, 100, 105, False),
])
def test_more_workgroups_than_cus(dcl, dh, heads, hkv, page, n, lo, hi, new, causal):
    """The kernels' form for many workgroups: one token or a block of each of many sequences, some of them empty, a missing page in
    one, NaN behind every end and in a key that only the last row sees."""
    lens = [lo + (37 * i) % (hi - lo + 1) for i in range(n)]
    counts = [new if new == 1 else 1 + (i * 7) % new if i % 3 == 0 else 0 for i in range(n)]
    counts = [min(c, max(1, x)) if new > 1 else c for c, x in zip(counts, lens)]
    assert n * hkv * (1 if new == 1 else (heads // hkv * max(counts) + 31) // 32) > 256
    pool = Pool4(dcl, lens, page, hkv, dh, seed=41, fill=0x7F)
    at = next(b for b in range(n) if lens[b] > 3 * page and counts[b])
    pool.vs[pool.table[at, (lens[at] - 1) // page].long(), 1, 0, (lens[at] - 1) % page] = 255
    gone = pool.table[at, 1].clone()
    pool.table[at, 1] = -1
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, causal, 0.1, pad=3)
    pool.table[at, 1] = gone

    def seen(b, m):
        return torch.arange(m) // page != 1 if b == at else torch.ones(m, dtype=torch.bool)
    check4(pool, out, lse, q, cu, counts, heads, causal, 0.1, seen=seen)
    assert bool((out[int(cu[-1]):] == 7).all())


@pytest.mark.parametrize("dh,heads,hkv,page,lens,counts,causal,width", [
    (128, 8, 2, 64, [1600, 100, 0, 3000, 40, 1537, 1535], [1] * 7, True, None),
    (64, 16, 1, 16, [2000, 1471, 1473, 5, 64], [1, 0, 1, 1, 1], True, 512),
    (128, 4, 2, 32, [0, 0, 1700, 0, 1530, 12, 0], [0, 1, 8, 2, 8, 0, 1], True, None),
    (128, 2, 2, 256, [9000], [2], False, 64),
    (64, 6, 3, 128, [6000, 20, 4000], [3, 3, 1], False, None),
    (128, 16, 2, 1024, [1024, 4096, 2048], [2, 1, 2], True, 16),
])
def test_parts_take_runs_in_turn(dcl, dh, heads, hkv, page, lens, counts, causal, width):
    """Sequences that end inside a run, with one, before the second part's first, and far below what the table could name; a
    missing page, and NaN behind every end."""
    pool = Pool4(dcl, lens, page, hkv, dh, seed=51, fill=0x7F, width=width)
    at = max(range(len(lens)), key=lambda b: lens[b])
    gone = pool.table[at, 1].clone()
    pool.table[at, 1] = -1
    out, lse, q, cu, args = attend(dcl, pool, counts, heads, causal, 0.1, pad=3)
    again = attend(dcl, pool, counts, heads, causal, 0.1, pad=3)
    pool.table[at, 1] = gone
    assert args[-1] > 256 and torch.equal(out, again[0]) and torch.equal(lse, again[1])

    def seen(b, m):
        return torch.arange(m) // page != 1 if b == at else torch.ones(m, dtype=torch.bool)
    check4(pool, out, lse, q, cu, counts, heads, causal, 0.1, seen=seen)
    assert bool((out[int(cu[-1]):] == 7).all())


@pytest.mark.parametrize("n", [63, 64, 65, 193, 256, 257])
def test_parts_of_many_sequences(dcl, n):
    lens = [2500 if i % 61 == 5 else 1540 if i % 61 == 7 else (29 * i) % 90 for i in range(n)]
    pool = Pool4(dcl, lens, 16, 2, 64, seed=52, fill=0x7F, width=1024)
    out, lse, q, cu, args = attend(dcl, pool, [1] * n, 2, True, 0.2)
    assert args[-1] > 256
    check4(pool, out, lse, q, cu, [1] * n, 2, True, 0.2)


def test_lengths_that_are_none_stay_in_bounds(dcl):
    """Borders and lengths out of any order: rows that no sequence has stay, those of the sound one are right."""
    lens = [2000, 1800, 40]
    pool = Pool4(dcl, lens, 64, 2, 128, seed=53, fill=0x7F)
    dev, table = pool.device(), pool.table.cuda()
    q = torch.randn(3, 4, 128, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    nb = dcl.dcl_pages_attention_workspace_bytes(dev, 4, 3, 3, 1, table.shape[1])
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")

    def run(length, cu):
        out = torch.full((3, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        dcl.dcl_pages_attention(dev, table, torch.tensor(length, dtype=torch.int32).cuda(),
                                torch.tensor(cu, dtype=torch.int32).cuda(), 3, 3, 1, q, 4, 0.1, True, out, None, ws, nb)
        return out.float().cpu()
    good = run(lens, [0, 1, 2, 3])
    assert torch.equal(run([2000, -5, 2 ** 31 - 1], [0, 1, 1, -7]), torch.cat([good[:1], torch.full((2, 4, 128), 7.0)]))
    assert torch.equal(run([2 ** 31 - 1, 1800, 40], [9, 1, 2, 2 ** 31 - 1])[1:], good[1:])
