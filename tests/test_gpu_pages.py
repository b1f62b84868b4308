"""The paged cache and attention over it against a plain float64 form: both element types, page sizes from 16 to 256,
lengths from nothing to more than one part, tokens that see nothing, pages that are missing, spoiled slots behind the
last key, NaN and infinities that only some rows see, strided operands, graphs, streams."""
import math

import pytest
import torch

from serving_reference import E4M3, Pool, attention_rows, e4m3_rows, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dcl():
    import paper_2607_20467_amd as m
    m.load_library()
    return m


def attend(dcl, pool, counts, heads, causal, scale, q=None, max_new=None, seed=3, pad=0, stream=None, q_std=1.5):
    """Runs the call; returns out, lse and the operands (CPU)."""
    g = torch.Generator().manual_seed(seed)
    cu = starts(counts)
    T = int(cu[-1]) + pad
    if q is None:
        q = (torch.randn(T, heads, pool.dh, generator=g) * q_std).to(torch.bfloat16)
    dev = pool.device()
    most = max(list(counts) + [0]) if max_new is None else max_new
    need = dcl.dcl_pages_attention_workspace_bytes(dev, heads, len(counts), T, most, pool.width)
    assert need > 0
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full((T, heads, pool.dh), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, heads), 7.0, device="cuda")
    args = (dev, pool.table.cuda(), pool.len.cuda(), cu.cuda(), len(counts), T, most, q.cuda(), heads, scale, causal, out,
            lse, ws, need)
    dcl.dcl_pages_attention(*args, stream)
    torch.cuda.synchronize()
    return out.double().cpu(), lse.double().cpu(), q, cu, args


def check(pool, out, lse, q, cu, counts, heads, causal, scale, max_new=None, seen=None):
    g = heads // pool.hkv
    for b, n in enumerate(counts):
        L = pool.lens[b]
        have = min(L, pool.width * pool.page)
        k, v = pool.rows(b, have)
        sees = torch.ones(n, have, dtype=torch.bool)
        if causal:
            sees &= torch.arange(have)[None, :] <= (L - n + torch.arange(n))[:, None]
        if seen is not None:
            sees &= seen(b, have)[None, :]
        for i in range(n if max_new is None else min(n, max_new)):
            t = int(cu[b]) + i
            for h in range(heads):
                o, s, eo, es = attention_rows(q[t, h].double()[None], k[:, h // g], v[:, h // g], scale, sees[i:i + 1])
                got, want = out[t, h], o[0]
                assert torch.equal(torch.isnan(got), torch.isnan(want)), (b, i, h)
                inf = torch.isinf(want)
                assert torch.equal(got[inf], want[inf]), (b, i, h)
                ok = torch.isfinite(want)
                err = (got - want).abs()
                assert bool((err[ok] <= eo[0][ok]).all()), (b, i, h, float((err / eo[0].clamp(min=1e-30))[ok].max()))
                if math.isfinite(float(s[0])):
                    assert abs(float(lse[t, h] - s[0])) <= float(es[0]), (b, i, h)
                else:
                    assert float(lse[t, h]) == float(s[0]) or math.isnan(float(s[0])), (b, i, h)


@pytest.mark.parametrize("e4m3", [False, True])
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
])
def test_attention_matches_float64(dcl, e4m3, dh, heads, hkv, page, lens, counts, causal):
    pool = Pool(dcl, lens, page, hkv, dh, e4m3, seed=5, fill=0x7F)
    scale = 1 / math.sqrt(dh)
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, causal, scale, pad=2)
    check(pool, out, lse, q, cu, counts, heads, causal, scale)
    assert bool((out[int(cu[-1]):] == 7).all()) and bool((lse[int(cu[-1]):] == 7).all())


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dh", [64, 128])
def test_many_rows_take_four_fragments(dcl, dh, e4m3):
    """Enough rows and workgroups for the layout of 64 rows: partial last tiles of rows and keys, NaN behind every end, an
    infinity (NaN in 8 bits) that only the last token sees, a missing page."""
    lens, counts = [70, 33, 20, 64, 65, 21, 40, 100], [20, 20, 20, 7, 20, 20, 3, 20]
    pool = Pool(dcl, lens, 16, 4, dh, e4m3, seed=12, fill=0x7F)
    pg, off = pool.places(0)
    pool.v[pg[69], 1, 5, off[69]] = 0x7F if e4m3 else math.inf
    pool.v[pg[69], 1, dh - 1, off[69]] = 0xFF if e4m3 else -math.inf
    gone = pool.table[7, 2].clone()
    pool.table[7, 2] = -1
    heads = 28
    assert (heads // 4 * 20 + 63) // 64 * 4 * 8 >= 96
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, True, 0.11)
    pool.table[7, 2] = gone

    def seen(b, n):
        return torch.arange(n) // 16 != 2 if b == 7 else torch.ones(n, dtype=torch.bool)
    check(pool, out, lse, q, cu, counts, heads, True, 0.11, seen=seen)
    assert not torch.isfinite(out[19, 7:14, 5]).any() and torch.isfinite(out[:19]).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_many_parts(dcl, e4m3):
    """More parts than one group of lanes joins, most of them empty for the short sequence, and a page missing from each."""
    pool = Pool(dcl, [6000, 300, 0], 32, 1, 128, e4m3, seed=13)
    missing = pool.table[:2, 3].clone()
    pool.table[:2, 3] = -1
    out, lse, q, cu, _ = attend(dcl, pool, [2, 1, 1], 3, True, 0.09)
    pool.table[:2, 3] = missing
    check(pool, out, lse, q, cu, [2, 1, 1], 3, True, 0.09, seen=lambda b, n: torch.arange(n) // 32 != 3)
    again = attend(dcl, pool, [2, 1, 1], 3, True, 0.09)[0]
    assert torch.equal(attend(dcl, pool, [2, 1, 1], 3, True, 0.09)[0], again)


@pytest.mark.parametrize("e4m3", [False, True])
def test_tokens_that_see_nothing(dcl, e4m3):
    """No key at all; fewer keys than new tokens (the first ones precede the sequence's start)."""
    pool = Pool(dcl, [0, 3, 20], 16, 2, 64, e4m3, fill=0xFF)
    counts = [2, 6, 0]
    out, lse, q, cu, _ = attend(dcl, pool, counts, 4, True, 0.125)
    assert bool((out[:2] == 0).all()) and bool((lse[:2] == -math.inf).all())
    assert bool((out[2:5] == 0).all()) and bool((lse[2:5] == -math.inf).all())
    check(pool, out, lse, q, cu, counts, 4, True, 0.125)


@pytest.mark.parametrize("e4m3", [False, True])
def test_missing_pages_take_no_part(dcl, e4m3):
    """Entries outside [0, n_pages) inside a sequence, all of them in another, and a table shorter than the length."""
    pool = Pool(dcl, [200, 90, 400], 32, 2, 128, e4m3, seed=2)
    for bad, (b, c) in zip((-1, pool.n_pages, 2 ** 31 - 1, -2 ** 31, -5), ((0, 1), (0, 3), (1, 0), (1, 1), (1, 2))):
        pool.table[b, c] = bad
    keep = pool.table.clone()
    out, lse, q, cu, _ = attend(dcl, pool, [2, 3, 1], 4, True, 0.09)
    pool.table = torch.where((keep < 0) | (keep >= pool.n_pages), torch.zeros_like(keep), keep)

    def seen(b, n):
        page = keep[b].long()[torch.arange(n) // 32]
        return (page >= 0) & (page < pool.n_pages)
    check(pool, out, lse, q, cu, [2, 3, 1], 4, True, 0.09, seen=seen)
    assert bool((out[2:5] == 0).all())
    pool.width = 3                                       # 96 of the positions
    pool.table = pool.table[:, :3].contiguous()
    pool.table[1] = torch.tensor([5, 6, 7])
    out, lse, q, cu, _ = attend(dcl, pool, [1, 1, 2], 4, True, 0.09)
    check(pool, out, lse, q, cu, [1, 1, 2], 4, True, 0.09)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("heads", [2, 8])
def test_odd_values_reach_only_rows_that_see_them(dcl, e4m3, heads):
    """NaN (and in bfloat16 +inf, -inf, both) in the values and keys of positions that only later tokens see."""
    pool = Pool(dcl, [150, 40], 32, 2, 64, e4m3, seed=9)
    vt, kt = pool.v.permute(0, 3, 1, 2), pool.k.permute(0, 2, 1, 3)

    def put(what, b, x, h, d, val):
        pg, off = pool.table[b, x // 32].long(), x % 32
        what[pg, off, h, d] = val
    inf = 0x7F if e4m3 else math.inf
    put(vt, 0, 146, 0, 3, inf)
    put(vt, 0, 147, 0, 3, 0xFF if e4m3 else -math.inf)
    put(vt, 0, 148, 1, 20, 0x7F if e4m3 else math.nan)
    put(vt, 0, 145, 1, 21, 0xFF if e4m3 else -math.inf)
    put(kt, 1, 38, 1, 5, 0x7F if e4m3 else math.nan)
    counts = [7, 5]
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, True, 0.125)
    check(pool, out, lse, q, cu, counts, heads, True, 0.125)
    assert torch.isfinite(out[:1]).all() and not torch.isfinite(out[6]).all()


def test_large_scores_and_rescaling(dcl):
    """Scores whose maximum keeps growing along the sequence, and a scale of either sign."""
    for scale in (1.0, -0.7, 0.0):
        pool = Pool(dcl, [700, 64], 64, 1, 128, False, seed=1)
        pool.k[pool.table[0].long()[:11]] *= torch.linspace(0.1, 4, 11)[:, None, None, None].to(torch.bfloat16)
        out, lse, q, cu, _ = attend(dcl, pool, [1, 1], 4, True, scale)
        check(pool, out, lse, q, cu, [1, 1], 4, True, scale)


def test_rows_past_max_new_are_left(dcl):
    pool = Pool(dcl, [100, 80], 32, 2, 64, False)
    out, lse, q, cu, _ = attend(dcl, pool, [5, 2], 2, True, 0.1, max_new=3)
    assert bool((out[3:5] == 7).all())
    check(pool, out, lse, q, cu, [5, 2], 2, True, 0.1, max_new=3)


def test_borders_and_lengths_out_of_range(dcl):
    """Borders that fall, leave [0, T] or are negative, and lengths below 0 or past the table, stay inside the buffers."""
    pool = Pool(dcl, [64, 64, 64, 64], 32, 1, 64, True)
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
    pool = Pool(dcl, [4], 16, 1, 64, False)
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


def strided(x, extra):
    """The same rows inside wider ones."""
    t, h, d = x.shape
    wide = torch.full((t, h * d + extra), 99.0, dtype=x.dtype, device=x.device)
    wide[:, :h * d] = x.reshape(t, h * d)
    return wide[:, :h * d].unflatten(1, (h, d)), wide


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dh,hkv,page,lens,counts", [
    (128, 2, 16, [1, 16, 17, 33, 0], [1, 3, 17, 20, 0]),
    (64, 3, 64, [200, 64, 130], [200, 1, 66]),
    (128, 1, 128, [129, 5], [129, 9]),
    (64, 1, 32, [1000], [777]),
])
def test_write_and_read(dcl, e4m3, dh, hkv, page, lens, counts):
    """Pages after a write: the tokens' places hold the rounded values, every other byte is as it was; reading gives the
    values back. Tokens before position 0 (more tokens than positions) are skipped and read as zeros."""
    pool = Pool(dcl, lens, page, hkv, dh, e4m3, seed=11)
    g = torch.Generator().manual_seed(4)
    cu = starts(counts)
    T = int(cu[-1]) + 2
    k = (torch.randn(T, hkv, dh, generator=g) * torch.exp(3 * torch.randn(T, hkv, 1, generator=g))).to(torch.bfloat16)
    v = torch.randn(T, hkv, dh, generator=g).to(torch.bfloat16)
    k[0, 0] = 0
    dev = pool.device()
    a = (dev, pool.table.cuda(), pool.len.cuda(), cu.cuda(), len(lens), T, max(counts))
    ks, _ = strided(k.cuda(), 8)
    dcl.dcl_pages_write(*a, ks, v.cuda())
    want = [x.clone() for x in (pool.k, pool.v)] + ([x.clone() for x in (pool.ks, pool.vs)] if e4m3 else [])
    back_k, back_v = torch.full((T, hkv, dh), 9.0).double(), torch.full((T, hkv, dh), 9.0).double()
    for b, n in enumerate(counts):
        for i in range(n):
            x, t = lens[b] - n + i, int(cu[b]) + i
            if x < 0:
                back_k[t] = back_v[t] = 0
                continue
            pg, off = int(pool.table[b, x // page]), x % page
            for src, pages, scales, back in ((k, 0, 2, back_k), (v, 1, 3, back_v)):
                at = want[pages][pg, :, off] if pages == 0 else want[pages][pg, :, :, off]
                if e4m3:
                    val, e = e4m3_rows(src[t].double())
                    at.copy_(val.float().to(torch.float8_e4m3fn).view(torch.uint8))
                    want[scales][pg, :, off] = e.to(torch.uint8)
                    back[t] = val * torch.exp2(e.double() - 127)[:, None]
                else:
                    at.copy_(src[t])
                    back[t] = src[t].double()
    got = [dev.k, dev.v] + ([dev.k_scale, dev.v_scale] if e4m3 else [])
    for name, x, y in zip(("k", "v", "k_scale", "v_scale"), got, want):
        x = x.cpu()
        same = (x == y) | ((x & 0x7F) == 0) & ((y & 0x7F) == 0) if e4m3 and name in "kv" else x == y
        assert bool(same.all()), (name, int((~same).sum()))
    rk, wide = strided(torch.full((T, hkv, dh), 9.0, dtype=torch.bfloat16, device="cuda"), 16)
    rv = torch.full((T, hkv, dh), 9.0, dtype=torch.bfloat16, device="cuda")
    dcl.dcl_pages_read(*a, rk, rv)
    assert torch.equal(rk.double().cpu(), back_k) and torch.equal(rv.double().cpu(), back_v)
    assert bool((wide[:, hkv * dh:] == 99).all())


def test_every_bfloat16_is_rounded_to_the_nearest_e4m3(dcl):
    """All 65536 bit patterns, each in a row whose largest magnitude fixes the scale: infinities, NaN, subnormals, the
    largest numbers, ties."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    rows = []
    for top in (448.0, 2.0 ** -100, 3e38, 1.9 * 2.0 ** -126, 0.0):
        x = bits.reshape(-1, 1, 64).clone()
        x[:, :, 63] = top
        fin = x.double().abs()
        x = torch.where((fin > top) & torch.isfinite(x.double()) & (top > 0), torch.zeros_like(x), x)
        rows.append(x)
    k = torch.cat(rows)
    T = len(k)
    pool = Pool(dcl, [T], 64, 1, 64, True)
    dev = pool.device()
    a = (dev, pool.table.cuda(), pool.len.cuda(), starts([T]).cuda(), 1, T, T)
    dcl.dcl_pages_write(*a, k.cuda(), k.cuda())
    pool.k, pool.v, pool.ks, pool.vs = (x.cpu() for x in (dev.k, dev.v, dev.k_scale, dev.v_scale))
    gk, gv = pool.rows(0)
    pg, off = pool.places(0)
    val, e = e4m3_rows(k.double())
    assert torch.equal(pool.ks[pg, 0, off].long(), e[:, 0])
    want = val * torch.exp2(e.double() - 127)[..., None]
    for got in (gk, gv):
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got.nan_to_num(0), want.nan_to_num(0))
    rk = torch.empty_like(k, device="cuda")
    rv = torch.empty_like(rk)
    dcl.dcl_pages_read(*a, rk, rv)
    # Read back they are those values in bfloat16, where two ends need its rounding: below its smallest step 2^-133, and
    # where four significant bits round up to 2^128 (the largest bfloat16, 255 * 2^120 under the scale 2^120, is stored
    # as 256), which bfloat16 does not have: infinity.
    got = rk.double().cpu()
    over = want.abs() >= 2.0 ** 128
    assert bool(over.any()) and torch.equal(got[over], torch.copysign(torch.full_like(want, math.inf), want)[over])
    err = (got - want).abs()[~over].nan_to_num(0, 1e300, 1e300)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert float(err.max()) <= 2.0 ** -133 / 2 and torch.equal(rk.view(torch.int16), rv.view(torch.int16))
    assert E4M3.nan_to_num(0).max() == 448


def test_replayed_graph_and_second_stream(dcl):
    """Captured calls replay bit for bit with eager work between them; two streams with a workspace each."""
    pool = Pool(dcl, [900, 300], 64, 2, 128, True, seed=8)
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
    """The last page of a pool of more than 2^32 bytes per array: its elements start past 2^31."""
    pages = 2 ** 31 // (8 * 64 * 128) + 9
    kp = torch.zeros((pages, 8, 64, 128), dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros((pages, 8, 128, 64), dtype=torch.bfloat16, device="cuda")
    dev = dcl.KVPages(pages, 64, 8, 128, k=kp, v=vp)
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32, device="cuda")
    ln, cu = torch.tensor([150], dtype=torch.int32, device="cuda"), starts([150]).cuda()
    g = torch.Generator().manual_seed(0)
    k, v = (torch.randn(150, 8, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    a = (dev, table, ln, cu, 1, 150, 150)
    dcl.dcl_pages_write(*a, k.cuda(), v.cuda())
    rk, rv = torch.empty_like(k, device="cuda"), torch.empty_like(v, device="cuda")
    dcl.dcl_pages_read(*a, rk, rv)
    assert torch.equal(rk.cpu(), k) and torch.equal(rv.cpu(), v)
    assert torch.equal(kp[pages - 1, :, :, :].cpu(), k[:64].transpose(0, 1))
    q = torch.randn(1, 8, 128, generator=g).to(torch.bfloat16)
    need = dcl.dcl_pages_attention_workspace_bytes(dev, 8, 1, 1, 1, 3)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = torch.empty(1, 8, 128, dtype=torch.bfloat16, device="cuda")
    dcl.dcl_pages_attention(dev, table, ln, starts([1]).cuda(), 1, 1, 1, q.cuda(), 8, 0.09, True, out, None, ws, need)
    for h in range(8):
        o, _, eo, _ = attention_rows(q[0, h].double()[None], k[:, h].double(), v[:, h].double(), 0.09,
                                     torch.ones(1, 150, dtype=torch.bool))
        assert bool(((out[0, h].double().cpu() - o[0]).abs() <= eo[0]).all())


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dh,heads,hkv,lens,new", [
    (64, 4, 4, [64, 900, 2000], 1), (128, 8, 2, [64, 1500], 1), (128, 4, 4, [640, 2000], 8), (64, 8, 4, [512], 16),
    (128, 16, 4, [256] * 12, 32), (128, 16, 4, [128] * 17, 32),
])
def test_probabilities_keep_sixteen_bits(dcl, e4m3, dh, heads, hkv, lens, new):
    """Half of the keys have the probability 1/2 (1 + 0.87 * 2^-8) of a reference's, half of them 1/2, with values 1 and -1: in
    bfloat16 the two are the same number, and rounded so they cancel. o is the difference, some 2^-10; two parts keep each
    probability to 2^-16, the scores to 2^-20 (four roundings of sums below 2) and the sums of m terms to m * 2^-23."""
    x = 1.25 * 2.0 ** -8                                     # a bfloat16 number, and with -1 a row of e4m3 at the scale 2^-8
    pool = Pool(dcl, lens, 64, hkv, dh, e4m3, seed=11)
    for t in (pool.k, pool.v):
        t.zero_()

    def put(t, at, byte, number):
        t[at] = byte if e4m3 else number
    if e4m3:
        pool.ks.fill_(119)
        pool.vs.fill_(127)
    byte = {float(v): i for i, v in enumerate(E4M3.tolist()) if v == v}
    slot = torch.arange(64) % 16                             # sixteen positions: a reference, a pair of each kind, ...
    kind = torch.where(slot < 2, 0, 1 + slot % 2)            # 0 reference, 1 and 2 the halves
    put(pool.k.movedim(3, 0), (0, slice(None), slice(None), kind > 0), byte[-256.0], -1.0)
    put(pool.k.movedim(3, 0), (1, slice(None), slice(None), kind == 1), byte[x * 256], x)
    put(pool.v.movedim(3, 0), (kind == 1,), byte[1.0], 1.0)
    put(pool.v.movedim(3, 0), (kind == 2,), byte[-1.0], -1.0)
    counts = [new] * len(lens)
    q = torch.zeros(sum(counts), heads, dh, dtype=torch.bfloat16)
    q[:, :, :2] = 1
    out, lse, *_ = attend(dcl, pool, counts, heads, False, math.log(2.0), q=q)
    for b, n in enumerate(lens):
        k, v = pool.rows(b)
        p = torch.exp2(k[:, 0, :2].sum(1))
        want = float((p * v[:, 0, 0]).sum() / p.sum())
        assert 2.0 ** -11 < want < 2.0 ** -9
        got = out[b * new:(b + 1) * new]
        assert float((got - want).abs().max()) <= want * 2.0 ** -8 + 2.0 ** -16 + 2.0 ** -20 + n * 2.0 ** -23, (b, want)
        assert float((lse[b * new:(b + 1) * new] - math.log(float(p.sum()))).abs().max()) <= (n + 64) * 2.0 ** -23


@pytest.mark.parametrize("dh,page", [(64, 16), (128, 32)])
def test_rows_of_more_than_128_workgroups_of_sixty_four(dcl, dh, page):
    """Enough of them for the layout of 64 rows whatever the sequences' lengths: bfloat16 pages, partial last tiles of rows and
    keys, NaN behind every end, an infinity that only the last token sees, a missing page, sequences without new tokens."""
    lens = [70, 33, 20, 64, 65, 21, 40, 100, 1, 300, 24]
    counts = [20, 20, 20, 7, 20, 20, 3, 20, 0, 20, 19]
    pool = Pool(dcl, lens, page, 4, dh, False, seed=14, fill=0x7F)
    pg, off = pool.places(0)
    pool.v[pg[69], 1, 5, off[69]] = math.inf
    pool.v[pg[69], 1, dh - 1, off[69]] = -math.inf
    gone = pool.table[7, 2].clone()
    pool.table[7, 2] = -1
    heads = 28
    assert (heads // 4 * 20 + 63) // 64 * 4 * len(lens) > 128
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, True, 0.11)
    pool.table[7, 2] = gone

    def seen(b, n):
        return torch.arange(n) // page != 2 if b == 7 else torch.ones(n, dtype=torch.bool)
    check(pool, out, lse, q, cu, counts, heads, True, 0.11, seen=seen)
    assert not torch.isfinite(out[19, 7:14, 5]).any() and torch.isfinite(out[:19]).all()
