"""Pages of 4 bits: the attention's forms for many workgroups that take a sequence in parts, guards around every buffer under borders and
lengths that are none, every scale byte, queries of the least sizes."""
import math

import pytest
import torch

from serving_reference import starts
from step_reference import E2M1, Pool4, attention_rows4, check4, e2m1_rows, key_bytes, scale_of, value_bytes
from test_gpu_pages import attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dcl():
    import paper_2607_20467_amd as m
    m.load_library()
    return m


def parts_of(args):
    """How many parts the call's workspace is for, and workgroups there are at least (16 rows each, or 32)."""
    dev, table, ln, cu, B, T, most, q, heads, scale, causal, out, lse, ws, need = args
    rows = heads // dev.n_kv_heads * most
    tiles = 1 if rows <= 16 else -(-rows // 32)
    parts = need // (T * heads * (dev.head_dim * 4 + 8))
    return parts, parts * B * dev.n_kv_heads * tiles


def run_and_check(dcl, pool, counts, heads, causal, max_new=None, least=256):
    """Against float64, with a page missing from the longest sequence; the same bits a second time; more than one part, more workgroups
    than CUs."""
    at = max(range(len(pool.lens)), key=lambda b: pool.lens[b])
    gone = pool.table[at, 1].clone()
    pool.table[at, 1] = -1
    out, lse, q, cu, args = attend(dcl, pool, counts, heads, causal, 0.1, max_new=max_new, pad=3)
    again = attend(dcl, pool, counts, heads, causal, 0.1, max_new=max_new, pad=3)
    pool.table[at, 1] = gone
    parts, workgroups = parts_of(args)
    assert parts > 1 and workgroups > least, (parts, workgroups)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])

    def seen(b, m):
        return torch.arange(m) // pool.page != 1 if b == at else torch.ones(m, dtype=torch.bool)
    check4(pool, out, lse, q, cu, counts, heads, causal, 0.1, max_new=max_new, seen=seen)
    assert bool((out[int(cu[-1]):] == 7).all()) and bool((lse[int(cu[-1]):] == 7).all())


@pytest.mark.parametrize("dh,heads,hkv,page,new,causal", [
    (128, 4, 4, 64, 1, True), (128, 16, 4, 16, 1, True), (128, 8, 4, 32, 3, True), (128, 4, 4, 1024, 2, False),
    (64, 8, 4, 64, 3, True), (64, 28, 4, 128, 1, True),
])
def test_a_few_tokens_of_many_sequences_in_parts(dcl, dh, heads, hkv, page, new, causal):
    """Runs of 2048 keys: sequences of one run, with one key more and one less, of all parts, of nothing."""
    long = {3: 2047, 11: 2048, 17: 2049, 30: 4097, 41: 6500, 63: 9000}
    lens = [long.get(i, (37 * i) % 150) for i in range(64)]
    counts = [min(new, 1 + i % 3) if i % 7 else 0 for i in range(64)]
    for i in long:
        counts[i] = new
    pool = Pool4(dcl, lens, page, hkv, dh, seed=61, fill=0x7F, width=10240 // page)
    run_and_check(dcl, pool, counts, heads, causal, max_new=new)


@pytest.mark.parametrize("dh,heads,page,causal", [(128, 4, 64, True), (64, 4, 16, True), (128, 4, 256, False), (64, 4, 1024, False)])
def test_blocks_of_many_sequences_in_parts(dcl, dh, heads, page, causal):
    """Runs of 16384 keys under two fragments: one run, with one key more and one less, of all parts, short blocks that need none."""
    lens, counts = [16383, 16384, 16385, 33000, 200, 64, 1, 0], [1, 2, 2, 1, 100, 33, 1, 0]
    pool = Pool4(dcl, lens, page, 4, dh, seed=62, fill=0x7F, width=40960 // page)
    run_and_check(dcl, pool, counts, heads, causal, max_new=256)


class Guarded:
    """Copies of tensors on the device, 64 KiB of a pattern on either side of each."""

    EDGE = 1 << 16

    def __init__(self):
        self.buffers = []

    def __call__(self, x):
        n = x.numel() * x.element_size()
        buffer = torch.full((n + 2 * self.EDGE,), 0xA5, dtype=torch.uint8, device="cuda")
        view = buffer[self.EDGE:self.EDGE + n].view(x.dtype).view(x.shape)
        view.copy_(x)
        self.buffers.append((buffer, n))
        return view

    def check(self):
        torch.cuda.synchronize()
        for buffer, n in self.buffers:
            assert bool((buffer[:self.EDGE] == 0xA5).all()) and bool((buffer[self.EDGE + n:] == 0xA5).all())


def rows_of(cu, T, length):
    """Of each sequence: its rows in the packed operand and its length, as the calls take borders and lengths of any value."""
    out = []
    for b, n in enumerate(length):
        lo = min(max(cu[b], 0), T)
        hi = max(lo, min(cu[b + 1], T))
        out.append((lo, hi - lo, min(max(n, 0), 1 << 30)))
    return out


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("cu", [[0, 2, 1, 4, 8], [-5, 2, 4, 6, 100], [8, 9, 10, 11, 12], [3, 2, 1, 0, -1], [0, 0, 5, 5, 7],
                                [-2 ** 31, 3, 2 ** 31 - 1, 3, 8]])
@pytest.mark.parametrize("length", [[64, -1, 2 ** 31 - 1, 5], [-2 ** 31, 0, 70, 1 << 20], [3, 64, 33, 2]])
def test_borders_and_lengths_that_are_none_touch_nothing_else(dcl, dh, cu, length):
    """Written are the places and rows that a border and a length name, in the buffers alone; all else keeps its contents. A row that
    two sequences claim holds, element by element, what one of them puts there."""
    T, W, page, hkv, heads, max_new = 8, 2, 32, 2, 4, 3
    pool = Pool4(dcl, [64] * 4, page, hkv, dh, seed=63)
    on = Guarded()
    dev = dcl.KVPages(pool.n_pages, page, hkv, dh, dcl.DCL_DTYPE_E2M1, k=on(pool.k), v=on(pool.v), k_scale=on(pool.ks), v_scale=on(pool.vs))
    g = torch.Generator().manual_seed(5)
    k, v, q = (torch.randn(T, h, dh, generator=g).bfloat16() for h in (hkv, hkv, heads))
    a = (dev, on(pool.table), on(torch.tensor(length, dtype=torch.int32)), on(torch.tensor(cu, dtype=torch.int32)), 4, T, max_new)
    spans = rows_of(cu, T, length)
    owners = [[] for _ in range(T)]                     # the (sequence, position, how many rows precede it) that a packed row belongs to
    for b, (first, n, ln) in enumerate(spans):
        for i in range(min(n, max_new)):
            owners[first + i].append((b, ln - n + i))

    # attention, over the pool as it is
    need = dcl.dcl_pages_attention_workspace_bytes(dev, heads, 4, T, max_new, W)
    out, lse = on(torch.full((T, heads, dh), 7.0).bfloat16()), on(torch.full((T, heads), 7.0))
    dcl.dcl_pages_attention(*a, on(q), heads, 0.1, True, out, lse, on(torch.zeros(need, dtype=torch.uint8)), need)
    on.check()
    got, got_l = out.double().cpu(), lse.double().cpu()
    for t in range(T):
        for h in range(heads):
            left = not owners[t]
            fits, near = (got[t, h] == 7) & left, float(got_l[t, h]) == 7 and left
            for b, x in owners[t]:
                keys = max(0, min(x + 1, W * page, spans[b][2]))
                kk, vv = pool.rows(b, keys)
                o, s, eo, es = attention_rows4(q[t, h].double()[None], kk[:, h // 2], vv[:, h // 2], 0.1, torch.ones(1, keys, dtype=torch.bool))
                near |= float(got_l[t, h]) == float(s[0]) if keys == 0 else abs(float(got_l[t, h] - s[0])) <= float(es[0])
                fits |= (got[t, h] - o[0]).abs() <= eo[0]
            assert near and bool(fits.all()), (t, h, owners[t])

    # write
    want = [x.clone() for x in (pool.k, pool.v, pool.ks, pool.vs)]
    (ck, ek), (cv, ev) = e2m1_rows(k.double()), e2m1_rows(v.double())
    for t in range(T):
        for b, x in owners[t]:
            if 0 <= x < W * page:
                pg, off = int(pool.table[b, x // page]), x % page
                want[0][pg, :, off], want[1][pg, :, :, off] = key_bytes(ck[t]), value_bytes(cv[t])
                want[2][pg, :, :, off], want[3][pg, :, :, off] = ek[t].to(torch.uint8), ev[t].to(torch.uint8)
    dcl.dcl_pages_write(*a, on(k), on(v))
    on.check()
    for name, x, y in zip(("k", "v", "k_scale", "v_scale"), (dev.k, dev.v, dev.k_scale, dev.v_scale), want):
        assert torch.equal(x.cpu(), y), name

    # read, what was written among it
    pool.k, pool.v, pool.ks, pool.vs = want
    rk, rv = on(torch.full((T, hkv, dh), 9.0).bfloat16()), on(torch.full((T, hkv, dh), 9.0).bfloat16())
    dcl.dcl_pages_read(*a, rk, rv)
    on.check()
    for got, which in ((rk, 0), (rv, 1)):
        got = got.double().cpu()
        for t in range(T):
            fits = (got[t] == 9) & (not owners[t])
            for b, x in owners[t]:
                back = pool.rows(b, W * page)[which][x] if 0 <= x < W * page else torch.zeros(hkv, dh).double()
                fits |= got[t] == back
            assert bool(fits.all()), (which, t, owners[t])


def test_every_scale_byte_reads_as_what_it_stands_for(dcl):
    """All codes under the bytes 1 to 255: bfloat16 numbers, infinities from 2^128 on, NaN under 255."""
    pool = Pool4(dcl, [255], 64, 1, 64, seed=64)
    code = (torch.arange(64) * 5 % 16)[None].expand(255, 64)
    e = torch.arange(1, 256)[:, None].expand(255, 2)
    pg, off = pool.places(0)
    pool.k.permute(0, 2, 1, 3)[pg, off] = key_bytes(code)[:, None]
    pool.v.permute(0, 3, 1, 2)[pg, off] = value_bytes(code)[:, None]
    for s in (pool.ks, pool.vs):
        s.permute(0, 3, 1, 2)[pg, off] = e.to(torch.uint8)[:, None]
    want = E2M1[code] * scale_of(e).repeat_interleave(32, -1)
    want = torch.where(want.abs() >= 2.0 ** 128, torch.copysign(torch.full_like(want, math.inf), want), want)
    rk, rv = (torch.zeros(255, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dcl.dcl_pages_read(pool.device(), pool.table.cuda(), pool.len.cuda(), starts([255]).cuda(), 1, 255, 255, rk, rv)
    for got in (rk, rv):
        got = got[:, 0].double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and int(torch.isnan(want).sum()) == 64
        assert torch.equal(got.nan_to_num(3, math.inf, -math.inf), want.nan_to_num(3, math.inf, -math.inf))


@pytest.mark.parametrize("least", [-108, -114, -117, -119])
def test_queries_of_the_least_sizes_are_held_to_the_same_bits(dcl, least):
    """Groups of a query whose largest element is down to 2^(least - 6), met by keys that are as large as those are small, so that
    every group moves the scores. The scale of a group stops at 2^-122, where the second part's step, 2^-9 of 2^-126, is below the
    last bit of any bfloat16 from 2^-126 on (2^-133): all of a query stays, and the bound is the one of larger queries."""
    pool = Pool4(dcl, [130, 40], 32, 2, 128, seed=65)
    heads, counts = 4, [2, 1]
    size = torch.tensor([least, least - 2, least - 4, least - 6])
    e = 127 - size - 3                                   # |q k| of some units a group
    assert int(e.max()) <= 252
    pool.ks[:] = e.to(torch.uint8)[None, None, :, None]
    g = torch.Generator().manual_seed(8)
    q = torch.randn(3, heads, 4, 32, generator=g).clamp(-2, 2)
    q[..., 7] = 1.9
    q = (q.double() * torch.exp2(size.double())[:, None]).flatten(2).to(torch.bfloat16)
    assert float(q.double().abs().max()) >= 2.0 ** least
    out, lse, q, cu, _ = attend(dcl, pool, counts, heads, True, 0.1, q=q)
    check4(pool, out, lse, q, cu, counts, heads, True, 0.1)
