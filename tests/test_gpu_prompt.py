"""Attention over packed prompts against a plain float64 form: lengths from one token to many tiles, grouped heads,
strided rows, NaN and infinities that only some rows see, hostile borders, graphs."""
import math

import pytest
import torch

from serving_reference import attention_rows, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dcl():
    import paper_2607_20467_amd as m
    m.load_library()
    return m


def operands(counts, heads, hkv, dh, pad=0, seed=0, q_std=1.5):
    g = torch.Generator().manual_seed(seed)
    T = sum(counts) + pad
    return [(torch.randn(T, h, dh, generator=g) * s).to(torch.bfloat16) for h, s in ((heads, q_std), (hkv, 1), (hkv, 1))]


def attend(dcl, q, k, v, cu, causal, scale, max_len=None, T=None, with_lse=True):
    T = q.shape[0] if T is None else T
    heads, dh, hkv = q.shape[1], q.shape[2], k.shape[1]
    B = len(cu) - 1
    most = int((cu[1:] - cu[:-1]).max()) if max_len is None else max_len
    out = torch.full((q.shape[0], heads, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((q.shape[0], heads), 7.0, device="cuda") if with_lse else None
    dcl.dcl_prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu.cuda(), B, T, most, heads, hkv, dh, scale, causal, out, lse)
    torch.cuda.synchronize()
    return out.double().cpu(), None if lse is None else lse.double().cpu()


def check(out, lse, q, k, v, cu, causal, scale, rows=None, heads=None):
    g = q.shape[1] // k.shape[1]
    for b in range(len(cu) - 1):
        lo, hi = int(cu[b]), int(cu[b + 1])
        n = hi - lo
        if n == 0:
            continue
        some = list(range(n)) if rows is None else sorted({r % n for r in rows})
        sees = torch.ones(n, n, dtype=torch.bool)
        if causal:
            sees = sees.tril()
        for h in range(q.shape[1]) if heads is None else heads:
            o, s, eo, es = attention_rows(q[lo:hi, h].double()[some], k[lo:hi, h // g].double(), v[lo:hi, h // g].double(),
                                          scale, sees[some])
            got, gl = out[lo:hi, h][some], lse[lo:hi, h][some]
            assert torch.equal(torch.isnan(got), torch.isnan(o)), (b, h)
            inf = torch.isinf(o)
            assert torch.equal(got[inf], o[inf]), (b, h)
            ok = torch.isfinite(o)
            err = (got - o).abs()
            assert bool((err[ok] <= eo[ok]).all()), (b, h, float((err / eo.clamp(min=1e-30))[ok].max()))
            fin = torch.isfinite(s)
            assert bool(((gl - s).abs()[fin] <= es[fin]).all()), (b, h)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,hkv,dh,counts", [
    (1, 1, 64, [1]),
    (4, 4, 64, [48, 2, 27, 19, 0, 7]),
    (4, 2, 128, [1, 63, 64, 65, 33]),
    (7, 1, 128, [127, 128, 129]),
    (2, 2, 128, [31, 32, 200]),
    (10, 5, 64, [130, 5]),
])
def test_matches_float64(dcl, heads, hkv, dh, counts, causal):
    q, k, v = operands(counts, heads, hkv, dh, pad=3)
    cu = starts(counts)
    out, lse = attend(dcl, q, k, v, cu, causal, 1 / math.sqrt(dh))
    check(out, lse, q, k, v, cu, causal, 1 / math.sqrt(dh))
    assert bool((out[int(cu[-1]):] == 7).all()) and bool((lse[int(cu[-1]):] == 7).all())


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dh,counts", [(128, [1000, 257, 640]), (64, [1500]), (128, [2049])])
def test_long_rows(dcl, dh, counts, causal):
    """Chosen rows of sequences of many tiles: first, last, around the tiles' borders."""
    heads, hkv = 16, 8
    q, k, v = operands(counts, heads, hkv, dh, seed=3)
    cu = starts(counts)
    out, lse = attend(dcl, q, k, v, cu, causal, 0.08)
    check(out, lse, q, k, v, cu, causal, 0.08, rows=[0, 1, 31, 32, 63, 64, 127, 128, 129, 255, 256, 511, 700, -1, -2, -65],
          heads=[0, 1, 7, 15])


def test_scales_and_growing_scores(dcl):
    counts = [300, 64]
    q, k, v = operands(counts, 2, 1, 128, seed=4)
    k *= torch.linspace(0.1, 5, 364)[:, None, None].to(torch.bfloat16)
    cu = starts(counts)
    for scale in (1.0, -0.5, 0.0):
        out, lse = attend(dcl, q, k, v, cu, True, scale)
        check(out, lse, q, k, v, cu, True, scale, rows=range(0, 300, 13))


@pytest.mark.parametrize("causal", [False, True])
def test_odd_values_reach_only_rows_that_see_them(dcl, causal):
    """NaN, +inf, -inf and both in values and keys: rows before them, and other sequences, are as without them."""
    counts = [150, 70, 64]
    q, k, v = operands(counts, 4, 2, 64, seed=6)
    v[100, 0, 3], v[130, 0, 3], v[149, 0, 9], v[149, 1, 63] = math.inf, -math.inf, math.nan, -math.inf
    k[210, 1, 5] = math.nan
    v[150, 1, 0] = math.inf
    v[219, 0, 7] = math.nan
    q[225, 2, 0] = math.nan
    cu = starts(counts)
    out, lse = attend(dcl, q, k, v, cu, causal, 0.125)
    check(out, lse, q, k, v, cu, causal, 0.125)
    assert torch.isfinite(out[226:]).all()
    if causal:
        assert torch.isfinite(out[:100]).all() and not torch.isfinite(out[149, 0]).all()


def test_parts_of_one_projection_and_far_rows(dcl):
    """q, k, v as views of one [T, (H + 2 Hkv) dh] tensor, and rows too far apart for 32-bit offsets inside a tile."""
    counts = [100, 33]
    heads, hkv, dh = 4, 2, 64
    q, k, v = operands(counts, heads, hkv, dh, seed=8)
    cu = starts(counts)
    ref, ref_l = attend(dcl, q, k, v, cu, True, 0.125)
    one = torch.cat([x.flatten(1) for x in (q, k, v)], 1).cuda()
    qs, ks, vs = (x.unflatten(1, (-1, dh)) for x in one.split([heads * dh, hkv * dh, hkv * dh], 1))
    out, lse = attend(dcl, qs, ks, vs, cu, True, 0.125)
    assert torch.equal(out, ref) and torch.equal(lse, ref_l)
    far = torch.zeros((133, (1 << 24) + 8), dtype=torch.bfloat16, device="cuda")     # 4.2 GiB
    far[:, 1024:1024 + hkv * dh] = k.flatten(1).cuda()
    kf = far[:, 1024:1024 + hkv * dh].unflatten(1, (hkv, dh))
    out, lse = attend(dcl, q, kf, v, cu, True, 0.125)
    assert torch.equal(out, ref) and torch.equal(lse, ref_l)


def test_rows_past_max_len_and_without_lse(dcl):
    counts = [200, 40]
    q, k, v = operands(counts, 2, 2, 128)
    cu = starts(counts)
    for causal in (False, True):
        ref, _ = attend(dcl, q, k, v, cu, causal, 0.1)
        out, _ = attend(dcl, q, k, v, cu, causal, 0.1, max_len=130, with_lse=False)
        assert torch.equal(out[:130], ref[:130]) and torch.equal(out[200:], ref[200:]) and bool((out[130:200] == 7).all())
        out, _ = attend(dcl, q, k, v, cu, causal, 0.1, max_len=0)
        assert bool((out == 7).all())


def test_borders_out_of_range_stay_inside(dcl):
    q, k, v = operands([70], 2, 1, 64)
    for cu in ([0, 20, 10, 70], [-7, 5, 60, 1000], [70, 71, 72, 73], [9, 6, 3, -1], [0, 0, 0, 0]):
        attend(dcl, q, k, v, torch.tensor(cu, dtype=torch.int32), True, 0.1, max_len=70)
    e = torch.empty(0, 2, 64, dtype=torch.bfloat16)
    attend(dcl, e, e, e, torch.zeros(2, dtype=torch.int32), True, 0.1)


def test_replays_and_streams(dcl):
    counts = [300, 17]
    q, k, v = (x.cuda() for x in operands(counts, 8, 4, 128))
    cu = starts(counts).cuda()
    out = torch.empty_like(q)
    lse = torch.empty(317, 8, device="cuda")

    def go(stream=None, to=out):
        dcl.dcl_prompt_attention(q, k, v, cu, 2, 317, 300, 8, 4, 128, 0.09, True, to, lse, stream)
    go()
    torch.cuda.synchronize()
    ref, ref_l = out.clone(), lse.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        go(side)
    for _ in range(3):
        out.fill_(3), lse.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(lse, ref_l)
    other = torch.empty_like(out)
    with torch.cuda.stream(side):
        go(to=other)
    go()
    torch.cuda.synchronize()
    assert torch.equal(other, ref) and torch.equal(out, ref)
