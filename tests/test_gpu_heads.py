"""Norm and rotation of heads against extended precision: both head sizes, whole and partial rotation, with and without gains,
far positions, rows of padding, strided operands, in place, graphs."""
import pytest
import torch

from step_reference import norm_rope

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dcl():
    import paper_2607_20467_amd as m
    m.load_library()
    return m


def normal(g, *shape):
    return torch.randn(*shape, generator=g)


def operands(T, H, Hkv, dh, seed=0):
    """Rows of one projection (queries, keys, values side by side), gains."""
    g = torch.Generator().manual_seed(seed)
    row = (normal(g, T, H + 2 * Hkv, dh) * torch.exp(normal(g, 1, H + 2 * Hkv, 1))).to(torch.bfloat16)
    return row, 1 + 0.3 * normal(g, dh), 1 + 0.3 * normal(g, dh)


def run(dcl, row, pos, H, Hkv, gq, gk, eps, base, rot, inplace=False, stream=None):
    T, _, dh = row.shape
    row = row.cuda()
    q, k = row[:, :H], row[:, H:H + Hkv]
    qo = q if inplace else torch.full((T, H, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    ko = k if inplace else torch.full((T, Hkv + 1, dh), 7.0, dtype=torch.bfloat16, device="cuda")[:, :Hkv]
    dcl.dcl_heads_norm_rope(q, k, pos.cuda(), T, H, Hkv, dh, None if gq is None else gq.cuda(),
                            None if gk is None else gk.cuda(), eps, base, rot, qo, ko, stream)
    torch.cuda.synchronize()
    return qo.double().cpu(), ko.double().cpu(), row.cpu()


def check(got, x, pos, gain, eps, base, rot, left=7.0):
    want, err = norm_rope(x.double(), pos, gain, eps, base, rot)
    live = pos >= 0
    off = (got - want).abs()[live]
    assert bool((off <= err[live]).all()), float((off / err[live]).max())
    assert torch.equal(got[~live], torch.full_like(got, left)[~live] if isinstance(left, float) else left[~live])


@pytest.mark.parametrize("T,H,Hkv,dh,rot,far", [
    (1, 1, 1, 64, 64, 1), (1, 28, 4, 128, 128, 131072), (7, 3, 1, 128, 64, 100), (33, 12, 12, 64, 16, 5000),
    (5, 32, 32, 128, 128, 2 ** 28), (300, 14, 2, 64, 32, 40000), (2100, 32, 8, 128, 128, 8192), (9, 5, 3, 64, 48, 900),
    (4, 2, 2, 128, 0, 10), (3, 0, 4, 64, 64, 10), (3, 9, 0, 128, 112, 10),
])
def test_matches_extended_precision(dcl, T, H, Hkv, dh, rot, far):
    row, gq, gk = operands(T, H, Hkv, dh, T)
    g = torch.Generator().manual_seed(1)
    pos = torch.randint(0, far, (T,), generator=g, dtype=torch.int32)
    pos[T // 2:T // 2 + T // 5] = -1
    pos[-1] = far - 1
    q, k, _ = run(dcl, row, pos, H, Hkv, gq, gk, 1e-6, 1e6, rot)
    check(q, row[:, :H], pos, gq, 1e-6, 1e6, rot)
    check(k, row[:, H:H + Hkv], pos, gk, 1e-6, 1e6, rot)


@pytest.mark.parametrize("base", [1.5, 10000.0, 5e5])
def test_the_farthest_positions(dcl, base):
    pos = torch.tensor([2 ** 31 - 1, 2 ** 31 - 2, 2 ** 30 + 1, 0, -1, -2 ** 31], dtype=torch.int32)
    row, gq, gk = operands(6, 4, 2, 128)
    q, k, _ = run(dcl, row, pos, 4, 2, gq, gk, 1e-5, base, 128)
    check(q, row[:, :4], pos, gq, 1e-5, base, 128)
    check(k, row[:, 4:6], pos, gk, 1e-5, base, 128)


def test_one_gain_or_none(dcl):
    row, gq, gk = operands(11, 6, 2, 64)
    pos = torch.arange(11, dtype=torch.int32) * 37
    for a, b in ((None, gk), (gq, None), (None, None)):
        q, k, _ = run(dcl, row, pos, 6, 2, a, b, 1e-6, 1e4, 64)
        check(q, row[:, :6], pos, a, 1e-6, 1e4, 64)
        check(k, row[:, 6:8], pos, b, 1e-6, 1e4, 64)
    q, k, _ = run(dcl, row, pos, 6, 2, None, None, 0.0, 1e4, 0)           # a copy
    assert torch.equal(q, row[:, :6].double()) and torch.equal(k, row[:, 6:8].double())


def test_in_place_inside_the_projection(dcl):
    """Outputs over the inputs: the same bits as beside them, values and skipped rows untouched."""
    row, gq, gk = operands(70, 8, 2, 128)
    pos = torch.arange(70, dtype=torch.int32) * 11
    pos[66:] = -1
    q, k, _ = run(dcl, row, pos, 8, 2, gq, gk, 1e-6, 1e6, 128)
    qi, ki, after = run(dcl, row, pos, 8, 2, gq, gk, 1e-6, 1e6, 128, inplace=True)
    assert torch.equal(qi[:66], q[:66]) and torch.equal(ki[:66], k[:66])
    assert torch.equal(after[:, 10:], row[:, 10:]) and torch.equal(after[66:], row[66:])


def test_rows_of_zeros_large_and_odd_values(dcl):
    row, gq, gk = operands(6, 2, 2, 64)
    row[0] = 0
    row[1] *= 1e-30
    row[2] *= 1e15
    row[3, 0, 5] = float("inf")
    row[4, 1, 40] = float("nan")
    pos = torch.arange(6, dtype=torch.int32)
    q, k, _ = run(dcl, row, pos, 2, 2, gq, gk, 1e-6, 1e4, 64)
    want, err = norm_rope(row[:, :2].double(), pos, gq, 1e-6, 1e4, 64)
    for t, h in ((0, 0), (0, 1), (1, 0), (1, 1), (2, 0), (2, 1), (3, 1), (4, 0), (5, 0), (5, 1)):
        assert bool(((q[t, h] - want[t, h]).abs() <= err[t, h]).all()), (t, h)
    assert bool((q[0] == 0).all())
    # an infinity or NaN makes its own head not a number, where and by its partner
    assert torch.isnan(q[3, 0, 5]) and torch.isnan(q[3, 0, 37]) and torch.isnan(q[4, 1]).all()
    check(k[5:], row[5:, 2:4], pos[5:], gk, 1e-6, 1e4, 64)


def test_no_rows(dcl):
    e = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    z = torch.empty(0, dtype=torch.int32, device="cuda")
    dcl.dcl_heads_norm_rope(e, e, z, 0, 4, 4, 64, None, None, 1e-6, 1e4, 64, e, e)
    torch.cuda.synchronize()


def test_replayed_graph_and_second_stream(dcl):
    row, gq, gk = operands(40, 8, 2, 128)
    row, gq, gk = row.cuda(), gq.cuda(), gk.cuda()
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    qo, ko = torch.zeros(40, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(40, 2, 128, dtype=torch.bfloat16, device="cuda")

    def call():
        dcl.dcl_heads_norm_rope(row[:, :8], row[:, 8:10], pos, 40, 8, 2, 128, gq, gk, 1e-6, 1e6, 128, qo, ko)
    call()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        call()
    for i in range(4):
        pos.copy_(torch.arange(40, dtype=torch.int32) * (i + 3))
        call()
        torch.cuda.synchronize()
        want = qo.clone(), ko.clone()
        qo.zero_(), ko.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
        qo.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            call()
        torch.cuda.synchronize()
        assert torch.equal(qo, want[0])
