"""The paged step's calls from Python in one native step: what it takes for sound gives what the interpreter's checks give, and whatever
is wrong with a call is refused by the same error, with the native step and without it."""
import inspect

import pytest
import torch

pytestmark = pytest.mark.gpu

B, P, W, HKV, H, DH, T = 3, 16, 6, 2, 4, 64, 9
LENS, COUNTS = [20, 33, 5], [2, 4, 3]


@pytest.fixture(scope="module")
def dcl():
    import paper_2607_20467_amd as m
    m.load_library()
    return m


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def rows(heads, seed, apart=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(T, heads + apart, DH, generator=g).bfloat16().cuda()[:, :heads]


def call(dcl, op):
    """The arguments of a sound call, new ones each time."""
    n = B * W
    g = torch.Generator().manual_seed(4)

    def some(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=g, dtype=torch.uint8).cuda()
    pool = dcl.KVPages(n + 4, P, HKV, DH, dcl.DCL_DTYPE_E2M1, k=some(0, 256, n + 4, HKV, P, DH // 2),
                       v=some(0, 256, n + 4, HKV, DH // 2, P), k_scale=some(124, 127, n + 4, HKV, DH // 32, P),
                       v_scale=some(124, 127, n + 4, HKV, DH // 32, P))
    table = torch.arange(n, dtype=torch.int32, device="cuda").view(B, W)
    batch = dict(pages=pool, table=table, length=ints(*LENS), cu=ints(0, 2, 6, 9), B=B, T=T, max_new=4)
    if op in ("extend", "shrink"):
        need = dcl.dcl_pages_turn_workspace_bytes(B)
        turn = dict(pages=pool, table=table, length=ints(*LENS), B=B, free_pages=ints(*range(n, n + 4), *[0] * n), n_free=ints(4),
                    ws=torch.empty(need, dtype=torch.uint8, device="cuda"), ws_bytes=need)
        if op == "shrink":
            return dcl.dcl_pages_shrink, dict(turn, keep=ints(4, 40, 0))
        return dcl.dcl_pages_extend, dict(turn, count=ints(13, 20, 3), T=40, cu=ints(0, 0, 0, 0), pos=ints(*[7] * 40),
                                          slot=torch.full((40,), 7, device="cuda"))
    if op == "heads":
        return dcl.dcl_heads_norm_rope, dict(
            q=rows(H, 1, 3), k=rows(HKV, 2), pos=ints(*range(T)), T=T, n_heads=H, n_kv_heads=HKV, head_dim=DH,
            g_q=torch.linspace(0.5, 2, DH, device="cuda"), g_k=None, eps=1e-6, rope_base=1e4, rot_dim=32, q_out=rows(H, 3), k_out=rows(HKV, 4, 1))
    if op in ("write", "read"):
        return getattr(dcl, "dcl_pages_" + op), dict(batch, k=rows(HKV, 1, 2), v=rows(HKV, 2))
    need = dcl.dcl_pages_attention_workspace_bytes(pool, H, B, T, 4, W)
    return dcl.dcl_pages_attention, dict(batch, q=rows(H, 1, 1), n_heads=H, scale=0.125, causal=True, out=rows(H, 2).contiguous(),
                                         lse=torch.zeros(T, H, device="cuda"), ws=torch.zeros(need, dtype=torch.uint8, device="cuda"),
                                         ws_bytes=need)


OPS = ["extend", "shrink", "heads", "write", "read", "attention"]


def state(args):
    """All that a call may have written: the tensors, and the pool's."""
    out = {k: v for k, v in args.items() if torch.is_tensor(v) and k != "ws"}
    pool = args.get("pages")
    if hasattr(pool, "k_scale"):
        out.update(pool_k=pool.k, pool_v=pool.v, pool_ks=pool.k_scale, pool_vs=pool.v_scale)
    return {k: v.clone() for k, v in out.items()}


def same(a, b):
    return a.dtype == b.dtype and a.shape == b.shape and bool(torch.all((a == b) | ((a != a) & (b != b))))


def outcome(f, args):
    try:
        f(**args)
    except Exception as e:
        return type(e).__name__, str(e)
    torch.cuda.synchronize()
    return "done", ""


@pytest.mark.parametrize("op", OPS)
def test_sound_calls_are_answered_natively_and_alike(dcl, op, monkeypatch):
    from paper_2607_20467_amd import binding
    f, args = call(dcl, op)
    assert binding._device() >= 0 and binding._native is not None, "the extension is not built"
    with monkeypatch.context() as m:
        m.setattr(binding, "load_library", lambda: pytest.fail("went through the interpreter's checks"))
        assert outcome(f, args) == ("done", "")
    got, before = state(args), state(call(dcl, op)[1])
    with monkeypatch.context() as m:
        m.setattr(binding, "_native", None)
        f, args = call(dcl, op)
        assert outcome(f, args) == ("done", "")
    want = state(args)
    assert any(not torch.equal(want[k], before[k]) for k in want)
    for k in want:
        assert torch.equal(got[k], want[k]), k
    # another stream, by its handle or as it is, and the current one
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        f, args = call(dcl, op)
        torch.cuda.synchronize()
        f(**args, stream=stream)
        side.synchronize()
        again = state(args)
        assert all(torch.equal(again[k], want[k]) for k in want)


def unsound(name, x):
    """What a caller may get wrong about an argument."""
    if torch.is_tensor(x):
        yield x.cpu()
        yield x.double()
        yield x.to(torch.int64) if x.dtype != torch.int64 else x.to(torch.int32)
        yield x.flatten()[:-1] if name != "table" else x[:, :-1]
        yield x.repeat_interleave(2, -1)[..., ::2]
        yield x[None]
        yield x[:-1]
        yield x.expand(2, *x.shape)[0]
    elif isinstance(x, bool):
        yield 2
    elif isinstance(x, int):
        yield from (0, -1, x - 1, x + 1, 2 ** 31 - 1, 2 ** 31, 2 ** 80, float(x))
    elif isinstance(x, float):
        yield from (-1.0, float("nan"), float("inf"), 2, "1")
    yield None
    yield "text"
    yield object()


@pytest.mark.parametrize("op", OPS)
def test_calls_are_refused_or_taken_alike(dcl, op, monkeypatch):
    from paper_2607_20467_amd import binding
    assert binding._device() >= 0
    native, refused, taken = binding._native, 0, 0
    assert native is not None, "the extension is not built"
    for name in call(dcl, op)[1]:
        i = 0
        while True:
            seen = []
            for module in (native, None):
                monkeypatch.setattr(binding, "_native", module)
                f, args = call(dcl, op)
                wrong = list(unsound(name, args[name]))
                if i == len(wrong):
                    break
                torch.cuda.synchronize()
                args[name] = wrong[i]
                print(op, name, i, type(wrong[i]).__name__, flush=True)
                seen.append((outcome(f, args), state(args)))
            if not seen:
                break
            (a, x), (b, y) = seen
            a, b = ((k, t.split(" object at ")[0]) for k, t in (a, b))
            assert a == b, (name, i)
            assert x.keys() == y.keys() and all(same(x[k], y[k]) for k in x), (name, i)
            refused += a[0] != "done"
            taken += a[0] == "done"
            i += 1
    assert refused > 40 and taken > 0, (refused, taken)


def test_every_call_is_in_the_native_step(dcl):
    from paper_2607_20467_amd import binding
    native = binding._load_native()
    for op in OPS:
        f, args = call(dcl, op)
        assert set(inspect.signature(f).parameters) == set(args) | {"stream"}
        assert hasattr(native, f.__name__[4:])
        assert getattr(native, f.__name__[4:])(0, 0) is None          # too few arguments: not its call
