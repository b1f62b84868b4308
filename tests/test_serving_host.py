"""The serving operators' refusals (host only: nothing is launched), and their index functions on hostile data."""
import ctypes
import os
import shutil
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def dcl():
    from paper_2607_20467_amd import build
    if build.is_stale():
        build.build()
    import paper_2607_20467_amd as m
    m.load_library()
    return m


def pool(dcl, **kw):
    f = dict(k=256, v=256, k_scale=0, v_scale=0, n_pages=4, page_len=16, n_kv_heads=2, head_dim=64, dtype=1)
    f.update(kw)
    return dcl.DclPages(*(f[n] for n, _ in dcl.DclPages._fields_))


BATCH = dict(table=256, max_pages=2, len=256, cu=256, B=1, T=4, max_new=4)


def call(dcl, name, pages, tail, **kw):
    b = dict(BATCH)
    b.update(kw)
    r = getattr(dcl.load_library(), name)(ctypes.byref(pages) if pages is not None else None,
                                          *(b[n] for n in BATCH), *tail)
    return r, dcl.dcl_last_error()


COPY = (256, 128, 256, 128, None)
ATTN = (256, 256, 4, 0.125, 1, 256, 256, 256, 1 << 40, None)


@pytest.mark.parametrize("name,tail", [("dcl_pages_write", COPY), ("dcl_pages_read", COPY), ("dcl_pages_attention", ATTN)])
@pytest.mark.parametrize("pages,batch,status,word", [
    (None, {}, 1, "pages"),
    (dict(dtype=0), {}, 2, "dtype"),
    (dict(head_dim=96), {}, 2, "head_dim"),
    (dict(n_kv_heads=0), {}, 1, "n_kv_heads"),
    (dict(page_len=24), {}, 1, "page_len"),
    (dict(page_len=8), {}, 1, "page_len"),
    (dict(page_len=2048), {}, 1, "page_len"),
    (dict(n_pages=0), {}, 1, "n_pages"),
    (dict(k=0), {}, 1, "k / v"),
    (dict(v=264), {}, 1, "aligned"),
    (dict(dtype=2), {}, 1, "k_scale"),
    (dict(dtype=2, k_scale=256, v_scale=257), {}, 1, "aligned"),
    ({}, dict(table=0), 1, "table"),
    ({}, dict(len=0), 1, "len"),
    ({}, dict(cu=0), 1, "cu"),
    ({}, dict(B=0), 1, "B=0"),
    ({}, dict(B=70000), 1, "B="),
    ({}, dict(T=-1), 1, "T="),
    ({}, dict(T=1 << 23), 1, "T="),
    ({}, dict(max_new=-1), 1, "max_new"),
    ({}, dict(max_pages=0), 1, "max_pages"),
    ({}, dict(max_pages=1 << 25), 1, "max_pages"),
])
def test_pages_refusals(dcl, name, tail, pages, batch, status, word):
    r, msg = call(dcl, name, None if pages is None else pool(dcl, **pages), tail, **batch)
    assert r == status and word in msg, (r, msg)


@pytest.mark.parametrize("tail,status,word", [
    ((0, 128, 256, 128, None), 1, "k is NULL"),
    ((256, 120, 256, 128, None), 1, "stride"),
    ((256, 132, 256, 128, None), 1, "stride"),
    ((256, 128, 264, 128, None), 1, "aligned"),
])
def test_pages_copy_refusals(dcl, tail, status, word):
    for name in ("dcl_pages_write", "dcl_pages_read"):
        r, msg = call(dcl, name, pool(dcl), tail)
        assert r == status and word in msg, (r, msg)


@pytest.mark.parametrize("change,status,word", [
    ({0: 0}, 1, "q is NULL"), ({1: 128}, 1, "stride"), ({2: 3}, 2, "n_heads"), ({2: 0}, 2, "n_heads"),
    ({3: float("nan")}, 1, "scale"), ({3: float("inf")}, 1, "scale"), ({4: 2}, 1, "causal"), ({5: 0}, 1, "out"),
    ({5: 8}, 1, "aligned"), ({7: 0}, 1, "workspace"), ({7: 64}, 1, "aligned"), ({8: 16}, 3, "workspace"),
])
def test_pages_attention_refusals(dcl, change, status, word):
    tail = [change.get(i, x) for i, x in enumerate(ATTN)]
    r, msg = call(dcl, "dcl_pages_attention", pool(dcl), tail)
    assert r == status and word in msg, (r, msg)


def test_pages_calls_of_too_many_workgroups(dcl):
    g = pool(dcl, n_kv_heads=1024)
    copy, attn = (256, 1 << 16, 256, 1 << 16, None), (256, 1 << 16, 1024, 0.125, 1, 256, 0, 256, 1 << 60, None)
    for name, tail, kw in (("dcl_pages_write", copy, dict(B=8192, max_new=0)), ("dcl_pages_read", copy, dict(max_new=1 << 22)),
                           ("dcl_pages_attention", attn, dict(B=1 << 14)),
                           ("dcl_pages_attention", attn, dict(max_new=1 << 20, T=1 << 20))):
        r, msg = call(dcl, name, g, tail, **kw)
        assert r == 2 and "too many" in msg, (name, kw, r, msg)
    assert dcl.load_library().dcl_pages_attention_workspace_bytes(ctypes.byref(g), 1024, 1 << 14, 4, 4, 2) == 0


def test_pages_workspace_sizes(dcl):
    f = dcl.load_library().dcl_pages_attention_workspace_bytes
    g = pool(dcl)
    assert f(ctypes.byref(g), 4, 1, 4, 4, 2) >= 256
    assert f(ctypes.byref(g), 4, 1, 0, 0, 2) >= 256               # nothing to do is no error
    for bad in ((3, 1, 4, 4, 2), (4, 0, 4, 4, 2), (4, 1, -1, 4, 2), (4, 1, 4, -1, 2), (4, 1, 4, 4, 0)):
        assert f(ctypes.byref(g), *bad) == 0
    assert f(None, 4, 1, 4, 4, 2) == 0
    # one token of a long sequence is split; the parts of many tokens need more
    one, many = f(ctypes.byref(g), 4, 1, 1, 1, 1 << 14), f(ctypes.byref(g), 4, 1, 2, 2, 1 << 14)
    assert 256 < one < many


def test_pools_and_operands_are_checked_by_the_binding(dcl):
    cpu = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(dcl.DclError, match="device"):
        dcl.KVPages(4, 16, 2, 64, k=cpu)
    with pytest.raises(dcl.DclError, match="shape"):
        dcl.KVPages(5, 16, 2, 64, k=cpu)
    with pytest.raises(dcl.DclError, match="positive"):
        dcl.KVPages(0, 16, 2, 64)
    with pytest.raises(dcl.DclError, match="dtype"):
        dcl.KVPages(4, 16, 2, 64, dtype=0)
    with pytest.raises(dcl.DclError, match="KVPages"):
        dcl.dcl_pages_write(None, cpu, cpu, cpu, 1, 4, 4, cpu, cpu)


PROBE = r"""
#include <cstdio>
#include <cstdlib>
#include "pages_index.h"
using namespace dcl;
int main() {
  unsigned s = 1;
  auto rnd = [&]() { s = s * 1664525u + 1013904223u; return (int)s; };
  const int odd[] = {0, 1, -1, 2147483647, -2147483647 - 1, 64, 63, 1 << 30, -(1 << 30)};
  auto any = [&]() { int r = rnd(); return (r & 3) ? odd[(unsigned)r % 9] : r >> ((unsigned)r % 31); };
  for (long i = 0; i < 2000000; ++i) {
    int cu[3] = {any(), any(), any()}, len[1] = {any()};
    const int T = (unsigned)any() % 4194305u;
    for (int b = 0; b < 2; ++b) {
      const SeqRows r = seq_rows(cu, b, T);
      if (r.first < 0 || r.n < 0 || r.first > T || r.n > T - r.first) return std::printf("rows %d %d of %d\n", r.first, r.n, T), 1;
      if (cu[b] >= 0 && cu[b] <= cu[b + 1] && cu[b + 1] <= T && (r.first != cu[b] || r.n != cu[b + 1] - cu[b])) return 2;
    }
    const int L = seq_len(len, 0);
    if (L < 0 || L > 1 << 30) return 3;
    int table[4] = {any(), any(), any(), any()};
    const int n_pages = 1 + (unsigned)any() % 1000, shift = 4 + (unsigned)rnd() % 7, width = 1 + (unsigned)rnd() % 4, c = any();
    const int p = page_of(table, width, n_pages, shift, c);
    if (p < -1 || p >= n_pages) return 4;
    if (p >= 0 && (c < 0 || (c >> (shift - 4)) >= width || table[c >> (shift - 4)] != p)) return 5;
  }
  std::puts("ok");
  return 0;
}
"""


def test_index_functions_stay_inside_for_any_device_data(tmp_path):
    """What the kernels make of borders, lengths and page numbers, compiled for the host with bounds checking."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ is not installed")
    src = tmp_path / "probe.cpp"
    src.write_text(PROBE)
    exe = tmp_path / "probe"
    subprocess.run([cxx, "-O1", "-g", "-std=c++17", "-fsanitize=undefined,bounds", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2607_20467_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "ok" in r.stdout, (r.returncode, r.stdout, r.stderr)


PROMPT = (256, 256, 256, 128, 256, 128, 256, 1, 4, 4, 4, 2, 64, 0.125, 1, 256, 0, None)


@pytest.mark.parametrize("change,status,word", [
    ({0: 0}, 1, "q is NULL"), ({1: 255}, 1, "stride"), ({1: 248}, 1, "stride"), ({2: 0}, 1, "k is NULL"), ({3: 64}, 1, "stride"),
    ({4: 8}, 1, "aligned"), ({5: 120}, 1, "stride"), ({6: 0}, 1, "cu"), ({7: 0}, 1, "B=0"), ({8: -1}, 1, "T="),
    ({9: -1}, 1, "max_len"), ({10: 3}, 2, "n_heads"), ({11: 0}, 2, "n_heads"), ({12: 80}, 2, "head_dim"),
    ({13: float("inf")}, 1, "scale"), ({14: 5}, 1, "causal"), ({15: 0}, 1, "out"),
    ({7: 60000, 9: 1 << 22, 8: 1 << 22}, 2, "too many"), ({7: 1 << 16, 8: 1 << 22, 9: 128 * 63}, 2, "too many"),
])
def test_prompt_refusals(dcl, change, status, word):
    r = dcl.load_library().dcl_prompt_attention(*[change.get(i, x) for i, x in enumerate(PROMPT)])
    assert r == status and word in dcl.dcl_last_error(), (r, dcl.dcl_last_error())


def sample_call(dcl, how=None, **kw):
    f = dict(logits=256, dtype=0, stride=1000, n=2, vocab=1000, token=256, conf=0, kept=0, ws=256, ws_bytes=1 << 40, stream=None)
    f.update(kw)
    s = dcl.DclSampling(0, 0, 0, 0, 256) if how is None else how
    r = dcl.load_library().dcl_sample_tokens(f["logits"], f["dtype"], f["stride"], f["n"], f["vocab"],
                                             ctypes.byref(s) if how != 0 else None, f["token"], f["conf"], f["kept"], f["ws"],
                                             f["ws_bytes"], f["stream"])
    return r, dcl.dcl_last_error()


@pytest.mark.parametrize("kw,status,word", [
    (dict(logits=0), 1, "logits is NULL"), (dict(dtype=2), 2, "dtype"), (dict(stride=999), 1, "stride"), (dict(n=-1), 1, "n=-1"),
    (dict(n=1 << 23), 1, "n="), (dict(vocab=0), 1, "vocab"), (dict(vocab=(1 << 20) + 1, stride=1 << 21), 1, "vocab"),
    (dict(token=0), 1, "token"), (dict(ws=0), 1, "workspace"), (dict(ws=128), 1, "aligned"), (dict(ws_bytes=0), 3, "workspace"),
    (dict(how=0), 1, "how"), (dict(logits=258), 1, "aligned"), (dict(logits=257, dtype=1), 1, "aligned"),
])
def test_sample_refusals(dcl, kw, status, word):
    r, msg = sample_call(dcl, **kw)
    assert r == status and word in msg, (r, msg)


def test_sample_needs_random_numbers_and_sizes(dcl):
    r, msg = sample_call(dcl, how=dcl.DclSampling(256, 256, 256, 256, 0))
    assert r == 1 and "uniform" in msg
    f = dcl.load_library().dcl_sample_workspace_bytes
    assert all(f(n, v) <= f(m, w) for n, m in ((1, 2), (4, 128), (128, 129), (128, 512), (512, 1 << 22))
               for v, w in ((1, 8191), (19999, 20000), (50000, 1 << 20), (1 << 20, 1 << 20)))
    assert f(1, 1) > 0 and f(0, 10) > 0 and f(-1, 10) == 0 and f(1, 0) == 0 and f(1, (1 << 20) + 1) == 0


def test_sample_hidden_refusals(dcl):
    import synth
    lib = dcl.load_library()
    m = dcl.dcl_model_create(dcl.config_from_geometry(synth.TINY, max_positions=64))
    s = dcl.DclSampling(0, 0, 0, 0, 256)
    try:
        assert lib.dcl_sample_hidden(None, 256, 1, ctypes.byref(s), 256, 0, 0, 256, 1 << 40, None) == 1
        assert lib.dcl_sample_hidden(m, 256, 1, ctypes.byref(s), 256, 0, 0, 256, 1 << 40, None) == 5
        assert lib.dcl_sample_hidden(m, 256, -1, ctypes.byref(s), 256, 0, 0, 256, 1 << 40, None) == 1
        assert lib.dcl_sample_hidden(m, 256, 1 << 20, ctypes.byref(s), 256, 0, 0, 256, 1 << 40, None) == 2
        assert lib.dcl_sample_hidden(m, 256, 1, None, 256, 0, 0, 256, 1 << 40, None) == 1
        assert dcl.dcl_sample_hidden_workspace_bytes(m, 3) >= 3 * synth.TINY.vocab * 4
        assert dcl.dcl_sample_hidden_workspace_bytes(m, 1 << 20) == 0 and dcl.dcl_sample_hidden_workspace_bytes(m, -1) == 0
    finally:
        dcl.dcl_model_destroy(m)


@pytest.mark.parametrize("given,place", [("side", "side"), (0x50, ("external", 0x50)), (0, "default")])
def test_a_runner_allocates_where_its_call_runs(dcl, monkeypatch, given, place):
    """Buffers of a call on another stream than the current one come from that stream's memory: the allocator hands them out
    again as soon as the call returns. A torch that writes down the stream under which it allocates stands for the device."""
    import contextlib
    import types
    now, made = ["current"], []

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    def empty(shape, dtype=None, device=None):
        made.append(now[-1])
        return torch.empty(shape, dtype=dtype)
    m, called = dcl.binding, []
    fake = types.SimpleNamespace(empty=empty, uint8=torch.uint8, int16=torch.int16, int32=torch.int32, float32=torch.float32,
                                 cuda=types.SimpleNamespace(stream=on, ExternalStream=lambda h: ("external", h),
                                                            default_stream=lambda: "default"))
    run = object.__new__(m.Runner)
    run.torch, run.model, run.ws, run.geom = fake, None, None, types.SimpleNamespace(vocab=8, d_model=4)
    for name in ("dcl_sample_hidden", "dcl_score_hidden", "dcl_debug_logits", "dcl_denoise_step", "dcl_kv_append"):
        monkeypatch.setattr(m, name, lambda *a, name=name: called.append((name, a[-1], len(now))))
    for name in ("dcl_sample_hidden_workspace_bytes", "dcl_score_workspace_bytes", "dcl_workspace_bytes"):
        monkeypatch.setattr(m, name, lambda *a: 64)
    rows, tokens = torch.zeros(3, 4, dtype=torch.int16), torch.zeros(1, 4, dtype=torch.int32)
    for stream, where in ((None, "current"), (given, place)):
        for go in (lambda: run.sample_hidden(rows, None, stream=stream), lambda: run.score_hidden(rows, stream=stream),
                   lambda: run.logits(tokens, tokens, stream=stream, with_hidden=True),
                   lambda: run.step(tokens, None, 4, stream=stream),
                   lambda: run.kv_append(tokens, ([], [], 0), stream=stream)):
            made.clear()
            run.ws = None
            go()
            assert made and set(made) == {where}, (called[-1], made)
            assert called[-1][1] is stream and now == ["current"]


def test_attention_calls_without_rows_need_no_workspace(dcl):
    """No tokens, or none that a call may take: accepted whatever the table and the batch, with the least workspace."""
    lib = dcl.load_library()
    for dtype, kw in ((1, {}), (2, dict(k_scale=256, v_scale=256))):
        for hkv, heads, B, max_pages in ((2, 4, 1, 2), (4, 32, 64, 1 << 14), (1024, 1024, 1 << 16, 1 << 22)):
            g = pool(dcl, dtype=dtype, n_kv_heads=hkv, head_dim=64, page_len=64, **kw)
            for T, max_new in ((0, 0), (0, 1), (0, 1 << 22), (64, 0), (1 << 22, 0)):
                assert lib.dcl_pages_attention_workspace_bytes(ctypes.byref(g), heads, B, T, max_new, max_pages) == 256
                r, msg = call(dcl, "dcl_pages_attention", g,
                              (256, heads * 64, heads, 0.125, 1, 256, 0, 256, 256, None), B=B, T=T, max_new=max_new,
                              max_pages=max_pages)
                assert r == 0, (dtype, hkv, T, max_new, msg)


@pytest.mark.parametrize("hkv,heads,B,max_new,max_pages", [
    (1024, 1024, 1 << 16, 1 << 16, 1 << 22),                       # units x capacity is 2^64
    (1024, 1024, 1 << 16, 1 << 22, 1 << 22), (1, 1 << 16, 1 << 16, 1 << 22, 1 << 22), (1, 1 << 16, 1, 1 << 22, 1),
    (1024, 1 << 16, 1 << 16, 1 << 22, 1), (512, 512, 1 << 16, 1 << 17, 1 << 22),
])
def test_the_largest_sizes_are_refused_not_computed_with(dcl, hkv, heads, B, max_new, max_pages):
    """Run apart: a division by a product that wrapped to 0 ends the process."""
    code = f"""
import ctypes, sys
sys.path.insert(0, {ROOT!r})
import paper_2607_20467_amd as dcl
lib = dcl.load_library()
g = dcl.DclPages(256, 256, 0, 0, 4, 64, {hkv}, 64, 1)
assert lib.dcl_pages_attention_workspace_bytes(ctypes.byref(g), {heads}, {B}, 1 << 22, {max_new}, {max_pages}) == 0
r = lib.dcl_pages_attention(ctypes.byref(g), 256, {max_pages}, 256, 256, {B}, 1 << 22, {max_new}, 256, {heads} * 64, {heads}, 0.125,
                            1, 256, 0, 256, (1 << 63) - 1, None)
assert r == 2 and "too many" in dcl.dcl_last_error(), r
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])


def test_missing_operands_are_refused_as_every_other_argument(dcl):
    """None goes to the library, which names what is missing; logits, whose type decides the call, have to be a tensor."""
    ws = dict(ws=256, ws_bytes=1 << 40)
    with pytest.raises(dcl.DclError, match="q is NULL"):
        dcl.dcl_prompt_attention(None, 256, 256, 256, 1, 4, 4, 4, 2, 64, 0.125, True, 256, stream=0)
    with pytest.raises(dcl.DclError, match="v is NULL"):
        dcl.dcl_prompt_attention(256, 256, None, 256, 1, 4, 4, 4, 2, 64, 0.125, True, 256, stream=0)
    with pytest.raises(dcl.DclError, match="out is NULL"):
        dcl.dcl_prompt_attention(256, 256, 256, 256, 1, 4, 4, 4, 2, 64, 0.125, True, None, stream=0)
    for logits in (None, 256, torch.zeros(2, 10)):
        with pytest.raises(dcl.DclError, match="logits"):
            dcl.dcl_sample_tokens(logits, 2, 10, None, None, None, None, 256, 256, None, None, **ws, stream=0)
