"""Refusals of the paged step's operators (host only: nothing is launched)."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from test_serving_host import ATTN, COPY, ROOT, call, pool


@pytest.fixture(scope="module")
def dcl():
    from paper_2607_20467_amd import build
    if build.is_stale():
        build.build()
    import paper_2607_20467_amd as m
    m.load_library()
    return m


def pool4(dcl, **kw):
    return pool(dcl, **{**dict(dtype=3, k_scale=256, v_scale=256), **kw})


@pytest.mark.parametrize("name,tail", [("dcl_pages_write", COPY), ("dcl_pages_read", COPY), ("dcl_pages_attention", ATTN)])
@pytest.mark.parametrize("pages,status,word", [
    (dict(dtype=4), 2, "dtype"), (dict(dtype=-1), 2, "dtype"), (dict(head_dim=96), 2, "head_dim"), (dict(k_scale=0), 1, "k_scale"),
    (dict(v_scale=0), 1, "v_scale"), (dict(v_scale=264), 1, "aligned"), (dict(k=8), 1, "aligned"), (dict(page_len=8), 1, "page_len"),
])
def test_pages_of_four_bits_are_checked_as_the_others(dcl, name, tail, pages, status, word):
    r, msg = call(dcl, name, pool4(dcl, **pages), tail)
    assert r == status and word in msg, (r, msg)


def test_an_attention_without_rows_launches_nothing(dcl):
    """A launch would fail where there is no device."""
    for kw in (dict(T=0, max_new=0), dict(T=0), dict(max_new=0)):
        r, msg = call(dcl, "dcl_pages_attention", pool4(dcl), ATTN, **kw)
        assert r == 0, (kw, r, msg)


def test_attention_workspace_of_four_bits(dcl):
    f = dcl.load_library().dcl_pages_attention_workspace_bytes
    g = ctypes.byref(pool4(dcl))
    assert f(g, 4, 1, 4, 4, 2) >= 256 and f(g, 3, 1, 4, 4, 2) == 0
    one, many = f(g, 4, 1, 1, 1, 1 << 14), f(g, 4, 1, 2, 2, 1 << 14)
    assert 256 < one < many
    r, msg = call(dcl, "dcl_pages_attention", pool4(dcl), ATTN[:8] + (16, None), max_pages=1 << 14)
    assert r == 3 and "workspace" in msg


@pytest.mark.parametrize("B,T,max_new,heads,hkv,tight,wide", [(8, 512, 64, 32, 32, 20, 2048), (128, 128, 1, 32, 8, 10, 2048)])
def test_a_wide_table_asks_for_the_workspace_of_parts(dcl, B, T, max_new, heads, hkv, tight, wide):
    """As the header has it: the lengths are the device's, so that parts and workspace follow from what the table could name."""
    def need(width):
        n = dcl.load_library().dcl_pages_attention_workspace_bytes(
            ctypes.byref(pool4(dcl, head_dim=128, n_kv_heads=hkv, page_len=64)), heads, B, T, max_new, width)
        return n // (T * heads * (128 * 4 + 8))           # outputs, and a reference and a sum, of each part
    assert need(tight) == 0 and need(wide) >= 2


EXTEND = dict(table=256, max_pages=2, len=256, count=256, B=1, T=4, free=256, n_free=256, cu=256, pos=256, slot=256, ws=256,
              ws_bytes=1 << 20, stream=None)
SHRINK = dict(table=256, max_pages=2, len=256, keep=256, B=1, free=256, n_free=256, ws=256, ws_bytes=1 << 20, stream=None)
BOTH = [
    (None, {}, 1, "pages"), (dict(dtype=0), {}, 2, "dtype"), (dict(page_len=24), {}, 1, "page_len"), (dict(n_pages=0), {}, 1, "n_pages"),
    (dict(n_pages=(1 << 30) + 1), {}, 2, "n_pages"), ({}, dict(table=0), 1, "table"), ({}, dict(len=0), 1, "len"),
    ({}, dict(free=0), 1, "free_pages"), ({}, dict(n_free=0), 1, "n_free"), ({}, dict(B=0), 1, "B=0"), ({}, dict(B=70000), 1, "B="),
    ({}, dict(max_pages=0), 1, "max_pages"), ({}, dict(max_pages=1 << 25), 1, "max_pages"),
    ({}, dict(B=1 << 16, max_pages=1 << 15), 2, "2^31"), ({}, dict(ws=0), 1, "workspace"), ({}, dict(ws=128), 1, "aligned"),
    ({}, dict(ws_bytes=255), 3, "workspace"),
]


@pytest.mark.parametrize("pages,kw,status,word", BOTH + [({}, dict(T=-1), 1, "T="), ({}, dict(T=1 << 23), 1, "T="), ({}, dict(cu=0), 1, "cu")])
def test_extend_refusals(dcl, pages, kw, status, word):
    g = None if pages is None else ctypes.byref(pool(dcl, **pages))
    r = dcl.load_library().dcl_pages_extend(g, *{**EXTEND, **kw}.values())
    assert r == status and word in dcl.dcl_last_error(), (r, dcl.dcl_last_error())


@pytest.mark.parametrize("pages,kw,status,word", BOTH + [({}, dict(keep=0), 1, "keep")])
def test_shrink_refusals(dcl, pages, kw, status, word):
    g = None if pages is None else ctypes.byref(pool(dcl, **pages))
    r = dcl.load_library().dcl_pages_shrink(g, *{**SHRINK, **kw}.values())
    assert r == status and word in dcl.dcl_last_error(), (r, dcl.dcl_last_error())


def test_turn_workspace_sizes(dcl):
    f = dcl.dcl_pages_turn_workspace_bytes
    assert f(0) == f(-1) == f((1 << 16) + 1) == 0
    assert f(1) % 256 == 0 and 256 <= f(1) < f(1 << 16) and f(1 << 16) >= 8 << 16


HEADS = dict(q=256, q_stride=128, k=256, k_stride=128, pos=256, T=4, n_heads=2, n_kv_heads=2, head_dim=64, g_q=256, g_k=256, eps=1e-6,
             base=1e4, rot=64, q_out=256, q_out_stride=128, k_out=256, k_out_stride=128, stream=None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(q=0), 1, "q is NULL"), (dict(k=0), 1, "k is NULL"), (dict(q_out=0), 1, "q_out"), (dict(k_out=264), 1, "aligned"),
    (dict(q_stride=120), 1, "stride"), (dict(k_stride=132), 1, "stride"), (dict(q_out_stride=64), 1, "stride"),
    (dict(k_out_stride=0), 1, "stride"), (dict(pos=0), 1, "pos"), (dict(T=-1), 1, "T="), (dict(T=1 << 23), 1, "T="),
    (dict(n_heads=-1), 1, "n_heads"), (dict(n_heads=0, n_kv_heads=0), 1, "n_heads"), (dict(n_kv_heads=1 << 17), 1, "n_kv_heads"),
    (dict(head_dim=96), 2, "head_dim"), (dict(g_q=8), 1, "g_q"), (dict(g_k=4), 1, "g_k"), (dict(eps=-1e-6), 1, "eps"),
    (dict(eps=float("nan")), 1, "eps"), (dict(eps=float("inf")), 1, "eps"), (dict(base=1.0), 1, "rope_base"),
    (dict(base=float("nan")), 1, "rope_base"), (dict(base=float("inf")), 1, "rope_base"), (dict(rot=-16), 1, "rot_dim"),
    (dict(rot=80), 1, "rot_dim"), (dict(rot=24), 1, "rot_dim"), (dict(q_out_stride=256), 1, "over its input"),
    (dict(k_stride=192), 1, "over its input"),
])
def test_heads_refusals(dcl, kw, status, word):
    r = dcl.load_library().dcl_heads_norm_rope(*{**HEADS, **kw}.values())
    assert r == status and word in dcl.dcl_last_error(), (r, dcl.dcl_last_error())


def test_heads_without_rows_return_at_once(dcl):
    assert dcl.load_library().dcl_heads_norm_rope(*{**HEADS, **dict(T=0, q=0, pos=0)}.values()) == 0


PROBE = r"""
#include <cstdio>
#include "pages_index.h"
using namespace dcl;
int main() {
  unsigned s = 1;
  auto rnd = [&]() { s = s * 1664525u + 1013904223u; return (int)s; };
  const int odd[] = {0, 1, -1, 2147483647, -2147483647 - 1, 64, 63, 1 << 30, -(1 << 30)};
  auto any = [&]() { int r = rnd(); return (r & 3) ? odd[(unsigned)r % 9] : r >> ((unsigned)r % 31); };
  for (long i = 0; i < 2000000; ++i) {
    int table[4] = {any(), any(), any(), any()};
    const int n_pages = 1 + (unsigned)any() % 1000, shift = 4 + (unsigned)rnd() % 7, width = 1 + (unsigned)rnd() % 4, c = any();
    const int at = page_entry(width, shift, c);
    if (at < 0 || at >= width) return 1;
    if (page_found(table[at], width, n_pages, shift, c) != page_of(table, width, n_pages, shift, c)) return 2;
  }
  std::puts("ok");
  return 0;
}
"""


def test_a_page_looked_up_in_two_steps_is_the_same(tmp_path):
    """Compiled for the host with bounds checking: the entry is always inside the row, the page what page_of gives."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ is not installed")
    src, exe = tmp_path / "probe.cpp", tmp_path / "probe"
    src.write_text(PROBE)
    subprocess.run([cxx, "-O1", "-g", "-std=c++17", "-fsanitize=undefined,bounds", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2607_20467_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "ok" in r.stdout, (r.returncode, r.stdout, r.stderr)


def test_the_binding_checks_pools_and_operands(dcl):
    k = torch.zeros(4, 2, 16, 32, dtype=torch.uint8)
    with pytest.raises(dcl.DclError, match="device"):
        dcl.KVPages(4, 16, 2, 64, dcl.DCL_DTYPE_E2M1, k=k)
    with pytest.raises(dcl.DclError, match="shape"):
        dcl.KVPages(4, 16, 2, 128, dcl.DCL_DTYPE_E2M1, k=k)
    with pytest.raises(dcl.DclError, match="head_dim"):
        dcl.KVPages(4, 16, 2, 80, dcl.DCL_DTYPE_E2M1)
    with pytest.raises(dcl.DclError, match="KVPages"):
        dcl.dcl_pages_extend(None, k, k, k, 1, 4, k, k, k, None, None, k, 256)
    with pytest.raises(dcl.DclError, match="KVPages"):
        dcl.dcl_pages_shrink(None, k, k, k, 1, k, k, k, 256)
    x, pos = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(dcl.DclError, match="device"):
        dcl.dcl_heads_norm_rope(x, x, pos, 4, 2, 2, 64, None, None, 1e-6, 1e4, 64, x, x)


def test_dtype_constants_match_the_header(dcl):
    header = open(os.path.join(ROOT, "include", "dcl.h")).read()
    for name, value in re.findall(r"(DCL_DTYPE_\w+) = (\d)", header):
        assert getattr(dcl, name) == int(value), name
