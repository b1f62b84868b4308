"""The native step of the paged calls from Python is optional: without it, or with one that does not load, every serving call goes through
the interpreter's checks (host only, in a copy of the package)."""
import os
import shutil
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PACKAGE = "paper_2607_20467_amd"

CALLS = r"""
import sys, warnings
import torch
import paper_2607_20467_amd as dcl
from paper_2607_20467_amd import binding

x, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
f = torch.zeros(4, 8)
calls = {
    "device": [lambda: dcl.dcl_prompt_attention(x, x, x, i, 1, 4, 4, 2, 2, 64, 0.1, True, x),
               lambda: dcl.dcl_heads_norm_rope(x, x, i, 4, 2, 2, 64, None, None, 1e-6, 1e4, 64, x, x),
               lambda: dcl.dcl_sample_tokens(f, 4, 8, None, None, None, None, None, i, None, None, f, 128)],
    "KVPages": [lambda: dcl.dcl_pages_write(None, i, i, i, 1, 4, 4, x, x),
                lambda: dcl.dcl_pages_attention(None, i, i, i, 1, 4, 4, x, 2, 0.1, True, x, None, f, 128),
                lambda: dcl.dcl_pages_extend(None, i, i, i, 1, 4, i, i, i, None, None, f, 128)],
}
with warnings.catch_warnings(record=True) as seen:
    warnings.simplefilter("always")
    for word, some in calls.items():
        for call in some:
            try:
                call()
            except dcl.DclError as e:
                assert word in str(e), e
            else:
                raise SystemExit("not refused")
print("native" if binding._native is not None else "none", len([w for w in seen if "extension" in str(w.message)]))
"""


def run_calls(at):
    r = subprocess.run([sys.executable, "-c", CALLS], cwd=at, capture_output=True, text=True, timeout=300,
                       env={**os.environ, "PYTHONPATH": str(at)})
    assert r.returncode == 0, r.stderr
    return r.stdout.split()


@pytest.fixture
def copy(tmp_path):
    """The package without the extension."""
    from paper_2607_20467_amd import build
    if build.is_stale():
        build.build()
    at = tmp_path / PACKAGE
    at.mkdir()
    for name in os.listdir(build.HERE):
        if name.endswith(".py"):
            shutil.copy(os.path.join(build.HERE, name), at)
    os.symlink(build.LIB, at / os.path.basename(build.LIB))
    return at


def name_of_extension():
    from paper_2607_20467_amd import build
    return os.path.basename(build.operands_path())


def test_without_the_extension_the_calls_are_checked_all_the_same(copy):
    assert run_calls(copy.parent) == ["none", "1"]


def test_an_extension_that_does_not_load_is_left_out(copy):
    (copy / name_of_extension()).write_bytes(b"no library")
    assert run_calls(copy.parent) == ["none", "1"]


def test_an_extension_that_misses_a_symbol_is_left_out(copy, tmp_path):
    """As one that was built against another torch may."""
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("gcc is not installed")
    src = tmp_path / "lacking.c"
    src.write_text("extern void *not_in_this_torch(void);\nvoid *PyInit__operands(void) { return not_in_this_torch(); }\n")
    subprocess.run([cc, "-shared", "-fPIC", str(src), "-o", str(copy / name_of_extension())], check=True)
    assert run_calls(copy.parent) == ["none", "1"]


def test_the_extension_of_another_torch_is_not_looked_at(copy, monkeypatch):
    from paper_2607_20467_amd import build
    own = build.operands_path()
    monkeypatch.setattr(torch, "__version__", "0.0.1+other")
    other = build.operands_path()
    assert os.path.basename(other) != os.path.basename(own)
    shutil.copy(own, copy / os.path.basename(other))
    shutil.copy(own, copy / "_operands.so")
    assert run_calls(copy.parent) == ["none", "1"]


def test_the_extension_that_fits_is_used(copy):
    from paper_2607_20467_amd import build
    shutil.copy(build.operands_path(), copy)
    assert run_calls(copy.parent) == ["native", "0"]


STAND_IN = """#!%s
import sys
open(sys.argv[sys.argv.index("-o") + 1], "wb").write(b"built")
"""


@pytest.mark.parametrize("how", ["compiler is missing", "compiler fails"])
def test_the_library_is_built_where_the_extension_is_not(tmp_path, monkeypatch, how):
    """With a stand-in for hipcc: the library is there, a warning says what is not, and no extension of an older build stays to enter the
    new library."""
    from paper_2607_20467_amd import build
    hipcc, cxx, at = (tmp_path / n for n in ("hipcc", "cxx", "package"))
    at.mkdir()
    hipcc.write_text(STAND_IN % sys.executable)
    cxx.write_text("#!/bin/sh\nexit 1\n")
    for f in (hipcc, cxx):
        f.chmod(0o755)
    if how == "compiler is missing":
        cxx = tmp_path / "none"
    monkeypatch.setenv("CXX", str(cxx))
    for name, value in (("HIPCC", str(hipcc)), ("HERE", str(at)), ("LIB", str(at / "libdcl.so"))):
        monkeypatch.setattr(build, name, value)
    with open(build.operands_path(), "wb") as f:
        f.write(b"older")
    with pytest.warns(RuntimeWarning, match="extension"):
        assert build.build() == str(at / "libdcl.so")
    assert (at / "libdcl.so").read_bytes() == b"built"
    assert os.listdir(at) == ["libdcl.so"]


def test_a_library_that_does_not_build_is_no_library(tmp_path, monkeypatch):
    from paper_2607_20467_amd import build
    """Nor does an extension for it stay."""
    hipcc, cxx = tmp_path / "hipcc", tmp_path / "cxx"
    hipcc.write_text("#!/bin/sh\nexit 1\n")
    cxx.write_text(STAND_IN % sys.executable)
    for f in (hipcc, cxx):
        f.chmod(0o755)
    monkeypatch.setenv("CXX", str(cxx))
    for name, value in (("HIPCC", str(hipcc)), ("HERE", str(tmp_path)), ("LIB", str(tmp_path / "libdcl.so"))):
        monkeypatch.setattr(build, name, value)
    with pytest.raises(subprocess.CalledProcessError):
        build.build()
    assert sorted(os.listdir(tmp_path)) == ["cxx", "hipcc"]
