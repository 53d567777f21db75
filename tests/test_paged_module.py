"""The compiled part of the binding: loaded with its first use, refused where it was built from other sources.  On the CPU."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _python(code, **env):
    return subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT, env=dict(os.environ, **env), timeout=300)


def test_a_module_from_other_sources_is_refused(monkeypatch):
    import paper_2405_12591_amd as dq
    from paper_2405_12591_amd import paged
    assert paged._load_module().stamp == paged._build.bind_stamp()
    monkeypatch.setattr(paged._build, "bind_stamp", lambda: "0" * 32)
    with pytest.raises(dq.DQError, match="rebuild"):
        paged._load_module()
    fresh = paged._Module()
    for name in ("rotate_heads", "paged_append", "paged_read", "paged_attention"):
        with pytest.raises(dq.DQError, match="rebuild"):
            getattr(fresh, name)


def test_the_stamp_follows_the_header_and_the_source(monkeypatch, tmp_path):
    from paper_2405_12591_amd import build as B
    was = B.bind_stamp()
    assert [os.path.basename(p) for p in B.BIND_SOURCES] == ["paged_bind.cpp", "decoquant.h"]
    for i in range(2):
        changed = tmp_path / os.path.basename(B.BIND_SOURCES[i])
        changed.write_text(open(B.BIND_SOURCES[i]).read() + "\n")
        monkeypatch.setattr(B, "BIND_SOURCES", [str(changed) if j == i else p for j, p in enumerate(B.BIND_SOURCES)])
        assert B.bind_stamp() != was
        monkeypatch.undo()
    assert B.bind_stamp() == was


def test_the_package_imports_without_the_compiled_part_and_without_a_compiler():
    """Callers of the DecoQuant cache alone need neither; the first call of the others says what is missing."""
    code = """
import importlib.util, os, sys, torch
spec = importlib.util.spec_from_file_location("paper_2405_12591_amd.build", os.path.join("paper_2405_12591_amd", "build.py"))
b = importlib.util.module_from_spec(spec)
sys.modules["paper_2405_12591_amd.build"] = b
spec.loader.exec_module(b)
b.BIND_PATH = os.path.join(os.sep, "nowhere", "_paged.so")
import paper_2405_12591_amd as dq
assert dq.version() == dq.ABI_VERSION and dq.KVCacheLayer and dq.PagedKVLayer
assert "paper_2405_12591_amd._paged" not in sys.modules
x = torch.zeros((1, 1, 64), dtype=torch.float16)
try:
    dq.paged._module.rotate_heads(x, x, None, None, None, None, None, None, 0.0, 0, 0)
except RuntimeError as e:
    print("refused:", str(e).splitlines()[0])
"""
    r = _python(code, CXX="/bin/false")
    assert r.returncode == 0 and "refused: the binding's compiled part does not build" in r.stdout, r.stdout + r.stderr


def test_a_library_that_lacks_functions_is_refused_by_name(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler here")
    src, lib = tmp_path / "old.c", tmp_path / "libold.so"
    src.write_text("int dq_version(void) { return 6; }\n")
    subprocess.run([gcc, "-shared", "-fPIC", str(src), "-o", str(lib)], check=True)
    r = _python("import paper_2405_12591_amd", DQ_LIBRARY_PATH=str(lib))
    assert r.returncode != 0 and "DQError" in r.stderr and "dq_paged_append" in r.stderr and "rebuild it" in r.stderr, r.stderr
