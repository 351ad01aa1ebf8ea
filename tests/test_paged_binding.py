"""The binding of the paged calls: the structs they are given, and the compiled checks behind them."""
import ctypes
import importlib.machinery
import os
import subprocess
import sys

import pytest
import torch

from paper_2507_08143_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

def _cache():
    k = torch.zeros(4, 16, 128, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    return B.PagedCache(k, k.clone(), i32(1, 2, 3, 2), mass=torch.zeros(4, 16), positions=i32(4, 16))


def test_calls_refuse_other_structs():
    """Every struct goes to the library by address: one of another kind would be read as what it is not."""
    c, shape, i32 = _cache(), B.Shape(1, 2, 128, 48, [4, 0, 3]), lambda *s: torch.zeros(*s, dtype=torch.int32)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    q, n = bf(3, 4, 128), i32(1, 2, 3)
    for cache, opt in ((c, B.options()), (c, c), (c, c.c), (c, None), (shape, B.decode_options(2, 20)), (c.c, B.decode_options(2, 20)),
                       (None, B.decode_options(2, 20))):
        with pytest.raises(TypeError):
            B.paged_attention(cache, 0, opt, q, n, bf(3, 4, 128), bf(100))
    kv = bf(1, 2, 7, 128)
    for cache, s in ((c, c), (c, shape.c), (c, B.options()), (shape, shape), (None, shape)):
        with pytest.raises(TypeError):
            B.paged_fill(cache, s, kv, kv, [2, 0, 3])
    for cache in (shape, c.c, None):
        with pytest.raises(TypeError):
            B.paged_evict(cache, n, n, n, 32)
    for cache, opt in ((c, B.options()), (shape, B.decode_options(2, 20)), (c, c)):
        with pytest.raises((TypeError, ctypes.ArgumentError)):
            B.paged_attention_workspace_bytes(cache, opt)


def _python(code, **env):
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, env={**os.environ, **env}, capture_output=True, text=True, timeout=300)


def test_other_entry_points_need_no_compiled_checks(tmp_path):
    """Built for another torch the checks are not loaded; where they cannot be built anew, the entry points that go through ctypes
    still work, and the paged calls say what is missing."""
    run = _python("""
import torch
torch.__version__ = "0.0.1+another"
from paper_2507_08143_b200 import binding as B
assert B.keep_count(10, 0.25) == 3 and B.make_sketch(1, 128, 48).shape == (128, 48)
k = torch.zeros(4, 16, 128, dtype=torch.bfloat16)
n = torch.zeros(1, 2, 3, dtype=torch.int32)
c = B.PagedCache(k, k.clone(), torch.zeros(1, 2, 3, 2, dtype=torch.int32), mass=torch.zeros(4, 16))
assert B.paged_attention_workspace_bytes(c, B.decode_options(2, 20)) > 0
try:
    B.paged_evict(c, n, n, n, 32)
except RuntimeError as e:
    assert "compiled argument checks" in str(e) and e.__cause__ is not None, e
    print("refused")
""", CXX=str(tmp_path / "no-such-compiler"))
    assert run.returncode == 0 and run.stdout.split() == ["refused"], run.stdout + run.stderr


def test_compiled_checks_are_named_for_what_they_were_built_against(monkeypatch):
    from paper_2507_08143_b200 import build
    here = build.fastcall_path()
    assert here.endswith(importlib.machinery.EXTENSION_SUFFIXES[0]) and torch.__version__.split("+")[0].replace(".", "_") in here
    assert B._fastcall.__file__ == here and os.path.exists(here)
    monkeypatch.setattr(torch, "__version__", torch.__version__ + ".post1")
    assert build.fastcall_path() != here


def test_a_build_that_fails_leaves_what_was_there(tmp_path):
    """The compiler writes beside the file that others may be loading; a failed run neither replaces nor removes it."""
    from paper_2507_08143_b200 import build
    out = tmp_path / "x.so"
    out.write_text("old")
    with pytest.raises(subprocess.CalledProcessError):
        build._compile([sys.executable, "-c", "import sys; open(sys.argv[2], 'w').write('half'); sys.exit(1)"], str(out))
    assert out.read_text() == "old" and os.listdir(tmp_path) == ["x.so"]
    build._compile([sys.executable, "-c", "import sys; open(sys.argv[2], 'w').write('new')"], str(out))
    assert out.read_text() == "new" and os.listdir(tmp_path) == ["x.so"]
