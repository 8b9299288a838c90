"""What of the binding needs what, on the host, each in a process of its own: the library does not need the compiled checks of tensor arguments."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _python(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout.split()


def test_compression_without_the_checks_of_cache_arguments():
    """Entry points that take no argument through them work where their module does not load; those that do say what is missing."""
    out = _python("""
import sys
sys.modules["paper_2605_23200_amd._args"] = None
from paper_2605_23200_amd import binding as B
p = B.make_params(n_layers=2, batch=1, n_kv_heads=2, group=2, window=8, t_max=1000, budget=100, n_segments=4)
assert B.lib().ams_status_string(0) and B.ams_workspace_bytes(p) > 0 and B.ams_attend_workspace_bytes(p) > 0
for call in (lambda: B._arg(None, None, 0, 0, "x"), lambda: B._token_rows(None, (1, 1, 1, 1, 1), None, 0, "x")):
    try:
        call()
    except ImportError as e:
        assert "_args.so" in str(e) and "paper_2605_23200_amd.build" in str(e), e
        print("named")
""")
    assert out == ["named", "named"]


def test_the_checks_are_loaded_with_the_first_argument():
    assert _python("""
import sys
from paper_2605_23200_amd import binding as B
B.lib()
print("paper_2605_23200_amd._args" in sys.modules, B._arg(None, None, 0, 0, "x"), "paper_2605_23200_amd._args" in sys.modules, B._arg.__name__)
""") == ["False", "None", "True", "arg"]


def test_the_library_is_linked_where_the_checks_do_not_compile(monkeypatch, tmp_path):
    """The build says what failed, after the library is there."""
    import pytest
    from paper_2605_23200_amd import build

    def fails():
        raise RuntimeError("g++ failed on args.cpp")
    done = []
    monkeypatch.setattr(build, "_compile_args", fails)
    monkeypatch.setattr(build, "_compile", lambda src: done.append(src) or src)
    monkeypatch.setattr(build, "OBJ_DIR", str(tmp_path))
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **kw: done.append(cmd[0]) or type("R", (), dict(returncode=0, stderr="")))
    with pytest.raises(RuntimeError, match="args.cpp"):
        build.build()
    assert done[-1] == "hipcc" and sorted(done[:-1]) == sorted(build.SOURCES)


def test_a_torch_without_types_of_4_bits():
    """uint8 codes and scales need no type of torch's own."""
    assert _python("""
import torch
for name in ("float4_e2m1fn_x2", "float8_e8m0fnu"):
    delattr(torch, name)
from paper_2605_23200_amd import binding as B
print(B.scale_shape(torch.empty((2, 3, 4, 100, 64), dtype=torch.uint8)), B._SCALE_DTYPES[B.E2M1], B._SCALE_DTYPES[B.INT8])
""") == "(2, 3, 4, 7, 4, 16) (torch.uint8,) (torch.float32,)".split()


def test_the_types_that_this_torch_has():
    import torch
    from paper_2605_23200_amd import binding as B
    assert B._CACHE_DTYPES[torch.float4_e2m1fn_x2] == B._CACHE_DTYPES[torch.uint8] == B.E2M1
    assert B._SCALE_DTYPES[B.E2M1] == (torch.uint8, torch.float8_e8m0fnu) and set(B._SCALE_DTYPES) == {B.INT8, B.E4M3, B.E2M1}
