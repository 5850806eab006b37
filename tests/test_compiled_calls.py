"""The compiled marshalling of the smallest calls is an addition: without it, or with one that was built for another Python or torch, the library and
every call are there all the same."""
import os
import subprocess
import sys
import textwrap

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def child(code):
    out = subprocess.run([sys.executable, "-W", "always", "-c", textwrap.dedent(code)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    return out.stdout, out.stderr


CALLS = """
    import ctypes
    assert B.conv_out_dims(B.conv_desc(1, 3, 8, 8, 8, 3, 3, 1, 1)) == (8, 8)
    P, NULL = ctypes.c_void_p, ctypes.c_void_p(0)
    assert B.lib().pcl_rms_norm_fwd(0, 8, 1, P(4096), NULL, P(4096), ctypes.c_float(1e-6), NULL, P(4096), NULL, NULL) == B.ERR_BAD_ARG
    x = torch.zeros(4, 8)
    for call in (lambda: B.rms_norm_fwd(4, 8, x, None, torch.zeros(8), 1e-6, None, x), lambda: B.quantize_rows(4, 8, x, x, x)):
        try:
            call()
        except ValueError:
            pass
        else:
            raise AssertionError("a tensor that is not on a CUDA device was taken")
"""


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_1602_06709_b200 import build
    build.build()


def test_used_where_it_is_there():
    out, err = child("import torch\nfrom paper_1602_06709_b200 import binding as B\nB.lib()\nprint(B._calls.built_for)")
    from paper_1602_06709_b200 import build
    assert out.strip() == build.calls_built_for() and "is not used" not in err


def test_missing():
    _, err = child("""
    import sys, torch
    sys.modules["paper_1602_06709_b200._pcl_calls"] = None
    from paper_1602_06709_b200 import binding as B
    B.lib()
    assert B._calls is None
    """ + CALLS)
    assert err.count("is not used") == 1


def test_built_for_another():
    _, err = child("""
    import sys, types, torch
    import paper_1602_06709_b200
    old = types.ModuleType("_pcl_calls")
    old.built_for = "cpython-39 torch-1.0"
    old.bind = lambda table: (_ for _ in ()).throw(AssertionError("bound"))
    paper_1602_06709_b200._pcl_calls = sys.modules["paper_1602_06709_b200._pcl_calls"] = old
    from paper_1602_06709_b200 import binding as B
    B.lib()
    assert B._calls is None
    """ + CALLS)
    assert err.count("cpython-39 torch-1.0") == 1


def test_the_library_is_built_without_it(monkeypatch, capsys):
    from paper_1602_06709_b200 import build

    def fails(force=False):
        raise FileNotFoundError("g++")

    monkeypatch.setattr(build, "build_calls", fails)
    assert os.path.exists(build.build())
    assert "was not built" in capsys.readouterr().err
