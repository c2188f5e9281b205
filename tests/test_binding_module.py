"""The binding with and without its extension module: host only, nothing is launched."""
import os
import shutil
import subprocess
import sys
import sysconfig

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE = 1, 3
P = 0x100000       # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_25120_amd import build
        build.build()
    binding.lib()
    return binding


CALLS = """
import sys
sys.path.insert(0, sys.argv[1])
from paper_2603_25120_amd import binding as B
assert B.__file__.startswith(sys.argv[1]), B.__file__
for call, status in ((lambda: B.mllm_op_keep8(None, 1 << 20, 2 << 20, 4, 64, 0, stream=1), 1),
                     (lambda: B.mllm_op_keep8(1 << 20, 2 << 20, 3 << 20, 4, 60, 0, stream=1), 3),
                     (lambda: B.mllm_op_norm_fwd(7, 1 << 20, 1 << 20, None, 1 << 20, 1 << 20, 4, 64, 1e-5, stream=1), 3)):
    try:
        call()
    except B.MllmError as e:
        assert e.status == status, str(e)
    else:
        raise AssertionError("not refused")
print("module" if hasattr(B._fast(), "bind") else "ctypes")
"""


def copy_of_the_package(B, tmp_path, keep):
    """The package as another build leaves it: only those of the extension module's files that `keep` takes."""
    to = tmp_path / "paper_2603_25120_amd"
    shutil.copytree(os.path.dirname(B.__file__), to, ignore=lambda _, names: [n for n in names if n == "__pycache__" or n.startswith("_calls") and not keep(n)])
    return to


def calls_from(path):
    r = subprocess.run([sys.executable, "-c", CALLS, str(path)], capture_output=True, text=True, cwd=str(path))
    assert r.returncode == 0, r.stderr
    return r.stdout.split()[-1]


def test_without_the_module(B, tmp_path):
    """Where there is no compiler for the host or no Python.h the calls go through ctypes, all of them."""
    copy_of_the_package(B, tmp_path, lambda name: False)
    assert calls_from(tmp_path) == "ctypes"


def test_with_the_module(B, tmp_path):
    copy_of_the_package(B, tmp_path, lambda name: True)
    assert calls_from(tmp_path) == "module"


def test_module_of_another_interpreter(B, tmp_path):
    """It has another name, and is not loaded: here files that no interpreter could load."""
    to = copy_of_the_package(B, tmp_path, lambda name: False)
    for name in ("_calls.so", "_calls.cpython-39-x86_64-linux-gnu.so", "_calls.abi3.so"):
        (to / name).write_bytes(b"made for another one")
    assert calls_from(tmp_path) == "ctypes"


def test_name_of_the_module(B):
    from paper_2603_25120_amd import build
    assert os.path.basename(build.CALLS) == "_calls" + sysconfig.get_config_var("EXT_SUFFIX")
    assert build.CALLS == B.CALLS_PATH


@pytest.mark.parametrize("lacks", ["compiler", "header"])
def test_build_where_the_module_cannot_be_built(lacks, tmp_path, monkeypatch, capsys):
    """No module then, and none of an older header either; hipcc alone builds the library."""
    from paper_2603_25120_amd import build
    old = tmp_path / "_calls.so"
    old.write_bytes(b"of an older header")
    monkeypatch.setattr(build, "CALLS", str(old))
    if lacks == "compiler":
        monkeypatch.setenv("CXX", str(tmp_path / "no-such-compiler"))
    else:
        monkeypatch.setattr(build, "python_headers", lambda: str(tmp_path))
    build.build_calls(force=True)
    assert not old.exists() and "_calls" in capsys.readouterr().err


def test_build_of_the_module(tmp_path, monkeypatch):
    """Made anew where its source or a header is newer; what an error in the source says is not lost."""
    from paper_2603_25120_amd import build
    out = tmp_path / "_calls.so"
    monkeypatch.setattr(build, "CALLS", str(out))
    build.build_calls(force=False)
    made = out.stat().st_mtime_ns
    build.build_calls(force=False)
    assert out.stat().st_mtime_ns == made
    os.utime(out, (1, 1))
    build.build_calls(force=False)
    assert out.stat().st_mtime > 1
    monkeypatch.setenv("CXX", "g++ -DMLLM_STAGE_H_ -include /no/such/header")
    with pytest.raises(RuntimeError):
        build.build_calls(force=True)


class Tensor:
    def data_ptr(self):
        return P


@pytest.mark.parametrize("through", ["module", "ctypes"])
def test_arguments(B, through):
    """Both ways take and refuse the same arguments."""
    calls = B._fast() if through == "module" else B._ThroughCtypes(B.lib())
    assert set(B.FAST) <= set(B.EXPORTS) and all(callable(getattr(calls, name)) for name in B.FAST)
    ok = (Tensor(), 2 * P, 3 * P, np.int64(0), np.int32(64), 64, 0, None)         # no rows: nothing is launched
    assert calls.mllm_op_keep8(*ok) == 0
    assert calls.mllm_op_keep8(None, None, None, *ok[3:]) == 0
    assert calls.mllm_op_keep8(None, 2 * P, 3 * P, 4, *ok[4:]) == NULL and "NULL" in B.mllm_last_error()
    assert calls.mllm_op_keep8(*ok[:3], True, *ok[4:6], 5, None) == SHAPE
    for bad, error in (((*ok[:-1],), TypeError), ((*ok, 0), TypeError), ((*ok[:4], 64.0, *ok[5:]), TypeError), (("x", *ok[1:]), AttributeError),
                       ((*ok[:6], 1 << 31, None), OverflowError), ((*ok[:3], 1 << 63, *ok[4:]), OverflowError)):
        with pytest.raises(error):
            calls.mllm_op_keep8(*bad)
    kept = (P, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, 0, 64, 64, 0, 0, 7 * P)
    with pytest.raises(OverflowError):
        calls.mllm_op_linear_bwd_keep8(*kept, -1, None)                            # a size is never negative
    assert calls.mllm_op_linear_bwd_keep8(*kept[:-4], -8, 0, 0, 7 * P, 0, None) == SHAPE
