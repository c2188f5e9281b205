"""Build the HIP library in-tree: `python -m paper_2603_25120_amd.build`.

Compiles every source under csrc/ for gfx950 with hipcc and links
`paper_2603_25120_amd/libmllm_stage.so`, and with g++ `_calls`, the binding's extension module for the interpreter that runs the build (host code; without it the
binding's calls go through ctypes).  Objects are cached under `_build/` (git-ignored); an object is rebuilt when its source or any header is newer.
"""
from __future__ import annotations

import os
import shlex
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libmllm_stage.so")
CALLS = os.path.join(HERE, "_calls" + sysconfig.get_config_var("EXT_SUFFIX"))   # an interpreter loads no other's
BUILD = os.path.join(ROOT, "_build")

SOURCES = ["gemm.hip", "gemm_fwd.hip", "gemm_dx.hip", "gemm_dw.hip", "gemm_pair.hip", "gemm_small.hip", "attention.hip", "elementwise.hip", "token.hip", "positions.hip", "residual.hip", "keep8.hip", "stage.hip", "ops_abi.hip", "profile.hip", "scheduler.hip", "planner.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=fast",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument"]


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("command failed: %s\n%s" % (" ".join(cmd), out))
    return out


def _newest_header() -> float:
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h")]
    headers.append(os.path.join(ROOT, "include", "mllm_stage.h"))
    return max(os.path.getmtime(h) for h in headers)


def python_headers() -> str:
    return sysconfig.get_paths()["include"]


def build_calls(force: bool) -> None:
    """The extension module, where its tools are there; a module of older headers does not stay in any case."""
    source = os.path.join(CSRC, "calls.cpp")
    if os.path.exists(CALLS):
        if not force and os.path.getmtime(CALLS) >= max(os.path.getmtime(source), _newest_header()):
            return
        os.remove(CALLS)
    compiler = shlex.split(os.environ.get("CXX", "g++"))
    if not shutil.which(compiler[0]) or not os.path.exists(os.path.join(python_headers(), "Python.h")):
        print("_calls, the binding's extension module, is not built: it takes a C++ compiler (%s) and Python.h; calls go through ctypes" % compiler[0], file=sys.stderr)
        return
    _run(compiler + ["-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-I" + python_headers(), source, "-o", CALLS])


def build(force: bool = False, verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(BUILD, exist_ok=True)
    newest_header = _newest_header()
    jobs, objs = [], []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(BUILD, src.replace(".hip", ".o"))
        objs.append(o)
        if force or not os.path.exists(o) or os.path.getmtime(o) < max(os.path.getmtime(s), newest_header):
            jobs.append([hipcc] + FLAGS + ["-c", s, "-o", o])
    with ThreadPoolExecutor(max_workers=min(8, max(1, len(jobs)))) as ex:
        for out in ex.map(_run, jobs):
            if verbose and out.strip():
                print(out)
    build_calls(force)
    if jobs or force or not os.path.exists(OUT):
        _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-pthread", "-o", OUT] + objs)
    return OUT


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
