"""The launches that a library call makes, without a GPU: a process of its own
loads ``launch_recorder.hip`` in the HIP runtime's place and then the library.

    for code, launched in launches.record([("convgemm_linear", (dtype, ...)), ...]):

``code`` is what the call returned, ``launched`` a list of dicts: the kernel's name
(demangled), its grid (workgroups), block, lds, and of the layer operators' kernels
what they were given.  Device addresses are never followed, so any number serves."""
from __future__ import annotations

import json
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
_built = None

CHILD = """
import ctypes, json, os, sys
recorder = ctypes.CDLL(sys.argv[1], mode=os.RTLD_GLOBAL | os.RTLD_NOW)
recorder.recorded.restype = ctypes.c_char_p
sys.path.insert(0, sys.argv[2])
import paper_2005_06410_amd as lt
lib = lt.load()
ARRAYS = {"p": ctypes.c_void_p, "q": ctypes.c_int64, "i": ctypes.c_int}
for name, args in json.load(sys.stdin):
    args = [(ARRAYS[a["of"]] * len(a["values"]))(*a["values"]) if isinstance(a, dict) else a for a in args]
    code = getattr(lib, name)(*args)
    print(json.dumps([code, [json.loads(v) for v in recorder.recorded().decode().splitlines()]]))
"""


def recorder():
    """The recorder's library, compiled once per process."""
    global _built
    if _built is None:
        from paper_2005_06410_amd import build
        _built = tempfile.TemporaryDirectory(prefix="launches_")
        out = os.path.join(_built.name, "recorder.so")
        subprocess.run([build.hipcc(), "--offload-arch=gfx950", "--offload-host-only", "-O1", "-fPIC", "-shared", "-std=c++17",
                        "-I" + build.INCLUDE, "-I" + build.CSRC, os.path.join(HERE, "launch_recorder.hip"), "-o", out],
                       check=True, capture_output=True, text=True)
    return os.path.join(_built.name, "recorder.so")


def record(calls):
    r = subprocess.run([sys.executable, "-c", CHILD, recorder(), ROOT], input=json.dumps(calls), capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    got = [json.loads(line) for line in r.stdout.splitlines()]
    assert len(got) == len(calls)
    return got
