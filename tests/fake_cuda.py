"""Runs calls of libfls.so in a child process whose CUDA runtime is tests/fake_runtime.cpp: no GPU, nothing launched."""
from __future__ import annotations

import json
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PRELUDE = """
import ctypes as C, json, os
from paper_2609_20359_b200 import _binding as fls
fake = C.CDLL(os.environ["LD_PRELOAD"])
for name in ("fake_grid", "fake_cleared"):
    getattr(fake, name).restype = C.POINTER(C.c_uint64)

def grids():
    return [list(fake.fake_grid(i)[:3]) for i in range(fake.fake_launches())]

def clears():
    return [list(fake.fake_cleared(i)[:2]) for i in range(fake.fake_clears())]

def buffers(rows, vocab, dim, layout, grads=True, f32=False, device=0):
    '''An fls_head_io over addresses of that device; nothing behind them is touched.'''
    io = fls.fls_head_io(rows=rows, ignore_label=-100, workspace_bytes=layout["workspace_bytes"])
    at = (device << 44) + (1 << 20)
    sizes = dict(hidden=2 * rows * dim, weight=2 * vocab * dim, labels=8 * rows, loss=4 * rows, lse=4 * rows,
                 workspace=layout["workspace_bytes"])
    if grads:
        sizes.update(grad_hidden=2 * rows * dim, grad_weight=(4 if f32 else 2) * vocab * dim)
    for name, size in sizes.items():
        setattr(io, name, at)
        at += (size + 4095) // 4096 * 4096
    return io

def code(f, *args, **kw):
    try:
        f(*args, **kw)
    except fls.FlsError as e:
        return e.code
    return 0
"""


def build(folder) -> str:
    from paper_2609_20359_b200 import build as b
    b.build()
    out = os.path.join(str(folder), "libfakecuda.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(b._nvcc())), "include")
    subprocess.run(["g++", "-shared", "-fPIC", "-std=c++17", "-w", "-I", cuda, "-I", b.CSRC, "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "fake_runtime.cpp"), "-o", out], check=True)
    return out


def run(fake: str, script: str):
    """What `script` assigns to `result`."""
    res = subprocess.run([sys.executable, "-c", PRELUDE + script + "\nprint('RESULT' + json.dumps(result))"], cwd=ROOT, text=True,
                         env={**os.environ, "LD_PRELOAD": fake}, capture_output=True)
    assert res.returncode == 0, res.stderr
    return json.loads(res.stdout.rsplit("RESULT", 1)[1])
