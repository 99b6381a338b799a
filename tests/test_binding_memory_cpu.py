"""Tensors without memory (inside ``torch.vmap``) in the binding's compiled part, without a GPU: a copy of it that takes
the current device to be 0, bound to a stand-in for the library, answers NotImplemented and leaves the interpreter whole."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2607_19438_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALLS = """
import ctypes, importlib.machinery, importlib.util, sys, threading, warnings
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
path = sys.argv[1]
spec = importlib.util.spec_from_file_location("_binding", path, loader=importlib.machinery.ExtensionFileLoader("_binding", path))
m = importlib.util.module_from_spec(spec)
spec.loader.exec_module(m)
done = ctypes.CFUNCTYPE(ctypes.c_int)(lambda: 0)
m.bind(lambda device: 0, *[ctypes.cast(done, ctypes.c_void_p).value] * 7)
with FakeTensorMode():
    def gpu(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda:0")
    many, x, freq = gpu(3, 4, 2, 64), gpu(4, 2, 64), gpu(32, dtype=torch.float64)
    i, cache = gpu(4, dtype=torch.int32), gpu(2, 2, 16 * 68, dtype=torch.uint8)
    for name, args in (("rope", lambda b: (b, i, freq, 1, False, 1.0, x)), ("rope", lambda b: (x, i, freq, 1, False, 1.0, b)),
                       ("kv4_store", lambda b: (b, x, i, cache)), ("kv4_store", lambda b: (x, b, i, cache)),
                       ("attention_packed", lambda b: (b, x, x, i, None, x)), ("attention_packed", lambda b: (x, b, b, i, None, x)),
                       ("attention_packed", lambda b: (x, x, x, i, None, b))):
        got = []
        torch.vmap(lambda b: (got.append(getattr(m, name)(*args(b))), b)[1])(many)
        assert got == [NotImplemented], (name, got)
        thread = threading.Thread(target=sum, args=(range(1000),))         # another thread can have the lock
        thread.start()
        thread.join()
    assert m.kv4_store(x, x, i, cache) is None                             # the stand-in is called where there is memory
print("whole")
"""


def test_tensors_without_memory(tmp_path, monkeypatch):
    if shutil.which(os.environ.get("CXX", "g++")) is None:
        pytest.skip("no host compiler")
    text = open(build.BINDING_SOURCE).read()
    for old, new in (("guard.getDevice().index()", "0"), ("../../include/qgemm.h", os.path.join(ROOT, "include", "qgemm.h"))):
        assert text.count(old) == 1
        text = text.replace(old, new)
    (tmp_path / "binding.cpp").write_text(text)
    (tmp_path / "calls.py").write_text(CALLS)
    monkeypatch.setattr(build, "BINDING_SOURCE", str(tmp_path / "binding.cpp"))
    monkeypatch.setattr(build, "BINDING", str(tmp_path / "_binding.so"))
    build.build_binding()
    res = subprocess.run([sys.executable, str(tmp_path / "calls.py"), str(tmp_path / "_binding.so")], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.strip() == "whole", (res.returncode, res.stderr[-2000:])
