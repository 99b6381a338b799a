"""The binding's compiled part of the operators for many continuations and many tenants, without a GPU: it answers
NotImplemented to whatever it does not take, and to everything where the library's functions were not given."""
import os
import shutil
import subprocess
import sys

import pytest

import torch


@pytest.fixture(scope="module")
def m():
    import paper_2607_19438_amd as q
    from paper_2607_19438_amd import build
    if not os.path.exists(q.lib_path()):
        build.build()
    if not os.path.exists(build.BINDING):
        build.build_binding()
    q.lib()
    return q


NAMES = ("attention_kv4_shared", "beam_select", "kv_reorder", "kv4_copy", "adapters")


def calls():
    i, x = torch.zeros(4, dtype=torch.int32), torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    c, f = torch.zeros((2, 2, 16 * 68), dtype=torch.uint8), torch.zeros((4, 8))
    t = i[:, None].contiguous()
    return {"attention_kv4_shared": (x, c, t, i, i, i[:3], None, None, None), "beam_select": (f, f[:2, :2].contiguous(), 2, None, 0),
            "kv_reorder": (t, i, i.view(2, 2), i, 16, None, None), "kv4_copy": (c, i, i, None),
            "adapters": (f, x[:, 0], x[:2], x.view(2, 8, 32), i, None, None)}


def test_it_has_them(m):
    if m._raw_stream is None or m._fast is None:
        pytest.skip("the library was loaded before the binding was built, or torch has no GPU streams")
    assert set(NAMES) <= set(dir(m._fast))


@pytest.mark.parametrize("name", NAMES)
def test_other_arguments_are_left_to_python(m, name):
    from paper_2607_19438_amd import _binding as b
    f, args = getattr(b, name), calls()[name]
    assert f(*args) is NotImplemented                          # host tensors
    for at in range(len(args)):                                # things that are no tensors or numbers
        for bad in (None, "x", object(), 1 << 80, float("nan"), [1]):
            assert f(*(bad if k == at else a for k, a in enumerate(args))) is NotImplemented
    assert f() is NotImplemented and f(*args, 1) is NotImplemented


def test_python_says_what_is_wrong(m):
    c = calls()
    for name in NAMES:
        with pytest.raises(ValueError, match="GPU tensor"):
            getattr(m, name)(*(a for a in c[name] if a is not None))
        with pytest.raises(TypeError, match="torch.Tensor"):
            getattr(m, name)(*[3] * (5 if name != "kv4_copy" else 3), *([3] if name == "attention_kv4_shared" else []))


STANDIN = """
import ctypes, importlib.machinery, importlib.util, sys, threading
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
path = sys.argv[1]
spec = importlib.util.spec_from_file_location("_binding", path, loader=importlib.machinery.ExtensionFileLoader("_binding", path))
m = importlib.util.module_from_spec(spec)
spec.loader.exec_module(m)
done = ctypes.CFUNCTYPE(ctypes.c_int)(lambda: 0)
address = ctypes.cast(done, ctypes.c_void_p).value
with FakeTensorMode():
    def gpu(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda:0")
    i, t, c = gpu(4, dtype=torch.int32), gpu(4, 3, dtype=torch.int32), gpu(2, 2, 16 * 68, dtype=torch.uint8)
    f, y, x = gpu(4, 8, dtype=torch.float32), gpu(4, 20, dtype=torch.float32), gpu(4, 2, 64)
    p, s, k = gpu(2, 2, dtype=torch.int32), gpu(2, 2, dtype=torch.float32), gpu(4, 64)
    a, b = gpu(3, 8, 64), gpu(3, 20, 8)
    calls = {"attention_kv4_shared": (x, c, t, i, i, gpu(3, dtype=torch.int32), None, None, x), "beam_select": (f, s, 2, None, 0),
             "kv_reorder": (t, i, p, i, 16, None, None), "kv4_copy": (c, i, i, None), "adapters": (y, k, a, b, i, None, None)}
    m.bind(lambda device: 0, *[address] * 7)
    for name, args in calls.items():                   # functions that were not given
        assert getattr(m, name)(*args) is NotImplemented, name
    m.bind(lambda device: 0, *[address] * 16)
    assert m.kv4_copy(*calls["kv4_copy"]) is None and m.adapters(*calls["adapters"]) is y      # the stand-in is called
    assert [tuple(o.shape) for o in m.beam_select(*calls["beam_select"])] == [(2, 2)] * 3
    assert [tuple(o.shape) for o in m.kv_reorder(*calls["kv_reorder"])] == [(4, 3), (4,), (4,), (4,), (1,), (12,), (1,)]
    for name, args in calls.items():                   # tensors without memory
        for at, arg in enumerate(args):
            if not isinstance(arg, torch.Tensor):
                continue
            got = []
            many = torch.empty((3, *arg.shape), dtype=arg.dtype, device="cuda:0")
            torch.vmap(lambda v: (got.append(getattr(m, name)(*(v if n == at else o for n, o in enumerate(args)))), v)[1])(many)
            assert got == [NotImplemented], (name, at, got)
            thread = threading.Thread(target=sum, args=(range(1000),))         # another thread can have the lock
            thread.start()
            thread.join()
print("whole")
"""


def test_with_a_stand_in_for_the_library(tmp_path, monkeypatch):
    """A copy of it that takes the current device to be 0: functions that were not given, tensors without memory, shapes."""
    from paper_2607_19438_amd import build
    if shutil.which(os.environ.get("CXX", "g++")) is None:
        pytest.skip("no host compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(build.BINDING_SOURCE).read()
    for old, new in (("guard.getDevice().index()", "0"), ("../../include/qgemm.h", os.path.join(root, "include", "qgemm.h"))):
        assert text.count(old) == 1
        text = text.replace(old, new)
    (tmp_path / "binding.cpp").write_text(text)
    (tmp_path / "calls.py").write_text(STANDIN)
    monkeypatch.setattr(build, "BINDING_SOURCE", str(tmp_path / "binding.cpp"))
    monkeypatch.setattr(build, "BINDING", str(tmp_path / "_binding.so"))
    build.build_binding()
    res = subprocess.run([sys.executable, str(tmp_path / "calls.py"), str(tmp_path / "_binding.so")], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.strip() == "whole", (res.returncode, res.stderr[-2000:])
