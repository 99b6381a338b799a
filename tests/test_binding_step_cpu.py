"""The binding's compiled part of the operators for many continuations and many tenants, without a GPU: it answers
NotImplemented to whatever it does not take, and to everything where the library's functions were not given."""
import importlib.machinery
import importlib.util
import os

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
