"""The binding's compiled part without a GPU: it answers NotImplemented to whatever it does not take, and the Python
functions then say what is wrong."""
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


def test_it_is_there_and_bound(m):
    if m._raw_stream is None or m._fast is None:
        pytest.skip("the library was loaded before the binding was built, or torch has no GPU streams")
    assert {"kv_plan", "rope", "kv4_store", "kv4_load", "attention_packed", "attention_kv4"} <= set(dir(m._fast))


def test_other_arguments_are_left_to_python(m):
    from paper_2607_19438_amd import _binding as b
    i, x = torch.zeros(4, dtype=torch.int32), torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    c = torch.zeros((2, 2, 16 * 68), dtype=torch.uint8)
    calls = [(b.kv_plan, (i, i, i[:, None], i, 16, 4)), (b.rope, (x, i, torch.ones(32, dtype=torch.float64), 1, False, 1.0, None)),
             (b.kv4_store, (x, x, i, c)), (b.kv4_load, (c, i, 64)), (b.attention_packed, (x, x, x, i, None, None)),
             (b.attention_kv4, (x, c, i[:, None], i, None, None, None))]
    for f, args in calls:
        assert f(*args) is NotImplemented                      # host tensors
        for at in range(len(args)):                            # things that are no tensors or numbers
            for bad in (None, "x", object(), 1 << 80, float("nan"), [1]):
                assert f(*(bad if k == at else a for k, a in enumerate(args))) is NotImplemented
        assert f() is NotImplemented and f(*args, 1) is NotImplemented
    with pytest.raises(TypeError):
        b.bind(1)


def test_python_says_what_is_wrong(m):
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="torch.Tensor"):
        m.rope(3, x, x, 1)
    with pytest.raises(ValueError, match="GPU tensor"):
        m.attention_packed(x, x, x, x)
