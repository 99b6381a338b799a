"""GPU: a tensor that ``adapters`` has added to says so to autograd, through the binding's compiled part and without it."""
import pytest

from gpu_util import torch_or_skip
from serve_util import dev_i32

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[True, False], ids=["compiled", "python"])
def m(request, monkeypatch):
    torch_or_skip()
    import paper_2607_19438_amd as q
    q.lib()
    assert q._fast is not None, "the binding's compiled part is not built (python -m paper_2607_19438_amd.build)"
    if not request.param:
        monkeypatch.setattr(q, "_fast", None)
    return q


def operands(torch):
    gen = torch.Generator(device="cuda").manual_seed(3)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, device="cuda", generator=gen).to(dtype)

    return normal(5, 24, dtype=torch.float32), (normal(5, 64), normal(2, 8, 64), normal(2, 24, 8), dev_i32(torch, [0, 1, 1, 0, -1]))


def test_a_tensor_that_is_added_to_has_a_new_version(m):
    torch = torch_or_skip()
    y, rest = operands(torch)
    want = m.adapters(y.clone(), *rest)
    v = y._version
    assert m.adapters(y, *rest) is y and y._version == v + 1 and torch.equal(y, want)
    wide = torch.zeros((5, 40), device="cuda")
    v = wide._version
    m.adapters(wide[:, 8:32], *rest)
    assert wide._version == v + 1                          # the base of a view too
    # a graph that has saved y refuses to go back through it
    y = want.clone()
    w = torch.ones((24,), device="cuda", requires_grad=True)
    z = (y * w).sum()
    m.adapters(y, *rest)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()
    y, _ = operands(torch)
    w = torch.ones((24,), device="cuda", requires_grad=True)
    m.adapters(y, *rest)
    (y * w).sum().backward()                               # and one that saves it afterwards does not
    assert torch.allclose(w.grad, want.sum(0))


def test_a_tensor_of_a_graph_is_refused(m):
    """y that requires a gradient would get one without the adapters' part."""
    torch = torch_or_skip()
    y, rest = operands(torch)
    want = m.adapters(y.clone(), *rest)
    leaf = y.clone().requires_grad_()
    inner = leaf * 1.0
    for t in (leaf, inner, inner[:, :24]):
        before = t.detach().clone()
        with pytest.raises(ValueError, match="requires a gradient"):
            m.adapters(t, *rest)
        assert torch.equal(t.detach(), before)
    with torch.no_grad():
        assert torch.equal(m.adapters(leaf, *rest), want)
    assert torch.equal(m.adapters(inner.detach(), *rest), want)
    with torch.inference_mode():
        t = y.clone()
        assert torch.equal(m.adapters(t, *rest), want)
    with torch.inference_mode():
        t = y.clone()
    m.adapters(t, *rest)                                   # an inference tensor outside of that mode has no version
    assert torch.equal(t, want)
