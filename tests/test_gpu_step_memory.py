"""GPU: the results of the operators for many continuations keep no scratch memory alive, through the binding's compiled part and
without it."""
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


def test_results_keep_no_scratch_memory(m):
    torch = torch_or_skip()
    for R, B, K, V in ((1, 4, 4, 3000), (6, 64, 128, 5000), (3, 2, 8, 90000)):
        out = m.beam_select(torch.randn((R * B, V), device="cuda"), torch.zeros((R, B), device="cuda"), K)
        assert all(t.untyped_storage().nbytes() <= 3 * 4 * R * K for t in out)
    p = m.kv_reorder(dev_i32(torch, [[1, 2, 3]] * 6), dev_i32(torch, [40] * 6), dev_i32(torch, [[0, 0, 1], [2, 1, 1]]), dev_i32(torch, range(10, 16)), 16)
    own = sum(getattr(p, n).numel() for n in m.KvReorder.__slots__)
    assert all(getattr(p, n).untyped_storage().nbytes() == 4 * own for n in m.KvReorder.__slots__)
