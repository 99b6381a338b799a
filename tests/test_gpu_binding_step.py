"""GPU: the operators for many continuations and many tenants give the same through the binding's compiled part and without
it, refuse the same, and keep no reference."""
import ctypes
import gc
import sys

import pytest

from gpu_util import torch_or_skip
from serve_util import dev_i32

pytestmark = pytest.mark.gpu


def q():
    import paper_2607_19438_amd as m
    m.lib()
    assert m._fast is not None, "the binding's compiled part is not built (python -m paper_2607_19438_amd.build)"
    return m


def calls(torch):
    """(function name, arguments as the Python function takes them, keywords) with fresh tensors."""
    gen = torch.Generator(device="cuda").manual_seed(2)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=gen, device="cuda").to(dtype)

    b = normal(9, 12, 64)
    cache = torch.randint(0, 120, (6, 2, 16 * 68), generator=gen, device="cuda").to(torch.uint8)
    table, kv = dev_i32(torch, [[0, 3, 1, 4, 5], [0, 3, 1, 4, 2]]), dev_i32(torch, [80, 77])
    cu, groups, prefix = dev_i32(torch, [0, 4, 9]), dev_i32(torch, [0, 2]), dev_i32(torch, [64])
    logits, scores = normal(6, 40, dtype=torch.float32), normal(2, 3, dtype=torch.float32)
    ended = torch.tensor([[False, True, False], [False, False, True]], device="cuda")
    beams, lens = dev_i32(torch, [[1, 2], [3, 4], [5, -1], [6, 7]]), dev_i32(torch, [20, 16, 3, 25])
    parents, free = dev_i32(torch, [[0, 0], [1, 1]]), dev_i32(torch, [9, 8, 10])
    y, x, wa, wb = normal(5, 24, dtype=torch.float32), normal(5, 64), normal(3, 8, 64), normal(3, 24, 8)
    ids, gain = dev_i32(torch, [2, 0, 0, -1, 1]), normal(3, dtype=torch.float32)
    wide = normal(5, 40, dtype=torch.float32)
    return [
        ("attention_kv4_shared", (b[:2, :8], cache, table, kv, groups, prefix), {}),
        ("attention_kv4_shared", (b[:, :8], cache, table, kv, groups, prefix, cu, 0.2),
         {"out": torch.zeros((9, 8, 64), dtype=torch.bfloat16, device="cuda")}),
        ("beam_select", (logits, scores), {}),
        ("beam_select", (normal(6, 64)[:, :37], scores, 5, ended, 36), {}),
        ("beam_select", (logits, scores, 5, ended.to(torch.uint8), 3), {}),
        ("kv_reorder", (beams, lens, parents, free, 16), {}),
        ("kv_reorder", (beams, lens, parents, free, 16, dev_i32(torch, [1, 0]), 3), {}),
        ("kv4_copy", (cache, dev_i32(torch, [0, -1, 9]), dev_i32(torch, [2, 3, 1])), {}),
        ("kv4_copy", (cache, dev_i32(torch, [0, -1, 3]), dev_i32(torch, [2, 3, 1]), 64), {}),
        ("kv4_copy", (torch.randint(0, 250, (6, 2, 16 * 136), generator=gen, device="cuda").to(torch.uint8), dev_i32(torch, [0]), dev_i32(torch, [5])), {}),
        ("adapters", (y, x, wa, wb, ids), {}),
        ("adapters", (wide[:, 8:32], x, wa, wb, ids[:2], gain, dev_i32(torch, [0, 3, 5])), {}),
    ]


def results(torch, m):
    out = []
    for name, args, kw in calls(torch):
        r = getattr(m, name)(*args, **kw)
        if "out" in kw:
            assert r is kw["out"]
        if name == "kv_reorder":
            r = tuple(getattr(r, n) for n in m.KvReorder.__slots__)
        elif name == "kv4_copy":
            assert r is None
            r = (args[0],)
        elif name == "adapters":
            assert r is args[0]
        out.append([x.clone() for x in (r if isinstance(r, tuple) else (r,))])
    return out


def test_both_ways_give_the_same(monkeypatch):
    torch = torch_or_skip()
    m = q()
    taken = []

    class Watch:
        def __getattr__(self, name):
            f = getattr(fast, name)

            def call(*a):
                r = f(*a)
                taken.append((name, r is not NotImplemented))
                return r
            return call

    fast = m._fast
    monkeypatch.setattr(m, "_fast", Watch())
    a = results(torch, m)
    assert [n for n, ok in taken if ok] == [n for n, _, _ in calls(torch)]
    monkeypatch.setattr(m, "_fast", None)
    b = results(torch, m)
    for x, y in zip(a, b):
        assert len(x) == len(y)
        for s, t in zip(x, y):
            assert s.shape == t.shape and s.dtype == t.dtype and s.stride() == t.stride() and torch.equal(s, t)


def test_refusals_are_the_same_either_way(monkeypatch):
    torch = torch_or_skip()
    m = q()

    def errors():
        got = []
        for name, args, kw in calls(torch):
            for at in range(len(args)):
                for change in ("host", "type", "float64", "transposed", "short", "negative", "none"):
                    a = list(args)
                    x = a[at]
                    if change == "none":
                        a[at] = None
                    elif not isinstance(x, torch.Tensor):
                        if change not in ("type", "negative", "float64"):
                            continue
                        a[at] = "x" if change == "type" else 1 << 33 if change == "float64" else -3
                    elif change == "host":
                        a[at] = x.cpu()
                    elif change == "type":
                        a[at] = "x"
                    elif change == "float64":
                        a[at] = x.to(torch.int64 if x.dtype == torch.float64 else torch.float64)
                    elif change == "transposed":
                        if x.dim() < 2:
                            continue
                        a[at] = x.transpose(-1, -2)
                    elif change == "short":
                        a[at] = x[:0] if x.dim() == 1 else x[..., :-1]
                    else:
                        continue
                    try:
                        getattr(m, name)(*a, **kw)
                        got.append((name, at, change, "fine"))
                    except (TypeError, ValueError, m.QGemmError, AttributeError, ctypes.ArgumentError) as e:
                        got.append((name, at, change, type(e).__name__))
        torch.cuda.synchronize()
        return got

    fast = errors()
    monkeypatch.setattr(m, "_fast", None)
    slow = errors()
    assert [e[:3] for e in fast] == [e[:3] for e in slow]
    for x, y in zip(fast, slow):
        assert (x[3] == "fine") == (y[3] == "fine"), (x, y)


def test_no_reference_is_kept():
    torch = torch_or_skip()
    m = q()
    args = calls(torch)
    for name, a, kw in args:
        getattr(m, name)(*a, **kw)
    torch.cuda.synchronize()
    gc.collect()

    def counted():                      # (small integers are the interpreter's own)
        return [[sys.getrefcount(x) for x in (*a, *kw.values()) if isinstance(x, torch.Tensor)] for _, a, kw in args]

    counts = counted()
    used = torch.cuda.memory_allocated()
    for _ in range(50):
        for name, a, kw in args:
            getattr(m, name)(*a, **kw)
    torch.cuda.synchronize()
    gc.collect()
    assert counted() == counts
    assert torch.cuda.memory_allocated() == used


@pytest.mark.parametrize("fast", [True, False])
def test_a_reordering_of_nothing(fast, monkeypatch):
    torch = torch_or_skip()
    m = q()
    if not fast:
        monkeypatch.setattr(m, "_fast", None)
    n = m.kv_reorder(torch.empty((0, 3), dtype=torch.int32, device="cuda"), dev_i32(torch, []), torch.empty((0, 4), dtype=torch.int32, device="cuda"),
                     dev_i32(torch, [5]), 16, released=2)
    assert n.block_table.shape == (0, 3) and int(n.used) == 0 and int(n.n_released) == 0 and n.released.tolist() == [-1, -1]


def test_the_current_stream_is_used():
    torch = torch_or_skip()
    m = q()
    y = torch.zeros((64, 32), device="cuda")
    x = torch.randn((64, 128), device="cuda").to(torch.bfloat16)
    a, b = torch.randn((2, 8, 128), device="cuda").to(torch.bfloat16), torch.randn((2, 32, 8), device="cuda").to(torch.bfloat16)
    ids = dev_i32(torch, [0, 1] * 32)
    want = m.adapters(y.clone(), x, a, b, ids)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late = torch.zeros_like(x)
        for _ in range(10):
            torch.mm(torch.ones((2048, 2048), device="cuda"), torch.ones((2048, 2048), device="cuda"))
        late.copy_(x)
        got = m.adapters(y.clone(), late, a, b, ids)
    side.synchronize()
    assert torch.equal(got, want)
