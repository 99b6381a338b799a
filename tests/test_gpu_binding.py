"""GPU: the two ways of the serving functions into the library, compiled and Python, give the same; the compiled one
takes what it should, leaves the rest and keeps no reference."""
import ctypes
import gc
import sys

import pytest

import oracle
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
    gen = torch.Generator(device="cuda").manual_seed(1)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=gen, device="cuda").to(dtype)

    rows = normal(21, 12, 64, dtype=torch.float32)
    f = torch.from_numpy(oracle.rope_frequencies(32, 10000.0)[0]).cuda()
    pos = torch.arange(21, dtype=torch.int32, device="cuda") * 3
    b = normal(21, 12, 64)
    cache = torch.randint(0, 120, (6, 2, 16 * 68), generator=gen, device="cuda").to(torch.uint8)
    slots = torch.randperm(96, generator=gen, device="cuda")[:21].to(torch.int32)
    table, kv = dev_i32(torch, [[0, 3, 1], [5, 2, 4]]), dev_i32(torch, [40, 17])
    cu = dev_i32(torch, [0, 13, 21])
    return [
        ("kv_plan", (dev_i32(torch, [3, 30]), dev_i32(torch, [20, 4]), dev_i32(torch, [[7, 0, 0], [1, 2, 0]]), dev_i32(torch, [9, 8, 5]), 16, 25), {}),
        ("rope", (rows, pos, f, 10), {}),
        ("rope", (rows, pos, f, 10), {"interleaved": True, "gain": 1.5}),
        ("rope", (b[:, 2:9], pos, f, 3), {"out": torch.zeros((21, 9, 64), dtype=torch.bfloat16, device="cuda")[:, 1:8]}),
        ("kv4_store", (b[:, 8:10], b[:, 10:], slots, cache), {}),
        ("kv4_load", (cache, slots, 64), {}),
        ("attention_packed", (b[:, :8], b[:, 8:10], b[:, 10:], cu), {}),
        ("attention_packed", (b[:, :8], b[:, 8:10], b[:, 10:], cu, 0.3), {"out": torch.zeros((21, 8, 64), dtype=torch.bfloat16, device="cuda")}),
        ("attention_kv4", (b[:2, :8], cache, table, kv), {}),
        ("attention_kv4", (b[:, :8], cache, table, kv, cu, 0.2), {"out": torch.zeros((21, 8, 64), dtype=torch.bfloat16, device="cuda")}),
    ]


def results(torch, m):
    out = []
    for name, args, kw in calls(torch):
        r = getattr(m, name)(*args, **kw)
        if "out" in kw:
            assert r is kw["out"]
        if name == "kv_plan":
            r = (r.cu_q, r.positions, r.slots, r.kv_len, r.used, args[2])
        elif name == "kv4_store":
            assert r is None
            r = (args[3],)
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
            assert s.shape == t.shape and s.dtype == t.dtype and torch.equal(s, t)


def test_refusals_are_the_same_either_way(monkeypatch):
    torch = torch_or_skip()
    m = q()

    def errors():
        got = []
        for name, args, kw in calls(torch):
            for at in range(len(args)):
                for change in ("host", "type", "float64", "transposed", "short", "negative"):
                    a = list(args)
                    x = a[at]
                    if not isinstance(x, torch.Tensor):
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
    counts = [[sys.getrefcount(x) for x in (*a, *kw.values())] for _, a, kw in args]
    used = torch.cuda.memory_allocated()
    for _ in range(50):
        for name, a, kw in args:
            getattr(m, name)(*a, **kw)
    torch.cuda.synchronize()
    gc.collect()
    assert [[sys.getrefcount(x) for x in (*a, *kw.values())] for _, a, kw in args] == counts
    assert torch.cuda.memory_allocated() == used


def test_the_current_stream_is_used():
    torch = torch_or_skip()
    m = q()
    x = torch.randn((64, 4, 64), device="cuda")
    f = torch.from_numpy(oracle.rope_frequencies(64, 10000.0)[0]).cuda()
    pos = torch.arange(64, dtype=torch.int32, device="cuda")
    want = m.rope(x, pos, f, 2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = torch.zeros_like(x)
        for _ in range(10):
            torch.mm(torch.ones((2048, 2048), device="cuda"), torch.ones((2048, 2048), device="cuda"))
        y.copy_(x)
        got = m.rope(y, pos, f, 2)
    side.synchronize()
    assert torch.equal(got, want)
