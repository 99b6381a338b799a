"""The entry points for many continuations and tenants without a GPU: refusals before anything touches the device."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def m():
    import paper_2607_19438_amd as q
    if not os.path.exists(q.lib_path()):
        from paper_2607_19438_amd import build
        build.build()
    return q


def caller(f, ok):
    return lambda **kw: f(*{**ok, **kw}.values(), None)


def test_attention_kv4_shared_refusals(m):
    ok = dict(q=16, cache=16, tab=16, kv=16, cu=16, groups=16, prefix=16, o=32, ws=16, bytes=1 << 40, T=4, R=3, G=2, H=4, Hkv=2, D=64, W=2, pages=4,
              page=16, qs=256, scale=0.1)
    call = caller(m.lib().qgemm_attention_kv4_shared, ok)
    for kw in ({"T": -1}, {"R": -1}, {"G": -1}, {"W": -1}, {"H": 3}, {"Hkv": 0}, {"page": 8}, {"page": 24}, {"pages": 0}, {"scale": 0.0},
               {"scale": float("nan")}, {"qs": 255}, {"cu": 0}, {"bytes": 0}, {"q": 0}, {"cache": 0}, {"tab": 0}, {"kv": 0}, {"groups": 0}, {"prefix": 0},
               {"o": 0}, {"ws": 0}):
        assert call(**kw) == -1, kw
    for kw in ({"D": 96}, {"R": 2049}, {"G": 2049}, {"W": 1 << 27}, {"T": 1 << 24, "H": 4, "D": 128}, {"T": 1 << 18, "H": 64, "Hkv": 64, "W": 1 << 20}):
        assert call(**kw) == -3, kw
    for kw in ({"q": 24}, {"cache": 24}, {"o": 24}, {"ws": 24}, {"tab": 18}, {"kv": 18}, {"cu": 18}, {"groups": 18}, {"prefix": 18}, {"qs": 260}):
        assert call(**kw) == -2, kw
    assert call(T=0) == 0 and call(R=0) == 0
    n = ctypes.c_int64(-1)
    w = m.lib().qgemm_attention_kv4_shared_workspace
    assert w(4, 3, 2, 4, 2, 64, 2, 16, None) == -1 and w(4, 3, 2, 4, 2, 96, 2, 16, ctypes.byref(n)) == -3
    assert w(4, 3, 2, 4, 2, 64, 2, 16, ctypes.byref(n)) == 0 and n.value > 0
    assert call(bytes=n.value - 1) == -1 and "workspace" in m.last_error()
    assert w(0, 3, 2, 4, 2, 64, 2, 16, ctypes.byref(n)) == 0 and n.value == 0


def test_beam_select_refusals(m):
    ok = dict(x=16, type=0, scores=16, fin=0, os=16, op=16, ot=16, ws=16, bytes=1 << 40, R=2, B=3, V=50, K=6, stride=50, end=0)
    call = caller(m.lib().qgemm_beam_select, ok)
    for kw in ({"type": 2}, {"R": -1}, {"B": 0}, {"V": 0}, {"K": 0}, {"stride": 49}, {"end": -1}, {"end": 50}, {"x": 0}, {"scores": 0}, {"os": 0}, {"op": 0},
               {"ot": 0}, {"ws": 0}, {"bytes": 0}):
        assert call(**kw) == -1, kw
    for kw in ({"B": 65}, {"K": 129}, {"V": (1 << 30) + 1, "stride": 1 << 31}, {"R": 1 << 20}):
        assert call(**kw) == -3, kw
    for kw in ({"x": 18}, {"scores": 18}, {"os": 18}, {"op": 18}, {"ot": 18}, {"ws": 24}, {"x": 17, "type": 1}):
        assert call(**kw) == -2, kw
    assert call(R=0) == 0
    n = ctypes.c_int64(-1)
    w = m.lib().qgemm_beam_select_workspace
    assert w(2, 3, 50, 6, None) == -1 and w(2, 65, 50, 6, ctypes.byref(n)) == -3
    assert w(2, 3, 50, 6, ctypes.byref(n)) == 0 and n.value > 0 and call(bytes=n.value - 1) == -1


def test_kv_reorder_refusals(m):
    names = ("tab", "kv", "par", "free", "keep", "new", "len", "src", "dst", "used", "rel", "nrel", "ws")
    size = dict(tab=24, kv=6, par=6, free=5, keep=2, new=24, len=6, src=6, dst=6, used=1, rel=7, nrel=1, ws=2 * (1 + 256 * 3))
    at = {name: (i + 1) << 14 for i, name in enumerate(names)}
    ok = dict(at, bytes=4 * size["ws"], R=2, B=3, W=4, F=5, Q=7, page=16)
    f = m.lib().qgemm_kv_reorder
    call = caller(f, ok)
    for kw in ({"R": -1}, {"B": 0}, {"W": -1}, {"F": -1}, {"Q": -1}, {"page": 8}, {"page": 24}, {"page": 2048}, {"bytes": 4 * size["ws"] - 1},
               *({n: 0} for n in names if n != "keep")):
        assert call(**kw) == -1, kw
    for kw in ({"B": 65}, {"R": 65536}, {"W": 1 << 30}):
        assert call(**kw) == -3, kw
    for n in names:
        assert call(**{n: at[n] + 2}) == -2, n
    assert call(R=0) == 0
    for a in ("new", "len", "src", "dst", "used", "rel", "nrel", "ws"):
        for b in names:
            for shift in () if a == b else (0, 4 * (size[b] - 1), -4 * (size[a] - 1)):
                assert call(**{a: at[b] + shift}) == -1, (a, b, shift)
                assert "overlap" in m.last_error(), (a, b, shift)
    n = ctypes.c_int64(-1)
    w = m.lib().qgemm_kv_reorder_workspace
    assert w(2, 3, 4, None) == -1 and w(-1, 3, 4, ctypes.byref(n)) == -1 and w(2, 65, 4, ctypes.byref(n)) == -3
    assert w(2, 3, 4, ctypes.byref(n)) == 0 and n.value == ok["bytes"]
    assert w(3, 1, 600, ctypes.byref(n)) == 0 and n.value == 4 * 9 * 257


def test_kv4_copy_refusals(m):
    ok = dict(cache=16, src=16, dst=16, n=2, Hkv=2, D=64, pages=4, page=16)
    call = caller(m.lib().qgemm_kv4_copy, ok)
    for kw in ({"cache": 0}, {"src": 0}, {"dst": 0}, {"n": -1}, {"Hkv": 0}, {"pages": 0}, {"page": 8}):
        assert call(**kw) == -1, kw
    assert call(D=96) == -3 and call(pages=1 << 27) == -3
    for kw in ({"cache": 24}, {"src": 18}, {"dst": 18}):
        assert call(**kw) == -2, kw
    assert call(n=0) == 0


def test_adapters_refusals(m):
    ok = dict(x=16, a=16, b=16, ids=16, cu=16, gain=0, y=32, ws=16, bytes=1 << 40, M=4, N=20, K=64, r=8, n=3, R=2, xs=64, ys=20)
    call = caller(m.lib().qgemm_adapters, ok)
    for kw in ({"M": -1}, {"R": -1}, {"N": 0}, {"n": 0}, {"K": 0}, {"K": 60}, {"r": 0}, {"r": 12}, {"xs": 56}, {"ys": 19}, {"cu": 0}, {"x": 0}, {"a": 0},
               {"b": 0}, {"ids": 0}, {"y": 0}, {"ws": 0}, {"bytes": 0}):
        assert call(**kw) == -1, kw
    for kw in ({"r": 136}, {"N": 1 << 29, "ys": 1 << 30}, {"K": 1 << 29, "xs": 1 << 29}, {"M": 1 << 29}, {"M": (1 << 25) + 1}, {"R": 1 << 29}):
        assert call(**kw) == -3, kw
    for kw in ({"x": 24}, {"a": 24}, {"b": 24}, {"ws": 24}, {"ids": 18}, {"cu": 18}, {"gain": 18}, {"y": 18}, {"xs": 68}):
        assert call(**kw) == -2, kw
    assert call(M=0) == 0 and call(R=0) == 0
    n = ctypes.c_int64(-1)
    w = m.lib().qgemm_adapters_workspace
    assert w(4, 20, 64, 8, None) == -1 and w(4, 20, 64, 12, ctypes.byref(n)) == -1
    assert w(4, 20, 64, 8, ctypes.byref(n)) == 0 and n.value > 0 and call(bytes=n.value - 1) == -1


def test_python_refuses_what_is_no_gpu_tensor(m):
    i, x = torch.zeros(4, dtype=torch.int32), torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    f, b = torch.zeros((4, 64)), torch.zeros((1, 8, 64), dtype=torch.bfloat16)
    c = torch.zeros((2, 2, 16 * 68), dtype=torch.uint8)
    for call in (lambda: m.attention_kv4_shared(x, c, i[:, None], i, i, i), lambda: m.beam_select(f, f), lambda: m.kv_reorder(i[:, None], i, i[:, None], i, 16),
                 lambda: m.kv4_copy(c, i, i), lambda: m.adapters(f, x[:, 0], b, b, i)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    for call in (lambda: m.attention_kv4_shared(1, c, i, i, i, i), lambda: m.beam_select(3, 4), lambda: m.kv_reorder(1, 2, 3, 4, 16), lambda: m.kv4_copy(1, 2, 3),
                 lambda: m.adapters(1, 2, 3, 4, 5)):
        with pytest.raises(TypeError, match="torch.Tensor"):
            call()
