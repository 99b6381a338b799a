"""The serving entry points without a GPU: refusals before anything touches the device, and the frequencies."""
import ctypes
import os

import numpy as np
import pytest

import oracle


@pytest.fixture(scope="module")
def m():
    import paper_2607_19438_amd as q
    if not os.path.exists(q.lib_path()):
        from paper_2607_19438_amd import build
        build.build()
    return q


def test_kv_plan_refusals(m):
    f = m.lib().qgemm_kv_plan
    ok = dict(kv=16, q=16, tab=16, free=16, cu=16, pos=16, slots=16, total=16, used=16, R=2, W=2, F=2, page=16, T=4)

    def call(**kw):
        return f(*{**ok, **kw}.values(), None)

    for kw in ({"R": -1}, {"W": -1}, {"F": -1}, {"T": -1}, {"page": 8}, {"page": 24}, {"page": 2048}, {"page": 0}, {"kv": 0}, {"q": 0},
               {"tab": 0}, {"free": 0}, {"cu": 0}, {"pos": 0}, {"slots": 0}, {"total": 0}, {"used": 0}):
        assert call(**kw) == -1, kw
    assert call(R=4097) == -3
    for name in ("kv", "q", "tab", "free", "cu", "pos", "slots", "total", "used"):
        assert call(**{name: 18}) == -2, name


def test_kv_plan_refuses_tables_that_overlap_what_it_writes(m):
    f = m.lib().qgemm_kv_plan
    n = dict(kv=3, q=3, tab=6, free=5, cu=4, pos=7, slots=7, total=3, used=1)
    at = {name: (i + 1) << 12 for i, name in enumerate(n)}
    written = ("tab", "cu", "pos", "slots", "total", "used")
    for a in written:
        for b in n:
            for shift in () if a == b else (0, 4 * (n[b] - 1), -4 * (n[a] - 1)):       # the same, and one entry in common
                p = {**at, a: at[b] + shift}
                assert f(*p.values(), 3, 2, 5, 16, 7, None) == -1, (a, b, shift)
                assert "overlap" in m.last_error(), (a, b, shift)


def test_rope_refusals(m):
    f = m.lib().qgemm_rope
    ok = dict(x=64, type=1, pos=64, freq=64, y=128, T=4, heads=3, rot_heads=2, D=64, rot=64, xs=192, ys=192, inter=0, gain=1.0)

    def call(**kw):
        return f(*{**ok, **kw}.values(), None)

    for kw in ({"type": 2}, {"T": -1}, {"heads": 0}, {"rot_heads": -1}, {"rot_heads": 4}, {"D": 63}, {"D": 0}, {"rot": 0}, {"rot": 63}, {"rot": 66},
               {"inter": 2}, {"gain": float("nan")}, {"gain": float("inf")}, {"xs": 191}, {"ys": 191}, {"x": 0}, {"pos": 0}, {"freq": 0},
               {"y": 0}, {"y": 64, "xs": 200}, {"y": 64, "type": 0}):
        assert call(**kw) == -1, kw
    assert call(D=1024, rot=514, xs=4096, ys=4096) == -3
    assert call(D=4096, heads=8192, xs=1 << 26, ys=1 << 26, rot_heads=1) == -3
    for kw in ({"x": 65}, {"y": 129}, {"pos": 66}, {"freq": 68}, {"x": 66, "type": 0}):
        assert call(**kw) == -2, kw
    assert call(T=0) == 0


def test_cache_refusals(m):
    st, ld = m.lib().qgemm_kv4_store, m.lib().qgemm_kv4_load
    ok = dict(k=16, v=16, slots=16, cache=16, T=4, Hkv=2, D=128, ks=256, vs=256, pages=3, page=16)

    def store(**kw):
        return st(*{**ok, **kw}.values(), None)

    def load(**kw):
        a = {**ok, **kw}
        return ld(a["cache"], a["slots"], a["k"], a["v"], a["T"], a["Hkv"], a["D"], a["pages"], a["page"], None)

    for f in (store, load):
        for kw in ({"T": -1}, {"Hkv": 0}, {"pages": 0}, {"page": 12}, {"page": 2048}, {"k": 0}, {"v": 0}, {"slots": 0}, {"cache": 0}):
            assert f(**kw) == -1, kw
        assert f(D=96) == -3 and f(pages=1 << 27) == -3
        for kw in ({"k": 24}, {"v": 24}, {"slots": 18}, {"cache": 24}):
            assert f(**kw) == -2, kw
        assert f(T=0) == 0
    assert store(ks=255) == -1 and store(vs=128) == -1 and store(ks=260) == -2 and store(vs=257) == -2


def test_attention_packed_refusals(m):
    f = m.lib().qgemm_attention_packed
    ok = dict(q=16, k=16, v=16, cu=16, o=16, T=8, R=2, H=4, Hkv=2, D=64, qs=256, ks=128, vs=128, os=256, scale=0.1)

    def call(**kw):
        return f(*{**ok, **kw}.values(), None)

    for kw in ({"T": -1}, {"R": -1}, {"H": 3}, {"Hkv": 0}, {"H": 0}, {"scale": 0.0}, {"scale": float("nan")}, {"scale": float("inf")},
               {"q": 0}, {"k": 0}, {"v": 0}, {"cu": 0}, {"o": 0}, {"qs": 248}, {"ks": 120}, {"vs": 120}, {"os": 248}):
        assert call(**kw) == -1, kw
    assert call(D=96) == -3 and call(T=1 << 24) == -3
    assert call(T=1 << 20, ks=1 << 11) == -3 and "4 GiB" in m.last_error()
    for kw in ({"q": 24}, {"k": 8}, {"v": 18}, {"o": 4}, {"cu": 18}, {"qs": 260}, {"ks": 132}, {"vs": 129}, {"os": 258}):
        assert call(**kw) == -2, kw
    assert call(T=0) == 0 and call(R=0) == 0


def test_attention_packed_refuses_strides_whose_product_with_the_rows_passes_64_bits(m):
    f = m.lib().qgemm_attention_packed
    for T in (1, 16, 384, 896):                     # 129, 144, 512 and 1024 strides with the block past the end
        for stride in (1 << 60, 1 << 59, 1 << 55, 1 << 54):
            for at in range(3):
                s = [256, 128, 128]
                s[at] = stride
                assert f(16, 16, 16, 16, 16, T, 2, 4, 2, 64, *s, 256, 0.1, None) == -3, (T, stride, at)
                assert "4 GiB" in m.last_error()


def test_attention_kv4_refusals(m):
    f, g = m.lib().qgemm_attention_kv4, m.lib().qgemm_attention_kv4_workspace
    ok = dict(q=16, cache=16, tab=16, kv=16, cu=16, o=16, ws=16, bytes=1 << 40, T=8, R=2, H=4, Hkv=2, D=64, W=4, pages=9, page=16, qs=256,
              scale=0.1)

    def call(**kw):
        return f(*{**ok, **kw}.values(), None)

    for kw in ({"T": -1}, {"R": -1}, {"W": -1}, {"H": 3}, {"Hkv": 0}, {"pages": 0}, {"page": 20}, {"scale": -1.0}, {"scale": float("nan")},
               {"q": 0}, {"cache": 0}, {"tab": 0}, {"kv": 0}, {"o": 0}, {"ws": 0}, {"qs": 248}, {"cu": 0}):
        assert call(**kw) == -1, kw
    assert call(bytes=100) == -1 and "workspace" in m.last_error()
    for kw in ({"D": 256}, {"T": 1 << 24}, {"W": (1 << 26) + 1}, {"R": (1 << 20) + 1}, {"pages": 1 << 27}):
        assert call(**kw) == -3, kw
    for kw in ({"q": 24}, {"cache": 24}, {"o": 24}, {"ws": 24}, {"tab": 18}, {"kv": 18}, {"cu": 18}, {"qs": 260}):
        assert call(**kw) == -2, kw
    assert call(T=0) == 0 and call(R=0) == 0
    n = ctypes.c_int64(-1)
    assert g(8, 2, 4, 2, 64, 4, 16, None) == -1
    assert g(8, 2, 4, 3, 64, 4, 16, ctypes.byref(n)) == -1 and g(8, 2, 4, 2, 80, 4, 16, ctypes.byref(n)) == -3
    assert g(0, 2, 4, 2, 64, 4, 16, ctypes.byref(n)) == 0 and n.value == 0
    assert g(8, 2, 4, 2, 64, 4, 16, ctypes.byref(n)) == 0 and 0 < n.value < 1 << 20
    assert g(1 << 16, 1 << 12, 16, 2, 128, 1 << 16, 16, ctypes.byref(n)) == 0 and 0 < n.value < 1 << 27
    assert g(1 << 16, 1 << 20, 16, 2, 128, 1 << 16, 16, ctypes.byref(n)) == -3 and "together" in m.last_error()


SCALED = [("none", {}), ("linear", {"factor": 4.0}), ("llama3", {"factor": 8.0, "low": 1.0, "high": 4.0, "length": 8192.0}),
          ("yarn", {"factor": 16.0, "low": 1.0, "high": 32.0, "length": 4096.0}), ("yarn", {"factor": 2.0, "low": 1.0, "high": 1.0001, "length": 100.0})]


@pytest.mark.parametrize("rot", [2, 6, 64, 128, 512])
@pytest.mark.parametrize("scaling,kw", SCALED)
def test_frequencies(m, rot, scaling, kw):
    f, gain = m.rope_frequencies(rot, 500000.0, scaling, device="cpu", **kw)
    ref, ref_gain = oracle.rope_frequencies(rot, 500000.0, scaling, **kw)
    assert f.shape == (rot // 2,) and np.allclose(f.numpy(), ref, rtol=1e-12) and gain == pytest.approx(ref_gain, rel=2.0 ** -23)


def test_frequency_refusals(m):
    for kw in ({"rot": 0}, {"rot": 7}, {"rot": 514}, {"rot": -2}, {"base": 1.0}, {"base": float("nan")}, {"base": float("inf")},
               {"scaling": "linear", "factor": 0.5}, {"scaling": "linear", "factor": float("nan")},
               {"scaling": "llama3", "factor": 2.0, "low": 4.0, "high": 1.0, "length": 100.0},
               {"scaling": "yarn", "factor": 2.0, "low": 0.0, "high": 1.0, "length": 100.0},
               {"scaling": "yarn", "factor": 2.0, "low": 1.0, "high": 32.0, "length": 0.0}):
        with pytest.raises(m.QGemmError):
            m.rope_frequencies(**{"rot": 64, "base": 10000.0, "device": "cpu", **kw})
    with pytest.raises(ValueError):
        m.rope_frequencies(64, scaling="ntk", device="cpu")


def test_calls_go_to_the_device_of_their_tensors(m, monkeypatch):
    """Tensors of another device than the current one: that device is made current around the call and its stream taken;
    tensors of two devices are refused."""
    import torch

    class Fake:
        def __init__(self, dev):
            self.dev = dev

        def get_device(self):
            return self.dev

    seen, current = [], [0]

    class Guard:
        def __init__(self, dev):
            self.dev = dev

        def __enter__(self):
            self.was, current[0] = current[0], self.dev

        def __exit__(self, *a):
            current[0] = self.was

    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(m, "_current_device", lambda: current[0])
    monkeypatch.setattr(m, "_stream_of", lambda dev: 100 + dev)
    for dev in (0, 3):
        m._enqueue(lambda *x: seen.append((current[0], *x)) or 0, m._device(Fake(dev), Fake(dev)), 7)
    assert seen == [(0, 7, 100), (3, 7, 103)] and current == [0]
    with pytest.raises(ValueError, match="one device"):
        m._device(Fake(0), Fake(1))


def test_sizes_past_31_bits_are_refused_not_cut(m):
    m._sizes(1, (1 << 31) - 1)
    with pytest.raises(ValueError, match="2\\^31"):
        m._sizes(1, 1 << 31)


def test_rotated_sizes_past_31_bits_are_refused_not_cut(m):
    for rot in ((1 << 32) + 64, 64 - (1 << 32), -(1 << 31)):
        with pytest.raises(ValueError, match="2\\^31"):
            m.rope_frequencies(rot, device="cpu")


def test_binding_refuses_host_tensors_and_shapes(m):
    import torch
    i = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    c = torch.zeros(m.kv4_cache_shape(2, 2, 64, 16), dtype=torch.uint8)
    for call in (lambda: m.kv_plan(i, i, i[:, None], i, 16, 4), lambda: m.rope(x, i, torch.ones(32, dtype=torch.float64), 1),
                 lambda: m.kv4_store(x, x, i, c), lambda: m.kv4_load(c, i, 64), lambda: m.attention_packed(x, x, x, i),
                 lambda: m.attention_kv4(x, c, i[:, None], i)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    assert m.kv4_cache_shape(3, 2, 128, 16) == (3, 2, 16 * 136)
