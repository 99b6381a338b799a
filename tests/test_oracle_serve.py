"""Pins of the serving oracle (``oracle/serve_oracle.py``): values derived by hand, closed forms and other
definitions of the same thing. No test here touches a GPU."""
import math

import numpy as np
import pytest

import oracle
from oracle import serve_oracle as so


def test_plan_by_hand():
    # pages of 16: request 0 has 15 tokens (one page) and gets 3 (a second page from its third token on);
    # request 1 nothing; request 2 starts with 33 tokens (three pages); request 3 fills its page exactly
    table = [[7, -5, -5], [-5, -5, -5], [-5, -5, -5], [9, -5, -5]]
    cu, pos, slots, tab, total, used = oracle.kv_plan([15, 0, 0, 8], [3, 0, 33, 8], table, [20, 21, 22, 23, 24], 16, 46)
    assert list(cu) == [0, 3, 3, 36, 44] and list(total) == [18, 0, 33, 16] and list(used) == [4]
    assert list(pos[:3]) == [15, 16, 17] and list(slots[:3]) == [7 * 16 + 15, 20 * 16, 20 * 16 + 1]
    assert list(slots[3:20]) == [21 * 16 + i for i in range(16)] + [22 * 16] and slots[35] == 23 * 16
    assert list(slots[36:]) == [9 * 16 + i for i in range(8, 16)] + [-1, -1] and list(pos[44:]) == [0, 0]
    assert tab.tolist() == [[7, 20, -5], [-5, -5, -5], [21, 22, 23], [9, -5, -5]]


def test_plan_short_of_pages_and_width():
    cu, pos, slots, tab, total, used = oracle.kv_plan([0, 0], [40, 40], [[-2] * 2, [-2] * 2], [3, 4, 5, 6], 16, 80)
    assert used[0] == 6
    assert list(slots[32:40]) == [-1] * 8                      # past the table's two pages
    assert tab[0].tolist() == [3, 4] and tab[1].tolist() == [6, -1]
    assert list(slots[40:56]) == [6 * 16 + i for i in range(16)] and list(slots[56:]) == [-1] * 24


def test_frequencies():
    f, g = oracle.rope_frequencies(8, 10000.0)
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001], rtol=1e-14) and g == 1.0
    assert np.allclose(oracle.rope_frequencies(8, 10000.0, "linear", 4.0)[0], f / 4, rtol=1e-15)
    # one pair turns more than `high` times over the length, one between, two fewer than `low` times
    L = 2 * math.pi * 30
    f3, _ = oracle.rope_frequencies(8, 10000.0, "llama3", 8.0, 1.0, 4.0, L)      # turns 30, 3, 0.3, 0.03
    w = (3.0 - 1) / 3
    assert np.allclose(f3, [1.0, 0.1 * (w + (1 - w) / 8), 0.01 / 8, 0.001 / 8], rtol=1e-14)
    # length 2 pi 500: pair i makes 500 / 10^i turns; 100 turns lie behind pair 0 and 1 turn before pair 3
    fy, gy = oracle.rope_frequencies(8, 10000.0, "yarn", 16.0, 1.0, 100.0, 2 * math.pi * 500)
    assert np.allclose(fy, [1.0, 0.1 * (2 / 3 + 1 / 48), 0.01 * (1 / 3 + 2 / 48), 0.001 / 16], rtol=1e-14)
    assert gy == pytest.approx(0.1 * math.log(16) + 1)


@pytest.mark.parametrize("inter", [False, True])
def test_rope_closed_forms(inter):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 3, 12))
    f = np.array([math.pi / 2, 0.3, 0.0])
    pos = [0, 1, 2, 3, 1000001]
    y = oracle.rope(x, pos, f, 2, inter, 1.5)
    assert np.array_equal(y[:, 2], x[:, 2]) and np.array_equal(y[..., 6:], x[..., 6:])     # other heads and dimensions
    assert np.allclose(y[0, :2, :6], 1.5 * x[0, :2, :6], rtol=1e-15)                       # position 0
    a, b = (0, 1) if inter else (0, 3)
    assert np.allclose(y[1, :2, a], -1.5 * x[1, :2, b]) and np.allclose(y[1, :2, b], 1.5 * x[1, :2, a])   # a quarter turn
    c, d = (2, 3) if inter else (1, 4)
    th = 0.3 * 1000001
    assert np.allclose(y[4, 0, c], 1.5 * (x[4, 0, c] * math.cos(th) - x[4, 0, d] * math.sin(th)), atol=1e-9)
    assert np.allclose(y[4, 0, d], 1.5 * (x[4, 0, c] * math.sin(th) + x[4, 0, d] * math.cos(th)), atol=1e-9)


def test_quantise_by_hand():
    b = np.zeros(32)
    b[:12] = [6.0, -6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.2, 0.3, -0.0]
    codes, E = oracle.quantise(b)                      # largest 6: levels as they are
    assert E == 127
    assert codes[:12].tolist() == [7, 15, 0, 2, 2, 4, 4, 6, 6, 8, 1, 8]
    b[0] = 7.0                                         # to 8 at two significant bits: the next power of two
    b[1] = 0.0
    codes, E = oracle.quantise(b)
    assert E == 128 and codes[0] == 6                  # 3.5 / level step 1: a tie, to 4
    b[0] = 6.99
    assert oracle.quantise(b)[1] == 127
    assert oracle.quantise(np.zeros(32))[1] == 1
    codes, E = oracle.quantise(np.full(32, 3.3895e38))          # no further than 6 * 2^125, the last below bf16's end
    assert E == 252 and np.all(codes == 7)
    for bad in (np.inf, -np.inf, np.nan):
        b[5] = bad
        assert oracle.quantise(b)[1] == 255


def test_quantised_error_is_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((200, 32)) * np.exp(rng.standard_normal((200, 1)) * 5)
    codes, E = oracle.quantise(x)
    y = so.dequantise(codes, E)
    a = np.abs(x) / 2.0 ** (E.astype(float) - 127)[:, None]
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    assert np.all(np.abs(x - y) / 2.0 ** (E.astype(float) - 127)[:, None] <= step / 2 + 1e-12)
    assert a.max() <= 7.0


def test_cache_layout_and_round_trip():
    D, page, Hkv = 64, 16, 2
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, 3 * page, Hkv, D))
    cache = oracle.encode_cache(k, v, page)
    assert cache.shape == (3, Hkv, page * 68)
    kd, vd = oracle.decode_cache(cache, D)
    for x, d in ((k, kd), (v, vd)):
        codes, E = oracle.quantise(x.reshape(-1, Hkv, 2, 32))
        assert np.array_equal(d, so.dequantise(codes, E).reshape(d.shape))
    # slot 20 (page 1, place 4), head 1, value element 33: the low or high nibble of byte 16 of its row
    by = cache[1, 1, (page + 4) * 32 + 16]
    codes, E = oracle.quantise(v[20, 1].reshape(2, 32))
    assert by == codes[1, 0] | codes[1, 1] << 4
    assert cache[1, 1, page * 64 + (page + 4) * 2 + 1] == E[1]


def test_packed_attention_is_prefill_attention_of_each_prompt():
    rng = np.random.default_rng(3)
    T, H, Hkv, D = 11, 4, 2, 8
    q, k, v = rng.standard_normal((T, H, D)), rng.standard_normal((T, Hkv, D)), rng.standard_normal((T, Hkv, D))
    o, _ = oracle.packed_attention(q, k, v, [0, 4, 4, 9], 0.4)
    for c0, c1 in ((0, 4), (4, 9)):
        for h in range(H):
            s = np.einsum("id,jd->ij", q[c0:c1, h], k[c0:c1, h // 2]) * 0.4
            s[np.triu_indices(c1 - c0, 1)] = -np.inf
            p = np.exp(s)
            assert np.allclose(o[c0:c1, h], (p / p.sum(1, keepdims=True)) @ v[c0:c1, h // 2])
    assert np.all(o[9:] == 0)


def test_cached_attention_limits():
    rng = np.random.default_rng(4)
    page, D = 16, 64
    k, v = rng.standard_normal((2, 4 * page, 1, D))
    q = rng.standard_normal((5, 2, D))
    table = [[2, 1], [3, 7]]
    o, _ = oracle.cached_attention(q, k, v, table, [1, 17], [0, 2, 5], page, 0.1)
    assert np.all(o[0] == 0)                              # position -1
    assert np.allclose(o[1], v[32, 0])                    # the only key
    assert np.isfinite(o[2:4]).all() and np.isnan(o[4]).all()       # the last row needs page 7 of 4
    ks = np.concatenate([k[48:64, 0]])
    p = np.exp(ks[:15] @ q[2, 1] * 0.1)
    assert np.allclose(o[2, 1], p @ v[48:63, 0] / p.sum())


@pytest.mark.parametrize("mistake", ["tie_down", "no_bump", "nibbles", "scale_index", "strict"])
def test_planted_mistakes_are_seen(mistake, monkeypatch):
    """Each pin above fails for a plausible mistake in the function that it pins."""
    if mistake == "tie_down":
        monkeypatch.setattr(so, "LEVELS", np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 5.0]))
        with pytest.raises(AssertionError):
            test_quantise_by_hand()
    elif mistake == "no_bump":
        real = so.quantise
        monkeypatch.setattr(oracle, "quantise", lambda x: real(np.where(np.abs(x) == 7.0, 6.0, x)))
        with pytest.raises(AssertionError):
            test_quantise_by_hand()
    elif mistake == "nibbles":
        real = so.encode_cache
        monkeypatch.setattr(oracle, "encode_cache", lambda *a: (real(*a) >> 4) | (real(*a) << 4))
        with pytest.raises(AssertionError):
            test_cache_layout_and_round_trip()
    elif mistake == "scale_index":
        real = so.decode_cache
        monkeypatch.setattr(oracle, "decode_cache", lambda c, D: real(np.roll(c, 1, -1), D))
        with pytest.raises(AssertionError):
            test_cache_layout_and_round_trip()
    else:
        real = so.cached_attention
        monkeypatch.setattr(oracle, "cached_attention", lambda q, k, v, t, n, *a: real(q, k, v, t, [x - 1 for x in n], *a))
        with pytest.raises(AssertionError):
            test_cached_attention_limits()
