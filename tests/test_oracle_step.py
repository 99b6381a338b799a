"""Pins of the oracle of the operators for many continuations and tenants (``oracle/step_oracle.py``): values derived by hand,
closed forms, other definitions of the same thing, and planted mistakes that the pins catch. No test here touches a GPU."""
import math

import numpy as np
import pytest

import oracle
from oracle import step_oracle as so


def attention_case(seed=0):
    rng = np.random.default_rng(seed)
    page, D, kv, new = 16, 64, [150, 139, 20, 70], [2, 1, 1, 3]
    pages = 40
    k, v = rng.standard_normal((pages * page, 2, D)), rng.standard_normal((pages * page, 2, D))
    table = rng.permutation(pages)[:40].reshape(4, 10)
    return rng.standard_normal((7, 4, D)), k, v, table, kv, [0, 2, 3, 4, 7], page


def pin_shared_is_cached_attention_with_the_leaders_pages():
    q, k, v, table, kv, cu, page = attention_case()
    o, a = so.shared_attention(q, k, v, table, kv, cu, [0, 2, 4], [140, 17], page, 0.1)
    same = table.copy()
    same[1, :8] = table[0, :8]                        # 140 and the shortest history of 138: 128 keys, 8 pages
    want, absv = oracle.cached_attention(q, k, v, same, kv, cu, page, 0.1)
    assert np.allclose(o, want, rtol=1e-12, atol=0) and np.allclose(a, absv, rtol=1e-12, atol=0)


def pin_shared_keys():
    kv, cu = [150, 139, 20, 70], [0, 2, 3, 4, 7]
    assert so.shared_keys(kv, cu, [0, 2, 4], [1000, 1000], 10, 16) == [(0, 128), (2, 0)]        # 138; 19
    assert so.shared_keys(kv, cu, [0, 1, 1, 2, 4], [-3, 5, 127, 64], 10, 16) == [(0, 0), (None, 0), (1, 64), (2, 0)]
    assert so.shared_keys([300, 300], [0, 0, 4], [0, 2], [290], 10, 16) == [(1, 128)]           # the table's 160
    assert so.shared_keys([128, 200], [0, 1, 2], [0, 2], [500], 100, 16) == [(0, 64)]           # 127 before the new token
    assert so.shared_keys([300, 5], [0, 0, 4], [0, 2], [290], 10, 16) == [(1, 0)]
    assert so.shared_keys([30, 330], [0, 0, 4], [0, 2], [290], 100, 16) == [(1, 256)]           # a request of no rows does not count


def pin_beams_by_hand():
    # beam 0: odds 1 : 2 : 1, beam 1: 6 : 1 : 1, worth a third of beam 0
    logits = np.log([[1, 2, 1], [6, 1, 1]])
    s, p, t = so.beam_select(logits, np.array([[0.0, -math.log(3)]]), 5)
    assert p.tolist() == [[0, 0, 0, 1, 1]] and t.tolist() == [[1, 0, 2, 0, 1]]
    assert np.allclose(np.exp(s), [[1 / 2, 1 / 4, 1 / 4, 1 / 4, 1 / 24]])
    s, p, t = so.beam_select(logits, np.array([[0.0, -math.log(3)]]), 7, np.array([[False, True]]), 2)
    assert p.tolist() == [[0, 1, 0, 0, -1, -1, -1]] and t.tolist() == [[1, 2, 0, 2, 2, 2, 2]]
    assert np.allclose(np.exp(s), [[1 / 2, 1 / 3, 1 / 4, 1 / 4, 0, 0, 0]])


def pin_beams_sum_to_one():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 50)) * 4
    val = so.beam_values(x, np.zeros(3), None, 0)
    assert np.allclose(np.exp(val).sum(1), 1.0, rtol=1e-13)
    assert np.allclose(so.beam_values(x + 700, np.zeros(3), None, 0), val, atol=1e-10)
    s, p, t = so.beam_select(x, np.zeros((1, 3)), 150)
    assert sorted(zip(p[0], t[0])) == [(b, v) for b in range(3) for v in range(50)] and np.all(np.diff(s[0]) <= 0)


def pin_no_candidates():
    x = np.zeros((5, 4))
    x[0, 1], x[1, 2], x[2] = np.nan, np.inf, -np.inf
    x[3, :3] = -np.inf
    s, p, t = so.beam_select(x, np.array([[0.0, 0.0, 0.0, -1.0, -np.inf]]), 3, None, 2)
    assert p.tolist() == [[3, -1, -1]] and t.tolist() == [[3, 2, 2]] and s.tolist() == [[-1.0, -np.inf, -np.inf]]


def pin_reorder_by_hand():
    # three beams of 18, 18 and 32 tokens in pages of 16, of which the first two share their first page
    table = [[5, 6, 9], [5, 7, 9], [8, 2, 9]]
    new, n, src, dst, used, gone = so.kv_reorder(table, [18, 18, 32], [[1, 1, 1]], [11, 12, 13], 16)
    assert new.tolist() == [[5, 7, -1], [5, 11, -1], [5, 12, -1]] and n == [18, 18, 18]
    assert src == [-1, 7, 7] and dst == [-1, 11, 12] and used == 2 and gone == [8, 6, 2]
    new, n, src, dst, used, gone = so.kv_reorder(table, [18, 18, 32], [[2, 2, -1]], [], 16, keep=[1])
    assert new.tolist() == [[8, 2, -1], [8, 2, -1], [-1, -1, -1]] and n == [32, 32, 0] and used == 0 and gone == [6, 7]
    assert so.kv_reorder(table, [18, 18, 32], [[2, 2, -1]], [], 16)[5] == [5, 6, 7]
    new, n, src, dst, used, gone = so.kv_reorder(table, [18, 18, 32], [[0, 0, 0]], [11], 16)
    assert new.tolist() == [[5, 6, -1], [5, 11, -1], [5, -1, -1]] and dst == [-1, 11, -1] and used == 2 and gone == [8, 7, 2]


def pin_reorder_pages_are_in_one_place():
    """Every old page is held by some new row or listed once; fresh pages are apart; no partly filled page is in two rows."""
    rng = np.random.default_rng(2)
    for _ in range(20):
        B, page = 4, 16
        n = [int(rng.integers(1, 100))] * B
        have = -(-n[0] // page)
        table = np.arange(B * have).reshape(B, have)
        table[1:, :have // 2] = table[0, :have // 2]
        par = rng.integers(-1, B, (1, B))
        new, length, src, dst, used, gone = so.kv_reorder(table, n, par, list(range(1000, 1004)), page)
        old, now = set(table.ravel().tolist()), set(new[new >= 0].tolist())
        assert now - old == set(d for d in dst if d >= 0) and len(gone) == len(set(gone)) and set(gone) == old - now
        if n[0] % page:
            last = [new[k, have - 1] for k in range(B) if par[0, k] >= 0]
            assert len(last) == len(set(last))


def pin_adapters():
    rng = np.random.default_rng(3)
    x, y = rng.standard_normal((6, 8)), rng.standard_normal((6, 5))
    a, b = rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 5, 2))
    out = so.adapters(y, x, a, b, [2, -1, 0, 3], np.array([1.0, 2.0, -0.5]), [0, 2, 3, 5, 6])
    for m, i, g in ((0, 2, -0.5), (1, 2, -0.5), (3, 0, 1.0), (4, 0, 1.0)):
        assert np.allclose(out[m] - y[m], [g * sum(b[i, c, j] * a[i, j, k] * x[m, k] for j in range(2) for k in range(8)) for c in range(5)])
    assert np.array_equal(out[[2, 5]], y[[2, 5]])
    assert np.array_equal(so.adapters(y, x, a, b, [0, 1, 2, 0, 1, 2]), so.adapters(y, x, a, b, [0, 1, 2, 0, 1, 2], np.ones(3), range(7)))
    tol = so.adapter_tolerance(y, x, a, b, [2, -1, 0, 3], np.array([1.0, 2.0, -0.5]), [0, 2, 3, 5, 6])
    assert (tol[[0, 1, 3, 4]] > 0).all() and not tol[[2, 5]].any() and tol.max() < 1e-4


PINS = [pin_shared_is_cached_attention_with_the_leaders_pages, pin_shared_keys, pin_beams_by_hand, pin_beams_sum_to_one, pin_no_candidates,
        pin_reorder_by_hand, pin_reorder_pages_are_in_one_place, pin_adapters]


@pytest.mark.parametrize("pin", PINS, ids=[p.__name__[4:] for p in PINS])
def test_pin(pin):
    pin()


def mutant(name, old, new):
    """The oracle's function with one piece of its source replaced."""
    import inspect
    src = inspect.getsource(getattr(so, name))
    assert src.count(old) >= 1, (name, old)
    scope = dict(so.__dict__)
    exec(src.replace(old, new, 1), scope)
    return scope[name]


@pytest.mark.parametrize("name,old,new", [
    ("shared_keys", "// 64 * 64", "// 1"), ("shared_keys", "- int(cu[r + 1] - cu[r])", ""), ("shared_keys", "[int(prefix[g]), W * page]", "[int(prefix[g])]"),
    ("shared_keys", "has[0]", "groups[g]"), ("shared_attention", "owner if p < common else r", "r"), ("shared_attention", "owner if p < common else r", "owner"),
    ("shared_attention", "p < common", "p <= common"), ("shared_attention", "- n + i + 1", "- n + i"),
    ("beam_values", "float(scores[b]) + ", ""), ("beam_values", "top + math.log", "math.log"), ("beam_values", "out[b, end] = scores[b]", "pass"),
    ("beam_select", "i // V, i % V", "i % V, i // V"), ("beam_select", "-val)", "val)"),
    ("kv_reorder", "and size[old] % page", ""), ("kv_reorder", "            seen.add(p)\n", ""), ("kv_reorder", "and at not in held", ""),
    ("kv_reorder", "                    held.add(at)\n", ""), ("kv_reorder", "used < len(free) and last", "last"), ("kv_reorder", "j < have[r * B + b] and", ""),
    ("adapters", "(1.0 if gain is None else float(gain[i])) * ", ""), ("adapters", "0 <= i < len(a)", "i < len(a)"),
])
def test_pins_bite(monkeypatch, name, old, new):
    monkeypatch.setattr(so, name, mutant(name, old, new))
    for other in ("shared_attention", "beam_select"):      # the copies of functions that call the changed one by name
        if name in ("shared_keys", "beam_values"):
            fn = getattr(so, other)
            scope = dict(fn.__globals__, **{name: getattr(so, name)})
            import types
            monkeypatch.setattr(so, other, types.FunctionType(fn.__code__, scope, other, fn.__defaults__))
    failed = 0
    with np.errstate(all="ignore"):
        for pin in PINS:
            try:
                pin()
            except Exception:
                failed += 1
    assert failed
