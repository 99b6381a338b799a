"""GPU: ``kv_reorder`` and ``kv4_copy`` against the oracle's integers: every table, list and byte equal."""
import numpy as np
import pytest

import oracle
from gpu_util import torch_or_skip
from serve_util import dev_i32

pytestmark = pytest.mark.gpu


def q():
    import paper_2607_19438_amd as m
    return m


def history(rng, R, B, page, most, width=None):
    """(table, kv_len, pages) of beams that share their first pages and, two and two, some of the later ones."""
    kv, rows, at = [], [], 0
    for _ in range(R):
        n = [int(rng.integers(0, most + 1))] * B if rng.random() < 0.7 else [int(x) for x in rng.integers(0, most + 1, B)]
        common = min(n) // page * int(rng.random() < 0.8)
        table = []
        for b in range(B):
            need = -(-n[b] // page)
            row = list(range(at, at + need))
            at += need
            row[:common] = table[0][:common] if b else row[:common]
            if b % 2:
                fork = int(rng.integers(0, min(n[b], n[b - 1]) // page + 1))
                row[:fork] = table[b - 1][:fork]
            table.append(row)
        kv += n
        rows += table
    W = max([len(r) for r in rows] + [1]) + 1 if width is None else width
    ids = rng.permutation(at + 7)
    out = np.full((R * B, W), -1, dtype=np.int64)
    for i, row in enumerate(rows):
        row = row[:W]
        out[i, :len(row)] = ids[row]
    return out, np.array(kv), at + 7


def run(torch, table, kv, parents, free, page, keep=None, released=None, out=None):
    return q().kv_reorder(dev_i32(torch, table), dev_i32(torch, kv), dev_i32(torch, parents), dev_i32(torch, free), page,
                          None if keep is None else dev_i32(torch, keep), released, out)


def check(torch, table, kv, parents, free, page, keep=None, released=None):
    p = run(torch, table, kv, parents, free, page, keep, released)
    new, length, src, dst, used, gone = oracle.kv_reorder(table, kv, parents, free, page, keep)
    assert p.block_table.cpu().tolist() == new.tolist()
    assert p.kv_len.cpu().tolist() == length and p.src.cpu().tolist() == src and p.dst.cpu().tolist() == dst
    assert p.used.item() == used and p.n_released.item() == len(gone)
    Q = table.size if released is None else released
    assert p.released.cpu().tolist() == (gone + [-1] * Q)[:Q]
    return p


@pytest.mark.parametrize("R,B,page,most,seed", [
    (1, 1, 16, 50, 0), (1, 4, 16, 16, 1), (3, 4, 16, 100, 2), (2, 8, 64, 500, 3), (5, 3, 32, 31, 4), (1, 64, 16, 300, 5), (700, 3, 16, 60, 6),
    (2, 5, 16, 9000, 7), (40, 16, 128, 1000, 8), (1, 2, 1024, 5000, 9)])
def test_random(R, B, page, most, seed):
    torch = torch_or_skip()
    rng = np.random.default_rng(seed)
    table, kv, pages = history(rng, R, B, page, most)
    for kind in range(4):
        parents = [rng.integers(0, B, (R, B)), np.tile(np.arange(B), (R, 1)), np.zeros((R, B), int), rng.integers(-1, B, (R, B))][kind]
        parents[rng.random(R) < 0.1] = -1
        free = pages + np.arange(R * B)
        keep = None if kind % 2 else rng.integers(0, table.shape[1] + 2, R)
        check(torch, table, kv, parents, free, page, keep)


def test_by_hand():
    """Three beams of 18, 18 and 32 tokens in pages of 16; the second has all children."""
    torch = torch_or_skip()
    table = [[5, 6, 9], [5, 7, 9], [8, 2, 9]]
    p = check(torch, np.array(table), [18, 18, 32], [[1, 1, 1]], [11, 12, 13], 16)
    assert p.block_table.cpu().tolist() == [[5, 7, -1], [5, 11, -1], [5, 12, -1]]
    assert p.src.cpu().tolist() == [-1, 7, 7] and p.dst.cpu().tolist() == [-1, 11, 12] and p.released.cpu().tolist()[:4] == [8, 6, 2, -1]
    p = check(torch, np.array(table), [18, 18, 32], [[2, 2, 2]], [11, 12, 13], 16)        # full pages need no copy
    assert p.used.item() == 0 and p.released.cpu().tolist()[:4] == [5, 6, 7, -1]


def test_short_lists_and_wrong_numbers():
    torch = torch_or_skip()
    rng = np.random.default_rng(10)
    table, kv, pages = history(rng, 4, 5, 16, 200)
    parents = rng.integers(0, 5, (4, 5))
    for free in ([], [pages], [pages, pages + 1, pages + 2]):
        check(torch, table, kv, parents, free, 16)
    for Q in (0, 1, 10):
        check(torch, table, kv, parents, pages + np.arange(20), 16, released=Q)
    parents[0] = [-5, 5, 2 ** 31 - 1, -2 ** 31, 3]
    check(torch, table, kv, parents, pages + np.arange(20), 16, keep=[-3, 2 ** 31 - 1, 0, 4])
    kv = kv.copy()
    kv[::3] = [-1, 2 ** 31 - 1, 100000, -2 ** 31, 0, 33, 1000][:len(kv[::3])]           # more tokens than the table has pages for
    check(torch, table, kv, parents, pages + np.arange(20), 16)
    wild = table.copy()
    wild[rng.random(table.shape) < 0.3] = -7
    check(torch, wild, kv, parents, pages + np.arange(20), 16)


def test_no_rows_no_columns():
    torch = torch_or_skip()
    p = run(torch, np.zeros((0, 3)), [], np.zeros((0, 2)), [], 16)
    assert p.block_table.shape == (0, 3)
    p = check(torch, np.zeros((4, 0), int), [0, 0, 5, 0], [[0, 0], [1, 0]], [3], 16)
    assert p.n_released.item() == 0


def test_result_written_into_an_earlier_one():
    torch = torch_or_skip()
    rng = np.random.default_rng(11)
    table, kv, pages = history(rng, 3, 4, 16, 100)
    parents = rng.integers(0, 4, (3, 4))
    a = run(torch, table, kv, parents, pages + np.arange(12), 16)
    b = run(torch, table, kv, np.zeros((3, 4)), pages + np.arange(12), 16, out=run(torch, table, kv, parents, [], 16))
    c = run(torch, table, kv, parents, pages + np.arange(12), 16, out=b)
    assert c is b
    for name in q().KvReorder.__slots__:
        assert torch.equal(getattr(a, name), getattr(c, name))
    with pytest.raises(q().QGemmError, match="overlap"):
        q().kv_reorder(c.block_table, c.kv_len, dev_i32(torch, parents), dev_i32(torch, [1]), 16, out=c)


def test_graph_replays():
    torch = torch_or_skip()
    rng = np.random.default_rng(12)
    table, kv, pages = history(rng, 6, 4, 16, 300)
    free = dev_i32(torch, pages + np.arange(24))
    t, n, par = dev_i32(torch, table), dev_i32(torch, kv), dev_i32(torch, np.zeros((6, 4)))
    cache = torch.randint(0, 256, (pages + 24, 2, 16 * 68), dtype=torch.uint8, device="cuda")
    m = q()
    m.kv_reorder(t, n, par, free, 16)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p = m.kv_reorder(t, n, par, free, 16)
        m.kv4_copy(cache, p.src, p.dst)
    for k in range(4):
        parents = rng.integers(-1, 4, (6, 4))
        par.copy_(dev_i32(torch, parents))
        want = cache.clone()
        g.replay()
        e = run(torch, table, kv, parents, pages + np.arange(24), 16)
        for name in m.KvReorder.__slots__:
            assert torch.equal(getattr(e, name), getattr(p, name))
        m.kv4_copy(want, e.src, e.dst)
        assert torch.equal(cache, want)


@pytest.mark.parametrize("pages,Hkv,D,page", [(9, 1, 64, 16), (7, 8, 128, 64), (5, 3, 64, 1024)])
def test_copy(pages, Hkv, D, page):
    torch = torch_or_skip()
    m = q()
    cache = torch.randint(0, 256, m.kv4_cache_shape(pages, Hkv, D, page), dtype=torch.uint8, device="cuda")
    src, dst = [0, -1, 3, 0, pages, 2, 2 ** 31 - 1, 1], [pages - 1, 2, -1, 4, 2, pages, 1, 1]
    want = cache.clone()
    for s, d in zip(src, dst):
        if 0 <= s < pages and 0 <= d < pages:
            want[d] = cache[s]
    for head in (None, D):
        got = cache.clone()
        m.kv4_copy(got, dev_i32(torch, src), dev_i32(torch, dst), head)
        assert torch.equal(got, want)
    m.kv4_copy(got, dev_i32(torch, []), dev_i32(torch, []))
    assert torch.equal(got, want)


def test_copy_past_32_bits():
    torch = torch_or_skip()
    m = q()
    pages = (5 << 30) // (2 * 16 * 136)
    big = torch.zeros(m.kv4_cache_shape(pages, 2, 128, 16), dtype=torch.uint8, device="cuda")
    big[pages - 1] = torch.randint(0, 256, big.shape[1:], dtype=torch.uint8, device="cuda")
    m.kv4_copy(big, dev_i32(torch, [pages - 1, pages - 1]), dev_i32(torch, [pages - 2, 3]))
    assert torch.equal(big[pages - 2], big[pages - 1]) and torch.equal(big[3], big[pages - 1])
    assert not big[pages - 3].any() and not big[2].any() and not big[4].any()
    del big
