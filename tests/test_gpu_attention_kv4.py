"""GPU: ``attention_kv4`` against the fp64 oracle on the values that the cache's bytes stand for. Bar: the oracle's
``attn_tolerance`` (2^-7 sum_j p_j |v_j| for the weights' rounding to bf16, 2^-8 |o| for the output's); the
unpacked keys and values are exact in bf16."""
import numpy as np
import pytest

import oracle
from gpu_util import torch_or_skip
from serve_util import bf16, dev_bf16, dev_i32, host_bf16, random_cache, starts, tables

pytestmark = pytest.mark.gpu


def q():
    import paper_2607_19438_amd as m
    return m


def make(kv, new, H, Hkv, D, page, seed=0, pad=0, std=1.0, width=None):
    rng = np.random.default_rng(seed)
    table, pages = tables(rng, kv, page, width=width)
    cache, k, v = random_cache(rng, pages, Hkv, D, page)
    qn, bits = bf16(rng.standard_normal((int(sum(new)) + pad, H, D)) * std)
    return table, cache, k, v, qn, bits, starts(new)


def run(torch, case, kv, cu, scale=None, out=None):
    table, cache, _, _, _, bits, _ = case
    return q().attention_kv4(dev_bf16(torch, bits), torch.from_numpy(cache).cuda(), dev_i32(torch, table), dev_i32(torch, kv),
                             None if cu is None else dev_i32(torch, cu), scale, out=out)


def check(torch, kv, new, H, Hkv, D, page, seed=0, pad=0, std=1.0, rows=None, width=None):
    case = make(kv, new, H, Hkv, D, page, seed, pad, std, width)
    table, cache, k, v, qn, bits, cu = case
    out = torch.full(qn.shape, 9.0, dtype=torch.bfloat16, device="cuda")
    run(torch, case, kv, None if list(new) == [1] * len(new) and not pad else cu, out=out)
    got = host_bf16(torch, out)
    assert np.all(got[cu[-1]:] == 9.0)                       # rows of no request
    scale = D ** -0.5
    if rows is None:
        ref, absv = oracle.cached_attention(qn, k, v, table, kv, cu, page, scale)
        sel = np.arange(cu[-1])
    else:
        ref, absv, sel = np.zeros(qn.shape), np.zeros(qn.shape), np.array(rows)
        for t in rows:
            r = int(np.searchsorted(cu, t, side="right") - 1)
            seen = int(kv[r]) - int(cu[r + 1] - 1 - t)
            kk, vv = oracle.gather_cache(k, v, table[r], seen, page)
            for h in range(H):
                g = h // (H // Hkv)
                s = kk[:, g] @ qn[t, h] * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                ref[t, h], absv[t, h] = p @ vv[:, g], p @ np.abs(vv[:, g])
    worst = oracle.attn_ratio(got[sel], ref[sel], absv[sel])
    print(f"[parity] kv4 {list(kv)[:6]} x {list(new)[:6]} {H}/{Hkv}x{D} page {page}: max |err| / bar = {worst:.3f}", flush=True)
    assert worst <= 1.0
    return out


DECODE = [  # kv lengths, H, Hkv, D, page
    ([1], 1, 1, 64, 16), ([1], 8, 2, 128, 16), ([2, 15, 16, 17], 4, 1, 128, 16), ([31, 32, 33, 127, 128, 129], 4, 4, 64, 32),
    ([300], 6, 2, 128, 64), ([1000, 1, 40], 16, 1, 128, 16), ([129, 513, 257], 32, 4, 64, 128), ([5] * 70, 2, 1, 64, 16),
    ([700], 40, 2, 128, 16), ([90, 1, 260], 66, 1, 64, 256), ([1025], 3, 1, 128, 1024),
]


@pytest.mark.parametrize("kv,H,Hkv,D,page", DECODE)
def test_single_tokens(kv, H, Hkv, D, page):
    check(torch_or_skip(), kv, [1] * len(kv), H, Hkv, D, page, seed=len(kv) + D)


SEVERAL = [  # kv lengths, new tokens, H, Hkv, D, page, rows behind
    ([5], [5], 2, 1, 64, 16, 0), ([40, 9], [3, 9], 4, 2, 128, 16, 2), ([100, 200, 33], [4, 0, 33], 8, 2, 64, 32, 0),
    ([260, 130], [17, 130], 2, 1, 128, 64, 0), ([129, 1, 64], [6, 1, 2], 12, 4, 128, 16, 5), ([300], [70], 4, 1, 64, 16, 0),
    ([0, 7, 0], [0, 1, 0], 2, 2, 128, 16, 3), ([600, 20], [9, 20], 16, 2, 64, 128, 0),
]


@pytest.mark.parametrize("kv,new,H,Hkv,D,page,pad", SEVERAL)
def test_several_tokens(kv, new, H, Hkv, D, page, pad):
    check(torch_or_skip(), kv, new, H, Hkv, D, page, seed=sum(new), pad=pad)


def test_rows_that_see_nothing_are_zero():
    """No key at all, and more new tokens than keys (the first ones are before the cache's start)."""
    torch = torch_or_skip()
    out = check(torch, [0, 3, 0, 40], [1, 5, 2, 1], 4, 2, 128, 16, seed=2)
    assert torch.all(out[0] == 0) and torch.all(out[1:3] == 0) and torch.all(out[6:8] == 0)
    out = check(torch, [0, 0], [1, 1], 2, 1, 64, 16, seed=3)
    assert torch.all(out == 0)


@pytest.mark.parametrize("D,page", [(128, 16), (64, 64)])
def test_long_and_short_together(D, page):
    """A cache long enough to be split over most workgroups, beside short ones: sampled rows."""
    torch = torch_or_skip()
    kv = [20000, 3, 700, 1, 5000, 64]
    check(torch, kv, [1] * 6, 16, 2, D, page, seed=7, rows=range(6))
    check(torch, kv, [4, 2, 5, 1, 3, 6], 16, 2, D, page, seed=8, rows=[0, 3, 4, 5, 6, 10, 11, 12, 14, 20])


@pytest.mark.parametrize("width", [15, 120])
def test_chunks_in_tables_of_either_length(width):
    """Two chunks of prompts; the table's length, not the requests', chooses how many workgroups share them."""
    check(torch_or_skip(), [900, 300], [300, 40], 32, 8, 64, 64, seed=18, rows=[0, 7, 150, 298, 299, 300, 301, 339], width=width)


CHUNKS = [  # kv lengths, new tokens, H, Hkv, D, page, table width: 128 query rows to a tile
    ([900, 500], [400, 433], 32, 8, 128, 16, None), ([1100], [833], 32, 4, 64, 64, 40), ([70, 0, 640, 9], [130, 0, 300, 9], 66, 2, 64, 16, None),
    ([600], [520], 64, 64, 128, 32, None), ([417, 100], [417, 416], 32, 8, 64, 256, 60), ([5000, 64], [800, 40], 32, 8, 128, 128, None),
]


@pytest.mark.parametrize("kv,new,H,Hkv,D,page,width", CHUNKS)
def test_chunks(kv, new, H, Hkv, D, page, width):
    """Every border of a request and some rows between; [417, 100] has rows before the cache's start."""
    cu = starts(new)
    rows = sorted({t for c in cu for t in (c - 1, c, c + 1, c + 31, c + 33) if 0 <= t < cu[-1]} | {cu[-1] // 3, cu[-1] // 2})
    rows = [t for t in rows if kv[int(np.searchsorted(cu, t, side="right") - 1)] - (cu[int(np.searchsorted(cu, t, side="right"))] - 1 - t) > 0]
    out = check(torch_or_skip(), kv, new, H, Hkv, D, page, seed=19, pad=3, rows=rows, width=width)
    for r, n in enumerate(new):
        blind = max(0, n - kv[r])
        assert not out[cu[r]:cu[r] + blind].any()


@pytest.mark.parametrize("D", [64, 128])
def test_what_pages_hold_behind_a_chunk_reaches_nothing(D):
    """As below for tiles of 128 rows: NaN behind the last key changes no bit; NaN keys, values and pages reach the rows
    that see them, a value block its own dimensions only."""
    torch = torch_or_skip()
    kv, new, H, Hkv, page = [470, 450], [430, 420], 32, 8, 16
    case = make(kv, new, H, Hkv, D, page, seed=20)
    table, cache, k, v, qn, bits, cu = case
    clean = run(torch, case, kv, cu)
    n0, sb = page * D, D // 32
    dirty = cache.copy()
    for r in range(2):
        for p in range(kv[r], len(table[r]) * page):
            if table[r, p // page] >= 0:
                at = n0 + (p % page) * sb
                dirty[table[r, p // page], :, at:at + sb] = 255
                dirty[table[r, p // page], :, at + page * sb:at + page * sb + sb] = 255
    assert torch.equal(run(torch, (table, dirty, k, v, qn, bits, cu), kv, cu), clean)
    # request 0: a NaN value block of position 100 (first seen by token 60); request 1: a NaN key of position 200 (170)
    for byte in (255, 254):
        dirty[table[0, 100 // page], :, n0 + (page + 100 % page) * sb + 1] = byte
        dirty[table[1, 200 // page], :, n0 + (200 % page) * sb] = 255
        o = run(torch, (table, dirty, k, v, qn, bits, cu), kv, cu).float()
        c = clean.float()
        assert torch.equal(o[:60], c[:60]) and torch.equal(o[430:600], c[430:600])
        assert torch.isnan(o[60:430, :, 32:64]).all() and torch.isnan(o[600:]).all()
        keep = [i for i in range(D) if not 32 <= i < 64]
        assert torch.equal(o[60:430][..., keep], c[60:430][..., keep])
    wild = table.copy()
    wild[0, 5] = len(cache)                      # positions 80 .. 95: token 40 is the first to see one
    o = run(torch, (wild, cache, k, v, qn, bits, cu), kv, cu).float()
    assert torch.equal(o[:40], clean[:40].float()) and torch.isnan(o[40:430]).all() and torch.equal(o[430:], clean[430:].float())


@pytest.mark.parametrize("kv,new,H,Hkv,D,page", [
    ([37, 5, 130], [4, 5, 1], 4, 2, 128, 16), ([3000, 200, 1], [1, 1, 1], 8, 1, 64, 16), ([900, 33], [30, 17], 16, 2, 64, 32),
    ([470, 450], [430, 420], 32, 8, 128, 16), ([2000, 700], [600, 240], 32, 8, 64, 16)])
def test_table_entries_behind_the_pages_of_a_request_may_be_anything(kv, new, H, Hkv, D, page):
    """Single and several tokens and tiles of 128 rows: entries that look-ups ahead of the keys may fetch, of either sign,
    just outside the pool, far outside and inside it."""
    torch = torch_or_skip()
    need = [-(-n // page) for n in kv]
    case = make(kv, new, H, Hkv, D, page, seed=24, width=max(need) + 9)
    table, cache, *rest = case
    clean = run(torch, case, kv, case[-1])
    assert torch.isfinite(clean.float()).all()
    free = np.arange(table.shape[1])[None, :] >= np.array(need)[:, None]
    values = [-2 ** 31, 2 ** 31 - 1, 10 ** 6, -1, len(cache), len(cache) - 1, 2 ** 30, 0]
    for shift in range(len(values)):                     # every value is the first behind a request's pages once
        wild = table.copy()
        for r in range(len(kv)):
            n = int(free[r].sum())
            wild[r, free[r]] = np.resize(np.roll(values, -shift - r), n)
        assert torch.equal(run(torch, (wild, cache, *rest), kv, case[-1]), clean)


def test_chunks_give_the_same_bits_every_time():
    torch = torch_or_skip()
    case = make([3000, 700], [600, 240], 32, 8, 64, 16, seed=21)
    first = run(torch, case, [3000, 700], case[-1])
    for _ in range(3):
        assert torch.equal(run(torch, case, [3000, 700], case[-1]), first)


@pytest.mark.parametrize("std", [4.0, 16.0])
def test_sharp(std):
    check(torch_or_skip(), [500, 77], [1, 1], 8, 2, 128, 16, seed=5, std=std)


def test_many_requests():
    """More requests than a workgroup has threads."""
    torch = torch_or_skip()
    rng = np.random.default_rng(10)
    kv = rng.integers(0, 60, 700)
    new = np.minimum(kv, rng.integers(0, 3, 700))
    check(torch, kv, [int(n) for n in new], 2, 1, 64, 16, seed=10)


def test_what_pages_hold_behind_a_row_reaches_nothing():
    """Slots behind a request's last key and spare pages full of NaN, table entries behind its pages of any value:
    the bits of a clean cache. And a NaN key or value of a later token leaves the rows before it alone."""
    torch = torch_or_skip()
    kv, new, H, Hkv, D, page = [37, 5, 130], [4, 5, 1], 4, 2, 128, 16
    case = make(kv, new, H, Hkv, D, page, seed=12)
    table, cache, k, v, qn, bits, cu = case
    clean = run(torch, case, kv, cu)
    used = np.zeros(len(cache) * page, bool)
    for r, n in enumerate(kv):
        for p in range(n):
            used[table[r, p // page] * page + p % page] = True
    dirty = cache.copy()
    n0 = page * D
    for s in np.nonzero(~used)[0]:
        p, o = divmod(int(s), page)
        for which in range(2):
            dirty[p, :, n0 + (which * page + o) * 4:n0 + (which * page + o) * 4 + 4] = 255
    wild = table.copy()
    wild[table < 0] = [-2 ** 31, 2 ** 31 - 1, 10 ** 6, -1][: 1] * int((table < 0).sum())
    o = run(torch, (wild, dirty, k, v, qn, bits, cu), kv, cu)
    assert torch.equal(o, clean)
    # request 0, its last token (position 36): NaN key; request 1, position 3: NaN values in one block of 32
    s0 = int(table[0, 36 // page] * page + 36 % page)
    s1 = int(table[1, 0] * page + 3)
    dirty[s0 // page, :, n0 + (s0 % page) * 4 + 1] = 255
    dirty[s1 // page, :, n0 + (page + s1 % page) * 4 + 2] = 255
    o = run(torch, (wild, dirty, k, v, qn, bits, cu), kv, cu).float()
    c = clean.float()
    assert torch.equal(o[:3], c[:3]) and torch.isnan(o[3]).all()
    assert torch.equal(o[4:7], c[4:7])
    assert torch.isnan(o[7:9, :, 64:96]).all()
    dirty[s1 // page, :, n0 + (page + s1 % page) * 4 + 2] = 254           # past bf16's range: the same
    assert torch.isnan(run(torch, (wild, dirty, k, v, qn, bits, cu), kv, cu).float()[7:9, :, 64:96]).all()
    keep = [i for i in range(128) if not 64 <= i < 96]
    assert torch.equal(o[7:9][..., keep], c[7:9][..., keep]) and torch.equal(o[9], c[9])


@pytest.mark.parametrize("kv,new,H,Hkv,D,page,width", [
    ([40, 300], [1, 1], 8, 2, 128, 16, None), ([3000, 5], [1, 1], 4, 4, 64, 16, None), ([700, 90], [9, 20], 16, 2, 64, 32, None),
    ([2500], [30], 8, 1, 128, 64, None), ([640], [600], 32, 8, 128, 32, 20), ([3000, 700], [600, 240], 32, 8, 64, 16, None)])
def test_rows_whose_scores_are_all_minus_infinity_are_nan(kv, new, H, Hkv, D, page, width):
    """Not zero as rows that see no key are: single and several tokens, tiles of 128 rows, split and whole, and no other row."""
    torch = torch_or_skip()
    table, cache, k, v, qn, bits, cu = make(kv, new, H, Hkv, D, page, seed=23, width=width)
    byte = np.arange(page) * (D // 2) + 2                     # element 5 of every key is 1.0 (code 2)
    cache[..., byte] = cache[..., byte] & 0x0f | 0x20
    k, v = oracle.decode_cache(cache, D)
    clean = run(torch, (table, cache, k, v, qn, bits, cu), kv, cu)
    bad = [(0, H - 1), (int(cu[-1]) - 1, 0), (int(cu[-1]) // 2, H // 2)]
    for t, h in bad:
        qn[t, h, 5] = -np.inf
        bits[t, h, 5] = 0xff80
    want = torch.zeros(clean.shape, dtype=torch.bool, device="cuda")
    for t, h in bad:
        r = int(np.searchsorted(cu, t, side="right") - 1)
        g = h // (H // Hkv)
        kk, _ = oracle.gather_cache(k, v, table[r], int(kv[r]) - int(cu[r + 1] - 1 - t), page)
        assert np.all(kk[:, g] @ qn[t, h] == -np.inf)
        want[t, h] = True
    o = run(torch, (table, cache, k, v, qn, bits, cu), kv, cu)
    assert torch.isnan(o[want]).all()
    # the others: both are within attn_tolerance, and sum_j p_j |v_j| is at most the largest value
    other, was = o[~want].float(), clean[~want].float()
    tol = 2 * (2.0 ** -7 * float(np.abs(v).max()) + 2.0 ** -8 * was.abs())
    assert torch.all((other - was).abs() <= tol)


def test_missing_pages_are_nan():
    torch = torch_or_skip()
    kv, H, Hkv, D, page = [40, 40, 200, 20], 4, 1, 64, 16
    case = make(kv, [1] * 4, H, Hkv, D, page, seed=13, width=13)
    table, cache, *_ = case
    table[1, 1] = len(cache)                       # one past the pool
    table[2, 7] = -1
    o = run(torch, case, kv, None).float()
    assert torch.isfinite(o[0]).all() and torch.isnan(o[1]).all() and torch.isnan(o[2]).all() and torch.isfinite(o[3]).all()
    o = run(torch, case, [40, 16, 112, 209], None).float()        # not needed; the table of 13 pages holds 208 keys
    assert torch.isfinite(o[:3]).all() and torch.isnan(o[3]).all()
    o = run(torch, case, [40, -5, 2 ** 31 - 1, 1], None).float()
    assert torch.isfinite(o[0]).all() and torch.all(o[1] == 0) and torch.isnan(o[2]).all() and torch.isfinite(o[3]).all()


@pytest.mark.parametrize("H,Hkv,new,pages", [(4, 1, 5, 13), (32, 8, 840, 53)])
def test_rows_before_the_end_of_a_short_table_are_whole(H, Hkv, new, pages):
    """Two keys more than the table has pages for: the last two rows are NaN, those before as in the oracle."""
    torch = torch_or_skip()
    kv = pages * 16
    case = make([kv], [new], H, Hkv, 64, 16, seed=22, width=pages)
    table, cache, k, v, qn, bits, cu = case
    o = host_bf16(torch, run(torch, case, [kv + 2], cu))
    assert np.isnan(o[-2:]).all() and np.isfinite(o[:-2]).all()
    kk, vv = oracle.gather_cache(k, v, table[0], kv, 16)
    t = new - 3                                             # sees exactly the table's keys
    ref, absv = np.zeros((1, H, 64)), np.zeros((1, H, 64))
    for h in range(H):
        g = h // (H // Hkv)
        s = kk[:, g] @ qn[t, h] * 64 ** -0.5
        p = np.exp(s - s.max())
        p /= p.sum()
        ref[0, h], absv[0, h] = p @ vv[:, g], p @ np.abs(vv[:, g])
    assert oracle.attn_ratio(o[t:t + 1], ref, absv) <= 1.0


def test_tables_of_no_pages():
    torch = torch_or_skip()
    m = q()
    x = torch.randn((3, 4, 64), device="cuda").to(torch.bfloat16)
    cache = torch.zeros(m.kv4_cache_shape(1, 2, 64, 16), dtype=torch.uint8, device="cuda")
    table = torch.empty((3, 0), dtype=torch.int32, device="cuda")
    o = m.attention_kv4(x, cache, table, dev_i32(torch, [0, 0, 0]))
    assert torch.all(o == 0)
    o = m.attention_kv4(x, cache, table, dev_i32(torch, [0, 1, 0])).float()
    assert torch.all(o[0] == 0) and torch.isnan(o[1]).all() and torch.all(o[2] == 0)
    none = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    assert m.attention_kv4(none, cache, table[:0], dev_i32(torch, [])).shape == (0, 4, 64)
    out = torch.full((3, 4, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    m.attention_kv4(x, cache, table[:0], dev_i32(torch, []), dev_i32(torch, [0]), out=out)       # rows of no request
    assert torch.all(out == 9)


def test_inconsistent_first_rows_stay_in_bounds():
    torch = torch_or_skip()
    case = make([40, 9, 33], [3, 4, 2], 4, 2, 64, 16, seed=14)
    buf = torch.full((9 + 64, 4, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    for cu in ([0, 100, 50, 9], [-5, 3, 2 ** 31 - 1, 9], [9, 9, 0, 4], [-1, -1, -1, -1]):
        run(torch, case, [40, 9, 33], cu, out=buf[32:41])
        torch.cuda.synchronize()
        assert torch.all(buf[:32] == 9) and torch.all(buf[41:] == 9)


def test_first_rows_that_descend_give_no_more_work_than_the_rows():
    """Requests that share their rows, every second one with all of them: 10^10 granules if they were taken as they
    are. The call ends, writes nothing outside its rows, and the next call is right."""
    torch = torch_or_skip()
    T, R, W = 4096, 2048, 1024
    buf = torch.full((T + 64, 8, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    cache = torch.zeros(q().kv4_cache_shape(1, 1, 64, 1024), dtype=torch.uint8, device="cuda")
    table = torch.zeros((R, W), dtype=torch.int32, device="cuda")
    kv = torch.full((R,), W * 1024, dtype=torch.int32, device="cuda")
    x = torch.zeros((T, 8, 64), dtype=torch.bfloat16, device="cuda")
    cu = dev_i32(torch, [T * (r & 1) for r in range(R + 1)])
    q().attention_kv4(x, cache, table, kv, cu, out=buf[32:-32])
    torch.cuda.synchronize()
    assert torch.all(buf[:32] == 9) and torch.all(buf[-32:] == 9)
    check(torch, [300, 41], [3, 1], 8, 1, 64, 16, seed=17)


def test_strided_queries_same_bits_every_time():
    torch = torch_or_skip()
    m = q()
    kv = [3000, 40, 1, 777]
    case = make(kv, [2, 1, 1, 3], 8, 2, 128, 16, seed=15)
    table, cache, _, _, _, bits, cu = case
    o = run(torch, case, kv, cu)
    wide = torch.zeros((7, 12, 128), dtype=torch.bfloat16, device="cuda")
    wide[:, :8] = dev_bf16(torch, bits)
    args = (torch.from_numpy(cache).cuda(), dev_i32(torch, table), dev_i32(torch, kv), dev_i32(torch, cu))
    for _ in range(3):
        assert torch.equal(m.attention_kv4(wide[:, :8], *args), o)


def test_cache_past_32_bits():
    """Pages whose byte offsets pass 2^32."""
    torch = torch_or_skip()
    m = q()
    pages = (5 << 30) // (2 * 16 * 136)
    big = torch.empty(m.kv4_cache_shape(pages, 2, 128, 16), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(16)
    small, k, v = random_cache(rng, 5, 2, 128, 16)
    at = [pages - 1, 3, pages - 2, pages // 2, pages - 7]
    for i, p in enumerate(at):
        big[p] = torch.from_numpy(small[i]).cuda()
    qn, bits = bf16(rng.standard_normal((1, 4, 128)))
    o = m.attention_kv4(dev_bf16(torch, bits), big, dev_i32(torch, [at]), dev_i32(torch, [77]))
    ref, absv = oracle.cached_attention(qn, k, v, [[0, 1, 2, 3, 4]], [77], [0, 1], 16, 128 ** -0.5)
    assert oracle.attn_ratio(host_bf16(torch, o), ref, absv) <= 1.0
    del big
