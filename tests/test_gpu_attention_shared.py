"""GPU: ``attention_kv4_shared`` against the fp64 oracle, within ``attn_tolerance`` as ``attention_kv4`` is: the keys that a group
shares are read through its first request's table, so in most cases here the other requests' entries for them are wrong on
purpose."""
import numpy as np
import pytest

import oracle
from gpu_util import torch_or_skip
from serve_util import bf16, dev_bf16, dev_i32, host_bf16, random_cache, starts

pytestmark = pytest.mark.gpu


def q():
    import paper_2607_19438_amd as m
    return m


def make(groups, prefix, own, new, H, Hkv, D, page, seed=0, pad=0, std=1.0, behind=1, wrong=True):
    """Requests of groups[g] .. groups[g+1]-1 with prefix[g] keys in common and own[r] more. A page that the prefix ends in is
    every request's own, and holds the same there; ``wrong``: entries of whole shared blocks are -1 in all but the first
    request that has rows."""
    rng = np.random.default_rng(seed)
    R = len(own)
    of = [next((g for g in range(len(prefix)) if groups[g] <= r < groups[g + 1]), None) for r in range(R)]
    kv = [(prefix[of[r]] if of[r] is not None else 0) + own[r] for r in range(R)]
    cu = starts(new)
    need = [-(-n // page) for n in kv]
    W = max(need + [1]) + behind
    ids = list(rng.permutation(sum(need) + 3))
    pages = len(ids)
    cache, _, _ = random_cache(rng, pages, Hkv, D, page)
    table = np.full((R, W), -1, dtype=np.int64)
    n0, first = page * D, {}
    for r in range(R):
        g = of[r]
        table[r, :need[r]] = [ids.pop() for _ in range(need[r])]
        if g is None:
            continue
        if g not in first:
            first[g] = r
            continue
        whole, part = divmod(prefix[g], page)
        table[r, :whole] = table[first[g], :whole]
        if part:                                          # the same keys and values in the page of its own
            a, b = table[first[g], whole], table[r, whole]
            for which in range(2):
                for lo, size in ((which * page * D // 2, D // 2), (n0 + which * page * (D // 32), D // 32)):
                    cache[b, :, lo:lo + part * size] = cache[a, :, lo:lo + part * size]
    if wrong:
        for (lead, common), g in zip(oracle.shared_keys(kv, cu, groups, prefix, W, page), range(len(prefix))):
            for r in range(groups[g], groups[g + 1]):
                if r != lead:
                    table[r, :common // page] = -1
    k, v = oracle.decode_cache(cache, D)
    qn, bits = bf16(rng.standard_normal((int(sum(new)) + pad, H, D)) * std)
    return dict(table=table, cache=cache, k=k, v=v, q=qn, bits=bits, cu=cu, kv=kv, groups=groups, prefix=prefix, page=page)


def run(torch, c, cu=True, out=None, **kw):
    c = {**c, **kw}
    return q().attention_kv4_shared(dev_bf16(torch, c["bits"]), torch.from_numpy(c["cache"]).cuda(), dev_i32(torch, c["table"]), dev_i32(torch, c["kv"]),
                                    dev_i32(torch, c["groups"]), dev_i32(torch, c["prefix"]), dev_i32(torch, c["cu"]) if cu else None, out=out)


def check(torch, c, cu=True, rows=None):
    out = torch.full(c["q"].shape, 9.0, dtype=torch.bfloat16, device="cuda")
    run(torch, c, cu, out)
    got = host_bf16(torch, out)
    T = int(c["cu"][-1])
    assert np.all(got[T:] == 9.0)
    D = c["q"].shape[2]
    ref, absv = oracle.shared_attention(c["q"], c["k"], c["v"], c["table"], c["kv"], c["cu"], c["groups"], c["prefix"], c["page"], D ** -0.5, rows)
    sel = np.arange(T) if rows is None else np.array(sorted(rows))
    worst = oracle.attn_ratio(got[sel], ref[sel], absv[sel])
    print(f"[parity] shared {list(c['groups'])[:5]} x {list(c['prefix'])[:5]} {c['q'].shape}: max |err| / bar = {worst:.3f}", flush=True)
    assert worst <= 1.0
    return out


SINGLE = [  # groups, prefix, own keys, H, Hkv, D, page
    ([0, 4], [100], [1, 5, 9, 30], 8, 2, 64, 16), ([0, 4], [128], [1, 1, 1, 1], 4, 1, 128, 16), ([0, 1], [300], [4], 6, 2, 128, 64),
    ([0, 3, 5], [64, 700], [1, 200, 3, 90, 17], 16, 2, 64, 32), ([0, 8], [1000], list(range(1, 9)), 32, 4, 128, 16),
    ([0, 2, 2, 6], [63, 5, 65], [9, 300, 1, 2, 1, 40], 8, 8, 128, 16), ([1, 4], [500], [40, 1, 2, 3, 600, 1], 4, 2, 64, 16),
    ([0, 40], [400], [1 + i % 7 for i in range(40)], 8, 2, 128, 64), ([0, 70], [260], [1 + i % 90 for i in range(70)], 40, 2, 64, 128),
    ([0, 24], [2100], [5] * 24, 32, 8, 64, 1024), ([0, 20, 60], [512, 1030], [1 + 9 * (i % 4) for i in range(60)], 12, 2, 128, 16),
    ([0, 3], [0], [1, 20, 300], 2, 1, 64, 16), ([0, 0, 2], [40, 0], [1, 1], 66, 1, 64, 16), ([0], [], [17, 1], 4, 4, 128, 16),
]


@pytest.mark.parametrize("groups,prefix,own,H,Hkv,D,page", SINGLE)
def test_single_tokens(groups, prefix, own, H, Hkv, D, page):
    torch = torch_or_skip()
    c = make(groups, prefix, own, [1] * len(own), H, Hkv, D, page, seed=len(own) + D)
    a = check(torch, c, cu=False)
    assert torch.equal(a, run(torch, c, cu=True))


SEVERAL = [  # groups, prefix, own keys, new tokens, H, Hkv, D, page, rows behind
    ([0, 2], [90], [5, 9], [5, 3], 4, 2, 128, 16, 2), ([0, 3], [200], [4, 0, 33], [4, 0, 33], 8, 2, 64, 32, 0),
    ([0, 3], [200], [0, 7, 33], [0, 7, 30], 8, 2, 64, 16, 3), ([0, 2, 4], [130, 640], [60, 2, 17, 9], [60, 1, 9, 9], 12, 4, 128, 16, 5),
    ([0, 12], [700], [20] * 12, [3 + i for i in range(12)], 16, 2, 128, 64, 1), ([0, 30], [200], [9] * 30, [i % 9 for i in range(30)], 8, 1, 64, 16, 0),
    ([0, 2], [150], [3, 5], [4, 5], 2, 1, 64, 16, 0), ([0, 2], [64], [0, 100], [0, 1], 2, 2, 128, 16, 3),
]


@pytest.mark.parametrize("groups,prefix,own,new,H,Hkv,D,page,pad", SEVERAL)
def test_several_tokens(groups, prefix, own, new, H, Hkv, D, page, pad):
    check(torch_or_skip(), make(groups, prefix, own, new, H, Hkv, D, page, seed=sum(new), pad=pad))


CHUNKS = [  # prompts behind a shared one: 128 rows to a tile of either kind
    ([0, 2], [700], [400, 433], [400, 433], 32, 8, 128, 16), ([0, 3], [300], [900, 140, 500], [833, 140, 440], 32, 4, 64, 64),
    ([0, 1, 2], [320, 64], [600, 520], [520, 520], 64, 64, 64, 32),
]


@pytest.mark.parametrize("groups,prefix,own,new,H,Hkv,D,page", CHUNKS)
def test_chunks(groups, prefix, own, new, H, Hkv, D, page):
    cu = starts(new)
    rows = {t for c in cu for t in (c - 1, c, c + 1, c + 31, c + 33) if 0 <= t < cu[-1]} | {int(cu[-1] // 3), int(cu[-1] // 2)}
    check(torch_or_skip(), make(groups, prefix, own, new, H, Hkv, D, page, seed=7, pad=2), rows={int(t) for t in rows})


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("groups,prefix,new,H,Hkv,page", [
    ([0, 170], [900], [1] * 170, 32, 8, 64), ([0, 170], [130], [1] * 170, 32, 8, 16),                # 128 rows to a tile of the shared keys,
    ([1, 90, 179], [700, 300], [1] * 180, 64, 8, 32), ([0, 44], [1500], [4 + i % 3 for i in range(44)], 32, 8, 128),   # 16 or 32 of the others
    ([0, 20, 41], [260, 640], [3 + i % 6 for i in range(43)], 64, 8, 16),
])
def test_many_rows_to_a_group(groups, prefix, new, H, Hkv, page, D):
    torch = torch_or_skip()
    own = [n + (41 * i) % 150 for i, n in enumerate(new)]
    c = make(groups, prefix, own, new, H, Hkv, D, page, seed=len(new), pad=1)
    rows = set(range(0, int(c["cu"][-1]), 7)) | {int(c["cu"][-1]) - 1}
    check(torch, c, rows=rows)


@pytest.mark.parametrize("D", [64, 128])
def test_long_prefix_split_over_the_chip(D):
    torch = torch_or_skip()
    own = [1 + (37 * i) % 500 for i in range(33)]
    c = make([0, 33], [9000], own, [1] * 33, 16, 2, D, 64, seed=8)
    check(torch, c, cu=False, rows={0, 7, 20, 32})
    c = make([0, 3, 6], [5000, 3000], [20, 3, 400, 1, 9, 70], [1] * 6, 16, 2, D, 64, seed=9)
    check(torch, c, cu=False)


def test_same_as_attention_over_the_cache():
    """With tables that are right for every request both calls compute the same; the difference is within twice the bar."""
    torch = torch_or_skip()
    c = make([0, 8, 16], [600, 90], [1 + 11 * i for i in range(16)], [1] * 16, 32, 8, 128, 16, seed=10, wrong=False)
    a = check(torch, c, cu=False)
    b = q().attention_kv4(dev_bf16(torch, c["bits"]), torch.from_numpy(c["cache"]).cuda(), dev_i32(torch, c["table"]), dev_i32(torch, c["kv"]))
    _, absv = oracle.shared_attention(c["q"], c["k"], c["v"], c["table"], c["kv"], c["cu"], [0], [], 16, 128 ** -0.5)
    assert oracle.attn_ratio(host_bf16(torch, a), host_bf16(torch, b), 2 * absv) <= 1.0


@pytest.mark.parametrize("std", [4.0, 16.0])
def test_sharp(std):
    """Rows that look at the shared keys alone, or at their own alone."""
    check(torch_or_skip(), make([0, 6], [300], [9] * 6, [1] * 6, 8, 2, 128, 16, seed=11, std=std), cu=False)


def test_rows_that_see_nothing_are_zero_and_prefixes_are_cut():
    torch = torch_or_skip()
    c = make([0, 3], [0], [0, 3, 40], [1, 5, 1], 4, 2, 128, 16, seed=12)
    out = check(torch, c)
    assert torch.all(out[0] == 0) and torch.all(out[1:3] == 0)
    # more than the shortest history, than the table, than nothing
    c = make([0, 3], [200], [1, 1, 1], [1, 1, 1], 4, 1, 64, 16, seed=13)
    want = check(torch, c, cu=False)
    for n in (2 ** 31 - 1, 10 ** 6):
        assert torch.equal(run(torch, c, cu=False, prefix=[n]), want)
    d = make([0, 3], [200], [1, 1, 1], [1, 1, 1], 4, 1, 64, 16, seed=13, wrong=False)
    for n in (0, -1, -2 ** 31, 63):
        d["prefix"] = [n]
        check(torch, d, cu=False)


@pytest.mark.parametrize("groups,prefix,own,new,H,Hkv", [([0, 3], [150], [20, 9, 30], [1, 1, 1], 4, 2), ([0, 20], [200], [20] * 20, [1] * 20, 32, 8),
                                                        ([0, 2], [320], [440, 420], [430, 420], 32, 8)])
def test_nan_reaches_the_rows_that_see_it(groups, prefix, own, new, H, Hkv):
    """A NaN key among the shared ones: the group's rows of its head. A value block of NaN: 32 of their dimensions. Slots behind
    a request's last key, and of no request, full of NaN: no bit. A page that is none: as NaN."""
    torch = torch_or_skip()
    D, page = 128, 16
    R = len(own)
    c = make(groups + [R + 1], prefix + [0], own + [70], new + [1], H, Hkv, D, page, seed=14)
    clean = run(torch, c)
    T = int(c["cu"][-1])
    n0, sb = page * D, D // 32
    used = set()
    for r in range(R + 1):
        used |= {int(c["table"][r, p // page]) * page + p % page for p in range(c["kv"][r]) if c["table"][r, p // page] >= 0}
    dirty = c["cache"].copy()
    for s in range(len(dirty) * page):
        if s not in used:
            p, o = divmod(s, page)
            for which in range(2):
                dirty[p, :, n0 + (which * page + o) * sb:n0 + (which * page + o + 1) * sb] = 255
    assert torch.equal(run(torch, c, cache=dirty), clean)
    lead = int(c["table"][0, 0]), 5                       # position 5 of the group
    G = H // Hkv
    bad = dirty.copy()
    bad[lead[0], 1, n0 + lead[1] * sb + 2] = 255          # key, head 1
    o = run(torch, c, cache=bad)
    assert torch.isnan(o[:T - 1, G:2 * G].float()).all() and torch.equal(o[T - 1], clean[T - 1])
    assert torch.equal(o[:T - 1, :G], clean[:T - 1, :G]) and torch.equal(o[:, 2 * G:], clean[:, 2 * G:])
    for byte in (255, 254):
        bad = dirty.copy()
        bad[lead[0], 1, n0 + (page + lead[1]) * sb + 2] = byte        # values, head 1
        o = run(torch, c, cache=bad)
        assert torch.isnan(o[:T - 1, G:2 * G, 64:96].float()).all()
        keep = [i for i in range(D) if not 64 <= i < 96]
        assert torch.equal(o[:T - 1, G:2 * G][..., keep], clean[:T - 1, G:2 * G][..., keep])
        assert torch.equal(o[:T - 1, :G], clean[:T - 1, :G]) and torch.equal(o[T - 1], clean[T - 1])
    wild = c["table"].copy()
    wild[0, 1] = len(dirty)
    o = run(torch, c, table=wild).float()
    assert torch.isnan(o[:T - 1]).all() and torch.isfinite(o[T - 1]).all()
    wild = c["table"].copy()
    wild[1, prefix[0] // page] = -5                       # of request 1 alone
    o = run(torch, c, table=wild).float()
    a, b = int(c["cu"][1]), int(c["cu"][2])
    first = max(0, (prefix[0] // page * page) - (c["kv"][1] - new[1]))
    assert torch.isnan(o[a + first:b]).all() and torch.isfinite(o[:a]).all() and torch.isfinite(o[b:]).all()


def test_keys_past_the_table():
    torch = torch_or_skip()
    c = make([0, 3], [128], [16, 32, 16], [1, 1, 1], 4, 1, 64, 16, seed=15, behind=0)
    o = run(torch, c, cu=False, kv=[144, 162, 144]).float()          # 10 pages: the table's 160 keys
    assert torch.isfinite(o[0]).all() and torch.isnan(o[1]).all() and torch.isfinite(o[2]).all()
    o = run(torch, c, cu=False, kv=[144, -5, 2 ** 31 - 1]).float()
    assert torch.all(o[1] == 0) and torch.isnan(o[2]).all()


def test_scores_of_minus_infinity_are_nan():
    """A row whose shared and own scores are all -inf; one whose own alone are is the softmax of the shared ones."""
    torch = torch_or_skip()
    D, page = 128, 16
    c = make([0, 5], [200], [30] * 5, [1] * 5, 8, 2, D, page, seed=16)
    byte = np.arange(page) * (D // 2) + 2                 # element 5 of every key is 1.0 (code 2)
    c["cache"][..., byte] = c["cache"][..., byte] & 0x0f | 0x20
    clean = run(torch, c, cu=False)
    c["bits"][2, 3, 5] = 0xff80
    o = run(torch, c, cu=False)
    assert torch.isnan(o[2, 3].float()).all()
    o[2, 3] = clean[2, 3]
    assert torch.equal(o, clean)


def test_groups_and_rows_that_descend_stay_in_bounds():
    torch = torch_or_skip()
    c = make([0, 3, 5], [100, 200], [9] * 5, [2] * 5, 4, 2, 64, 16, seed=17, wrong=False)
    buf = torch.full((10 + 64, 4, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    for groups in ([5, 2, 0], [0, 5, 3], [-4, 2 ** 31 - 1, 1], [3, 1, 9]):
        run(torch, c, out=buf[32:42], groups=groups)
        torch.cuda.synchronize()
        assert torch.all(buf[:32] == 9) and torch.all(buf[42:] == 9)
    for cu in ([0, 100, 50, 9, 2, 1], [-5, 3, 2 ** 31 - 1, 9, 9, 10], [9, 9, 0, 4, 7, 10], [-1] * 6):
        q().attention_kv4_shared(
            dev_bf16(torch, c["bits"]), torch.from_numpy(c["cache"]).cuda(), dev_i32(torch, c["table"]), dev_i32(torch, c["kv"]),
            dev_i32(torch, c["groups"]), dev_i32(torch, c["prefix"]), dev_i32(torch, cu), out=buf[32:42])
        torch.cuda.synchronize()
        assert torch.all(buf[:32] == 9) and torch.all(buf[42:] == 9)
    check(torch, c)


def test_many_requests_and_groups():
    torch = torch_or_skip()
    rng = np.random.default_rng(18)
    groups = [0] + sorted(rng.integers(0, 701, 299).tolist()) + [700]
    own = [int(n) for n in rng.integers(1, 40, 700)]
    new = [int(min(n, m)) for n, m in zip(own, rng.integers(0, 3, 700))]
    check(torch, make(groups, [int(n) for n in rng.integers(0, 300, 300)], own, new, 2, 1, 64, 16, seed=18))
    for groups, prefix in (([0, 2048], [70]), (list(range(2049)), [70] * 2048)):        # as many as there may be
        c = make(groups, prefix, [1] * 2048, [1] * 2048, 2, 1, 64, 16, seed=19)
        check(torch, c, cu=False, rows={0, 1, 1023, 2047})


def test_tables_of_no_pages_and_no_requests():
    torch = torch_or_skip()
    m = q()
    x = torch.randn((3, 4, 64), device="cuda").to(torch.bfloat16)
    cache = torch.zeros(m.kv4_cache_shape(1, 2, 64, 16), dtype=torch.uint8, device="cuda")
    table = torch.empty((3, 0), dtype=torch.int32, device="cuda")
    g, p = dev_i32(torch, [0, 3]), dev_i32(torch, [50])
    assert torch.all(m.attention_kv4_shared(x, cache, table, dev_i32(torch, [0, 0, 0]), g, p) == 0)
    o = m.attention_kv4_shared(x, cache, table, dev_i32(torch, [0, 1, 0]), g, p).float()
    assert torch.all(o[0] == 0) and torch.isnan(o[1]).all() and torch.all(o[2] == 0)
    none = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    assert m.attention_kv4_shared(none, cache, table[:0], dev_i32(torch, []), dev_i32(torch, [0, 0]), p).shape == (0, 4, 64)


def test_strided_queries_streams_and_graphs():
    torch = torch_or_skip()
    m = q()
    c = make([0, 4, 9], [900, 300], [1 + 40 * (i % 5) for i in range(9)], [1] * 9, 8, 2, 128, 16, seed=20, behind=40)
    want = run(torch, c, cu=False)
    wide = torch.zeros((9, 12, 128), dtype=torch.bfloat16, device="cuda")
    wide[:, :8] = dev_bf16(torch, c["bits"])
    args = [torch.from_numpy(c["cache"]).cuda(), dev_i32(torch, c["table"]), dev_i32(torch, c["kv"]), dev_i32(torch, c["groups"]),
            dev_i32(torch, c["prefix"])]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(m.attention_kv4_shared(wide[:, :8], *args))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = m.attention_kv4_shared(wide[:, :8], *args)
    g2 = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g2):                            # a second graph with a workspace of its own
        o2 = m.attention_kv4_shared(wide[:, :8], *args)
    for pre, shorter in (([900, 300], 0), ([64, 0], 0), ([500, 128], 1), ([900, 300], 0)):
        args[2].copy_(dev_i32(torch, np.array(c["kv"]) - shorter))
        args[4].copy_(dev_i32(torch, pre))
        if pre != [900, 300]:
            args[1].copy_(dev_i32(torch, full_table(c)))
        g.replay()
        g2.replay()
        e = m.attention_kv4_shared(wide[:, :8], *args)
        assert torch.equal(o, e) and torch.equal(o2, e)


def full_table(c):
    """The table with the shared entries of every request."""
    t = c["table"].copy()
    for g in range(len(c["prefix"])):
        for r in range(c["groups"][g], c["groups"][g + 1]):
            bad = t[r] < 0
            bad[-(-c["kv"][r] // c["page"]):] = False
            t[r, bad] = t[c["groups"][g], bad]
    return t


def test_cache_past_32_bits():
    torch = torch_or_skip()
    m = q()
    pages = (5 << 30) // (2 * 16 * 136)
    big = torch.empty(m.kv4_cache_shape(pages, 2, 128, 16), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(21)
    small, k, v = random_cache(rng, 9, 2, 128, 16)
    at = [pages - 1, 3, pages - 2, pages // 2, pages - 7, pages - 9, pages - 11, 5, 6]
    for i, p in enumerate(at):
        big[p] = torch.from_numpy(small[i]).cuda()
    qn, bits = bf16(rng.standard_normal((2, 4, 128)))
    t = np.array([[0, 1, 2, 3, 4, 5], [0, 1, 2, 3, 4, 7]])
    o = m.attention_kv4_shared(dev_bf16(torch, bits), big, dev_i32(torch, np.array(at)[t]), dev_i32(torch, [90, 83]), dev_i32(torch, [0, 2]), dev_i32(torch, [80]))
    ref, absv = oracle.shared_attention(qn, k, v, t, [90, 83], [0, 1, 2], [0, 2], [80], 16, 128 ** -0.5)
    assert oracle.attn_ratio(host_bf16(torch, o), ref, absv) <= 1.0
    del big
