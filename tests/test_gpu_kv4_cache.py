"""GPU: ``kv4_store`` / ``kv4_load`` against the oracle's blocks; every code, exponent and value is equal."""
import numpy as np
import pytest

import oracle
from oracle import serve_oracle as so
from gpu_util import torch_or_skip
from serve_util import bf16, dev_bf16, dev_i32, host_bf16

pytestmark = pytest.mark.gpu


def q():
    import paper_2607_19438_amd as m
    return m


def store_ref(cache, k, v, slots, page):
    """The cache's bytes after the store, by the oracle's encoding of one-token caches."""
    cache = cache.copy()
    T, Hkv, D = k.shape
    for which, x in enumerate((k, v)):
        codes, E = oracle.quantise(x.reshape(T, Hkv, D // 32, 32))
        codes = codes.reshape(T, Hkv, D)
        for t, s in enumerate(slots):
            if 0 <= s < len(cache) * page:
                p, o = divmod(int(s), page)
                c0, s0 = (which * page + o) * (D // 2), page * D + (which * page + o) * (D // 32)
                cache[p, :, c0:c0 + D // 2] = codes[t, :, 0::2] | (codes[t, :, 1::2] << 4)
                cache[p, :, s0:s0 + D // 32] = E[t]
    return cache


CASES = [  # T, Hkv, D, page, pages
    (1, 1, 64, 16, 1), (1, 4, 128, 16, 5), (13, 2, 64, 32, 3), (40, 3, 128, 64, 2), (65, 8, 64, 16, 7), (129, 1, 128, 128, 2),
    (20, 2, 128, 1024, 1),
]


@pytest.mark.parametrize("T,Hkv,D,page,pages", CASES)
def test_store_and_load(T, Hkv, D, page, pages):
    torch = torch_or_skip()
    m = q()
    rng = np.random.default_rng(T + D)
    scale = np.exp(rng.standard_normal((T, Hkv, 1)) * 8)         # blocks over many binades
    k, kb = bf16(rng.standard_normal((T, Hkv, D)) * scale)
    v, vb = bf16(rng.standard_normal((T, Hkv, D)) / scale)
    slots = rng.permutation(pages * page)[:T] if T <= pages * page else np.arange(T)
    if T > 5:
        slots[2], slots[4] = -1, pages * page                    # skipped
    cache = rng.integers(0, 256, m.kv4_cache_shape(pages, Hkv, D, page)).astype(np.uint8)
    dc = torch.from_numpy(cache).cuda()
    m.kv4_store(dev_bf16(torch, kb), dev_bf16(torch, vb), dev_i32(torch, slots), dc)
    want = store_ref(cache, k, v, slots, page)
    assert np.array_equal(dc.cpu().numpy(), want)
    # every slot back, and slots that are none leave their rows
    every = list(range(pages * page)) + [-1, pages * page, 2 ** 31 - 1, -2 ** 31]
    kk = torch.full((len(every), Hkv, D), 3.0, dtype=torch.bfloat16, device="cuda")
    vv = kk.clone()
    m.kv4_load(dc, dev_i32(torch, every), D, kk, vv)
    for got, ref in zip((kk, vv), oracle.decode_cache(want, D)):
        got = host_bf16(torch, got)
        fits = ~(np.abs(ref) > 3.3895e38)                        # (random exponents: beyond bf16's range)
        tiny = np.abs(ref) < 2.0 ** -126
        assert np.array_equal(got[:-4][fits & ~tiny], ref[fits & ~tiny], equal_nan=True)
        assert np.all(np.abs(got[:-4][tiny] - ref[tiny]) <= 2.0 ** -133)
        assert np.all(got[-4:] == 3.0)


def test_every_bf16_number_is_held_as_the_oracle_holds_it():
    """All finite bf16 patterns, as the largest of a block and beside a fixed largest; ties, subnormals, zeros."""
    torch = torch_or_skip()
    m = q()
    bits = np.arange(65536, dtype=np.uint32).astype(np.uint16)
    rows = np.zeros((65536 // 16, 1, 64), dtype=np.uint16)
    rows[:, 0, :16] = bits.reshape(-1, 16)
    rows[:, 0, 32:48] = bits.reshape(-1, 16)
    rows[:, 0, 50] = np.uint16(0x40E0)                           # 7: the block counts as one of 8
    x = oracle.decode_bf16(rows)
    T, page = len(rows), 1024
    cache = torch.zeros(m.kv4_cache_shape(T // page, 1, 64, page), dtype=torch.uint8, device="cuda")
    d = dev_bf16(torch, rows)
    m.kv4_store(d, d, torch.arange(T, dtype=torch.int32, device="cuda"), cache)
    c = cache.cpu().numpy()
    with np.errstate(invalid="ignore"):
        codes, E = oracle.quantise(x.reshape(T, 2, 32))
    got_E = c[:, 0, page * 64:page * 64 + page * 2].reshape(T, 2)
    assert np.array_equal(got_E, E)
    by = c[:, 0, :page * 32].reshape(T, 32)
    got = np.stack([by & 15, by >> 4], -1).reshape(T, 2, 32)
    assert np.array_equal(got[E != 255], codes[E != 255])


def test_all_codes_and_exponents_load():
    torch = torch_or_skip()
    m = q()
    page, D = 128, 64
    cache = np.zeros(m.kv4_cache_shape(2, 1, D, page), dtype=np.uint8)
    cache[:, 0, :page * D] = np.tile(np.arange(256, dtype=np.uint8), page * D // 256)
    cache[0, 0, page * D:] = np.arange(512).astype(np.uint8)
    cache[1, 0, page * D:] = np.arange(512)[::-1].astype(np.uint8)
    k, v = m.kv4_load(torch.from_numpy(cache).cuda(), torch.arange(2 * page, dtype=torch.int32, device="cuda"), D)
    for got, ref in zip((k, v), oracle.decode_cache(cache, D)):
        got = host_bf16(torch, got)
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        ok = np.isfinite(ref) & (np.abs(ref) >= 2.0 ** -126) & (np.abs(ref) < 2.0 ** 128)
        assert np.array_equal(got[ok], ref[ok])


def test_a_slot_given_twice_touches_no_other():
    """Which of the tokens it holds is not specified; every other slot is as without the second one."""
    torch = torch_or_skip()
    m = q()
    x = torch.randn((8, 2, 64), device="cuda").to(torch.bfloat16)
    slots = dev_i32(torch, [3, 9, 3, 20, 31, 9, 0, 3])
    cache = torch.randint(0, 255, m.kv4_cache_shape(2, 2, 64, 16), device="cuda").to(torch.uint8)
    before = [y.clone() for y in m.kv4_load(cache, torch.arange(32, dtype=torch.int32, device="cuda"), 64)]
    m.kv4_store(x, x, slots, cache)
    once = torch.zeros(m.kv4_cache_shape(2, 2, 64, 16), dtype=torch.uint8, device="cuda")
    m.kv4_store(x, x, torch.arange(8, dtype=torch.int32, device="cuda"), once)
    alone = m.kv4_load(once, torch.arange(8, dtype=torch.int32, device="cuda"), 64)
    after = m.kv4_load(cache, torch.arange(32, dtype=torch.int32, device="cuda"), 64)
    for b, a, o in zip(before, after, alone):
        keep = [s for s in range(32) if s not in (3, 9, 20, 31, 0)]
        assert torch.equal(a[keep].view(torch.int16), b[keep].view(torch.int16))
        for s, t in ((20, 3), (31, 4), (0, 6)):
            assert torch.equal(a[s], o[t])


def test_nonfinite_blocks_are_nan_and_alone():
    torch = torch_or_skip()
    m = q()
    x = torch.randn((6, 2, 128), device="cuda").to(torch.bfloat16)
    x[1, 0, 40], x[3, 1, 127], x[4, 0, 0] = float("nan"), float("inf"), float("-inf")
    cache = torch.zeros(m.kv4_cache_shape(1, 2, 128, 16), dtype=torch.uint8, device="cuda")
    slots = torch.arange(6, dtype=torch.int32, device="cuda") + 4
    m.kv4_store(x, x, slots, cache)
    for y in m.kv4_load(cache, slots, 128):
        bad = torch.isnan(y).view(6, 2, 4, 32)
        want = torch.zeros_like(bad)
        want[1, 0, 1], want[3, 1, 3], want[4, 0, 0] = True, True, True
        assert torch.equal(bad, want)


def test_strided_rows_and_large_offsets():
    """Views of one projection row; and a cache of more than 4 GiB, whose last page is read and written."""
    torch = torch_or_skip()
    m = q()
    qkv = torch.randn((9, 7, 128), device="cuda").to(torch.bfloat16)
    k, v = qkv[:, 3:5], qkv[:, 5:7]
    slots = dev_i32(torch, [5, 40, 3, 17, 16, 15, 0, 63, 33])
    a = torch.zeros(m.kv4_cache_shape(4, 2, 128, 16), dtype=torch.uint8, device="cuda")
    b = torch.zeros_like(a)
    m.kv4_store(k, v, slots, a)
    m.kv4_store(k.contiguous(), v.contiguous(), slots, b)
    assert torch.equal(a, b) and a.any()
    pages = (5 << 30) // (2 * 16 * 136)
    big = torch.empty(m.kv4_cache_shape(pages, 2, 128, 16), dtype=torch.uint8, device="cuda")
    at = dev_i32(torch, [pages * 16 - 1 - i for i in range(9)])
    m.kv4_store(k, v, at, big)
    for x, y in zip(m.kv4_load(big, at, 128), m.kv4_load(a, slots, 128)):
        assert torch.equal(x, y)
    del big


def test_the_largest_numbers_stay_finite():
    torch = torch_or_skip()
    m = q()
    x = torch.full((3, 1, 64), 3.3895e38, device="cuda").to(torch.bfloat16)
    x[1], x[2] = -x[1], 2.9e38
    cache = torch.zeros(m.kv4_cache_shape(1, 1, 64, 16), dtype=torch.uint8, device="cuda")
    slots = torch.arange(3, dtype=torch.int32, device="cuda")
    m.kv4_store(x, x, slots, cache)
    for y in m.kv4_load(cache, slots, 64):
        y = host_bf16(torch, y)
        assert np.all(y[0] == 6 * 2.0 ** 125) and np.all(y[1] == -6 * 2.0 ** 125) and np.all(y[2] == 6 * 2.0 ** 125)


def test_values_of_one_step():
    """What is read back is within half a level step of what was stored (the largest magnitude of a block at most
    7 level units, steps of 0.5, 1 and 2)."""
    torch = torch_or_skip()
    m = q()
    rng = np.random.default_rng(9)
    x, bits = bf16(rng.standard_normal((64, 2, 128)))
    cache = torch.zeros(m.kv4_cache_shape(4, 2, 128, 16), dtype=torch.uint8, device="cuda")
    slots = torch.arange(64, dtype=torch.int32, device="cuda")
    m.kv4_store(dev_bf16(torch, bits), dev_bf16(torch, bits), slots, cache)
    codes, E = oracle.quantise(x.reshape(64, 2, 4, 32))
    unit = 2.0 ** (E.astype(float) - 127)[..., None]
    step = np.where(np.abs(x.reshape(codes.shape)) < 2 * unit, 0.5, np.where(np.abs(x.reshape(codes.shape)) < 4 * unit, 1, 2)) * unit
    for y in m.kv4_load(cache, slots, 128):
        y = host_bf16(torch, y).reshape(codes.shape)
        assert np.all(np.abs(y - x.reshape(codes.shape)) <= step / 2)
        assert np.array_equal(y, so.dequantise(codes, E))
