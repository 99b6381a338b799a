"""GPU: ``attention_packed`` against the fp64 oracle, prompt by prompt. Bar: the oracle's ``attn_tolerance``
(2^-7 sum_j p_j |v_j| for the weights' rounding to bf16, 2^-8 |o| for the output's), as for ``attention_prefill``."""
import numpy as np
import pytest

import oracle
from gpu_util import torch_or_skip
from serve_util import bf16, dev_bf16, dev_i32, host_bf16, starts

pytestmark = pytest.mark.gpu


def q():
    import paper_2607_19438_amd as m
    return m


def make(lens, H, Hkv, D, pad=0, seed=0, std=1.0):
    rng = np.random.default_rng(seed)
    T = int(sum(lens)) + pad
    row, bits = bf16(rng.standard_normal((T, H + 2 * Hkv, D)) * np.r_[np.full(H, std), np.ones(2 * Hkv)][None, :, None])
    return row, bits, starts(lens)


def views(t, H, Hkv):
    return t[:, :H], t[:, H:H + Hkv], t[:, H + Hkv:]


def check(torch, lens, H, Hkv, D, pad=0, seed=0, std=1.0, rows=None):
    row, bits, cu = make(lens, H, Hkv, D, pad, seed, std)
    d = dev_bf16(torch, bits)
    out = torch.full((len(row), H, D), 9.0, dtype=torch.bfloat16, device="cuda")
    scale = 1.0 / np.sqrt(D)
    o = q().attention_packed(*views(d, H, Hkv), dev_i32(torch, cu), scale, out=out)
    assert o is out
    got = host_bf16(torch, o)
    assert np.all(got[cu[-1]:] == 9.0)                       # rows of no prompt
    qn, kn, vn = views(row, H, Hkv)
    worst = 0.0
    if rows is None:
        ref, absv = oracle.packed_attention(qn, kn, vn, cu, scale)
        worst = oracle.attn_ratio(got[:cu[-1]], ref[:cu[-1]], absv[:cu[-1]])
    else:
        for t in rows:
            c0 = cu[np.searchsorted(cu, t, side="right") - 1]
            for h in range(H):
                g = h // (H // Hkv)
                s = kn[c0:t + 1, g] @ qn[t, h] * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                worst = max(worst, oracle.attn_ratio(got[t, h], p @ vn[c0:t + 1, g], p @ np.abs(vn[c0:t + 1, g])))
    print(f"[parity] packed {lens[:8]} {H}/{Hkv}x{D}: max |err| / bar = {worst:.3f}", flush=True)
    assert worst <= 1.0
    return o


CASES = [  # lengths, H, Hkv, D, rows behind
    ([1], 1, 1, 64, 0), ([1], 4, 2, 128, 3), ([1, 1, 1], 2, 1, 128, 0), ([0, 5, 0, 0, 7, 0], 2, 2, 64, 2),
    ([63, 1, 64, 65], 4, 1, 128, 0), ([128, 128], 2, 2, 64, 0), ([127, 129, 2], 2, 1, 64, 1), ([31, 33, 32, 64, 1, 95], 2, 1, 128, 200),
    ([200], 6, 2, 128, 0), ([300, 17], 8, 8, 64, 0), ([1] * 150, 2, 1, 64, 0), ([3, 250, 3], 3, 1, 128, 70),
]


@pytest.mark.parametrize("lens,H,Hkv,D,pad", CASES)
def test_packed(lens, H, Hkv, D, pad):
    check(torch_or_skip(), lens, H, Hkv, D, pad, seed=len(lens))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,lens", [(2, [700, 5, 900, 64, 1, 331]), (32, [513, 1500, 1, 2200])])
def test_packed_both_forms_sampled(H, lens, D):
    """Few and many workgroups (keys of a query over two waves, or not): rows at the borders and in between."""
    torch = torch_or_skip()
    cu = starts(lens)
    rows = sorted({int(c) + d for c in cu for d in (-1, 0, 1, 63, 130) if 0 <= c + d < cu[-1]})
    check(torch, lens, H, max(1, H // 8), D, 40, seed=D, rows=rows)


@pytest.mark.parametrize("std", [4.0, 16.0])
def test_packed_sharp(std):
    check(torch_or_skip(), [150, 90, 1, 200], 2, 1, 128, seed=3, std=std)


def test_many_prompts():
    """More prompts than a workgroup has threads, most of them empty: the first one of a tile is found in steps."""
    torch = torch_or_skip()
    rng = np.random.default_rng(8)
    lens = np.where(rng.random(3000) < 0.9, 0, rng.integers(1, 4, 3000))
    check(torch, [int(n) for n in lens], 1, 1, 64, 5, seed=5)
    big = np.zeros(70001, dtype=np.int64)                     # a third step of the search
    big[[0, 300, 65536, 69999]] = [40, 130, 77, 3]
    check(torch, [int(n) for n in big], 1, 1, 64, seed=6)


def test_one_prompt_equals_attention_prefill():
    """A single prompt through both entry points: the same weights and sums, so the outputs agree to fp32 order."""
    torch = torch_or_skip()
    m = q()
    for S, H, Hkv, D in ((257, 4, 2, 128), (1000, 8, 8, 64)):
        row, bits, cu = make([S], H, Hkv, D, seed=S)
        d = dev_bf16(torch, bits)
        a, b, c = (x.contiguous() for x in views(d, H, Hkv))
        o = host_bf16(torch, m.attention_packed(a, b, c, dev_i32(torch, cu)))
        p = host_bf16(torch, m.attention_prefill(a[None], b[None], c[None])[0])
        ref, absv = oracle.packed_attention(*views(row, H, Hkv), cu, D ** -0.5) if S < 300 else (p, np.abs(p) + 1)
        assert np.all(np.abs(o - p) <= 2 * oracle.attn_tolerance(ref, absv))


@pytest.mark.parametrize("H", [1, 32, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_prompts_do_not_touch_each_other(bad, H):
    """Infinite and NaN queries, keys and values of one prompt (and of rows of none) reach no other prompt's rows,
    nor rows before them of their own."""
    torch = torch_or_skip()
    m = q()
    lens, D = [70, 20, 1, 45, 130, 9], 128
    Hkv = max(1, H // 8)
    row, bits, cu = make(lens, H, Hkv, D, 50, seed=11)
    d = dev_bf16(torch, bits)
    clean = m.attention_packed(*views(d, H, Hkv), dev_i32(torch, cu))
    e = d.clone()
    e[cu[1]:cu[2], :] = bad                       # a prompt as a whole
    e[cu[3] + 30, H + Hkv:, 5] = bad              # one value of another, from its row 30 on
    e[cu[4] + 60, H:H + Hkv, 7] = bad             # one key
    e[cu[-1]:] = bad                              # rows of no prompt
    o = m.attention_packed(*views(e, H, Hkv), dev_i32(torch, cu))
    for r0, r1 in ((cu[0], cu[1]), (cu[2], cu[3] + 30), (cu[4], cu[4] + 60), (cu[5], cu[6])):
        assert torch.isfinite(o[r0:r1].float()).all()
        diff = (o[r0:r1].float() - clean[r0:r1].float()).abs()
        assert torch.all(diff <= 2.0 ** -6 * clean[r0:r1].float().abs() + 2.0 ** -7 * 4)
    assert not torch.isfinite(o[cu[1]:cu[2]].float()).any()
    assert not torch.isfinite(o[cu[3] + 30:cu[4], :, 5].float()).any()
    assert torch.isfinite(o[cu[3] + 30:cu[4], :, 6].float()).all()


@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 64), (32, 4, 128)])
def test_an_early_infinite_value_stays_cheap_and_in_its_element(H, Hkv, D):
    """One infinite value near the start of a long prompt: its element of the rows that see it is infinite, everything else
    as without it. And the call takes a few times as long, for looking at the keys that those rows do not see, not 200
    times, for computing each of them by itself."""
    torch = torch_or_skip()
    m = q()
    lens = [5, 4000, 40, 700]
    row, bits, cu = make(lens, H, Hkv, D, seed=13)
    d, cud = dev_bf16(torch, bits), dev_i32(torch, cu)

    def us(x):
        best = 1e9
        for _ in range(3):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            o = m.attention_packed(*views(x, H, Hkv), cud)
            b.record()
            torch.cuda.synchronize()
            best = min(best, 1e3 * a.elapsed_time(b))
        return o.float(), best

    us(d)
    clean, t0 = us(d)
    e = d.clone()
    at = int(cu[1]) + 3
    e[at, H + Hkv:, 5] = float("inf")
    o, t1 = us(e)
    print(f"[time] {H}/{Hkv}x{D}: {t0:.1f} us, with an infinite value {t1:.1f}", flush=True)
    assert torch.all(o[at:cu[2], :, 5] == float("inf"))
    o[at:cu[2], :, 5] = clean[at:cu[2], :, 5]
    assert torch.all((o - clean).abs() <= 2.0 ** -6 * clean.abs() + 2.0 ** -7 * 4)
    assert t1 < 20 * t0 + 100


def test_strides_of_every_operand_and_determinism():
    torch = torch_or_skip()
    m = q()
    lens, H, Hkv, D = [90, 3, 61], 4, 2, 64
    row, bits, cu = make(lens, H, Hkv, D, seed=4)
    d = dev_bf16(torch, bits)
    a, b, c = (x.contiguous() for x in views(d, H, Hkv))
    cud = dev_i32(torch, cu)
    o = m.attention_packed(a, b, c, cud)

    def wider(x, extra):
        w = torch.zeros((x.shape[0], x.shape[1] * D + extra), dtype=torch.bfloat16, device="cuda")
        w[:, :x.shape[1] * D] = x.flatten(1)
        return w[:, :x.shape[1] * D].unflatten(1, (x.shape[1], D))

    out = wider(torch.zeros_like(o), 24)
    p = m.attention_packed(wider(a, 8), wider(b, 16), wider(c, 40), cud, out=out)
    assert torch.equal(o, p)
    for _ in range(3):
        assert torch.equal(m.attention_packed(a, b, c, cud), o)


def test_inconsistent_table_stays_in_bounds():
    """Tables that do not ascend or pass T: some rows come out, nothing else is written."""
    torch = torch_or_skip()
    m = q()
    T, H, D = 300, 2, 64
    x = torch.randn((T, 4, D), device="cuda").to(torch.bfloat16)
    buf = torch.full((T + 64, H, D), 9.0, dtype=torch.bfloat16, device="cuda")
    for cu in ([0, 100, 50, 900], [0, -5, 300], [7, 200], [0, 2 ** 31 - 1], [-9, -3], [300, 0], [0]):
        m.attention_packed(x[:, :2], x[:, 2:3], x[:, 3:], dev_i32(torch, cu), out=buf[32:32 + T])
        torch.cuda.synchronize()
        assert torch.all(buf[:32] == 9) and torch.all(buf[32 + T:] == 9)
