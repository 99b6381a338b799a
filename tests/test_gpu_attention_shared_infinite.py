"""GPU: ``attention_kv4_shared`` where a row's scores overflow to -inf over its own keys alone, or over the shared ones alone: the
softmax of the others, in each form of the kernel; over all of them: NaN."""
import numpy as np
import pytest

import oracle
from gpu_util import torch_or_skip
from serve_util import bf16, host_bf16
from test_gpu_attention_shared import make, run

pytestmark = pytest.mark.gpu

HUGE = -2.0 ** 127


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("prefix,own,new,H,Hkv", [
    (128, [30] * 5, [1] * 5, 8, 2), (192, [20 + i % 9 for i in range(40)], [1] * 40, 32, 8), (256, [20 + i % 9 for i in range(170)], [1] * 170, 32, 8),
    (192, [60, 47, 33], [9, 5, 7], 16, 2), (192, [400, 433], [400, 433], 32, 4),
])
def test_part_of_the_scores_is_minus_infinity(prefix, own, new, H, Hkv, D):
    torch = torch_or_skip()
    page, R = 16, len(own)
    c = make([0, R], [prefix], own, new, H, Hkv, D, page, seed=R + D, wrong=False)
    # of the first block of every key only elements 5 and 6 are left: 1024 and 0 behind the shared keys, 0 and 1024 among them
    n0, sb = page * D, D // 32
    shared = [int(p) for p in c["table"][0, :prefix // page]]
    cache = c["cache"]
    for p in range(len(cache)):
        for o in range(page):
            at = o * (D // 2)
            cache[p, :, at:at + 16] = 0
            cache[p, :, n0 + o * sb] = 137                 # 2^10
            if p in shared:
                cache[p, :, at + 3] = 0x02                 # element 6: 1.0
            else:
                cache[p, :, at + 2] = 0x20                 # element 5
    c["k"], c["v"] = oracle.decode_cache(cache, D)
    T = int(c["cu"][-1])
    q = c["q"]
    q[:, :, 5:7] = 0.0
    rows = sorted({0, 1, 2, 3, T // 2, T // 2 + 1, T - 2, T - 1})
    for i, t in enumerate(rows):
        if i % 3 == 0:
            q[t, :, 5] = HUGE                              # own keys: -2^137
        elif i % 3 == 1:
            q[t, :, 6] = HUGE                              # shared keys
    both = rows[2]
    q[both, :, 5:7] = HUGE
    c["q"], c["bits"] = bf16(q)
    got = host_bf16(torch, run(torch, c))
    keep = [t for t in rows if t != both]
    ref, absv = oracle.shared_attention(c["q"], c["k"], c["v"], c["table"], c["kv"], c["cu"], [0, R], [prefix], page, D ** -0.5, set(keep))
    worst = oracle.attn_ratio(got[keep], ref[keep], absv[keep])
    print(f"[parity] shared, part of the scores -inf, {q.shape}: max |err| / bar = {worst:.3f}", flush=True)
    assert worst <= 1.0 and np.isnan(got[both]).all()
    assert np.isfinite(np.delete(got, both, 0)).all()
