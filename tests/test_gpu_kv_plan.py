"""GPU: ``kv_plan`` against the oracle's token-by-token plan; every output is a whole number and equal."""
import numpy as np
import pytest

import oracle
from gpu_util import torch_or_skip
from serve_util import dev_i32, starts

pytestmark = pytest.mark.gpu


def q():
    import paper_2607_19438_amd as m
    return m


def check(torch, kv, new, table, free, page, T):
    want = oracle.kv_plan(kv, new, table, free, page, T)
    tab = dev_i32(torch, table)
    p = q().kv_plan(dev_i32(torch, kv), dev_i32(torch, new), tab, dev_i32(torch, free), page, T)
    torch.cuda.synchronize()
    for name, got, ref in zip(("cu_q", "positions", "slots", "table", "kv_len", "used"),
                              (p.cu_q, p.positions, p.slots, tab, p.kv_len, p.used), want):
        assert np.array_equal(got.cpu().numpy(), ref), name


CASES = [  # requests, page, largest kv, largest q, rows behind the last token, free pages less than needed
    (1, 16, 0, 1, 0, 0), (1, 16, 100, 1, 3, 0), (3, 16, 40, 40, 0, 0), (64, 16, 8000, 1, 0, 0), (65, 32, 500, 9, 17, 0),
    (256, 64, 1000, 1, 0, 0), (257, 128, 1000, 30, 5, 0), (700, 16, 300, 12, 100, 0), (4096, 1024, 5000, 2, 1, 0),
    (9, 16, 64, 200, 0, 5), (2, 16, 3, 3000, 0, 1000),
]


@pytest.mark.parametrize("R,page,kv_max,q_max,pad,short", CASES)
def test_plan(R, page, kv_max, q_max, pad, short):
    torch = torch_or_skip()
    rng = np.random.default_rng(R + page)
    kv = rng.integers(0, kv_max + 1, R)
    new = rng.integers(0, q_max + 1, R)
    new[rng.random(R) < 0.2] = 0
    kv[rng.random(R) < 0.2] //= page
    kv[0] = kv[0] // page * page                 # a request whose pages are full
    need = -(-(kv + new) // page)
    have = -(-kv // page)
    W = int(need.max()) + 1
    table = rng.integers(0, 10000, (R, W))
    free = rng.permutation(int((need - have).sum()) + 4)[:max(0, int((need - have).sum()) + 4 - short)] + 20000
    check(torch, kv, new, table, free, page, int(new.sum()) + pad)


def test_plan_edges():
    torch = torch_or_skip()
    # nothing at all; no request; requests without tokens; a narrow table; bad entries; more tokens than rows
    check(torch, [5, 0], [0, 0], [[3], [4]], [9], 16, 0)
    check(torch, [5, 0], [0, 0], [[3], [4]], [9], 16, 7)
    check(torch, [0, 31, 15], [50, 2, 1], [[-1] * 2, [5, 6], [8, 9]], [1, 2, 3, 4], 16, 53)
    check(torch, [10, 20], [4, 4], [[-7, -1], [3, -9]], [1], 16, 8)
    check(torch, [16, 0, 5], [40, 40, 1], [[1, -1, -1, -1], [-1] * 4, [2, -1, -1, -1]], list(range(30, 40)), 16, 50)
    check(torch, [-3, 4], [2, -1], [[-1], [6]], [11], 16, 4)
    m = q()
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    p = m.kv_plan(e, e, torch.empty((0, 4), dtype=torch.int32, device="cuda"), e, 16, 5)
    torch.cuda.synchronize()
    assert p.cu_q.tolist() == [0] and p.slots.tolist() == [-1] * 5 and p.positions.tolist() == [0] * 5 and p.used.tolist() == [0]


def test_plan_slots_past_31_bits_are_refused():
    torch = torch_or_skip()
    check(torch, [0, 3], [1, 1], [[0], [2 ** 27 - 1]], [2 ** 27], 16, 2)


def test_a_plan_is_not_written_over_its_own_input():
    """Lengths fed back into the plan that they come from: refused, nothing written. Two plans in turn: as the oracle."""
    torch = torch_or_skip()
    m = q()
    R, T, W, page = 300, 900, 40, 16
    rng = np.random.default_rng(5)
    kv = rng.integers(0, 400, R)
    new = np.full(R, 3)
    table = np.full((R, W), -1)
    table[:, :25] = np.arange(R * 25).reshape(R, 25)
    free = np.arange(1000) + 20000
    tab, freed, newd = dev_i32(torch, table), dev_i32(torch, free), dev_i32(torch, new)
    plans, kvd, at = (m.KvPlan(R, T, "cuda"), m.KvPlan(R, T, "cuda")), dev_i32(torch, kv), 0
    for step in range(6):
        want = oracle.kv_plan(kv, new, table, free[at:], page, T)
        p = m.kv_plan(kvd, newd, tab, freed[at:].contiguous(), page, T, out=plans[step & 1])
        for got, ref in zip((p.cu_q, p.positions, p.slots, tab, p.kv_len, p.used), want):
            assert np.array_equal(got.cpu().numpy(), ref)
        table, kv, kvd, at = want[3], want[4], p.kv_len, at + int(want[5][0])
        before = [t.clone() for t in (p.cu_q, p.positions, p.slots, p.kv_len, p.used, tab)]
        for bad in (lambda: m.kv_plan(p.kv_len, newd, tab, freed, page, T, out=p), lambda: m.kv_plan(kvd, p.kv_len, tab, freed, page, T, out=p),
                    lambda: m.kv_plan(kvd, newd, tab, p.slots, page, T, out=p), lambda: m.kv_plan(kvd, newd, tab, tab.view(-1), page, T)):
            with pytest.raises(m.QGemmError, match="overlap"):
                bad()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(before, (p.cu_q, p.positions, p.slots, p.kv_len, p.used, tab)))


def test_plan_writes_its_outputs_only():
    torch = torch_or_skip()
    m = q()
    R, T, W = 5, 33, 4
    kv, new = [3, 0, 17, 40, 16], [5, 9, 1, 3, 15]
    buf = torch.full((400,), 77, dtype=torch.int32, device="cuda")
    out = m.KvPlan(R, T, "cuda")
    off = 3                                       # 4-byte aligned only
    for name, n in (("cu_q", R + 1), ("positions", T), ("slots", T), ("kv_len", R), ("used", 1)):
        setattr(out, name, buf[off:off + n])
        off += n + 5
    table = torch.full((R, W), -1, dtype=torch.int32, device="cuda")
    table[:, 0], table[2:4, 1], table[3, 2] = 1, 2, 3
    before = table.cpu().numpy().copy()
    free = dev_i32(torch, range(50, 60))
    m.kv_plan(dev_i32(torch, kv), dev_i32(torch, new), table, free, 16, T, out=out)
    want = oracle.kv_plan(kv, new, before, list(range(50, 60)), 16, T)
    assert np.array_equal(table.cpu().numpy(), want[3])
    b = buf.cpu().numpy()
    off = 3
    for ref in (want[0], want[1], want[2], want[4], want[5]):
        assert np.array_equal(b[off:off + len(ref)], ref)
        assert np.all(b[off + len(ref):off + len(ref) + 5] == 77)
        off += len(ref) + 5
    assert np.all(b[:3] == 77)
    assert np.array_equal(starts(new), want[0])
