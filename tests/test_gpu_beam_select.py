"""GPU: ``beam_select`` against the fp64 oracle. A value may be off by the oracle's ``beam_tolerance``; which candidate stands at a
place may differ from the oracle's only where their values lie within twice that. Ties are exact."""
import numpy as np
import pytest

import oracle
from gpu_util import torch_or_skip

pytestmark = pytest.mark.gpu


def q():
    import paper_2607_19438_amd as m
    return m


def dev(torch, a, bf=False):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if bf else t


def call(torch, logits, scores, K, finished=None, end=0, bf=False):
    """The call's results and the logits as the device holds them."""
    x = dev(torch, logits, bf)
    f = None if finished is None else torch.from_numpy(np.asarray(finished)).cuda()
    s, p, t = q().beam_select(x, dev(torch, scores), K, finished=f, end=end)
    return s.cpu().numpy(), p.cpu().numpy(), t.cpu().numpy(), x.float().cpu().numpy().astype(np.float64)


def check(torch, logits, scores, K, finished=None, end=0, bf=False):
    got, par, tok, x = call(torch, logits, scores, K, finished, end, bf)
    scores = np.asarray(scores, dtype=np.float32).astype(np.float64)
    R, B = scores.shape
    want, _, _ = oracle.beam_select(x, scores, K, finished, end)
    worst = 0.0
    for r in range(R):
        val = oracle.beam_values(x[r * B:(r + 1) * B], scores[r], None if finished is None else finished[r], end)
        taken = set()
        for k in range(K):
            if want[r, k] == -np.inf:
                assert got[r, k] == -np.inf and par[r, k] == -1 and tok[r, k] == end
                continue
            b, v = int(par[r, k]), int(tok[r, k])
            assert 0 <= b < B and 0 <= v < x.shape[1] and (b, v) not in taken
            taken.add((b, v))
            if finished is not None and finished[r][b]:                     # the beam's own score, to the bit
                assert v == end and got[r, k] == scores[r, b]
                tol = 2.0 ** -23 * abs(val[b, v]) + 1e-37
            else:
                tol = oracle.beam_tolerance(x[r * B + b], val[b, v])
            assert abs(val[b, v] - want[r, k]) <= 2 * tol                   # a candidate worth what the oracle's is
            worst = max(worst, abs(got[r, k] - val[b, v]) / tol)
    print(f"[parity] beam {R}x{B} V={x.shape[1]} K={K} {'bf16' if bf else 'fp32'}: max |err| / tol = {worst:.3f}", flush=True)
    assert worst <= 1.0
    return got, par, tok, x


SIZES = [  # R, B, K, V, bf16
    (1, 1, 1, 1, False), (1, 4, 4, 3, False), (2, 3, 6, 5, True), (1, 1, 7, 100, False), (3, 4, 4, 1000, True), (1, 4, 4, 4095, False),
    (2, 2, 4, 4096, True), (1, 5, 10, 4097, False), (2, 1, 1, 8193, True), (1, 4, 8, 32000, False), (3, 5, 10, 50021, True),
    (1, 64, 128, 5000, False), (2, 8, 128, 4500, True), (300, 4, 4, 300, False), (260, 4, 8, 9001, True),
]


@pytest.mark.parametrize("R,B,K,V,bf", SIZES)
def test_sizes(R, B, K, V, bf):
    rng = np.random.default_rng(R + V)
    check(torch_or_skip(), 3 * rng.standard_normal((R * B, V)), -10 * rng.random((R, B)), K, bf=bf)


@pytest.mark.parametrize("bf", [False, True])
def test_ended_beams_and_beams_that_are_not_there(bf):
    torch = torch_or_skip()
    rng = np.random.default_rng(1)
    R, B, V = 6, 4, 5000
    scores = -8 * rng.random((R, B))
    scores[0, 1:] = -np.inf
    scores[1, 2] = np.nan
    scores[3] = -np.inf
    done = rng.random((R, B)) < 0.4
    done[0] = [False, True, True, True]
    done[2] = True
    logits = 2 * rng.standard_normal((R * B, V))
    logits[done.ravel()] = np.nan                         # not read
    got, par, tok, _ = check(torch, logits, scores, 8, done, 7, bf)
    assert (par[3] == -1).all() and (tok[3] == 7).all() and (got[3] == -np.inf).all()
    assert sorted(par[2, :4]) == [0, 1, 2, 3] and (tok[2] == 7).all() and (par[2, 4:] == -1).all()
    flags = call(torch, logits, scores, 8, done.astype(np.uint8), 7, bf)
    assert np.array_equal(flags[0], got) and np.array_equal(flags[1], par) and np.array_equal(flags[2], tok)


def test_infinities_and_nan_stay_in_their_beam():
    torch = torch_or_skip()
    rng = np.random.default_rng(2)
    V = 9000
    logits = 2 * rng.standard_normal((8, V))
    logits[1, 8999] = np.nan
    logits[2, 17] = np.inf
    logits[3] = -np.inf
    logits[4, ::2] = -np.inf                              # tokens that are masked out
    logits[5] = -np.inf
    logits[5, 4444] = 1e30                                # a single token
    logits[6] *= 1e30
    got, par, tok, _ = check(torch, logits, np.zeros((1, 8)), 128)
    assert not set(par[0]) & {1, 2, 3} and set(par[0]) >= {0, 4, 5, 6}
    assert (tok[0][par[0] == 4] % 2 == 1).all() and (tok[0][par[0] == 5] == 4444).all()
    alone, par, tok, _ = check(torch, logits[5:6], np.zeros((1, 1)), 4)
    assert alone[0].tolist() == [0.0] + [-np.inf] * 3 and tok[0].tolist() == [4444, 0, 0, 0]


@pytest.mark.parametrize("bf,V", [(False, 300), (True, 4096), (False, 20000), (True, 60001)])
def test_ties_go_to_the_lower_beam_and_token(bf, V):
    """Equal logits, and equal rows of equal scores: exactly the order of the numbers, in one piece of a row and in several."""
    torch = torch_or_skip()
    rng = np.random.default_rng(3)
    for logits in (np.zeros((6, V)), np.tile(rng.integers(0, 3, V), (6, 1)).astype(float), np.tile(-np.abs(np.arange(V) % 7 - 3.0), (6, 1))):
        logits[logits == 0] = np.where(rng.random((logits == 0).sum()) < 0.5, 0.0, -0.0)      # zeros of either sign are equal
        got, par, tok, x = call(torch, logits, np.zeros((2, 3)), 20, bf=bf)
        _, p, t = oracle.beam_select(x, np.zeros((2, 3)), 20)
        assert np.array_equal(par, p) and np.array_equal(tok, t)
        assert len(set(got[0])) == len(set(got[1])) and np.array_equal(got[0], got[1])


@pytest.mark.parametrize("order", ["ascending", "descending", "late", "comb"])
def test_orders_that_fill_the_list(order):
    """Rows in one piece whose best come last, first, in a run, or all in one thread's places."""
    torch = torch_or_skip()
    V, B = 13000, 64
    rng = np.random.default_rng(4)
    x = {"ascending": np.arange(V) * 1e-3, "descending": -np.arange(V) * 1e-3, "late": np.where(np.arange(V) > V - 3000, 5.0 + np.arange(V) * 1e-3, 0.0),
         "comb": np.where(np.arange(V) % 1024 < 4, 3.0 + np.arange(V) * 1e-4, 0.0)}[order]
    check(torch, np.tile(x, (B, 1)) + 1e-5 * rng.standard_normal((B, V)), -rng.random((1, B)), 128)


def test_rows_at_any_stride_and_past_32_bits():
    torch = torch_or_skip()
    rng = np.random.default_rng(5)
    x = 3 * rng.standard_normal((3, 777))
    for dtype, bf, step in ((torch.bfloat16, True, (1 << 30) + 5), (torch.float32, False, 901)):
        buf = torch.empty(2 * step + 800, dtype=dtype, device="cuda")
        rows = buf[1:].as_strided((3, 777), (step, 1))
        rows.copy_(dev(torch, x, bf))
        s, p, t = q().beam_select(rows, torch.zeros((1, 3), device="cuda"), 5)
        a, b, c, _ = call(torch, x, np.zeros((1, 3)), 5, bf=bf)
        assert np.array_equal(s.cpu().numpy(), a) and np.array_equal(p.cpu().numpy(), b) and np.array_equal(t.cpu().numpy(), c)
        del rows, buf


def test_no_requests():
    torch = torch_or_skip()
    s, p, t = q().beam_select(torch.zeros((0, 50), device="cuda"), torch.zeros((0, 4), device="cuda"), 8)
    assert s.shape == p.shape == t.shape == (0, 8)


def test_same_bits_on_other_streams_and_from_a_graph():
    torch = torch_or_skip()
    rng = np.random.default_rng(6)
    m = q()
    cases = [(dev(torch, 3 * rng.standard_normal((12, 30011)), bf), dev(torch, -5 * rng.random((3, 4)))) for bf in (False, True)]
    first = [m.beam_select(x, s, 8) for x, s in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    outs = [[] for _ in cases]
    for _ in range(3):                                    # two streams at once, each call with a workspace of its own
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                outs[i].append(m.beam_select(*cases[i], 8))
    torch.cuda.synchronize()
    for i, want in enumerate(first):
        for o in outs[i]:
            assert all(torch.equal(a, b) for a, b in zip(o, want))
    x, s = cases[0][0].clone(), cases[0][1].clone()
    with torch.cuda.stream(streams[0]):
        m.beam_select(x, s, 8)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = m.beam_select(x, s, 8)
    for k in range(4):
        x.copy_(cases[0][0] if k % 2 else -cases[0][0])
        g.replay()
        want = m.beam_select(x, s, 8)
        assert all(torch.equal(a, b) for a, b in zip(o, want))
