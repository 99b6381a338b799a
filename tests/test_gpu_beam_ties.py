"""GPU: the order of ``beam_select``'s candidates where values are equal. Of a beam the order is that of the logits, equal ones
the lower token first, also where the score is so large that logits of different size give one value in 64 bits; between
beams equal values go to the lower beam. It does not depend on the pieces that a row is cut into, so every order here is
exact."""
import numpy as np
import pytest

import oracle
from gpu_util import torch_or_skip

pytestmark = pytest.mark.gpu


def call(torch, logits, scores, K, bf=False):
    import paper_2607_19438_amd as m
    x = torch.from_numpy(np.asarray(logits, dtype=np.float32)).cuda()
    x = x.to(torch.bfloat16) if bf else x
    s, p, t = m.beam_select(x, torch.from_numpy(np.asarray(scores, dtype=np.float32)).cuda(), K)
    return s.cpu().numpy(), p.cpu().numpy(), t.cpu().numpy(), x.float().cpu().numpy().astype(np.float64)


def by_logit(x, K):
    """The tokens of a row: larger logits first, of equal ones the lower token."""
    return np.argsort(-x, kind="stable")[:K]


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("V", [4, 4096, 20000, 120001])
@pytest.mark.parametrize("score", [-1e30, -1e10, 1e20, np.inf])
def test_scores_that_hide_the_logits(score, V, bf):
    """One beam and three of equal scores, alone and among 400 requests: 1 to 30 pieces of a row, and one."""
    torch = torch_or_skip()
    rng = np.random.default_rng(V)
    row = 3 * rng.standard_normal(V)
    if V == 4:
        row = np.array([1.0, 1.5, 2.0, 0.0])
    K = min(V, 24)
    s, p, t, x = call(torch, row[None], [[score]], K, bf)
    assert t[0].tolist() == by_logit(x[0], K).tolist() and (p == 0).all() and (s == np.float32(score)).all()
    if np.isfinite(score):
        assert np.array_equal(t, oracle.beam_select(x, np.array([[score]]), K)[2])
    # three beams: at -1e30 and 1e20 all candidates are worth the same, and the first beam has them all
    s, p, t, x = call(torch, np.stack([row, row[::-1], row]), [[score] * 3], K, bf)
    if score != -1e10:
        assert (p == 0).all() and t[0].tolist() == by_logit(x[0], K).tolist()
    for b in range(3):
        mine = t[0][p[0] == b]
        assert mine.tolist() == by_logit(x[b], len(mine)).tolist()
    if V <= 20000 and score != -1e10:
        many, pm, tm, _ = call(torch, np.tile(np.stack([row, row[::-1], row]), (400, 1)), [[score] * 3] * 400, K, bf)
        assert (tm[[0, 77, 399]] == t[0]).all() and (pm[[0, 77, 399]] == p[0]).all()


@pytest.mark.parametrize("V", [300, 30000])
def test_logits_too_small_to_show(V):
    """Logits of 1e-30 beside zeros: one value in 64 bits, and the larger logit first all the same, whichever piece it is in."""
    torch = torch_or_skip()
    row = np.zeros(V)
    row[[V - 1, V // 2, 7]] = [3e-30, 2e-30, 1e-30]
    row[[5, V - 2]] = -1e-30
    want = [V - 1, V // 2, 7] + [v for v in range(V) if row[v] == 0][:9]
    s, p, t, x = call(torch, np.stack([row, row]), [[0.0, 0.0]], 12)
    assert t[0].tolist() == want and (p == 0).all()
    assert np.array_equal(t, oracle.beam_select(x, np.zeros((1, 2)), 12)[2])


def test_equal_beams_of_few_tokens():
    """Values that tie within beams and between them, with fewer tokens to a beam than are taken."""
    torch = torch_or_skip()
    rng = np.random.default_rng(5)
    x = rng.integers(-3, 4, (8, 40)).astype(float)
    x[1, 3:] = -np.inf
    s, p, t, x = call(torch, x, [[-1e30] * 8], 128)
    want = [(b, int(v)) for b in range(8) for v in by_logit(x[b], 40) if x[b, v] > -np.inf][:128]
    assert list(zip(p[0].tolist(), t[0].tolist())) == want
    _, po, to = oracle.beam_select(x, np.full((1, 8), -1e30), 128)
    assert np.array_equal(p, po) and np.array_equal(t, to)
