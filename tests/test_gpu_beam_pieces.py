"""GPU: ``beam_select`` over rows of up to 74 pieces, whose maxima and sums a lane, a part of a wave or a wave's lanes in turn
join: among them pieces with no candidate at all, and a NaN or an infinity in the last piece only."""
import numpy as np
import pytest

from gpu_util import torch_or_skip
from test_gpu_beam_select import check

pytestmark = pytest.mark.gpu


def pieces(R, B, V, K):
    import paper_2607_19438_amd as m
    return m._workspace("beam_select", R, B, V, K) // (R * B * (16 + 8 * K))         # maximum and sum, and K candidates


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("R,B,K,V,n", [(1, 1, 4, 300001, 74), (1, 3, 4, 300001, 74), (2, 2, 2, 270000, 66), (1, 1, 7, 262144, 64), (1, 5, 3, 150001, 37),
                                       (3, 2, 4, 100003, 25), (1, 4, 8, 70000, 18)])
def test_many_pieces(R, B, K, V, n, bf):
    torch = torch_or_skip()
    assert pieces(R, B, V, K) == n
    rng = np.random.default_rng(n + B)
    x = 3 * rng.standard_normal((R * B, V))
    check(torch, x, -5 * rng.random((R, B)), K, bf=bf)
    x[:, :V * 9 // 10] = -np.inf                           # nothing in all pieces but the last few
    check(torch, x, -5 * rng.random((R, B)), K, bf=bf)
    x[:, :] = -np.inf
    x[:, V - 1] = rng.standard_normal(R * B)               # one candidate, in the last
    got, par, tok, _ = check(torch, x, np.zeros((R, B)), K, bf=bf)
    assert (tok[got > -np.inf] == V - 1).all() and (got[got > -np.inf] == 0).all()


@pytest.mark.parametrize("V,n", [(300001, 74), (150001, 37), (70000, 18)])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_what_only_the_last_piece_holds(V, n, bad):
    torch = torch_or_skip()
    assert pieces(1, 3, V, 4) == n
    rng = np.random.default_rng(n)
    x = 2 * rng.standard_normal((3, V))
    x[1, V - 3] = bad
    got, par, tok, _ = check(torch, x, [[-1.0, 0.0, -2.0]], 4)
    assert 1 not in par[0] and (par[0] >= 0).all()
    x[:, V - 2] = bad
    got, par, tok, _ = check(torch, x, [[-1.0, 0.0, -2.0]], 4, end=3)
    assert (par == -1).all() and (tok == 3).all()
    # a beam's largest logit in the last piece, far above the sums before it
    x = 2 * rng.standard_normal((3, V))
    x[:, V - 1] = [200.0, -200.0, 80.0]
    got, par, tok, _ = check(torch, x, [[-1.0, 0.0, -2.0]], 4)
    assert tok[0, 0] == V - 1 and par[0, 0] == 0 and got[0, 0] == -1.0
