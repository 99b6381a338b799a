"""GPU: ``adapters`` where an adapter's weights or its inner sums are infinite: y += gain b (a x) as the formula has it, an
infinity times a number an infinity of the product's sign, and NaN only where the formula gives it (0 times infinity, infinity
less infinity, NaN itself), whatever bits the inner sum has."""
import numpy as np
import pytest

from gpu_util import dev_f32, torch_or_skip
from serve_util import bf16, dev_bf16, dev_i32

pytestmark = pytest.mark.gpu

INF, NAN = np.inf, np.nan
# inner sums, each the sum of two bf16 products: of few bits and of all 24, of either sign
SUMS = [(1.0, 0.0), (1.0, 2.0 ** -23), (1.0, 2.0 ** -8), (1.0, 2.0 ** -16), (-1.0, 0.0), (-3.0, -2.0 ** -15), (0.5, 0.0), (2.0 ** -80, 0.0), (-2.0 ** -80, 0.0),
        (2.0 ** 100, 2.0 ** 77), (255.0, 255 * 2.0 ** -16), (0.0, 0.0), (INF, 1.0), (-INF, 1.0), (NAN, 0.0)]
WEIGHTS = [INF, -INF, 1.0, -2.0, 0.0, NAN]


@pytest.mark.parametrize("M,r,N", [(16, 8, 6), (16, 40, 70), (250, 128, 6), (300, 8, 70), (300, 24, 6), (300, 64, 70), (300, 128, 40), (33000, 16, 6)])
@pytest.mark.parametrize("gain", [None, -0.5])
def test_infinities_are_the_formulas(M, r, N, gain):
    import paper_2607_19438_amd as m
    torch = torch_or_skip()
    K, j = 16, r - 3                                       # the only rank with a sum other than 0
    x, xb = bf16(np.array([SUMS[i % len(SUMS)] + (0.0,) * (K - 2) for i in range(M)]))
    a, ab = bf16(np.zeros((1, r, K)))
    a[0, j, :2], ab[0, j, :2] = bf16([1.0, 1.0])
    a[0, :, 2:], ab[0, :, 2:] = bf16(np.ones((r, K - 2)))
    xf = np.where(np.isfinite(x), x, 0.0)
    rows = np.isfinite(x).all(1)                           # (in the others every rank's sum is infinity times 0)
    b, bb = bf16(np.ones((1, N, r)))
    b[0, :, j], bb[0, :, j] = bf16([WEIGHTS[c % len(WEIGHTS)] for c in range(N)])
    y = np.arange(M * N).reshape(M, N) % 7 - 3.0
    got = m.adapters(dev_f32(torch, y), dev_bf16(torch, xb), dev_bf16(torch, ab), dev_bf16(torch, bb), dev_i32(torch, np.zeros(M)),
                     None if gain is None else dev_f32(torch, [gain])).cpu().numpy().astype(np.float64)
    g = 1.0 if gain is None else gain
    mid = xf[:, :2].sum(1) * g
    with np.errstate(invalid="ignore"):
        want = y + mid[:, None] * b[0, :, j][None]
    odd = ~np.isfinite(want)
    for p in (INF, -INF):
        assert np.array_equal((got == p)[rows], (want == p)[rows])
    assert np.array_equal(np.isnan(got)[rows], np.isnan(want)[rows])
    near = rows[:, None] & ~odd
    tol = 2.0 ** -22 * (np.abs(y) + np.abs(np.where(odd, 0.0, want)))      # exact products; y's addition, and gain's, once each
    assert (np.abs(got - want)[near] <= tol[near]).all()
    assert np.isnan(got[~rows]).all()


@pytest.mark.parametrize("M,r", [(20, 8), (300, 64)])
def test_infinite_inner_sums(M, r):
    """a's only rank other than 0 is one of all-infinite sums: infinity times a number, and NaN at 0 alone."""
    import paper_2607_19438_amd as m
    torch = torch_or_skip()
    K = 8
    x, xb = bf16(np.ones((M, K)))
    a, ab = bf16(np.zeros((1, r, K)))
    a[0, 2, 0], ab[0, 2, 0] = (v[0] for v in bf16([-INF]))
    weights = [1.0, -2.0, 0.0, INF, -INF, NAN]
    b, bb = bf16(np.zeros((1, 6, r)))
    b[0, :, 2], bb[0, :, 2] = bf16(weights)
    got = m.adapters(torch.zeros((M, 6), device="cuda"), dev_bf16(torch, xb), dev_bf16(torch, ab), dev_bf16(torch, bb), dev_i32(torch, np.zeros(M))).cpu().numpy()
    assert np.array_equal(got, np.tile(np.array([-INF, INF, NAN, -INF, INF, NAN]), (M, 1)), equal_nan=True)
