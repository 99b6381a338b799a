"""GPU: ``kv_reorder`` over so many columns and requests that a workgroup takes several blocks of columns, in either kernel: every
table and list equal to the oracle's integers."""
import numpy as np
import pytest

from gpu_util import torch_or_skip
from test_gpu_kv_reorder import check, history

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,B,W,page,most", [(1100, 2, 600, 16, 9000), (3, 1, 300000, 16, 4700000), (700, 3, 700, 64, 40000), (2100, 1, 270, 16, 4300), (5000, 1, 40, 16, 640),
                                             (1, 2, 250000, 16, 3900000), (30, 4, 20000, 128, 2500000)])
def test_several_blocks_to_a_workgroup(R, B, W, page, most):
    torch = torch_or_skip()
    rng = np.random.default_rng(R + W)
    table, kv, pages = history(rng, R, B, page, most, width=W)
    parents = rng.integers(-1, B, (R, B))
    parents[rng.random(R) < 0.2] = -1                    # whose pages are all released
    free = pages + np.arange(R * B)
    check(torch, table, kv, parents, free, page, keep=rng.integers(0, W // 2, R))
    check(torch, table, kv, parents, free, page, released=int(rng.integers(1, table.size // 3)))
