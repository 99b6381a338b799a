"""GPU: ``adapters`` against the fp64 oracle, within its ``adapter_tolerance`` (fp32 summation alone: the inner sums enter the
second product whole)."""
import numpy as np
import pytest

import oracle
from gpu_util import dev_f32, torch_or_skip
from serve_util import bf16, dev_bf16, dev_i32, starts

pytestmark = pytest.mark.gpu


def q():
    import paper_2607_19438_amd as m
    return m


def make(lens, N, K, r, n, seed=0, pad=0):
    rng = np.random.default_rng(seed)
    M = int(sum(lens)) + pad
    x, xb = bf16(rng.standard_normal((M, K)))
    a, ab = bf16(rng.standard_normal((n, r, K)) * K ** -0.5)
    b, bb = bf16(rng.standard_normal((n, N, r)))
    y = rng.standard_normal((M, N)).astype(np.float32)
    return dict(x=x, xb=xb, a=a, ab=ab, b=b, bb=bb, y=y, gain=rng.uniform(-2, 2, n).astype(np.float32), ids=rng.integers(-1, n, len(lens)),
                cu=starts(lens))


def run(torch, c, ragged, gain=True, y=None):
    y = dev_f32(torch, c["y"]) if y is None else y
    o = q().adapters(y, dev_bf16(torch, c["xb"]), dev_bf16(torch, c["ab"]), dev_bf16(torch, c["bb"]), dev_i32(torch, c["ids"]),
                     dev_f32(torch, c["gain"]) if gain else None, dev_i32(torch, c["cu"]) if ragged else None)
    assert o is y
    return o


def check(torch, c, ragged, gain=True):
    got = run(torch, c, ragged, gain).cpu().numpy()
    args = (c["y"].astype(np.float64), c["x"], c["a"], c["b"], c["ids"], c["gain"] if gain else None, c["cu"] if ragged else None)
    ref, tol = oracle.adapters(*args), oracle.adapter_tolerance(*args)
    none = tol.sum(1) == 0
    assert np.array_equal(got[none], c["y"][none])                       # rows of no adapter: not a bit
    worst = float(np.max(np.abs(got - ref)[~none] / tol[~none])) if (~none).any() else 0.0
    print(f"[parity] adapters {got.shape} r={c['a'].shape[1]} n={len(c['a'])}: max |err| / tol = {worst:.3f}", flush=True)
    assert worst <= 1.0
    return got


SIZES = [  # lens, N, K, r, n, rows behind
    ([1], 1, 8, 8, 1, 0), ([1, 1, 1], 17, 40, 16, 2, 0), ([1] * 16, 64, 256, 8, 16, 0), ([1] * 33, 130, 512, 24, 40, 0), ([1] * 300, 257, 128, 32, 7, 0),
    ([5, 0, 1, 40, 3], 100, 264, 16, 3, 4), ([70], 65, 1000, 64, 1, 0), ([130, 7, 300], 515, 384, 40, 3, 9), ([1, 2, 0, 0, 15, 16, 17], 48, 72, 128, 4, 1),
    ([600, 1, 500, 3], 260, 520, 16, 2, 3), ([2000, 300], 96, 128, 104, 2, 0), ([0, 0], 16, 16, 8, 1, 5), ([1] * 1100, 33, 64, 72, 1100, 0),
    ([700, 700], 1030, 2048, 32, 2, 0),
]


@pytest.mark.parametrize("lens,N,K,r,n,pad", SIZES)
def test_sizes(lens, N, K, r, n, pad):
    torch = torch_or_skip()
    c = make(lens, N, K, r, n, seed=N + K, pad=pad)
    check(torch, c, True)
    if all(x == 1 for x in lens) and not pad:
        check(torch, c, False, gain=False)


@pytest.mark.parametrize("R,most,N,K,r,pad", [(63, 9, 40, 64, 8, 3), (64, 9, 40, 64, 40, 0), (65, 9, 40, 64, 16, 1), (130, 3, 33, 40, 8, 0), (1000, 2, 20, 16, 24, 5),
                                             (4100, 1, 20, 16, 8, 0), (300, 60, 1030, 64, 48, 7), (300, 60, 1030, 64, 8, 0), (90, 60, 1030, 264, 16, 2)])
def test_many_requests(R, most, N, K, r, pad):
    """Requests of no row up to `most`, in every part of a look-up among up to thousands, and tiles of several adapters whose
    workgroups go through more than one piece of the columns."""
    torch = torch_or_skip()
    lens = np.random.default_rng(R).integers(0, most + 1, R)
    lens[[0, R // 2, R - 1]] = [0, most, 0]
    c = make(list(lens), N, K, r, 5, seed=R, pad=pad)
    check(torch, c, True)


def test_interleaved_tenants():
    """Rows that change their adapter at every step, in a batch large enough for tiles of several rows."""
    torch = torch_or_skip()
    c = make([1] * 1500, 70, 256, 16, 9, seed=3)
    check(torch, c, False)


@pytest.mark.parametrize("M,N", [(40, 99), (1300, 140)])
def test_strided_rows(M, N):
    """The columns of one projection within wider rows, at strides of any alignment; nothing beside them is written."""
    torch = torch_or_skip()
    c = make([M - 3, 3], N, 128, 16, 2, seed=4)
    c["ids"] = np.array([1, 0])
    want = run(torch, c, True)
    for width, off in ((N + 11, 5), (4 * N + 4, 8), (N, 0)):
        wide = torch.full((M, width), 7.0, device="cuda")
        view = wide[:, off:off + N]
        view.copy_(dev_f32(torch, c["y"]))
        xs = torch.zeros((M, 128 + 24), dtype=torch.bfloat16, device="cuda")
        xs[:, 8:136] = dev_bf16(torch, c["xb"])
        q().adapters(view, xs[:, 8:136], dev_bf16(torch, c["ab"]), dev_bf16(torch, c["bb"]), dev_i32(torch, c["ids"]), dev_f32(torch, c["gain"]),
                     dev_i32(torch, c["cu"]))
        assert torch.equal(view, want)
        assert torch.all(wide[:, :off] == 7) and torch.all(wide[:, off + N:] == 7)


@pytest.mark.parametrize("lens", [[1] * 20, [9, 3, 5, 3], [600, 500, 200, 40]])
def test_what_one_tenant_holds_reaches_no_other(lens):
    torch = torch_or_skip()
    c = make(lens, 80, 256, 16, 4, seed=5)
    c["ids"] = np.arange(len(lens)) % 4
    clean = run(torch, c, True)
    d = {k: v.copy() for k, v in c.items()}
    d["ab"][1, 3, 100] = 0x7fc0                       # NaN, infinity and -infinity in the weights of adapters 1 and 2,
    d["bb"][1, 7, :] = 0x7f80
    d["bb"][2] = 0xff80
    hit = [r for r in range(len(lens)) if d["ids"][r] == 3][0]
    d["xb"][d["cu"][hit], 9] = 0x7f80                 # and in a row of a request of adapter 3
    o = run(torch, d, True)
    fine = np.ones(len(c["y"]), bool)
    for r in range(len(lens)):
        if d["ids"][r] in (1, 2):
            fine[d["cu"][r]:d["cu"][r + 1]] = False
    fine[d["cu"][hit]] = False
    keep = torch.from_numpy(fine).cuda()
    assert torch.equal(o[keep], clean[keep])
    assert not torch.isfinite(o[~keep]).all(dim=1).any()


def test_large_and_small_inner_sums():
    """Inner sums beyond bf16's largest number stay finite, and those of 2^-100 keep their value."""
    torch = torch_or_skip()
    c = make([2], 4, 8, 8, 1)
    c["ids"] = np.array([0])
    c["y"][:] = 0
    c["gain"][:] = 1
    c["x"], c["xb"] = bf16(np.zeros((2, 8)))
    c["a"], c["ab"] = bf16(np.zeros((1, 8, 8)))
    c["b"], c["bb"] = bf16(np.zeros((1, 4, 8)))
    c["x"][0, 0], c["xb"][0, 0] = (v[0] for v in bf16([2.0 ** 126]))
    c["a"][0, 0, 0], c["ab"][0, 0, 0] = (v[0] for v in bf16([3.984375]))       # 2^126 times that: more than bf16 rounds to
    c["x"][0, 1], c["xb"][0, 1] = (v[0] for v in bf16([2.0 ** 111]))
    c["a"][0, 0, 1], c["ab"][0, 0, 1] = (v[0] for v in bf16([255.0]))
    c["x"][1, 2], c["xb"][1, 2] = (v[0] for v in bf16([2.0 ** -100]))
    c["a"][0, 0, 2], c["ab"][0, 0, 2] = (v[0] for v in bf16([1.0078125]))
    c["b"][0, :, 0], c["bb"][0, :, 0] = bf16([2.0 ** -3, 1.0, -0.5, 2.0 ** 3])
    got = run(torch, c, True).cpu().numpy().astype(np.float64)
    mid = c["a"][0] @ c["x"].T
    assert mid[0, 0] < np.finfo(np.float32).max and oracle.decode_bf16(np.array([0x7f7f]))[0] < mid[0, 0]
    want = (c["b"][0] @ mid).T
    assert np.allclose(got[0, [0, 1, 2]], want[0, [0, 1, 2]], rtol=2.0 ** -22) and got[0, 3] == np.inf
    assert np.allclose(got[1], want[1], rtol=2.0 ** -22)


def test_past_32_bits():
    torch = torch_or_skip()
    c = make([1, 1, 1], 50, 64, 8, 2, seed=6)
    c["ids"] = np.array([1, 0, 1])
    want = run(torch, c, False)
    for step in ((1 << 30) + 12, (1 << 30) + 3):
        buf = torch.empty(2 * step + 64, device="cuda")
        y = buf.as_strided((3, 50), (step, 1))
        y.copy_(dev_f32(torch, c["y"]))
        assert torch.equal(run(torch, c, False, y=y), want)
        del y, buf
    # an adapter behind 2^31 elements of others
    n, r, K, N = 2100, 64, 16384, 64
    a = torch.zeros((n, r, K), dtype=torch.bfloat16, device="cuda")
    b = torch.zeros((n, N, r), dtype=torch.bfloat16, device="cuda")
    assert (n - 1) * r * K > 2 ** 31
    a[n - 1, 5, 17] = 2.0
    b[n - 1, 9, 5] = 3.0
    x = torch.ones((1, K), dtype=torch.bfloat16, device="cuda")
    y = q().adapters(torch.zeros((1, N), device="cuda"), x, a, b, dev_i32(torch, [n - 1]))
    assert y[0, 9] == 6.0 and y.sum() == 6.0


def test_first_rows_that_descend_and_ids_out_of_range():
    torch = torch_or_skip()
    c = make([3, 4, 2], 40, 64, 8, 2, seed=7)
    for ids in ([2, -1, 5], [2 ** 31 - 1, -2 ** 31, 100]):
        c["ids"] = np.array(ids)
        assert np.array_equal(run(torch, c, True).cpu().numpy(), c["y"])
    c["ids"] = np.array([0, 1, 0])
    buf = torch.full((9 + 64, 40), 9.0, device="cuda")
    for cu in ([0, 100, 50, 9], [-5, 3, 2 ** 31 - 1, 9], [9, 9, 0, 4], [-1, -1, -1, -1], [2, 4, 5, 7]):
        c["cu"] = np.array(cu)
        buf[32:41] = dev_f32(torch, c["y"])
        run(torch, c, True, y=buf[32:41])
        torch.cuda.synchronize()
        assert torch.all(buf[:32] == 9) and torch.all(buf[41:] == 9)
    assert torch.equal(buf[32:34], dev_f32(torch, c["y"])[:2]) and torch.equal(buf[39:41], dev_f32(torch, c["y"])[7:])     # the last: rows of none


def test_no_rows():
    torch = torch_or_skip()
    c = make([], 40, 64, 8, 2)
    assert run(torch, c, True).shape == (0, 40)
    c = make([0, 0], 40, 64, 8, 2, pad=3)
    assert np.array_equal(run(torch, c, True).cpu().numpy(), c["y"])
    c["ids"], c["cu"] = np.array([], int), np.array([0])
    assert np.array_equal(run(torch, c, True).cpu().numpy(), c["y"])


@pytest.mark.parametrize("lens", [[1] * 40, [900, 400, 2]])
def test_same_bits_on_other_streams_and_from_a_graph(lens):
    torch = torch_or_skip()
    c = make(lens, 300, 512, 32, 5, seed=8)
    c["ids"] = np.arange(len(lens)) % 5
    want = run(torch, c, True)
    t = [dev_bf16(torch, c[k]) for k in ("xb", "ab", "bb")] + [dev_i32(torch, c["ids"]), dev_f32(torch, c["gain"]), dev_i32(torch, c["cu"])]
    y0 = dev_f32(torch, c["y"])
    streams = [torch.cuda.Stream() for _ in range(2)]
    ys = [y0.clone() for _ in range(6)]
    torch.cuda.synchronize()
    for i, y in enumerate(ys):
        with torch.cuda.stream(streams[i % 2]):
            q().adapters(y, *t)
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in ys)
    y = y0.clone()
    q().adapters(y, *t)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        q().adapters(y, *t)
    for _ in range(3):
        y.copy_(y0)
        g.replay()
        assert torch.equal(y, want)
        run(torch, c, True)
