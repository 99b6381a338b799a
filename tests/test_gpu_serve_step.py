"""GPU: the serving operators together, as a program uses them: a step of new prompts, then decode steps over the
cache that it filled; captured into a graph and replayed; on several streams at once."""
import numpy as np
import pytest

import oracle
import synth
from gpu_util import torch_or_skip
from serve_util import dev_i32, host_bf16, starts

pytestmark = pytest.mark.gpu

H, Hkv, D, PAGE, HIDDEN = 8, 2, 128, 16, 512


def q():
    import paper_2607_19438_amd as m
    return m


class Layer:
    """QKV projection weights (Q8), a cache and its free list."""

    def __init__(self, torch, seed, R, pages, width):
        m = q()
        w = synth.make_qweight(synth.rng_for(seed), (H + 2 * Hkv) * D, HIDDEN, synth.FMT_Q8, keep_q=False)
        self.wq, self.sc = torch.from_numpy(w.wq).cuda(), torch.from_numpy(w.scales).cuda()
        self.cache = torch.full(m.kv4_cache_shape(pages, Hkv, D, PAGE), 255, dtype=torch.uint8, device="cuda")   # NaN until stored
        self.free = dev_i32(torch, np.random.default_rng(seed).permutation(pages))
        self.table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
        self.freq, self.gain = m.rope_frequencies(D, 10000.0, "linear", factor=2.0)

    def qkv(self, x):
        return q().dense(x, self.wq, self.sc, synth.FMT_Q8).view(-1, H + 2 * Hkv, D)

    def step(self, x, kv_len, q_len, free, packed, single=False):
        """One step's attention output; packed: the requests are new, attend over the rows themselves."""
        m = q()
        plan = m.kv_plan(kv_len, q_len, self.table, free, PAGE, x.shape[0])
        rows = m.rope(self.qkv(x), plan.positions, self.freq, H + Hkv, gain=self.gain)
        k, v = rows[:, H:H + Hkv], rows[:, H + Hkv:]
        m.kv4_store(k, v, plan.slots, self.cache)
        if packed:
            return plan, rows, m.attention_packed(rows[:, :H], k, v, plan.cu_q)
        return plan, rows, m.attention_kv4(rows[:, :H], self.cache, self.table, plan.kv_len, None if single else plan.cu_q)


def activations(torch, T, seed):
    return torch.randn((T, HIDDEN), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


def test_prompts_then_tokens_against_the_oracle():
    torch = torch_or_skip()
    lens = [37, 1, 16, 130]
    R, pad = len(lens), 3
    s = Layer(torch, 1, R, 40, 12)
    zero = torch.zeros(R, dtype=torch.int32, device="cuda")
    x = activations(torch, sum(lens) + pad, 2)
    qkv = s.qkv(x).cpu().numpy().astype(np.float64)
    plan, rows, o = s.step(x, zero, dev_i32(torch, lens), s.free, packed=True)
    cu = starts(lens)
    # rotary rows from the projection's own fp32 rows
    want = oracle.kv_plan([0] * R, lens, np.full((R, 12), -1), s.free.cpu().numpy(), PAGE, len(qkv))
    assert np.array_equal(plan.positions.cpu().numpy(), want[1]) and np.array_equal(s.table.cpu().numpy(), want[3])
    f, gain = oracle.rope_frequencies(D, 10000.0, "linear", 2.0)
    ref = oracle.rope(qkv, want[1], f, H + Hkv, gain=gain)
    got = host_bf16(torch, rows)
    assert np.all(np.abs(got - ref) <= oracle.rope_tolerance(qkv, ref, f, H + Hkv, gain=gain))
    # packed attention over the same bf16 rows
    qn, kn, vn = got[:, :H], got[:, H:H + Hkv], got[:, H + Hkv:]
    ref, absv = oracle.packed_attention(qn, kn, vn, cu, D ** -0.5)
    assert oracle.attn_ratio(host_bf16(torch, o)[:cu[-1]], ref[:cu[-1]], absv[:cu[-1]]) <= 1.0
    # the cache holds the quantised rows where the plan put them, and nothing elsewhere
    ck, cv = oracle.decode_cache(s.cache.cpu().numpy(), D)
    slots = want[2][:cu[-1]]
    for held, rows_of in ((ck, kn), (cv, vn)):
        codes, E = oracle.quantise(rows_of[:cu[-1]].reshape(-1, Hkv, D // 32, 32))
        assert np.array_equal(held[slots], oracle.serve_oracle.dequantise(codes, E).reshape(-1, Hkv, D))
        other = np.ones(len(held), bool)
        other[slots] = False
        assert np.isnan(held[other]).all()
    # three decode steps and one of drafted tokens
    kv, taken = list(lens), int(want[5][0])
    for step, new in enumerate(([1] * R, [1] * R, [4, 1, 3, 2], [1] * R)):
        single = new == [1] * R
        x = activations(torch, sum(new), 10 + step)
        plan, rows, o = s.step(x, dev_i32(torch, kv), dev_i32(torch, new), s.free[taken:].contiguous(), False, single)
        want = oracle.kv_plan(kv, new, s.table.cpu().numpy(), s.free.cpu().numpy()[taken:], PAGE, sum(new))
        kv = [a + b for a, b in zip(kv, new)]
        taken += int(want[5][0])
        assert plan.kv_len.tolist() == kv and int(plan.used) == int(want[5][0])
        ck, cv = oracle.decode_cache(s.cache.cpu().numpy(), D)
        ref, absv = oracle.cached_attention(host_bf16(torch, rows)[:, :H], ck, cv, s.table.cpu().numpy(), kv, starts(new), PAGE, D ** -0.5)
        r = oracle.attn_ratio(host_bf16(torch, o), ref, absv)
        print(f"[parity] decode step {step}: max |err| / bar = {r:.3f}", flush=True)
        assert r <= 1.0


def test_decode_step_captured_and_replayed():
    """A whole decode step in a graph; every replay, with eager work and synchronisations between, gives the eager
    step's bits for the inputs that are in its buffers then. Two graphs of different sizes in turn."""
    torch = torch_or_skip()
    graphs = []
    for R, seed in ((5, 3), (40, 4)):
        s = Layer(torch, seed, R, 40 * R, 40)
        rng = np.random.default_rng(seed)
        kv0 = rng.integers(1, 500, R)
        x0 = activations(torch, int(kv0.sum()), seed)
        plan, _, _ = s.step(x0, torch.zeros(R, dtype=torch.int32, device="cuda"), dev_i32(torch, kv0), s.free, packed=True)
        free = s.free[int(plan.used):].contiguous()
        kv, new, x = plan.kv_len.clone(), torch.ones(R, dtype=torch.int32, device="cuda"), activations(torch, R, seed + 50)
        s.step(x, kv, new, free, False, True)                    # (grows the library's workspaces)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _, rows, o = s.step(x, kv, new, free, False, True)
        graphs.append((s, g, kv, new, free, x, rows, o, R))
    for i in range(5):
        for s, g, kv, new, free, x, rows, o, R in graphs:
            x.copy_(activations(torch, R, 100 + i))
            g.replay()
            torch.cuda.synchronize()
            cache, table, got = s.cache.clone(), s.table.clone(), o.clone()
            _, _, want = s.step(x, kv, new, free, False, True)
            torch.cuda.synchronize()
            assert torch.equal(got, want) and torch.equal(cache, s.cache) and torch.equal(table, s.table)
            kv += 1                                               # the next replay's token goes one further
            torch.randn(1000, device="cuda").sum().item()


def test_calls_on_two_streams():
    """Attention over the cache on two streams at once, each on its own data, split over all workgroups: each call
    has its own workspace, so both give the bits of a call by itself."""
    torch = torch_or_skip()
    m = q()
    sides = []
    for seed in (5, 6):
        rng = np.random.default_rng(seed)
        kv = [9000 + seed, 40, 3000]
        need = [-(-n // 64) for n in kv]
        pages = sum(need)
        cache = torch.zeros(m.kv4_cache_shape(pages, 4, 128, 64), dtype=torch.uint8, device="cuda")
        k = torch.from_numpy(rng.standard_normal((pages * 64, 4, 128)).astype(np.float32)).cuda().to(torch.bfloat16)
        m.kv4_store(k, k.flip(0).contiguous(), torch.arange(pages * 64, dtype=torch.int32, device="cuda"), cache)
        table = np.full((3, max(need)), -1)
        ids, at = rng.permutation(pages), 0
        for r, n in enumerate(need):
            table[r, :n] = ids[at:at + n]
            at += n
        qd = torch.from_numpy(rng.standard_normal((3, 16, 128)).astype(np.float32)).cuda().to(torch.bfloat16)
        sides.append((qd, cache, dev_i32(torch, table), dev_i32(torch, kv)))
    want = [m.attention_kv4(*a) for a in sides]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(10):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i].append(m.attention_kv4(*sides[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(o, want[i]) for o in got[i])


def test_outputs_on_a_side_stream_follow_its_work():
    """Inputs produced on the same side stream just before the calls: nothing runs on another stream."""
    torch = torch_or_skip()
    m = q()
    s = Layer(torch, 7, 4, 200, 60)
    lens = dev_i32(torch, [100, 200, 30, 400])
    zero = torch.zeros(4, dtype=torch.int32, device="cuda")
    x = activations(torch, 730, 8)
    _, _, want = s.step(x, zero, lens, s.free, packed=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = torch.zeros_like(x)
        for _ in range(20):
            torch.mm(torch.ones((2048, 2048), device="cuda"), torch.ones((2048, 2048), device="cuda"))
        y.copy_(x)
        _, _, got = s.step(y, zero, lens, s.free, packed=True)
    side.synchronize()
    assert torch.equal(got, want)
