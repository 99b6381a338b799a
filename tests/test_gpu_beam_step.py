"""GPU: steps of beam search with an adapter to each request, as a server makes them: plan, projection with adapters, rotary
positions, 4-bit cache, attention over the shared prompts, logits, selection, table reordering and page copies. Every
operator of every step is held to its oracle on what it was given, the beams' histories to a record kept beside them,
and replays of a captured step to the eager ones."""
import numpy as np
import pytest

import oracle
import synth
from gpu_util import torch_or_skip
from serve_util import bf16, dev_bf16, dev_i32, host_bf16

pytestmark = pytest.mark.gpu

R, B, H, HKV, D, PAGE, V, K, RANK, END = 2, 3, 8, 2, 64, 16, 200, 512, 8, 7
ROWS = R * B


def q():
    import paper_2607_19438_amd as m
    return m


class Server:
    """What is on the GPU between steps; a step changes it in place, so that it can be captured."""

    def __init__(self, torch, lens, steps):
        m = q()
        self.torch, self.lens = torch, lens
        rng = np.random.default_rng(5)
        qkv = synth.dense_case("beam_qkv", synth.FMT_Q8, 1, (H + 2 * HKV) * D, K, seed=21, stream=(1,))
        head = synth.dense_case("beam_head", synth.FMT_Q8, 1, V, H * D, seed=22, stream=(2,))
        self.fmt = qkv.fmt
        self.qkv, self.head = ([torch.from_numpy(np.ascontiguousarray(t)).cuda() for t in (c.w.wq, c.w.scales)] for c in (qkv, head))
        self.embed = dev_bf16(torch, bf16(rng.standard_normal((V, K)) * 0.3)[1])
        self.a = dev_bf16(torch, bf16(rng.standard_normal((R, RANK, K)) * 0.05)[1])
        self.b = dev_bf16(torch, bf16(rng.standard_normal((R, (H + 2 * HKV) * D, RANK)) * 0.2)[1])
        self.gain = torch.tensor([0.5, 2.0], device="cuda")
        self.ids = dev_i32(torch, np.repeat([1, 0], B))
        self.freq, _ = m.rope_frequencies(D, 10000.0)
        self.W = -(-(max(lens) + steps + 1) // PAGE)
        prompt = [-(-n // PAGE) for n in lens]
        pages = sum(prompt) + ROWS * (steps + 2)
        order = list(rng.permutation(pages))
        table = np.full((ROWS, self.W), -1)
        for r in range(R):
            table[r * B:(r + 1) * B, :prompt[r]] = [order.pop() for _ in range(prompt[r])]
        self.cache = torch.zeros(m.kv4_cache_shape(pages, HKV, D, PAGE), dtype=torch.uint8, device="cuda")
        slots = [table[r * B, p // PAGE] * PAGE + p % PAGE for r in range(R) for p in range(lens[r])]
        kv = [dev_bf16(torch, bf16(rng.standard_normal((sum(lens), HKV, D)))[1]) for _ in range(2)]
        m.kv4_store(*kv, dev_i32(torch, slots), self.cache)
        self.table = dev_i32(torch, table)
        self.kv_len = dev_i32(torch, np.repeat(lens, B))
        self.free = dev_i32(torch, order)
        self.groups, self.prefix = dev_i32(torch, np.arange(R + 1) * B), dev_i32(torch, lens)
        self.keep = dev_i32(torch, [n // PAGE for n in lens])
        self.one = dev_i32(torch, np.ones(ROWS))
        self.tokens = dev_i32(torch, np.repeat([11, 150], B).reshape(R, B))
        # before the first selection a request has one beam
        self.scores = torch.full((R, B), -float("inf"), device="cuda")
        self.scores[:, 0] = 0.0
        self.turn = torch.arange(len(order), dtype=torch.int64, device="cuda")

    def step(self, see=lambda **kw: None):
        m, torch = q(), self.torch
        finished = self.tokens == END
        x = self.embed.index_select(0, self.tokens.view(-1))
        before = dict(kv_len=self.kv_len.clone(), table=self.table.clone())
        plan = m.kv_plan(self.kv_len, self.one, self.table, self.free, PAGE, ROWS)
        y = m.dense(x, *self.qkv, self.fmt)
        base = y.clone()
        assert m.adapters(y, x, self.a, self.b, self.ids, self.gain) is y
        rows = m.rope(y.view(ROWS, H + 2 * HKV, D), plan.positions, self.freq, H + HKV)
        m.kv4_store(rows[:, H:H + HKV], rows[:, H + HKV:], plan.slots, self.cache)
        o = m.attention_kv4_shared(rows[:, :H], self.cache, self.table, plan.kv_len, self.groups, self.prefix)
        logits = m.dense(o.view(ROWS, H * D), *self.head, self.fmt)
        best, parents, tokens = m.beam_select(logits, self.scores, finished=finished, end=END)
        free = self.free[(self.turn + plan.used) % len(self.turn)].contiguous()
        new = m.kv_reorder(self.table, plan.kv_len, parents, free, PAGE, keep=self.keep)
        see(x=x, base=base, y=y, rows=rows, o=o, logits=logits, finished=finished, scores=self.scores, best=best, parents=parents,
            tokens=tokens, free=free, new=new, plan=plan, **before)
        m.kv4_copy(self.cache, new.src, new.dst)
        self.free.copy_(free[(self.turn + new.used) % len(self.turn)])
        self.table.copy_(new.block_table)
        self.kv_len.copy_(new.kv_len)
        self.scores.copy_(best)
        self.tokens.copy_(tokens)

    def state(self):
        return [t.clone() for t in (self.table, self.kv_len, self.scores, self.tokens, self.free, self.cache)]


@pytest.mark.parametrize("lens,steps", [((70, 203), 6), ((64, 16), 18), ((1, 15), 3)])
def test_steps_of_beam_search(lens, steps):
    torch = torch_or_skip()
    m = q()
    s = Server(torch, list(lens), steps)
    table = s.table.cpu().numpy()

    def keys(row_table, n):
        """The keys and values of a row's n tokens as the cache has them."""
        slots = [int(row_table[p // PAGE]) * PAGE + p % PAGE for p in range(n)]
        assert min(slots) >= 0
        return torch.cat(m.kv4_load(s.cache, dev_i32(torch, slots), D), 1).cpu()

    histories = [keys(table[r], lens[r // B]) for r in range(ROWS)]
    seen = {}

    def see(**kw):
        seen.update(kw)

    a, b = host_bf16(torch, s.a), host_bf16(torch, s.b)
    gain, ids = s.gain.cpu().numpy().astype(np.float64), s.ids.cpu().numpy()
    cu = np.arange(ROWS + 1)
    for at in range(steps):
        s.step(see)
        old_table, old_len = seen["table"].cpu().numpy(), seen["kv_len"].cpu().numpy()
        plan, new = seen["plan"], seen["new"]
        now = plan.kv_len.cpu().numpy()
        assert np.array_equal(now, old_len + 1)
        # adapters
        base, x = seen["base"].double().cpu().numpy(), host_bf16(torch, seen["x"])
        want = oracle.adapters(base, x, a, b, ids, gain)
        assert (np.abs(seen["y"].double().cpu().numpy() - want) <= oracle.adapter_tolerance(base, x, a, b, ids, gain)).all()
        # selection
        logits = seen["logits"].double().cpu().numpy()
        scores, fin = seen["scores"], seen["finished"].cpu().numpy()
        parents, tokens, best = seen["parents"].cpu().numpy(), seen["tokens"].cpu().numpy(), seen["best"].double().cpu().numpy()
        was = seen["was"].cpu().numpy() if "was" in seen else np.where(np.arange(B) == 0, 0.0, -np.inf)[None].repeat(R, 0).astype(np.float32)
        want_best, _, _ = oracle.beam_select(logits, was, B, fin, END)
        for r in range(R):
            value = oracle.beam_values(logits[r * B:(r + 1) * B], was[r], fin[r], END)
            assert len({(p, t) for p, t in zip(parents[r], tokens[r])}) == B
            for k in range(B):
                tol = oracle.beam_tolerance(logits[r * B + parents[r, k]], want_best[r, k])
                assert abs(best[r, k] - want_best[r, k]) <= tol and abs(value[parents[r, k], tokens[r, k]] - best[r, k]) <= tol
        seen["was"] = s.scores.clone()
        # tables: the plan's new entries are in the table that was reordered
        planned = old_table.copy()
        for r in range(ROWS):
            if old_len[r] % PAGE == 0:
                j = old_len[r] // PAGE
                planned[r, j] = plan.slots.cpu().numpy()[r] // PAGE
        t, n, src, dst, used, released = oracle.kv_reorder(planned, now, parents, seen["free"].cpu().numpy(), PAGE, [v // PAGE for v in lens])
        assert np.array_equal(new.block_table.cpu().numpy(), t) and new.kv_len.tolist() == list(n)
        assert new.src.tolist() == list(src) and new.dst.tolist() == list(dst) and int(new.used) == used
        assert int(new.n_released) == len(released) and new.released.tolist()[:len(released)] == released
        # a row's history is its parent's with the token that was just stored; pages that are filled in part have one holder
        rows = seen["rows"]
        fresh = torch.cat(m.kv4_load(s.cache, plan.slots, D), 1).cpu()
        histories = [torch.cat([histories[r // B * B + parents.reshape(-1)[r]], fresh[r // B * B + parents.reshape(-1)[r]][None]]) for r in range(ROWS)]
        holders = []
        for r in range(ROWS):
            assert torch.equal(keys(t[r], int(n[r])), histories[r]), (at, r)
            if n[r] % PAGE:
                holders.append(int(t[r, n[r] // PAGE]))
        assert len(set(holders)) == len(holders)
        # attention, over the cache as it is after the copies: they change no page that a row had
        ck, cv = oracle.decode_cache(s.cache.cpu().numpy(), D)
        o, absv = oracle.shared_attention(host_bf16(torch, rows)[:, :H], ck, cv, planned, now, cu, list(np.arange(R + 1) * B), list(lens), PAGE,
                                          D ** -0.5)
        assert oracle.attn_ratio(host_bf16(torch, seen["o"]), o, absv) <= 1.0


def test_a_captured_step_replays_as_the_eager_one():
    torch = torch_or_skip()
    steps = 8
    eager = Server(torch, [70, 203], steps + 3)
    want = []
    for _ in range(steps):
        eager.step()
        want.append(eager.state())
    s = Server(torch, [70, 203], steps + 3)
    start = s.state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    for again in range(2):
        for t, v in zip((s.table, s.kv_len, s.scores, s.tokens, s.free, s.cache), start):
            t.copy_(v)
        for i in range(steps):
            graph.replay()
            torch.cuda.synchronize()
            for x, y in zip(s.state(), want[i]):
                assert torch.equal(x, y), (again, i)
            torch.ones((512, 512), device="cuda").mm(torch.ones((512, 512), device="cuda"))
