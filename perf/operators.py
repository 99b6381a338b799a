"""The operators of one serving step around the projections, as timed cases with their plain forms.

A step over a ragged batch of requests makes these calls, each the way an inference program does (tensors,
cache and tables in hand, one pass on the current stream):

* ``plan``: block tables, slots and positions of the step's tokens from the requests' lengths (``kv_plan``);
* ``rope``: the QKV projection's rows to bf16 with rotary positions on the query and key heads (``rope``);
* ``store``: keys and values into the paged 4-bit cache, and the cache read back (``kv4_store``, ``kv4_load``);
* ``packed``: causal attention over new prompts packed end to end (``attention_packed``);
* ``kv4``: attention of new tokens over the paged 4-bit cache (``attention_kv4``).

The cache is ``uint8 [pages][Hkv][page * (D + D/16)]``: per page and head the key codes ``[page][D/2]``, the value
codes ``[page][D/2]``, the key scales ``[page][D/32]`` and the value scales ``[page][D/32]``. Codes are e2m1 (bit 3
the sign; 0, 0.5, 1, 1.5, 2, 3, 4, 6), element 2j in the low nibble; a scale byte E stands for 2^(E-127), 255 for NaN.
"""
from __future__ import annotations

import math
import random

import torch

own = False

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------

def listed():
    return [
        # the plan of a decode step of 64 running requests: the smallest call
        {"name": "plan_decode", "kind": "plan", "R": 64, "page": 16, "kv_lo": 1, "kv_hi": 8000, "q_lo": 1, "q_hi": 1, "fresh": 0.0, "pad": 0, "shape": 1},
        # a step that mixes running requests with the chunks of new prompts
        {"name": "plan_mixed", "kind": "plan", "R": 500, "page": 64, "kv_lo": 1, "kv_hi": 16000, "q_lo": 1, "q_hi": 400, "fresh": 0.3, "pad": 100, "shape": 2},
        # the QKV rows of a decode step of 16 requests, 32 query and 4 key/value heads
        {"name": "rope_decode", "kind": "rope", "T": 16, "heads": 40, "turned": 36, "D": 128, "rot": 128, "x": "fp32", "pairs": "half", "scaling": "none", "far": 8000},
        # the same rows of a long prompt
        {"name": "rope_prompt", "kind": "rope", "T": 8192, "heads": 40, "turned": 36, "D": 128, "rot": 128, "x": "fp32", "pairs": "half", "scaling": "llama3", "far": 8192},
        # an odd number of tokens far into a long context, half of each head turned, neighbouring pairs
        {"name": "rope_far", "kind": "rope", "T": 1777, "heads": 48, "turned": 40, "D": 64, "rot": 32, "x": "bf16", "pairs": "neighbours", "scaling": "yarn", "far": 1000000},
        # the new keys and values of a decode step, one slot in every request's page
        {"name": "store_decode", "kind": "store", "T": 64, "Hkv": 8, "D": 128, "page": 16, "run": 1, "spare": 64},
        # a prompt's keys and values, pages in free-list order
        {"name": "store_prompt", "kind": "store", "T": 8191, "Hkv": 8, "D": 64, "page": 64, "run": 8191, "spare": 0},
        # short prompts of one token up to a few hundred, packed
        {"name": "packed_short", "kind": "packed", "R": 37, "len_lo": 1, "len_hi": 300, "H": 32, "Hkv": 8, "D": 64, "pad": 13, "shape": 3},
        # long and short prompts together
        {"name": "packed_long", "kind": "packed", "R": 4, "len_lo": 100, "len_hi": 6000, "H": 32, "Hkv": 4, "D": 128, "pad": 0, "shape": 15},
        # a single request's next token
        {"name": "kv4_one", "kind": "kv4", "R": 1, "kv_lo": 4097, "kv_hi": 4097, "q_lo": 1, "q_hi": 1, "H": 32, "Hkv": 4, "D": 128, "page": 16, "shape": 5},
        # a decode step of 64 requests of very different lengths
        {"name": "kv4_batch", "kind": "kv4", "R": 64, "kv_lo": 20, "kv_hi": 16000, "q_lo": 1, "q_hi": 1, "H": 32, "Hkv": 8, "D": 128, "page": 64, "shape": 6},
        # drafted tokens verified, or the last rows of a chunked prompt
        {"name": "kv4_drafts", "kind": "kv4", "R": 9, "kv_lo": 500, "kv_hi": 5000, "q_lo": 3, "q_hi": 9, "H": 32, "Hkv": 8, "D": 64, "page": 32, "shape": 7},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "rope", "store", "packed", "kv4", "kv4"])
    shape = rng.randint(100, 10 ** 6)
    if kind == "plan":
        R = _log_uniform(rng, 1, 500)
        return {"kind": kind, "R": R, "page": rng.choice([16, 32, 64, 128]), "kv_lo": 1, "kv_hi": _log_uniform(rng, 50, 16000),
                "q_lo": 1, "q_hi": rng.choice([1, 1, 5, _log_uniform(rng, 2, 400)]), "fresh": rng.choice([0.0, 0.2]),
                "pad": rng.choice([0, 0, 7, 64]), "shape": shape}
    if kind == "rope":
        D = rng.choice([64, 128])
        rot = rng.choice([D, D, D // 2, D // 4])
        H, Hkv = rng.choice([(8, 8), (16, 4), (24, 8), (32, 4), (32, 8)])
        return {"kind": kind, "T": _log_uniform(rng, 1, 8000), "heads": H + 2 * Hkv, "turned": H + Hkv, "D": D, "rot": rot,
                "x": rng.choice(["fp32", "fp32", "bf16"]), "pairs": rng.choice(["half", "neighbours"]),
                "scaling": rng.choice(["none", "linear", "llama3", "yarn"]), "far": _log_uniform(rng, 1000, 1000000)}
    if kind == "store":
        T = _log_uniform(rng, 1, 8000)
        D = rng.choice([64, 128])
        Hkv = rng.choice([1, 2, 4, 8] if D == 64 else [1, 2, 4])
        return {"kind": kind, "T": T, "Hkv": Hkv, "D": D, "page": rng.choice([16, 32, 64, 128]),
                "run": rng.choice([1, _log_uniform(rng, 1, T), T]) if T <= 200 else rng.choice([T // 3, T]),
                "spare": rng.choice([0, 3])}
    H, Hkv = rng.choice([(8, 8), (16, 4), (24, 8), (32, 4), (32, 8)])
    D = rng.choice([64, 128])
    if kind == "packed":
        top = _log_uniform(rng, 20, 3000)
        return {"kind": kind, "R": max(1, min(rng.randint(1, 40), 5000 // top)), "len_lo": 1, "len_hi": top, "H": H, "Hkv": Hkv, "D": D,
                "pad": rng.choice([0, 5, 130]), "shape": shape}
    top = _log_uniform(rng, 30, 16000)
    lo, hi = rng.choice([(1, 1), (1, 1), (1, 6), (8, 32)])
    R = _log_uniform(rng, 1, 64)
    return {"kind": kind, "R": min(R, 8) if hi > 6 else R, "kv_lo": max(hi, top // 30), "kv_hi": max(hi, top), "q_lo": lo, "q_hi": hi,
            "H": H, "Hkv": Hkv, "D": D, "page": rng.choice([16, 32, 64, 128]), "shape": shape}


def _spread(rng, n, lo, hi):
    """n lengths between lo and hi, spread over their logarithm where that spans more than a factor of ten."""
    if hi <= 10 * lo:
        return [rng.randint(lo, hi) for _ in range(n)]
    return [_log_uniform(rng, lo, hi) for _ in range(n)]


def _lengths(case):
    """(new, kv) lengths of the requests: new tokens, and tokens in the cache (plan: before them, kv4: with them)."""
    rng = random.Random(case["shape"])
    R = case["R"]
    if case["kind"] == "packed":
        new = _spread(rng, R, case["len_lo"], case["len_hi"])
        return new, new
    new = _spread(rng, R, case["q_lo"], case["q_hi"])
    kv = _spread(rng, R, case["kv_lo"], case["kv_hi"])
    if case["kind"] == "plan":
        kv = [0 if rng.random() < case["fresh"] else n for n in kv]
    return new, kv


def _ceil(a, b):
    return -(-a // b)


# ---------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------

def _quantised(x):
    """(codes' values, scale exponents E) of blocks of 32 along the last axis: x ~ value * 2^(E-127)."""
    b = x.float().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1)
    E = (((top.view(torch.int32) + 0x200000) >> 23) - 2).clamp(1, 253)
    a = b * ((254 - E) << 23).view(torch.float32).unsqueeze(-1)
    mag = a.abs()
    step = torch.where(mag < 2, 0.5, torch.where(mag < 4, 1.0, 2.0))
    return torch.copysign((torch.round(mag / step) * step).clamp(max=6.0), a), E


def _cache_of(k, v, pages, page):
    """The cache that holds k, v [pages*page][Hkv][D]."""
    Hkv, D = k.shape[1:]
    parts = []
    scales = []
    for x in (k, v):
        val, E = _quantised(x.view(pages, page, Hkv, D).transpose(1, 2))
        mag = val.abs()
        code = torch.where(mag < 2, mag * 2, torch.where(mag < 4, mag + 2, mag / 2 + 4)).to(torch.uint8)
        code = (code | (torch.signbit(val).to(torch.uint8) << 3)).flatten(-2)
        parts.append((code[..., 0::2] | (code[..., 1::2] << 4)).flatten(-2))
        scales.append(E.to(torch.uint8).flatten(-2))
    return torch.cat(parts + scales, -1).contiguous()


def _frequencies(rot, scaling):
    """(float64 frequencies of the rot/2 pairs, factor on the sine and cosine); the context grows eight times."""
    base, factor, before = 500000.0, 8.0, 8192.0
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [x / factor for x in f], 1.0
    if scaling == "llama3":
        low, high, out = 1.0, 4.0, []
        for x in f:
            turns = before * x / (2 * math.pi)
            s = min(1.0, max(0.0, (turns - low) / (high - low)))
            out.append((1 - s) * x / factor + s * x)
        return out, 1.0
    if scaling == "yarn":
        dim = lambda turns: rot * math.log(before / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        low, high = max(math.floor(dim(32.0)), 0), min(math.ceil(dim(1.0)), rot - 1)
        out = []
        for i, x in enumerate(f):
            s = min(1.0, max(0.0, (i - low) / (high - low if high > low else 0.001)))
            out.append(x / factor * s + x * (1 - s))
        return out, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, dtype=torch.float32, device="cuda", generator=gen).to(dtype)

    def shuffled(n):
        return torch.randperm(n, device="cuda", generator=gen).to(torch.int32)

    if kind == "plan":
        new, kv = _lengths(case)
        page = case["page"]
        have = [_ceil(n, page) for n in kv]
        need = [_ceil(n + m, page) for n, m in zip(kv, new)]
        width = max(need) + 2
        used = _i32(have)
        extra = sum(need) - sum(have) + 32
        ids = shuffled(sum(have) + extra)
        slot = torch.arange(width, device="cuda", dtype=torch.int32)[None, :]
        at = (torch.cumsum(used, 0).to(torch.int32) - used)[:, None] + slot
        table = torch.where(slot < used[:, None], ids[at.clamp(max=len(ids) - 1).long()], -1).to(torch.int32)
        return {"case": case, "kv_len": _i32(kv), "q_len": _i32(new), "table": table, "free": ids[sum(have):].contiguous(),
                "T": sum(new) + case["pad"]}
    if kind == "rope":
        T, heads, D = case["T"], case["heads"], case["D"]
        f, gain = _frequencies(case["rot"], case["scaling"])
        x = normal(T, heads, D, dtype=torch.float32 if case["x"] == "fp32" else torch.bfloat16)
        first = torch.randint(0, max(1, case["far"] - T), (1,), device="cuda", generator=gen)
        pos = (first + torch.arange(T, device="cuda")).to(torch.int32)
        return {"case": case, "x": x, "positions": pos, "inv_freq": torch.tensor(f, dtype=torch.float64, device="cuda"), "gain": gain}
    if kind == "store":
        T, Hkv, D, page = case["T"], case["Hkv"], case["D"], case["page"]
        # every run of tokens starts in a page of its own
        runs = _ceil(T, case["run"])
        per = _ceil(case["run"], page)
        pages = runs * per + case["spare"]
        ids = shuffled(pages)
        t = torch.arange(T, device="cuda")
        at = t % case["run"]
        first = torch.randint(0, page, (runs,), device="cuda", generator=gen) if case["run"] == 1 else torch.zeros(runs, dtype=torch.long, device="cuda")
        slots = (ids[t // case["run"] * per + at // page] * page + at % page + first[t // case["run"]]).to(torch.int32)
        # keys and values as the views of one row of projections that they are in use
        qkv = normal(T, 4 * Hkv, D)
        cache = _cache_of(normal(pages * page, Hkv, D), normal(pages * page, Hkv, D), pages, page)
        return {"case": case, "k": qkv[:, 2 * Hkv:3 * Hkv], "v": qkv[:, 3 * Hkv:], "slots": slots, "cache": cache,
                "all": torch.arange(pages * page, dtype=torch.int32, device="cuda")}
    H, Hkv, D = case["H"], case["Hkv"], case["D"]
    new, kv = _lengths(case)
    scale = 1.0 / math.sqrt(D)
    if kind == "packed":
        T = sum(new) + case["pad"]
        qkv = normal(T, H + 2 * Hkv, D)
        return {"case": case, "q": qkv[:, :H], "k": qkv[:, H:H + Hkv], "v": qkv[:, H + Hkv:], "cu": _i32(_starts(new)),
                "scale": scale, "out": torch.zeros((T, H, D), dtype=torch.bfloat16, device="cuda")}
    page = case["page"]
    need = [_ceil(n, page) for n in kv]
    pages = sum(need) + 1
    ids = shuffled(pages)
    width = max(need)
    slot = torch.arange(width, device="cuda", dtype=torch.int32)[None, :]
    used = _i32(need)
    at = (torch.cumsum(used, 0).to(torch.int32) - used)[:, None] + slot
    table = torch.where(slot < used[:, None], ids[at.clamp(max=pages - 1).long()], -1).to(torch.int32)
    cache = _cache_of(normal(pages * page, Hkv, D), normal(pages * page, Hkv, D), pages, page)
    return {"case": case, "q": normal(sum(new), H, D), "cache": cache, "table": table, "kv_len": _i32(kv), "cu": _i32(_starts(new)),
            "most": max(new), "scale": scale}


# ---------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if own:
        import paper_2607_19438_amd as qg
        if kind == "plan":
            p = qg.kv_plan(s["kv_len"], s["q_len"], s["table"], s["free"], s["case"]["page"], s["T"])
            return {"cu_q": p.cu_q, "positions": p.positions, "slots": p.slots, "table": s["table"], "kv_len": p.kv_len, "used": p.used}
        if kind == "rope":
            return qg.rope(s["x"], s["positions"], s["inv_freq"], s["case"]["turned"], interleaved=s["case"]["pairs"] == "neighbours",
                           gain=s["gain"])
        if kind == "store":
            qg.kv4_store(s["k"], s["v"], s["slots"], s["cache"])
            return qg.kv4_load(s["cache"], s["all"], s["case"]["D"])
        if kind == "packed":
            return qg.attention_packed(s["q"], s["k"], s["v"], s["cu"], s["scale"], out=s["out"])
        return qg.attention_kv4(s["q"], s["cache"], s["table"], s["kv_len"], None if s["case"]["q_hi"] == 1 else s["cu"], s["scale"])
    return {"plan": _plan, "rope": _rope, "store": _store, "packed": _packed, "kv4": _kv4}[kind](s)


def _plan(s):
    page, T = s["case"]["page"], s["T"]
    kv, q, table, free = s["kv_len"], s["q_len"], s["table"], s["free"]
    ends = torch.cumsum(q, 0)
    have, need = (kv + (page - 1)) // page, (kv + q + (page - 1)) // page
    before = torch.cumsum(need - have, 0) - (need - have)
    t = torch.arange(T, device=q.device)
    r = torch.searchsorted(ends, t, right=True).clamp(max=len(q) - 1)
    real = t < ends[-1]
    pos = kv[r] + t - (ends - q)[r]
    j = (pos // page).clamp(max=table.shape[1] - 1)
    fresh = (before[r] + j - have[r]).clamp(0, len(free) - 1)
    at = torch.where(j < have[r], table[r, j], free[fresh])
    c = torch.arange(table.shape[1], device=q.device)[None, :]
    f = (before[:, None] + c - have[:, None]).clamp(0, len(free) - 1)
    out = torch.where((c >= have[:, None]) & (c < need[:, None]), free[f], table)
    cu = torch.cat([torch.zeros_like(ends[:1]), ends])
    return {"cu_q": cu.to(torch.int32), "positions": torch.where(real, pos, 0).to(torch.int32),
            "slots": torch.where(real, at * page + pos % page, -1).to(torch.int32), "table": out.to(torch.int32),
            "kv_len": kv + q, "used": (need - have).sum().reshape(1).to(torch.int32)}


def _rope(s):
    c = s["case"]
    x, rot, n = s["x"].float(), c["rot"], c["turned"]
    angle = s["positions"].double()[:, None, None] * s["inv_freq"]
    cos, sin = (torch.cos(angle) * s["gain"]).float(), (torch.sin(angle) * s["gain"]).float()
    part = x[:, :n, :rot]
    if c["pairs"] == "half":
        a, b = part[..., :rot // 2], part[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    out = x.to(torch.bfloat16)
    out[:, :n, :rot] = turned.to(torch.bfloat16)
    return out


def _values(cache, D):
    """The keys and values [pages][Hkv][page][D] that a cache holds, fp32."""
    page = cache.shape[-1] * 16 // (17 * D)
    n = page * D // 2
    level = torch.arange(256, device=cache.device)
    nibble = torch.stack([level & 15, level >> 4], -1)
    mag = nibble & 7
    value = torch.where(mag < 4, mag * 0.5, torch.where(mag < 6, mag - 2.0, mag * 2.0 - 8.0))
    pair = torch.where(nibble > 7, -value, value).float()
    power = torch.where(level == 255, math.nan, torch.ldexp(torch.ones((), device=cache.device, dtype=torch.float64), level - 127)).float()
    codes = pair[cache[..., :2 * n].int()].view(*cache.shape[:2], 2, page, D // 32, 32)
    scale = power[cache[..., 2 * n:].int()].view(*cache.shape[:2], 2, page, D // 32, 1)
    kv = (codes * scale).flatten(-2)
    return kv[:, :, 0], kv[:, :, 1]


def _store(s):
    D = s["case"]["D"]
    out = []
    for held, x in zip(_values(s["cache"], D), (s["k"], s["v"])):
        val, E = _quantised(x)
        new = (val * (E << 23).view(torch.float32).unsqueeze(-1)).flatten(-2)
        held = held.transpose(1, 2).flatten(0, 1).contiguous()
        held[s["slots"].long()] = new
        out.append(held.to(torch.bfloat16))
    return tuple(out)


def _packed(s):
    T, H, D = s["q"].shape
    Hkv = s["k"].shape[1]
    q = s["q"].float().view(T, Hkv, H // Hkv, D).permute(1, 2, 0, 3)
    k, v = (x.float().transpose(0, 1).contiguous() for x in (s["k"], s["v"]))
    t = torch.arange(T, device=q.device)
    seq = torch.searchsorted(s["cu"][1:].contiguous(), t, right=True)
    sees = (seq[:, None] == seq[None, :]) & (t[None, :] <= t[:, None])
    score = torch.matmul(q.reshape(Hkv, -1, D), k.transpose(1, 2).contiguous()).view(Hkv, H // Hkv, T, T)
    score = score.mul_(s["scale"]).masked_fill_(~sees, -math.inf)
    score = score.sub_(score.amax(-1, keepdim=True)).exp_()
    total = score.sum(-1, keepdim=True)
    o = torch.matmul(score.view(Hkv, -1, T), v).view(Hkv, H // Hkv, T, D) / total
    o = o.permute(2, 0, 1, 3).reshape(T, H, D)
    return torch.where((seq < len(s["cu"]) - 1)[:, None, None], o, 0.0).to(torch.bfloat16)


def _kv4(s):
    T, H, D = s["q"].shape
    R, most = len(s["kv_len"]), s["most"]
    k, v = _values(s["cache"], D)
    Hkv, page = k.shape[1], k.shape[2]
    at = s["table"].clamp(min=0).flatten()
    k, v = (x[at].view(R, -1, Hkv, page, D).transpose(1, 2).reshape(R, Hkv, -1, D) for x in (k, v))
    cu = s["cu"].long()
    n = cu[1:] - cu[:-1]
    i = torch.arange(most, device=cu.device)
    rows = (cu[:-1, None] + i).clamp(max=T - 1)
    q = s["q"].float()[rows].view(R, most, Hkv, H // Hkv, D).transpose(1, 2).reshape(R, Hkv, -1, D)
    key = torch.arange(k.shape[2], device=cu.device)
    v = torch.where((key < s["kv_len"][:, None])[:, None, :, None], v, 0.0)
    sees = key <= (s["kv_len"] - n)[:, None, None] + i[:, None]
    score = torch.matmul(q, k.transpose(2, 3)).view(R, Hkv, most, H // Hkv, -1) * s["scale"]
    score = torch.where(sees[:, None, :, None, :], score, -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(R, Hkv, -1, p.shape[-1]), v).view(R, Hkv, most, H // Hkv, D) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 2, 1, 3, 4).reshape(R, most, H, D)
    t = torch.arange(T, device=cu.device)
    r = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=R - 1)
    return o[r, t - cu[r]].to(torch.bfloat16)


# ---------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its result in 64 bits
# ---------------------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "plan":
        new, kv = _lengths(case)
        page = case["page"]
        touched = sum(_ceil(n + m, page) - n // page for n, m in zip(kv, new))
        fresh = sum(_ceil(n + m, page) - _ceil(n, page) for n, m in zip(kv, new))
        return {"bytes": 4 * (4 * case["R"] + 2 + 2 * (sum(new) + case["pad"]) + touched + fresh), "flops": sum(new)}
    if kind == "rope":
        n = case["T"] * case["heads"] * case["D"]
        return {"bytes": n * (6 if case["x"] == "fp32" else 4) + 4 * case["T"] + 4 * case["rot"],
                "flops": 3 * case["T"] * case["turned"] * case["rot"]}
    if kind == "store":
        # both ways: bf16 keys and values in, codes and scales out; the cache read back, bf16 out
        T, n, D = case["T"], case["Hkv"] * case["D"], case["D"]
        runs = _ceil(T, case["run"])
        held = (runs * _ceil(case["run"], case["page"]) + case["spare"]) * case["page"]
        return {"bytes": T * (4 * n + n * 17 // 16 + 4) + held * (4 * n + n * 17 // 16 + 4), "flops": 4 * T * n + 2 * held * n}
    new, kv = _lengths(case)
    H, Hkv, D = case["H"], case["Hkv"], case["D"]
    rows = sum(new) * H * D * 2
    if kind == "packed":
        return {"bytes": 2 * rows + sum(new) * Hkv * D * 4 + 4 * len(new) + 4, "flops": sum(2 * n * (n + 1) * D * H for n in new)}
    keys = sum(kv) * Hkv * D * 17 // 16
    pages = sum(_ceil(n, case["page"]) for n in kv)
    seen = sum(m * n - m * (m - 1) // 2 for n, m in zip(kv, new))
    return {"bytes": 2 * rows + keys + 4 * pages + 8 * len(new), "flops": 4 * seen * D * H}


def _level64(x):
    """x [..., n*32] float64 as blocks of 32 hold it: the level next to x / 2^E, ties to the even code."""
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)                       # top = m 2^e, m in [0.5, 1)
    e = torch.where(m >= 0.875, e + 1, e) - 3     # 1.75 and up counts as the next power; the largest level is 6 < 2^3
    e = torch.where(top > 0, e, -126).clamp(min=-126)
    unit = torch.ldexp(torch.ones_like(top), e)
    a = (b / unit).abs()
    code = torch.zeros_like(a)
    for c in range(7):
        edge = (LEVELS[c] + LEVELS[c + 1]) / 2
        code = torch.where((a > edge) if c % 2 == 0 else (a >= edge), c + 1.0, code)
    level = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)[code.long()]
    return (torch.copysign(level, b) * unit).flatten(-2)


def _cache64(cache, D, h, which):
    """Keys (0) or values (1) of head h of a cache, float64 [pages*page][D], element by element of its layout."""
    page = cache.shape[-1] * 16 // (17 * D)
    rec = cache[:, h].long()
    codes = rec[:, which * page * D // 2:(which + 1) * page * D // 2].reshape(-1, page, D // 2)
    first = page * D + which * page * D // 32
    E = rec[:, first:first + page * D // 32].reshape(-1, page, D // 32)
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), dtype=torch.float64, device=cache.device)
    val = torch.empty((*codes.shape[:2], D), dtype=torch.float64, device=cache.device)
    val[..., 0::2] = level[codes % 16]
    val[..., 1::2] = level[codes // 16]
    return (val * torch.ldexp(torch.ones_like(E, dtype=torch.float64), E - 127).repeat_interleave(32, -1)).flatten(0, 1)


def exact(case, seed):
    kind = case["kind"]
    if kind == "plan":
        return None      # whole numbers
    s = prepare(case, seed)
    if kind == "rope":
        n, rot = case["turned"], case["rot"]
        x = s["x"].double()
        first = torch.arange(rot // 2, device=x.device) * (2 if case["pairs"] == "neighbours" else 1)
        second = first + (1 if case["pairs"] == "neighbours" else rot // 2)
        turn = torch.polar(torch.full((), s["gain"], dtype=torch.float64, device=x.device), s["positions"].double()[:, None] * s["inv_freq"][None, :])
        z = torch.complex(x[:, :n, first], x[:, :n, second]) * turn[:, None, :]
        x[:, :n, first], x[:, :n, second] = z.real, z.imag
        return x
    if kind == "store":
        D, out = case["D"], []
        for which, x in enumerate((s["k"], s["v"])):
            held = torch.stack([_cache64(s["cache"], D, h, which) for h in range(case["Hkv"])], 1)
            held[s["slots"].long()] = _level64(x.double())
            out.append(held)
        return tuple(out)
    H, Hkv, D = case["H"], case["Hkv"], case["D"]
    new, kv = _lengths(case)
    at = _starts(new)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for g in range(Hkv):
        if kind == "kv4":
            keys, values = _cache64(s["cache"], D, g, 0), _cache64(s["cache"], D, g, 1)
        for r, (n, m) in enumerate(zip(new, kv)):
            rows = slice(at[r], at[r + 1])
            if kind == "packed":
                k, v = s["k"][rows, g].double(), s["v"][rows, g].double()
            else:
                page = case["page"]
                slots = (s["table"][r, :_ceil(m, page)].long()[:, None] * page + torch.arange(page, device="cuda")).flatten()[:m]
                k, v = keys[slots], values[slots]
            q = s["q"][rows, g * (H // Hkv):(g + 1) * (H // Hkv)].double().transpose(0, 1)
            w = torch.matmul(q, k.T.contiguous()) * s["scale"]
            hidden = torch.arange(m, device="cuda")[None, :] > m - n + torch.arange(n, device="cuda")[:, None]
            w = torch.softmax(w.masked_fill(hidden, -math.inf), -1)
            out[rows, g * (H // Hkv):(g + 1) * (H // Hkv)] = torch.matmul(w, v).transpose(0, 1)
    return out
