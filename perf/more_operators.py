"""The operators of a serving step with many continuations of a prompt and many tenants, as timed cases with their plain forms.

Beam search and batches that share a prompt make these calls around the projections and the paged 4-bit cache, each the
way an inference program does (tensors, cache and tables in hand, one pass on the current stream):

* ``shared``: attention of new tokens over the cache for groups of requests that share their first keys
  (``attention_kv4_shared``);
* ``beam``: the best continuations of every request's beams over the vocabulary (``beam_select``);
* ``reorder``: block tables after a selection, and the pages of the cache that it has copied (``kv_reorder``, ``kv4_copy``);
* ``adapters``: low-rank adapters of many requests beside a shared projection (``adapters``).

The cache is ``uint8 [pages][Hkv][page * (D + D/16)]``: per page and head the key codes ``[page][D/2]``, the value
codes ``[page][D/2]``, the key scales ``[page][D/32]`` and the value scales ``[page][D/32]``. Codes are e2m1 (bit 3
the sign; 0, 0.5, 1, 1.5, 2, 3, 4, 6), element 2j in the low nibble; a scale byte E stands for 2^(E-127).
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
        # the next token of four beams over one prompt: the smallest call
        {"name": "shared_beams", "kind": "shared", "G": 1, "each": 4, "pre_lo": 1000, "pre_hi": 1000, "own_lo": 1, "own_hi": 60, "q_lo": 1, "q_hi": 1, "H": 32, "Hkv": 8, "D": 128, "page": 16, "shape": 1},
        # a decode step of 64 requests behind one long system prompt
        {"name": "shared_prompt", "kind": "shared", "G": 1, "each": 64, "pre_lo": 7919, "pre_hi": 7919, "own_lo": 10, "own_hi": 600, "q_lo": 1, "q_hi": 1, "H": 32, "Hkv": 8, "D": 128, "page": 64, "shape": 2},
        # a decode step of 24 requests of eight beams each, prompts of very different lengths
        {"name": "shared_groups", "kind": "shared", "G": 24, "each": 8, "pre_lo": 200, "pre_hi": 5000, "own_lo": 1, "own_hi": 300, "q_lo": 1, "q_hi": 1, "H": 32, "Hkv": 4, "D": 64, "page": 32, "shape": 3},
        # one request of four beams: the smallest selection
        {"name": "beam_one", "kind": "beam", "R": 1, "B": 4, "K": 4, "V": 32000, "x": "fp32", "done": 0.0},
        # an odd vocabulary in bf16, twice as many candidates as beams
        {"name": "beam_odd", "kind": "beam", "R": 17, "B": 5, "K": 10, "V": 50021, "x": "bf16", "done": 0.1},
        # a full batch over a large vocabulary
        {"name": "beam_batch", "kind": "beam", "R": 48, "B": 8, "K": 16, "V": 128000, "x": "fp32", "done": 0.1},
        # four requests of four beams, one layer's cache
        {"name": "reorder_few", "kind": "reorder", "R": 4, "B": 4, "kv_lo": 300, "kv_hi": 3000, "gen": 100, "page": 16, "Hkv": 8, "D": 128, "dead": 0.0, "shape": 7},
        # a full batch with requests that have ended, one layer's cache
        {"name": "reorder_batch", "kind": "reorder", "R": 64, "B": 8, "kv_lo": 100, "kv_hi": 6000, "gen": 200, "page": 32, "Hkv": 8, "D": 128, "dead": 0.1, "shape": 8},
        # a decode step of 16 requests over eight adapters
        {"name": "adapters_decode", "kind": "adapters", "R": 16, "len_lo": 1, "len_hi": 1, "N": 2048, "K": 2048, "r": 16, "n": 8, "none": 0.1, "shape": 4},
        # a decode step of 96 requests, most with an adapter of their own
        {"name": "adapters_many", "kind": "adapters", "R": 96, "len_lo": 1, "len_hi": 1, "N": 8192, "K": 2048, "r": 32, "n": 64, "none": 0.0, "shape": 5},
        # prompts of one token up to some hundred, an odd number of output columns
        {"name": "adapters_ragged", "kind": "adapters", "R": 21, "len_lo": 1, "len_hi": 400, "N": 5003, "K": 2048, "r": 8, "n": 5, "none": 0.2, "shape": 6},
        # long prompts of a few tenants with adapters of high rank
        {"name": "adapters_long", "kind": "adapters", "R": 4, "len_lo": 500, "len_hi": 4000, "N": 8192, "K": 2048, "r": 64, "n": 4, "none": 0.0, "shape": 9},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["shared", "shared", "beam", "reorder", "adapters", "adapters"])
    shape = rng.randint(100, 10 ** 6)
    if kind == "shared":
        H, Hkv = rng.choice([(8, 8), (16, 4), (28, 4), (32, 4), (32, 8)])
        G = _log_uniform(rng, 1, 24)
        each = max(1, min(_log_uniform(rng, 1, 64), 192 // G))
        top = _log_uniform(rng, 40, min(8000, 480000 // (G * each)))
        lo, hi = rng.choice([(1, 1), (1, 1), (1, 5), (1, 40)])
        hi = min(hi, max(1, 1000 // (G * each)))
        return {"kind": kind, "G": G, "each": each, "pre_lo": rng.choice([top, max(1, top // 20)]), "pre_hi": top, "own_lo": hi,
                "own_hi": hi + _log_uniform(rng, 1, 500), "q_lo": min(lo, hi), "q_hi": hi, "H": H, "Hkv": Hkv, "D": rng.choice([64, 128]),
                "page": rng.choice([16, 32, 64, 128]), "shape": shape}
    if kind == "beam":
        R, B = _log_uniform(rng, 1, 48), rng.randint(1, 8)
        V = _log_uniform(rng, 1000, min(128000, 40_000_000 // (R * B)))
        return {"kind": kind, "R": R, "B": B, "K": rng.choice([B, B, 2 * B]), "V": V, "x": rng.choice(["fp32", "bf16"]),
                "done": rng.choice([0.0, 0.3])}
    if kind == "reorder":
        D = rng.choice([64, 128])
        return {"kind": kind, "R": _log_uniform(rng, 1, 64), "B": rng.randint(2, 8), "kv_lo": 1, "kv_hi": _log_uniform(rng, 20, 4000),
                "gen": _log_uniform(rng, 1, 200), "page": rng.choice([16, 32, 64]), "Hkv": rng.choice([1, 4, 8]), "D": D,
                "dead": rng.choice([0.0, 0.2]), "shape": shape}
    R = _log_uniform(rng, 1, 100)
    top = rng.choice([1, 1, _log_uniform(rng, 2, max(2, 8000 // R))])
    return {"kind": kind, "R": R, "len_lo": 1, "len_hi": top, "N": _log_uniform(rng, 64, 8192), "K": 32 * _log_uniform(rng, 4, 128),
            "r": rng.choice([8, 16, 24, 32, 64]), "n": _log_uniform(rng, 1, 32), "none": rng.choice([0.0, 0.3]), "shape": shape}


def _spread(rng, n, lo, hi):
    """n lengths between lo and hi, spread over their logarithm where that spans more than a factor of ten."""
    if hi <= 10 * lo:
        return [rng.randint(lo, hi) for _ in range(n)]
    return [_log_uniform(rng, lo, hi) for _ in range(n)]


def _lengths(case):
    """shared: (prefix lengths of the groups, new tokens and own keys of the requests); reorder: (prompt lengths and
    generated tokens of the requests, their beams' parents); adapters: (rows of the requests, their adapters)."""
    rng = random.Random(case["shape"])
    if case["kind"] == "adapters":
        lens = _spread(rng, case["R"], case["len_lo"], case["len_hi"])
        return lens, [-1 if rng.random() < case["none"] else rng.randrange(case["n"]) for _ in lens]
    if case["kind"] == "reorder":
        prompt, made = _spread(rng, case["R"], case["kv_lo"], case["kv_hi"]), _spread(rng, case["R"], 1, case["gen"])
        # a few beams have most of the children, and an ended request has none
        return prompt, made, [[-1] * case["B"] if rng.random() < case["dead"] else [min(int(rng.expovariate(0.8)), case["B"] - 1) for _ in range(case["B"])]
                              for _ in prompt]
    n = case["G"] * case["each"]
    return (_spread(rng, case["G"], case["pre_lo"], case["pre_hi"]), _spread(rng, n, case["q_lo"], case["q_hi"]),
            _spread(rng, n, case["own_lo"], case["own_hi"]))


def _ceil(a, b):
    return -(-a // b)


def _starts(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out


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


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rng = random.Random(int(seed))
    kind = case["kind"]

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, dtype=torch.float32, device="cuda", generator=gen).to(dtype)

    def uniform(*shape):
        return torch.rand(shape, dtype=torch.float32, device="cuda", generator=gen)

    def shuffled(n):
        return torch.randperm(n, device="cuda", generator=gen).to(torch.int32).tolist()

    if kind == "shared":
        H, Hkv, D, page, each = case["H"], case["Hkv"], case["D"], case["page"], case["each"]
        pre, new, mine = _lengths(case)
        kv = [pre[r // each] + n for r, n in enumerate(mine)]
        # a group's full pages of the prefix are one for all; the page that the prefix ends in and those behind it are each request's own
        pages = sum(p // page for p in pre) + sum(_ceil(n, page) - pre[r // each] // page for r, n in enumerate(kv))
        ids = shuffled(pages)
        width = max(_ceil(n, page) for n in kv)
        rows, copies = [], []
        for g, p in enumerate(pre):
            common = [ids.pop() for _ in range(p // page)]
            first = None
            for r in range(g * each, (g + 1) * each):
                row = common + [ids.pop() for _ in range(_ceil(kv[r], page) - p // page)]
                if p % page:
                    first = row[p // page] if first is None else first
                    copies.append((row[p // page], first))
                rows.append(row + [-1] * (width - len(row)))
        cache = _cache_of(normal(pages * page, Hkv, D), normal(pages * page, Hkv, D), pages, page)
        if copies:      # the prefix's last keys, in every request's own page
            to, of = (torch.tensor(x, device="cuda") for x in zip(*copies))
            cache[to] = cache[of]
        return {"case": case, "q": normal(sum(new), H, D), "cache": cache, "table": _i32(rows), "kv_len": _i32(kv), "cu": _i32(_starts(new)),
                "groups": _i32([each * g for g in range(case["G"] + 1)]), "prefix": _i32(pre), "most": max(new), "scale": 1.0 / math.sqrt(D)}
    if kind == "beam":
        R, B, V = case["R"], case["B"], case["V"]
        logits = normal(R * B, V, dtype=torch.float32).mul_(3.0).to(torch.float32 if case["x"] == "fp32" else torch.bfloat16)
        scores = -10.0 * uniform(R, B)
        if R > 1:
            scores[0, 1:] = -math.inf                 # a request's first step: one live beam
        finished = uniform(R, B) < case["done"]
        return {"case": case, "logits": logits, "scores": scores, "finished": finished if case["done"] else None, "end": min(2, V - 1)}
    if kind == "reorder":
        R, B, page, Hkv, D = case["R"], case["B"], case["page"], case["Hkv"], case["D"]
        prompt, made, parents = _lengths(case)
        # beams 2i and 2i+1 have some of their generated pages in common; a beam's last, partly filled page is its own
        cols = [_ceil(p + n, page) for p, n in zip(prompt, made)]
        spare = R * B
        width = max(cols) + 1
        ids = shuffled(sum(p // page + B * (c - p // page) for p, c in zip(prompt, cols)) + spare)
        pages = len(ids)
        table, kv = [], []
        for p, n, c in zip(prompt, made, cols):
            common = [ids.pop() for _ in range(p // page)]
            rows = []
            for b in range(B):
                row = common + [ids.pop() for _ in range(c - p // page)]
                if b % 2:
                    fork = rng.randint(p // page, (p + n) // page)
                    row[:fork] = rows[-1][:fork]
                rows.append(row)
            table += [row + [-1] * (width - c) for row in rows]
            kv += [p + n] * B
        cache = torch.randint(0, 256, (pages, Hkv, page * (D + D // 16)), dtype=torch.uint8, device="cuda", generator=gen)
        return {"case": case, "table": _i32(table), "kv_len": _i32(kv), "parents": _i32(parents), "free": _i32(ids[:spare]), "cache": cache,
                "keep": _i32([p // page for p in prompt])}
    lens, ids = _lengths(case)
    M, N, K, r, n = sum(lens), case["N"], case["K"], case["r"], case["n"]
    return {"case": case, "x": normal(M, K), "y": normal(M, N, dtype=torch.float32), "a": normal(n, r, K, dtype=torch.float32).mul_(K ** -0.5).to(torch.bfloat16),
            "b": normal(n, N, r, dtype=torch.float32).mul_(0.5).to(torch.bfloat16), "ids": _i32(ids), "gain": 0.5 + uniform(n), "cu": _i32(_starts(lens))}


# ---------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        import paper_2607_19438_amd as qg
        if kind == "shared":
            return qg.attention_kv4_shared(s["q"], s["cache"], s["table"], s["kv_len"], s["groups"], s["prefix"],
                                           None if case["q_hi"] == 1 else s["cu"], s["scale"])
        if kind == "beam":
            scores, parents, tokens = qg.beam_select(s["logits"], s["scores"], case["K"], finished=s["finished"], end=s["end"])
            return {"scores": scores, "parents": parents, "tokens": tokens}
        if kind == "reorder":
            p = qg.kv_reorder(s["table"], s["kv_len"], s["parents"], s["free"], case["page"], keep=s["keep"])
            qg.kv4_copy(s["cache"], p.src, p.dst)
            return {"table": p.block_table, "kv_len": p.kv_len, "src": p.src, "dst": p.dst, "used": p.used, "released": p.released,
                    "count": p.n_released, "cache": s["cache"]}
        return qg.adapters(s["y"], s["x"], s["a"], s["b"], s["ids"], s["gain"], None if case["len_hi"] == 1 else s["cu"])
    return {"shared": _shared, "beam": _beam, "reorder": _reorder, "adapters": _adapters}[kind](s)


def _values(cache, D):
    """The keys and values [pages][Hkv][page][D] that a cache holds, fp32."""
    page = cache.shape[-1] * 16 // (17 * D)
    n = page * D // 2
    level = torch.arange(256, device=cache.device)
    nibble = torch.stack([level & 15, level >> 4], -1)
    mag = nibble & 7
    value = torch.where(mag < 4, mag * 0.5, torch.where(mag < 6, mag - 2.0, mag * 2.0 - 8.0))
    pair = torch.where(nibble > 7, -value, value).float()
    power = torch.ldexp(torch.ones((), device=cache.device, dtype=torch.float64), level - 127).float()
    codes = pair[cache[..., :2 * n].int()].view(*cache.shape[:2], 2, page, D // 32, 32)
    scale = power[cache[..., 2 * n:].int()].view(*cache.shape[:2], 2, page, D // 32, 1)
    kv = (codes * scale).flatten(-2)
    return kv[:, :, 0], kv[:, :, 1]


def _shared(s):
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
    sees = key <= (s["kv_len"] - n)[:, None, None] + i[:, None]
    score = torch.matmul(q, k.transpose(2, 3)).view(R, Hkv, most, H // Hkv, -1) * s["scale"]
    score = score.masked_fill_(~sees[:, None, :, None, :], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    o = torch.matmul(p.view(R, Hkv, -1, p.shape[-1]), v).view(R, Hkv, most, H // Hkv, D) / p.sum(-1, keepdim=True)
    o = o.permute(0, 2, 1, 3, 4).reshape(R, most, H, D)
    t = torch.arange(T, device=cu.device)
    r = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    return o[r, t - cu[r]].to(torch.bfloat16)


def _beam(s):
    # in 64 bits: candidates of different beams can lie close together, and a difference decides which is taken
    c = s["case"]
    R, B, V = c["R"], c["B"], c["V"]
    x = s["logits"].double()
    top = x.amax(-1, keepdim=True)
    value = s["scores"].double().view(-1, 1) + (x - (top + torch.log(torch.exp(x - top).sum(-1, keepdim=True))))
    if s["finished"] is not None:
        only = torch.full_like(value, -math.inf)
        only[:, s["end"]] = s["scores"].double().flatten()
        value = torch.where(s["finished"].view(-1, 1), only, value)
    best, at = torch.sort(value.view(R, B * V), dim=-1, descending=True, stable=True)
    best, at = best[:, :c["K"]], at[:, :c["K"]]
    real = best > -math.inf
    return {"scores": best.float(), "parents": torch.where(real, at // V, -1).to(torch.int32),
            "tokens": torch.where(real, at % V, s["end"]).to(torch.int32)}


def _reorder(s):
    c = s["case"]
    R, B, page = c["R"], c["B"], c["page"]
    old = s["table"].view(R, B, -1)
    kv = s["kv_len"].view(R, B)
    W = old.shape[-1]
    par = s["parents"].long()
    lives = par >= 0
    p = par.clamp(min=0)
    k = torch.arange(B, device=old.device)
    again = ((par[:, :, None] == par[:, None, :]) & (k[None, :] < k[:, None])).any(-1) & lives     # not its parent's first child
    kv_new = torch.where(lives, kv.gather(1, p), 0)
    have = (kv + page - 1) // page
    have_new = (kv_new + page - 1) // page
    fresh = again & (kv_new % page != 0)
    nth = torch.cumsum(fresh.flatten().int(), 0).view(R, B) - 1
    page_at = torch.where(fresh, s["free"][nth.clamp(0, len(s["free"]) - 1)], -1)
    col = torch.arange(W, device=old.device)
    table = old.gather(1, p[:, :, None].expand(R, B, W))
    last = (kv_new // page)[:, :, None]
    src = torch.where(fresh, table.gather(2, last.clamp(max=W - 1)).squeeze(-1), -1)
    table = torch.where(fresh[:, :, None] & (col == last), page_at[:, :, None], table)
    table = torch.where(col < have_new[:, :, None], table, -1)
    # a page of the old rows that no new row of the request holds, in the lowest row that held it
    has = (col < have[:, :, None]) & (col >= s["keep"][:, None, None])
    held = (old[:, :, None] == table[:, None]).any(2)
    twice = ((old[:, :, None] == old[:, None]) & (k[None, :] < k[:, None])[None, :, :, None] & (col < have[:, None, :, None])).any(2)
    gone = (has & ~held & ~twice).transpose(1, 2).flatten()
    count = gone.sum()
    place = torch.where(gone, torch.cumsum(gone, 0) - 1, gone.numel())
    released = torch.full((gone.numel() + 1,), -1, dtype=torch.int32, device=old.device)
    released[place] = old.transpose(1, 2).flatten()
    released[-1] = -1
    dst = page_at.flatten()
    cache = s["cache"]
    moved = fresh.flatten()
    cache[dst[moved].long()] = cache[src.flatten()[moved].long()]
    return {"table": table.view(R * B, W).to(torch.int32), "kv_len": kv_new.flatten().to(torch.int32), "src": src.flatten().to(torch.int32),
            "dst": dst.to(torch.int32), "used": fresh.sum().reshape(1).to(torch.int32), "released": released[:-1],
            "count": count.reshape(1).to(torch.int32), "cache": cache}


def _adapters(s):
    # every row through every adapter, and its own kept
    n, r, K = s["a"].shape
    M = len(s["x"])
    t = torch.arange(M, device="cuda")
    mine = s["ids"][torch.searchsorted(s["cu"][1:].contiguous(), t, right=True)]
    keep = torch.where(mine[:, None] == torch.arange(n, device="cuda"), s["gain"], 0.0)
    mid = torch.matmul(s["x"].float(), s["a"].float().view(n * r, K).t()).view(M, n, r) * keep[:, :, None]
    delta = torch.matmul(mid.view(M, n * r), s["b"].float().transpose(1, 2).reshape(n * r, -1))
    return s["y"].add_(delta)


# ---------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its result in 64 bits
# ---------------------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "shared":
        H, Hkv, D, page, each = case["H"], case["Hkv"], case["D"], case["page"], case["each"]
        pre, new, mine = _lengths(case)
        keys = sum(pre) + sum(mine)
        entries = sum(_ceil(p, page) for p in pre) + sum(_ceil(n, page) for n in mine)
        seen = sum(m * (pre[r // each] + n) - m * (m - 1) // 2 for r, (m, n) in enumerate(zip(new, mine)))
        return {"bytes": 4 * sum(new) * H * D + keys * Hkv * D * 17 // 16 + 4 * entries + 8 * len(new), "flops": 4 * seen * D * H}
    if kind == "beam":
        n = case["R"] * case["B"] * case["V"]
        return {"bytes": n * (4 if case["x"] == "fp32" else 2) + case["R"] * (5 * case["B"] + 12 * case["K"]), "flops": 3 * n}
    if kind == "reorder":
        # the old rows' entries, the new rows' whole tables, and the pages that are copied, read and written
        R, B, page = case["R"], case["B"], case["page"]
        prompt, made, parents = _lengths(case)
        cols = [_ceil(p + n, page) for p, n in zip(prompt, made)]
        held = B * sum(cols)
        record = case["Hkv"] * page * (case["D"] + case["D"] // 16)
        copied = sum(B - len(set(of)) for p, n, of in zip(prompt, made, parents) if (p + n) % page and of[0] >= 0)
        return {"bytes": 4 * (held + R * B * (max(cols) + 1) + 5 * R * B) + copied * 2 * record, "flops": 0}
    lens, ids = _lengths(case)
    M, N, K, r = sum(lens), case["N"], case["K"], case["r"]
    used = len(set(ids) - {-1})
    M = sum(n for n, a in zip(lens, ids) if a >= 0)
    return {"bytes": 2 * M * K + 8 * M * N + 2 * used * r * (K + N), "flops": 2 * M * r * (K + N)}


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
    if kind == "reorder":
        return None      # whole numbers
    s = prepare(case, seed)
    if kind == "shared":
        H, Hkv, D, page = case["H"], case["Hkv"], case["D"], case["page"]
        pre, new, mine = _lengths(case)
        at = _starts(new)
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for g in range(Hkv):
            keys, values = _cache64(s["cache"], D, g, 0), _cache64(s["cache"], D, g, 1)
            for r, (n, m) in enumerate(zip(new, mine)):
                m += pre[r // case["each"]]
                slots = (s["table"][r, :_ceil(m, page)].long()[:, None] * page + torch.arange(page, device="cuda")).flatten()[:m]
                heads = slice(g * (H // Hkv), (g + 1) * (H // Hkv))
                q = s["q"][at[r]:at[r + 1], heads].double().transpose(0, 1)
                w = torch.matmul(q, keys[slots].T.contiguous()) * s["scale"]
                hidden = torch.arange(m, device="cuda")[None, :] > m - n + torch.arange(n, device="cuda")[:, None]
                w = torch.softmax(w.masked_fill(hidden, -math.inf), -1)
                out[at[r]:at[r + 1], heads] = torch.matmul(w, values[slots]).transpose(0, 1)
        return out
    if kind == "beam":
        # the values of every request's candidates alone: which they are is whole numbers
        R, B, V = case["R"], case["B"], case["V"]
        best = torch.full((R, case["K"]), -math.inf, dtype=torch.float64, device="cuda")
        for r in range(R):
            found = []
            for b in range(B):
                score, row = s["scores"][r, b].double(), s["logits"][r * B + b].double()
                if s["finished"] is not None and bool(s["finished"][r, b]):
                    found.append(score.reshape(1))
                else:
                    found.append(torch.log_softmax(row, 0).topk(min(V, case["K"])).values + score)
            found = torch.cat(found).sort(descending=True).values[:case["K"]]
            best[r, :len(found)] = found
        return {"scores": best, "parents": None, "tokens": None}
    out = s["y"].double()
    at = _starts(_lengths(case)[0])
    for r, a in enumerate(s["ids"].tolist()):
        if a >= 0:
            rows = slice(at[r], at[r + 1])
            mid = torch.matmul(s["x"][rows].double(), s["a"][a].double().T.contiguous())
            out[rows] += s["gain"][a].double() * torch.matmul(mid, s["b"][a].double().T.contiguous())
    return out
