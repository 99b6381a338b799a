"""Shared helpers of the serving tests: bf16 arrays, requests with pages of a shuffled pool, packed rows."""
import numpy as np

import oracle
import synth


def bf16(x):
    """x rounded to bf16, as float64 and as bits."""
    bits = synth.bf16_bits(np.asarray(x, dtype=np.float32))
    return oracle.decode_bf16(bits), bits


def dev_bf16(torch, bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16).cuda()


def host_bf16(torch, t):
    """A bf16 tensor as float64."""
    return oracle.decode_bf16(t.detach().contiguous().cpu().view(torch.int16).numpy().view(np.uint16))


def dev_i32(torch, a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).cuda()


def starts(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def tables(rng, kv_len, page, spare=2, width=None):
    """(block table [R][W] with -1 behind each request's pages, pages in all) over a shuffled pool."""
    need = [-(-int(n) // page) for n in kv_len]
    pages = sum(need) + spare
    ids = rng.permutation(pages)
    W = width if width is not None else max(need + [1]) + 1
    t = np.full((len(kv_len), W), -1, dtype=np.int64)
    at = 0
    for r, n in enumerate(need):
        t[r, :n] = ids[at:at + n]
        at += n
    return t, pages


def random_cache(rng, pages, Hkv, D, page, std=1.0):
    """(cache bytes, key values, value values) of random rows; codes and exponents drawn directly, near std."""
    cache = np.zeros((pages, Hkv, page * (D + D // 16)), dtype=np.uint8)
    n = page * D
    cache[..., :n] = rng.integers(0, 256, cache[..., :n].shape)
    cache[..., n:] = 126 + int(round(np.log2(std))) - (rng.random(cache[..., n:].shape) < 0.4)
    k, v = oracle.decode_cache(cache, D)
    return cache, k, v
