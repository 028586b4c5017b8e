"""A key/value cache held in 4 bits, and log probabilities of given tokens, from their definitions.

A group is 32 dims of a token's head; with a = max |x| of its values the scale s is the least number of five
significant bits with 7 s >= a, and x is held as the whole number c in -7..7 nearest x / s, ties to even.  The
bytes of a (layer, page, head) are the codes c + 8 of all its slots, then their scales in bfloat16.
"""
from __future__ import annotations

import numpy as np

GROUP = 32


def scales(x):
    """Of groups x [..., 32], fp64: m 2^e with m = 16..31, or a multiple of 2^-130 below 2^-126."""
    a = np.abs(x).max(-1)
    out = np.zeros(a.shape)
    for i, v in np.ndenumerate(a):
        if v == 0:
            continue
        e = max(int(np.floor(np.log2(v / 7))) - 4, -130)
        e -= 2                                       # (the logarithm may be off by one)
        e = max(e, -130)
        m = int(np.ceil(v / 7 / 2.0 ** e))
        while m > 31:
            e += 1
            m = int(np.ceil(v / 7 / 2.0 ** e))
        s = m * 2.0 ** e
        assert 7 * s >= v
        out[i] = s
    return out


def quantise(x):
    """x [..., d] -> (whole numbers [..., d / 32, 32], scales [..., d / 32]), exact in fp64."""
    y = np.asarray(x, np.float64).reshape(x.shape[:-1] + (-1, GROUP))
    s = scales(y)
    q = np.divide(y, s[..., None], out=np.zeros_like(y), where=s[..., None] > 0)
    c = np.rint(q)                                   # (ties to even; |q| <= 7, and a quotient next to a tie differs in fp64)
    return c.astype(np.int64), s


def values(x):
    """What rows x [..., d] read back as."""
    c, s = quantise(x)
    return (c * s[..., None]).reshape(x.shape)


def pack(rows):
    """[..., page, d] -> bytes [..., page * d * 9 / 16] of blocks."""
    c, s = quantise(rows)
    lead, page, d = rows.shape[:-2], rows.shape[-2], rows.shape[-1]
    c = (c + 8).reshape(lead + (page, d // 8, 4, 2))             # element 8 w + 2 k + h
    shift = 16 * np.arange(2) + 4 * np.arange(4)[:, None]
    words = (c << shift).sum((-1, -2)).astype("<u4")
    codes = words.view(np.uint8).reshape(lead + (page * d // 2,))
    bits = (s.astype("<f4").view("<u4") >> 16).astype("<u2").view(np.uint8).reshape(lead + (page * d // 16,))
    return np.concatenate([codes, bits], -1)


def unpack(block, page, d):
    """bytes [..., page * d * 9 / 16] -> fp32 [..., page, d]."""
    lead = block.shape[:-1]
    words = np.ascontiguousarray(block[..., :page * d // 2]).view("<u4").astype(np.int64).reshape(lead + (page, d // 8))
    shift = 16 * np.arange(2) + 4 * np.arange(4)[:, None]
    c = ((words[..., None, None] >> shift) & 15).reshape(lead + (page, d // GROUP, GROUP)) - 8
    bits = np.ascontiguousarray(block[..., page * d // 2:]).view("<u2").astype("<u4") << 16
    s = bits.view("<f4").reshape(lead + (page, d // GROUP, 1))
    with np.errstate(invalid="ignore"):
        return (c.astype(np.float32) * s).reshape(lead + (page, d))


def logprobs(z, tokens, temperature, k):
    """z [rows][V] -> (logprob, entropy, top, top_logprob), fp64; rows without a token (-1), and rows without a
    distribution (their largest logit infinite, a NaN in them)."""
    rows, V = z.shape
    logprob, entropy = np.full(rows, -np.inf), np.zeros(rows)
    top, top_logprob = np.full((rows, k), -1), np.full((rows, k), -np.inf)
    for r, t in enumerate(tokens):
        if not 0 <= t < V:
            continue
        x = np.asarray(z[r], np.float64) / temperature
        m = np.max(x)
        if not np.isfinite(m):
            logprob[r] = entropy[r] = np.nan
            top_logprob[r] = np.nan
            continue
        x = x - m
        lse = np.log(np.exp(x).sum())
        p = np.exp(x - lse)
        logprob[r] = x[t] - lse
        entropy[r] = -(p[p > 0] * (x[p > 0] - lse)).sum()
        order = np.argsort(-np.asarray(z[r], np.float64), kind="stable")[:k]
        top[r], top_logprob[r] = order, x[order] - lse
    return logprob, entropy, top, top_logprob
