"""Helpers of the tests of a cache held in 4 bits: pools of bytes, and the values they stand for."""
import numpy as np
import torch

from oracle import cache_q4
from oracle.target import PagedCache


def make_pool(layers, pages, nkv, page, d, g, device="cpu", order="dense", lean=0.0):
    """Two uint8 pools [layers][pages][nkv][page][9 d / 16] of quantised normal values; order "pages": layers
    inside the pages and both pools side by side."""
    out = []
    for _ in range(2):
        x = torch.randn(layers, pages, nkv, page, d, generator=g).numpy() + lean
        out.append(torch.from_numpy(cache_q4.pack(x)).unflatten(-1, (page, d * 9 // 16)))
    if order == "dense":
        return tuple(x.to(device) for x in out)
    both = torch.stack(out).permute(2, 0, 3, 1, 4, 5).contiguous().to(device)        # [pages][2][nkv][layers][page][held]
    return tuple(both[:, i].permute(2, 0, 1, 3, 4) for i in range(2))


def held(pool):
    """fp32 [layers][pages][nkv][page][d] of a pool of bytes."""
    page, width = pool.shape[3:]
    return cache_q4.unpack(pool.contiguous().flatten(3).cpu().numpy(), page, width * 16 // 9)


def oracle_cache(k, v, table, lens, refs):
    return PagedCache(held(k), held(v), *(t.cpu().numpy() for t in (table, lens, refs)))


def same_tokens(oc, k, v, table, lens, refs):
    """The bookkeeping, and every token of every sequence (what lies in unused slots may be anything)."""
    np.testing.assert_array_equal(table.cpu().numpy(), oc.table)
    np.testing.assert_array_equal(lens.cpu().numpy(), oc.len)
    np.testing.assert_array_equal(refs.cpu().numpy(), oc.refs)
    here = oracle_cache(k, v, table, lens, refs)
    for s in range(len(oc.len)):
        for layer in range(k.shape[0]):
            for a, b in zip(here.tokens(layer, s), oc.tokens(layer, s)):
                np.testing.assert_array_equal(a, b)
