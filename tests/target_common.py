"""Shared helpers of the tests of the target side: caches as tensors and as the oracle's."""
import numpy as np
import torch

from oracle.target import PagedCache

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def up(t):
    return t.detach().float().cpu().numpy()


def make_pool(layers, pages, nkv, page, d, dtype, g, order="dense", device="cpu"):
    """k, v [layers][pages][nkv][page][d]; order "tokens": slots outside the heads in memory, k and v beside each other."""
    def rnd(*shape):
        return torch.randn(*shape, generator=g).to(DT[dtype]).to(device)
    if order == "dense":
        return rnd(layers, pages, nkv, page, d), rnd(layers, pages, nkv, page, d)
    both = rnd(pages, layers, page, 2, nkv, d)
    return both[:, :, :, 0].permute(1, 0, 3, 2, 4), both[:, :, :, 1].permute(1, 0, 3, 2, 4)


def make_cache(lens, shared, page, pool, seqs=None, spare=2, seed=0):
    """Sequences of `lens` tokens, the first `shared` tokens' whole pages held by all, at shuffled places.
    -> (table, len, refs) int32; rows of the table beyond the lens are empty sequences."""
    pages = pool[0].shape[1]
    rng = np.random.RandomState(seed)
    place = list(rng.permutation(pages))
    n = len(lens)
    width = max([-(-x // page) for x in lens] + [1]) + spare
    table, refs = np.full((n, width), -1, np.int32), np.zeros(pages, np.int32)
    common = [place.pop() for _ in range(shared // page)]
    for b, x in enumerate(lens):
        for i in range(-(-x // page)):
            table[b, i] = common[i] if i < len(common) else place.pop()
            refs[table[b, i]] += 1
    return torch.from_numpy(table), torch.tensor(lens, dtype=torch.int32), torch.from_numpy(refs)


def oracle_cache(k, v, table, lens, refs):
    return PagedCache(up(k), up(v), *(t.cpu().numpy() for t in (table, lens, refs)))


def same_cache(oc, k, v, table, lens, refs):
    np.testing.assert_array_equal(table.cpu().numpy(), oc.table)
    np.testing.assert_array_equal(lens.cpu().numpy(), oc.len)
    np.testing.assert_array_equal(refs.cpu().numpy(), oc.refs)
    np.testing.assert_array_equal(up(k), oc.k)
    np.testing.assert_array_equal(up(v), oc.v)


def holders(table, lens, refs, page):
    """Every page's count is the number of sequences that hold it."""
    want = np.zeros(len(refs), np.int64)
    for s, n in enumerate(lens.tolist()):
        for pg in table[s, :-(-n // page)].tolist():
            want[pg] += 1
    np.testing.assert_array_equal(refs.cpu().numpy(), want)
