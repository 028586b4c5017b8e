"""A cache held in 4 bits against the oracle: quantising writes, reads, and the page operators over it.  Every stored
code and scale has one right value, so everything is compared for equality."""
import numpy as np
import pytest
import torch

from oracle import cache_q4
from tests.gpu_common import lsp_lib
from tests.q4_common import held, make_pool, oracle_cache, same_tokens
from tests.target_common import DT, holders, make_cache, make_pool as make_plain_pool, oracle_cache as plain_oracle, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


def ints(x):
    return torch.tensor([int(i) for i in x], dtype=torch.int32, device="cuda")


def starts(rows):
    return ints(np.concatenate([[0], np.cumsum(rows)]))


def gen(seed):
    return torch.Generator().manual_seed(seed)


def write(lsp, c, layer, seqs, rows, k, v, bits=0):
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    lsp.lsp_pages_write_q4(c, layer, ints(seqs), starts(rows), k, v, err)
    assert int(err.item()) == bits


def read(lsp, c, layer, seqs, rows, dtype, bits=0, pad=0, fill=7.0):
    shape = (int(sum(rows)), c.nkv * c.d + pad)
    k, v = (torch.full(shape, fill, dtype=DT[dtype], device="cuda")[:, :c.nkv * c.d].unflatten(1, (c.nkv, c.d)) for _ in range(2))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    lsp.lsp_pages_read(c, layer, ints(seqs), starts(rows), k, v, err)
    assert int(err.item()) == bits
    return k, v


# rows whose values are hard to place: ties, the largest and smallest numbers, empty groups
def hard_rows(total, nkv, d, dtype, g):
    x = torch.randn(total, nkv, d, generator=g) * torch.exp(3 * torch.randn(total, nkv, 1, generator=g))
    flat = x.view(-1, 32)
    n = flat.shape[0]
    flat[0] = 0
    if n > 6:
        flat[1] = torch.tensor([7.0] + [(i - 15) / 2.2 // 1 + 0.5 for i in range(31)]).clamp(-7, 7)      # ties at scale 1
        flat[2] = torch.tensor([7 * 19.0] + [19 * ((i % 14) - 7 + 0.5) for i in range(31)])              # ... at scale 19
        flat[3] = torch.tensor([2.0 ** -133 * (i - 9) for i in range(32)])                               # below the normal numbers
        flat[4] = torch.tensor([3.3e38 if i == 5 else -2e37 * i / 32 for i in range(32)])
        flat[5] = torch.tensor([1e-30 * (i - 16) for i in range(32)])
        flat[6] = torch.tensor([-(2.0 ** -149) if i == 31 else 0.0 for i in range(32)])
    return x.to(DT[dtype]).cuda()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("nkv,d,page,order", [(1, 64, 16, "dense"), (3, 64, 32, "pages"), (8, 128, 64, "dense"), (2, 128, 256, "pages"),
                                              (5, 128, 16, "dense")])
def test_written_rows_read_back_as_the_nearest_values(lsp, nkv, d, page, order, dtype):
    g = gen(3)
    lens, rows, seqs = [1, 2 * page, 3 * page + 5, 40, 0], [1, 17, 2 * page + 3, 0, 0], [0, 1, 2, 3, 4]
    pool = make_pool(2, 20, nkv, page, d, g, "cuda", order)
    t = [x.cuda() for x in make_cache(lens, 0, page, pool)]
    oc, before = oracle_cache(*pool, *t), [x.clone() for x in pool]
    c = lsp.make_kv_cache(*pool, *t)
    total = sum(rows)
    wide = hard_rows(total, 2 * nkv + 1, d, dtype, g)
    k, v = wide[:, :nkv], wide[:, nkv:2 * nkv]       # slices of a fused row
    write(lsp, c, 1, seqs, rows, k, v)
    start = np.concatenate([[0], np.cumsum(rows)])
    oc.write(1, seqs, start, cache_q4.values(up(k).astype(np.float64)), cache_q4.values(up(v).astype(np.float64)))
    same_tokens(oc, *pool, *t)
    # nothing else was touched: the other layer, and the codes of every other slot
    for x, y, z in zip(pool, before, (oc.k, oc.v)):
        assert torch.equal(x[0], y[0])
        np.testing.assert_array_equal(held(x), z)
    for out, pad in ((dtype, 0), ("f32", 16), ("bf16", 8)):
        kr, vr = read(lsp, c, 1, seqs, rows, out, pad=pad)
        np.testing.assert_array_equal(up(kr), cache_q4.values(up(k).astype(np.float64)))
        np.testing.assert_array_equal(up(vr), cache_q4.values(up(v).astype(np.float64)))
    # what was read back is held as it is: it writes the same values again
    write(lsp, c, 1, seqs, rows, kr, vr)
    same_tokens(oc, *pool, *t)


def test_every_scale_and_its_ties(lsp):
    """Sixteen mantissas of the scale, with every half step and its two neighbours in fp32."""
    page, d, nkv = 64, 128, 1
    rows = []
    for m in range(16, 32):
        for e in (-40, 0, 33):
            s = np.float32(m * 2.0 ** (e - 4))
            x = [7 * s]
            for n in range(7):
                y = np.float32((n + 0.5) * s)
                x += [y, -y, np.nextafter(y, np.float32(0)), -np.nextafter(y, np.float32(np.inf))]
            rows.append(x + [0.0] * 3)
    x = torch.from_numpy(np.float32(rows)).view(-1, nkv, d).cuda()        # 48 groups: 12 rows
    pool = make_pool(1, 2, nkv, page, d, gen(1), "cuda")
    t = [y.cuda() for y in make_cache([12], 0, page, pool)]
    c = lsp.make_kv_cache(*pool, *t)
    write(lsp, c, 0, [0], [12], x, x)
    k, v = read(lsp, c, 0, [0], [12], "f32")
    want = cache_q4.values(up(x).astype(np.float64))
    np.testing.assert_array_equal(up(k), want)
    np.testing.assert_array_equal(up(v), want)


@pytest.mark.parametrize("dtype", list(DT))
def test_a_group_that_is_not_finite_is_nan_and_the_others_are_not(lsp, dtype):
    page, d, nkv = 16, 64, 2
    x = torch.randn(3, nkv, d, generator=gen(2)).to(DT[dtype]).cuda()
    x[0, 0, 3], x[1, 1, 40], x[2, 0, 63] = float("nan"), float("inf"), float("-inf")
    pool = make_pool(1, 2, nkv, page, d, gen(1), "cuda")
    t = [y.cuda() for y in make_cache([3], 0, page, pool)]
    c = lsp.make_kv_cache(*pool, *t)
    write(lsp, c, 0, [0], [3], x, x)
    k, _ = read(lsp, c, 0, [0], [3], "f32")
    bad = ~torch.isfinite(x.float()).view(3, nkv, 2, 32).all(-1, keepdim=True).expand(-1, -1, -1, 32).reshape(x.shape)
    assert torch.equal(torch.isnan(k), bad)
    clean = torch.where(bad, torch.zeros_like(x), x)
    np.testing.assert_array_equal(up(torch.where(bad, torch.zeros_like(k), k)), cache_q4.values(up(clean).astype(np.float64)))


@pytest.mark.parametrize("kind", ["q4", "bf16", "f32"])
def test_entries_that_cannot_be_used(lsp, kind):
    """Sequences and ranges outside the cache leave rows as they were, pages outside the pool read as zero."""
    page, d, nkv = 16, 64, 2
    g = gen(4)
    lens = [20, 33, 40, 5, 50]
    pool = make_pool(1, 20, nkv, page, d, g, "cuda") if kind == "q4" else make_plain_pool(1, 20, nkv, page, d, kind, g, device="cuda")
    t = [x.cuda() for x in make_cache(lens, 0, page, pool)]
    t[0][1, 1] = 20
    t[0][2, 0] = -1
    t[1][4] = 10 ** 6
    oc = (oracle_cache if kind == "q4" else plain_oracle)(*pool, *t)
    before = [x.clone() for x in pool]
    c = lsp.make_kv_cache(*pool, *t)
    seqs, rows = [0, 1, 9, 2, -1, 3, 4], [3, 33, 2, 40, 1, 8, 2]          # (sequence 3 is shorter than its rows)
    dtype = "f32" if kind == "q4" else kind
    k, v = read(lsp, c, 0, seqs, rows, dtype, bits=lsp.LSP_DEV_BAD_SEQ)
    at = 0
    for s, r in zip(seqs, rows):
        here = up(k[at:at + r]), up(v[at:at + r])
        if s in (0, 1, 2):
            for a, b in zip(here, oc.tokens(0, s)):
                np.testing.assert_array_equal(a, b[len(b) - r:])
        elif s == 3:
            for a, b in zip(here, oc.tokens(0, s)):
                np.testing.assert_array_equal(a[3:], b)
                assert (a[:3] == 7).all()
        else:
            assert (here[0] == 7).all() and (here[1] == 7).all()
        at += r
    if kind == "q4":
        x = torch.randn(sum(rows), nkv, d, generator=g).cuda()
        write(lsp, c, 0, seqs, rows, x, x, bits=lsp.LSP_DEV_BAD_SEQ)
        y = cache_q4.values(up(x).astype(np.float64))
        oc.write(0, seqs, np.concatenate([[0], np.cumsum(rows)]), y, y)
        np.testing.assert_array_equal(held(pool[0]), oc.k)
        np.testing.assert_array_equal(held(pool[1]), oc.v)
    else:
        assert all(torch.equal(a, b) for a, b in zip(pool, before))


@pytest.mark.parametrize("dtype,order", [("bf16", "dense"), ("f32", "tokens"), ("bf16", "tokens")])
def test_reading_caches_of_elements(lsp, dtype, order):
    lens, rows, seqs = [100, 1, 64, 17], [3, 1, 16, 100], [2, 1, 3, 0]
    pool = make_plain_pool(3, 20, 3, 32, 64, dtype, gen(6), order, "cuda")
    t = [x.cuda() for x in make_cache(lens, 0, 32, pool)]
    oc = plain_oracle(*pool, *t)
    c = lsp.make_kv_cache(*pool, *t)
    k, v = read(lsp, c, 2, seqs, rows, dtype, pad=8)
    at = 0
    for s, r in zip(seqs, rows):
        want = oc.tokens(2, s)
        for a, b in zip((k, v), want):
            np.testing.assert_array_equal(up(a[at:at + r]), b[len(b) - r:])
        at += r
    # rows before the first entry and behind the last are nobody's
    out = [torch.full((10, 3, 64), 7.0, dtype=DT[dtype], device="cuda") for _ in range(2)]
    lsp.lsp_pages_read(c, 0, ints([0]), ints([4, 8]), *out)
    for x in out:
        assert bool((x[:4] == 7).all()) and bool((x[8:] == 7).all()) and not bool((x[4:8] == 7).any())


class Both:
    """A cache in 4 bits on the GPU and the oracle's copy of its values."""

    def __init__(self, lsp, pool, table, lens, refs):
        self.lsp, self.pool = lsp, pool
        self.t = [x.cuda() for x in (table, lens, refs)]
        self.o = oracle_cache(*pool, *self.t)
        self.c = lsp.make_kv_cache(*pool, *self.t)
        self.ws = torch.empty(lsp.lsp_pages_workspace_bytes(self.c), dtype=torch.uint8, device="cuda").fill_(0xAB)
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def check(self):
        torch.cuda.synchronize()
        same_tokens(self.o, *self.pool, *self.t)
        holders(*self.t, self.o.page)


@pytest.mark.parametrize("d,nkv,page,order", [(128, 2, 16, "dense"), (64, 3, 32, "pages"), (64, 1, 16, "dense")])
def test_a_long_run_of_random_operations(lsp, d, nkv, page, order):
    g, rng = gen(5), np.random.RandomState(7)
    seqs, layers, pages = 7, 2, 30
    pool = make_pool(layers, pages, nkv, page, d, g, "cuda", order)
    b = Both(lsp, pool, *make_cache([0] * seqs, 0, page, pool, spare=4))
    for step in range(90):
        op = rng.randint(5)
        some = [int(x) for x in rng.permutation(seqs)[:rng.randint(1, 5)]]
        if op == 0 and len(some) > 1:
            half = len(some) // 2
            src, dst = [int(x) for x in rng.choice(some[half:], half)], some[:half]
            lsp.lsp_pages_fork(b.c, ints(src), ints(dst), b.err)
            b.o.fork(src, dst)
        elif op in (1, 2):
            add = [int(x) for x in rng.randint(0, 2 * page + 3, len(some))]
            lsp.lsp_pages_reserve(b.c, ints(some), ints(add), b.ws, b.err)
            bad, short = b.o.reserve(some, add)
            ok = [i for i in range(len(some)) if i not in bad + short]
            rows = [add[i] for i in ok]
            if ok and sum(rows):
                layer = int(rng.randint(layers))
                k, v = (torch.randn(sum(rows), nkv, d, generator=g).cuda() for _ in range(2))
                for x in range(layers):              # (a page's slots hold nothing that was written before)
                    write(lsp, b.c, x, [some[i] for i in ok], rows, k, v) if x != layer else None
                write(lsp, b.c, layer, [some[i] for i in ok], rows, v, k)
                start = np.concatenate([[0], np.cumsum(rows)]).astype(int)
                kk, vv = (cache_q4.values(up(x).astype(np.float64)) for x in (k, v))
                for x in range(layers):
                    b.o.write(x, [some[i] for i in ok], start, *((vv, kk) if x == layer else (kk, vv)))
        elif op == 3:
            new = [int(x) for x in rng.randint(0, 4 * page, len(some))]
            lsp.lsp_pages_trim(b.c, ints(some), ints(new), b.err)
            b.o.trim(some, new)
        elif step % 3 == 0:
            live = torch.zeros(1, dtype=torch.int32, device="cuda")
            lsp.lsp_pages_compact(b.c, live, b.ws)
            assert int(live.item()) == b.o.compact()
        if step % 9 == 8:
            b.check()
    b.check()


def test_offsets_beyond_32_bits(lsp):
    """Pages more than 2^31 bytes from the pool's start (one head of a page every 72 MB, nothing between is written)."""
    page, d, nkv, pages = 16, 64, 1, 60
    step = 72 << 20
    raw = torch.empty(2 * pages * step, dtype=torch.uint8, device="cuda")
    pool = [raw[i * step:].as_strided((1, pages, nkv, page, 36), (step, 2 * step, page * 36, 36, 1)) for i in range(2)]
    t = [x.cuda() for x in make_cache([50 * page], 0, page, pool)]
    c = lsp.make_kv_cache(*pool, *t)
    k, v = (torch.randn(50 * page, nkv, d, generator=gen(8)).cuda() for _ in range(2))
    write(lsp, c, 0, [0], [50 * page], k, v)
    for a, b in zip(read(lsp, c, 0, [0], [50 * page], "bf16"), (k, v)):
        np.testing.assert_array_equal(up(a), cache_q4.values(up(b).astype(np.float64)))
    ws = torch.empty(lsp.lsp_pages_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    lsp.lsp_pages_compact(c, None, ws)
    for a, b in zip(read(lsp, c, 0, [0], [50 * page], "bf16"), (k, v)):
        np.testing.assert_array_equal(up(a), cache_q4.values(up(b).astype(np.float64)))


def test_captured_writes_and_reads_follow_their_tensors(lsp):
    page, d, nkv = 16, 128, 2
    pool = make_pool(1, 12, nkv, page, d, gen(1), "cuda")
    t = [x.cuda() for x in make_cache([30, 40], 0, page, pool)]
    c = lsp.make_kv_cache(*pool, *t)
    k, v = (torch.zeros(9, nkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    seqs, start = ints([1, 0]), ints([0, 4, 9])
    lsp.lsp_pages_write_q4(c, 0, seqs, start, k, v)
    lsp.lsp_pages_read(c, 0, seqs, start, ko, vo)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lsp.lsp_pages_write_q4(c, 0, seqs, start, k, v)
        lsp.lsp_pages_read(c, 0, seqs, start, ko, vo)
    for seed in range(3):
        k.copy_(torch.randn(k.shape, generator=gen(seed)))
        v.copy_(torch.randn(v.shape, generator=gen(seed + 9)))
        t[1].copy_(ints([30 + seed, 40 - 9 * seed]))
        graph.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(up(ko), cache_q4.values(up(k).astype(np.float64)))
        np.testing.assert_array_equal(up(vo), cache_q4.values(up(v).astype(np.float64)))
