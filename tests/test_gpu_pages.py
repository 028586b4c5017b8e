"""Page operators of the target's cache against the oracle: every table entry, length, count of
holders and stored value equal (nothing is computed, so nothing may differ)."""
import numpy as np
import pytest
import torch

from tests.gpu_common import lsp_lib
from tests.target_common import DT, holders, make_cache, make_pool, oracle_cache, same_cache, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


class Both:
    """A cache on the GPU and the oracle's copy of it."""

    def __init__(self, lsp, pool, table, lens, refs):
        self.lsp, (self.k, self.v) = lsp, pool
        self.t = [x.cuda() for x in (table, lens, refs)]
        self.o = oracle_cache(self.k, self.v, *self.t)
        self.c = lsp.make_kv_cache(self.k, self.v, *self.t)
        self.ws = torch.empty(lsp.lsp_pages_workspace_bytes(self.c), dtype=torch.uint8, device="cuda").fill_(0xAB)
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def bits(self):
        e = int(self.err.item())
        self.err.zero_()
        return e

    def check(self):
        torch.cuda.synchronize()
        same_cache(self.o, self.k, self.v, *self.t)
        holders(*self.t, self.o.page)

    def ints(self, x):
        return torch.tensor(list(map(int, x)), dtype=torch.int32, device="cuda")

    def fork(self, src, dst):
        self.lsp.lsp_pages_fork(self.c, self.ints(src), self.ints(dst), self.err)
        bad = self.o.fork(list(src), list(dst))
        assert self.bits() == (self.lsp.LSP_DEV_BAD_SEQ if bad else 0)

    def trim(self, seqs, new):
        self.lsp.lsp_pages_trim(self.c, self.ints(seqs), self.ints(new), self.err)
        bad = self.o.trim(list(seqs), list(new))
        assert self.bits() == (self.lsp.LSP_DEV_BAD_SEQ if bad else 0)

    def reserve(self, seqs, add):
        self.lsp.lsp_pages_reserve(self.c, self.ints(seqs), self.ints(add), self.ws, self.err)
        bad, short = self.o.reserve(list(seqs), list(add))
        want = (self.lsp.LSP_DEV_BAD_SEQ if bad else 0) | (self.lsp.LSP_DEV_NO_PAGE if short else 0)
        assert self.bits() == want
        return bad, short

    def write(self, layer, seqs, rows, g, stride_pad=0):
        start = np.concatenate([[0], np.cumsum(rows)]).astype(int)
        nkv, d = self.c.nkv, self.c.d
        shape = (int(start[-1]), nkv * d + stride_pad)
        kn, vn = (torch.randn(shape, generator=g).to(self.k.dtype).cuda() for _ in range(2))
        kn, vn = (x[:, :nkv * d].unflatten(1, (nkv, d)) for x in (kn, vn))
        self.lsp.lsp_pages_write(self.c, layer, self.ints(seqs), self.ints(start), kn, vn, self.err)
        self.o.write(layer, list(seqs), start, up(kn), up(vn))
        assert self.bits() == 0

    def compact(self):
        live = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.lsp.lsp_pages_compact(self.c, live, self.ws)
        assert int(live.item()) == self.o.compact()


def gen(seed):
    return torch.Generator().manual_seed(seed)


@pytest.mark.parametrize("dtype,d,nkv,page,order", [("bf16", 128, 2, 16, "dense"), ("bf16", 64, 3, 32, "tokens"),
                                                    ("f32", 64, 1, 64, "dense"), ("f32", 128, 2, 16, "tokens")])
def test_a_long_run_of_random_operations(lsp, dtype, d, nkv, page, order):
    g, rng = gen(5), np.random.RandomState(7)
    seqs, layers, pages = 9, 2, 40
    pool = make_pool(layers, pages, nkv, page, d, dtype, g, order, "cuda")
    table, lens, refs = make_cache([0] * seqs, 0, page, pool, spare=5)
    b = Both(lsp, pool, table, lens, refs)
    for step in range(120):
        op = rng.randint(5)
        some = list(rng.permutation(seqs)[:rng.randint(1, 5)])
        if op == 0:
            half = len(some) // 2
            b.fork(list(rng.choice(some[half:], half)), some[:half]) if half else None
        elif op in (1, 2):
            add = list(rng.randint(0, 2 * page + 3, len(some)))
            bad, short = b.reserve(some, add)
            ok = [i for i in range(len(some)) if i not in bad + short]
            if ok and sum(add[i] for i in ok):
                b.write(int(rng.randint(layers)), [some[i] for i in ok], [add[i] for i in ok], g, 64 if step % 2 else 0)
        elif op == 3:
            b.trim(some, list(rng.randint(0, 4 * page, len(some))))
        elif step % 3 == 0:
            b.compact()
        if step % 10 == 9:
            b.check()
    b.check()


def test_the_last_holder_keeps_a_shared_page_and_the_others_copy_it(lsp):
    g = gen(1)
    pool = make_pool(3, 12, 2, 16, 128, "bf16", g, device="cuda")
    b = Both(lsp, pool, *make_cache([21, 0, 0, 0], 0, 16, pool))
    b.fork([0, 0, 0], [1, 2, 3])
    b.check()
    b.reserve([2, 0, 3, 1], [1, 17, 0, 1])           # sequence 3 takes nothing: it keeps sharing, so all three copy
    b.check()
    page = b.t[0][:, 1].cpu().tolist()
    assert len(set(page)) == 4
    b.fork([0, 0], [1, 2])
    b.trim([0, 1, 2], [20, 20, 20])
    b.reserve([1, 0, 2], [1, 1, 1])                  # all three: the last listed keeps it
    b.check()


def test_a_sequence_cut_into_a_shared_page_copies_it_before_it_grows(lsp):
    g = gen(2)
    pool = make_pool(1, 12, 1, 16, 64, "f32", g, device="cuda")
    b = Both(lsp, pool, *make_cache([48, 0], 0, 16, pool))
    b.fork([0], [1])
    b.trim([1], [20])                                # its second page is full in sequence 0, and shared
    b.reserve([1], [3])
    b.write(0, [1], [3], g)
    b.check()
    b.trim([1], [32])
    b.trim([0, 1], [0, 0])
    b.check()
    assert int(b.t[2].sum()) == 0


def test_refusals_on_the_device_leave_the_entry_alone(lsp):
    g = gen(3)
    pool = make_pool(1, 8, 1, 16, 64, "bf16", g, device="cuda")
    b = Both(lsp, pool, *make_cache([30, 5, 0, 0], 0, 16, pool, spare=1))
    b.fork([0, 1, 9, 0], [2, 2, 3, -1])              # a dst twice, a src and a dst outside
    b.check()
    b.fork([0, 1], [1, 3])                           # sequence 1 is both
    b.check()
    b.trim([0, 0, 7, 1], [16, 3, 1, -2])
    b.check()
    b.reserve([1, 1, -4, 0, 3], [2, 2, 1, -1, 1000])
    b.check()
    b.reserve([3, 1, 0], [16, 40, 1])                # pages run out at the second; the third is left too
    b.check()
    b.reserve([0], [0])
    b.check()
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    lsp.lsp_pages_fork(b.c, empty, empty)
    lsp.lsp_pages_trim(b.c, empty, empty)
    lsp.lsp_pages_reserve(b.c, empty, empty, b.ws)
    b.check()


def test_rows_that_have_no_place_are_dropped(lsp):
    g = gen(4)
    pool = make_pool(1, 6, 1, 16, 64, "bf16", g, device="cuda")
    b = Both(lsp, pool, *make_cache([3, 20], 0, 16, pool))
    rows = torch.randn(9, 1, 64, generator=g).bfloat16().cuda()
    b.lsp.lsp_pages_write(b.c, 0, b.ints([0, 77, 1]), b.ints([0, 5, 7, 9]), rows, rows, b.err)   # 5 rows for 3 tokens, none for 77
    assert b.bits() == lsp.LSP_DEV_BAD_SEQ
    b.o.write(0, [0], [2, 5], up(rows), up(rows))
    b.o.write(0, [1], [7, 9], up(rows), up(rows))
    b.check()


def test_many_entries_and_many_pages(lsp):
    """The most entries of a call, and a pool of several scan steps; free pages start late."""
    g, rng = gen(6), np.random.RandomState(2)
    n, pages = lsp_max_seqs(), 20001
    pool = make_pool(1, pages, 1, 16, 64, "bf16", g, device="cuda")
    lens = [int(x) for x in rng.randint(0, 200, n)]
    b = Both(lsp, pool, *make_cache(lens + [0] * n, 0, 16, pool, spare=3))
    b.fork(range(n), range(n, 2 * n))
    b.reserve(range(n, 2 * n), rng.randint(0, 40, n))
    b.check()
    b.trim(range(n), rng.randint(0, 100, n))
    b.compact()
    b.check()
    b.compact()                                      # nothing left to move
    b.check()


def lsp_max_seqs():
    return 1024


def test_the_same_calls_give_the_same_pages_on_another_stream(lsp):
    g = gen(8)
    k, v = make_pool(2, 30, 2, 16, 128, "bf16", g, device="cuda")
    table, lens, refs = make_cache([25, 40, 0, 0], 16, 16, (k, v), spare=4)
    got = []
    side = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), side):
        kk, vv, t = k.clone(), v.clone(), [x.cuda() for x in (table, lens, refs)]
        c = lsp.make_kv_cache(kk, vv, *t)
        ws = torch.empty(lsp.lsp_pages_workspace_bytes(c), dtype=torch.uint8, device="cuda")
        src, dst, add = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 1], [2, 3], [9, 30]))
        torch.cuda.synchronize()
        lsp.lsp_pages_fork(c, src, dst, stream=stream)
        lsp.lsp_pages_reserve(c, dst, add, ws, stream=stream)
        lsp.lsp_pages_trim(c, src, add, stream=stream)
        lsp.lsp_pages_compact(c, None, ws, stream=stream)
        torch.cuda.synchronize()
        got.append([kk, vv] + t)
    assert all(torch.equal(x, y) for x, y in zip(*got))


def test_a_captured_round_of_pages_replays(lsp):
    """fork, reserve and trim in a CUDA graph: the same pages on every replay."""
    g = gen(9)
    pool = make_pool(1, 30, 1, 16, 64, "bf16", g, device="cuda")
    b = Both(lsp, pool, *make_cache([25, 0, 0], 0, 16, pool, spare=4))
    src, dst, add, new = b.ints([0, 0]), b.ints([1, 2]), b.ints([9, 30]), b.ints([30, 33])

    def calls():
        lsp.lsp_pages_fork(b.c, src, dst)
        lsp.lsp_pages_reserve(b.c, dst, add, b.ws)
        lsp.lsp_pages_trim(b.c, dst, new)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        b.o.fork([0, 0], [1, 2])
        b.o.reserve([1, 2], [9, 30])
        b.o.trim([1, 2], [30, 33])
        b.check()


@pytest.mark.parametrize("dtype", list(DT))
def test_pages_past_32_bit_offsets(lsp, dtype):
    """A pool of more than 2^32 bytes a tensor whose live pages lie at both ends."""
    es = 2 if dtype == "bf16" else 4
    page, d, nkv = 256, 128, 8
    per = page * d * nkv * es
    pages = 2 ** 32 // per + 40
    k = torch.empty(1, pages, nkv, page, d, dtype=DT[dtype], device="cuda")
    v = torch.empty_like(k)
    refs = torch.ones(pages, dtype=torch.int32, device="cuda")     # held elsewhere
    refs[-20:] = 0
    table = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    c = lsp.make_kv_cache(k, v, table, lens, refs)
    ws = torch.empty(lsp.lsp_pages_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    one = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    lsp.lsp_pages_reserve(c, one(0), one(300), ws)
    rows = torch.randn(300, nkv, d, generator=gen(1)).to(DT[dtype]).cuda()
    lsp.lsp_pages_write(c, 0, one(0), one(0, 300), rows, -rows)
    lsp.lsp_pages_fork(c, one(0), one(1))
    lsp.lsp_pages_reserve(c, one(1), one(1), ws)                   # copies page 2 to another far one
    torch.cuda.synchronize()
    assert table.tolist() == [[pages - 20, pages - 19, -1, -1], [pages - 20, pages - 18, -1, -1]]
    assert torch.equal(k[0, pages - 20].transpose(0, 1), rows[:256])
    assert torch.equal(v[0, pages - 18, :, :44].transpose(0, 1), -rows[256:])
    refs[:pages - 20] = 0
    lsp.lsp_pages_compact(c, None, ws)
    torch.cuda.synchronize()
    assert table.tolist() == [[0, 1, -1, -1], [0, 2, -1, -1]] and refs.tolist()[:4] == [2, 1, 1, 0]
    assert torch.equal(k[0, 0].transpose(0, 1), rows[:256]) and torch.equal(k[0, 2, :, :44].transpose(0, 1), rows[256:])
