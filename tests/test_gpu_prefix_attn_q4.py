"""lsp_prefix_attention_q4 against the oracle's fp64 attention over the values that the cache stands for.

Tolerances, from the arithmetic.  bf16: those of lsp_prefix_attention, for the same reasons (keys and values are bf16
exactly).  f32: q and the weights are taken to 24 bits (2^-24 of each), products are exact, fp32 sums of up to 128
terms of |score| < 20 move a weight by at most about 1e-5; 4e-5 of sum_j w_j |v_j|.  lse: 2e-5 + 2e-6 |lse|.
"""
import numpy as np
import pytest
import torch

from oracle.target import cache_attention
from tests.gpu_common import lsp_lib
from tests.q4_common import make_pool, oracle_cache
from tests.target_common import DT, make_cache, up
from tests.test_gpu_prefix_attn import CASES, compare

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


def ints(x):
    return torch.tensor([int(i) for i in x], dtype=torch.int32, device="cuda")


def attend(lsp, pool, t, q, seqs, rows, shared, layer=0, scale=None, lse=True, stream=None, bits=0, fill=0xFF):
    """-> (out, lse) of one call; the workspace starts as NaN patterns."""
    c = lsp.make_kv_cache(*pool, *t)
    ws = torch.empty(max(256, lsp.lsp_prefix_attention_q4_workspace_bytes(c, q.dtype, q.shape[1], len(seqs), q.shape[0])),
                     dtype=torch.uint8, device="cuda").fill_(fill)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    z = torch.full(q.shape[:2], float("nan"), device="cuda") if lse else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ids, start = ints(seqs), ints(np.concatenate([[0], np.cumsum(rows)]))
    torch.cuda.synchronize()
    lsp.lsp_prefix_attention_q4(c, layer, q, ids, start, out, z, shared_len=shared, scale=scale or q.shape[2] ** -0.5,
                                workspace=ws, dev_error=err, stream=stream)
    torch.cuda.synchronize()
    assert int(err.item()) == bits
    return out, z


def case(lens, rows, shared, *, nq, nkv, d, dtype, page, layers=1, order="dense", seed=0, extra=3, spare=2):
    g = torch.Generator().manual_seed(seed)
    need = shared // page + sum(-(-n // page) - min(-(-n // page), shared // page) for n in lens)
    pool = make_pool(layers, need + extra, nkv, page, d, g, "cuda", order)
    t = make_cache(lens, shared, page, pool, spare=spare, seed=seed)
    q = (torch.randn(sum(rows), nq, d, generator=g) * 1.5).to(DT[dtype]).cuda()
    return pool, [x.cuda() for x in t], q


MORE = {
    # rows of an item around the numbers that a warp and its row groups take: 8, 16, 32, 64
    "8 and 9 rows": dict(lens=[300, 301], rows=[8, 9], shared=0, nq=2, nkv=2, d=128, page=16),
    "16 and 17 rows": dict(lens=[300, 301], rows=[16, 17], shared=0, nq=2, nkv=2, d=64, page=64),
    "32, 33 and 65 rows": dict(lens=[300, 301, 310], rows=[32, 33, 65], shared=128, nq=1, nkv=1, d=128, page=128),
    "three heads a key head": dict(lens=[300, 301, 310], rows=[21, 22, 43], shared=0, nq=6, nkv=2, d=64, page=32),
    "33 heads a key head": dict(lens=[140, 150], rows=[1, 3], shared=128, nq=33, nkv=1, d=128, page=32),
    "pages of 256": dict(lens=[700, 513, 256], rows=[1, 2, 1], shared=256, nq=8, nkv=2, d=64, page=256),
    "a block and one token": dict(lens=[129, 257], rows=[1, 1], shared=128, nq=4, nkv=4, d=128, page=64),
}


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("name", list(CASES) + list(MORE))
def test_equals_the_oracle(lsp, name, dtype):
    kw = dict(CASES.get(name) or MORE[name], dtype=dtype)
    pool, t, q = case(**kw)
    seqs = list(range(len(kw["lens"])))
    oc = oracle_cache(*pool, *t)
    out, z = attend(lsp, pool, t, q, seqs, kw["rows"], kw["shared"])
    compare(oc, q, seqs, kw["rows"], out, z)
    again, z2 = attend(lsp, pool, t, q, seqs, kw["rows"], kw["shared"], fill=0)
    assert torch.equal(out, again) and torch.equal(z, z2)
    # the same rows with nothing said to be shared
    out, z = attend(lsp, pool, t, q, seqs, kw["rows"], 0)
    compare(oc, q, seqs, kw["rows"], out, z)


@pytest.mark.parametrize("dtype", list(DT))
def test_other_strides_layers_orders_and_streams(lsp, dtype):
    lens, rows, shared = [90, 100, 77, 130], [2, 1, 5, 3], 70
    pool, t, _ = case(lens, rows, shared, nq=4, nkv=2, d=64, dtype=dtype, page=16, layers=3, order="pages")
    g = torch.Generator().manual_seed(5)
    fused = torch.randn(sum(rows), 8, 64, generator=g).to(DT[dtype]).cuda()
    q = fused[:, 2:6]                                # a slice of a q/k/v row
    seqs = [2, 0, 3, 1]
    oc = oracle_cache(*pool, *t)
    for layer, stream in ((2, None), (0, torch.cuda.Stream())):
        out, _ = attend(lsp, pool, t, q, seqs, rows, shared, layer=layer, scale=0.2, lse=False, stream=stream)
        compare(oc, q, seqs, rows, out, None, layer=layer, scale=0.2)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("page,d", [(16, 128), (128, 128), (256, 64), (32, 64)])
def test_what_lies_in_unused_places_is_never_seen(lsp, page, d, dtype):
    """Codes and scales of slots without a token are any bits, scales NaN and infinite among them."""
    lens, rows, shared = [page * 3 + 5, page * 4 + 1, 7], [4, 21, 2], 0
    pool, t, q = case(lens, rows, shared, nq=8, nkv=2, d=d, dtype=dtype, page=page)
    seqs = [0, 1, 2]
    oc = oracle_cache(*pool, *t)
    used = torch.zeros(pool[0].shape[1], page, dtype=torch.bool)
    for s, n in enumerate(lens):
        for i in range(n):
            used[t[0][s, i // page], i % page] = True
    free = ~used.cuda()
    g = torch.Generator().manual_seed(1)
    bad = torch.tensor([0x7FC0, 0x7F80, -128, 0x7F7F, -1], dtype=torch.int16)       # NaN, inf, -inf, the largest, NaN
    for x in pool:
        block = x.flatten(3)
        codes = block[..., :page * d // 2].unflatten(-1, (page, -1))
        scales = block[..., page * d // 2:].view(torch.int16).unflatten(-1, (page, -1))
        where = free[None, :, None, :, None]
        codes.copy_(torch.where(where, torch.randint(0, 256, codes.shape, generator=g, dtype=torch.uint8).cuda(), codes))
        scales.copy_(torch.where(where, bad[torch.randint(0, 5, scales.shape, generator=g)].cuda(), scales))
    out, z = attend(lsp, pool, t, q, seqs, rows, shared)
    compare(oc, q, seqs, rows, out, z)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows", [[5, 3], [40, 35]])
def test_large_scores_that_rise_from_block_to_block(lsp, rows, dtype):
    lens, shared = [700, 640], 512
    pool, t, q = case(lens, rows, shared, nq=4, nkv=2, d=128, dtype=dtype, page=16, seed=3)
    q = q * 12
    oc = oracle_cache(*pool, *t)
    start = np.concatenate([[0], np.cumsum(rows)])
    want, lse, _ = cache_attention(oc, 0, up(q), [0, 1], start, 128 ** -0.5)
    out, z = attend(lsp, pool, t, q, [0, 1], rows, shared)
    # scores of some tens: their fp32 error (2^-23 of the sum of |terms|, below 500) moves a weight by up to 1e-4
    np.testing.assert_allclose(out.double().cpu().numpy(), want, rtol=0,
                               atol=(2 ** -7 if dtype == "bf16" else 2e-4) * np.abs(want).max())
    np.testing.assert_allclose(z.cpu().numpy(), lse, rtol=2e-6, atol=2e-4)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("page", [16, 64])
def test_entries_outside_the_cache_are_reported(lsp, page, dtype):
    lens, rows = [3 * page + 2, 4 * page, 2 * page + 8], [2, 3, 1]
    pool, t, q = case(lens, rows, 0, nq=4, nkv=2, d=64, dtype=dtype, page=page)
    for x in pool:                                   # (what the ring held before is not what a page of none reads as)
        x.flatten(3)[..., page * 32:].view(torch.int16).fill_(0x4000)
    oc = oracle_cache(*pool, *t)
    bad = lsp.LSP_DEV_BAD_SEQ
    out, z = attend(lsp, pool, t, q, [0, 99, -1], rows, 0, bits=bad)     # sequences that are none
    compare(oc, q, [0, 99, -1], rows, out, z)
    t[0][1, 2] = 10 ** 6                                                 # a page that is none reads as zeros
    t[0][0, 0] = -5
    oc = oracle_cache(*pool, *t)
    out, z = attend(lsp, pool, t, q, [0, 1, 2], rows, 0, bits=bad)
    compare(oc, q, [0, 1, 2], rows, out, z)
    t[1][2] = -3                                                         # a length that is none
    out, z = attend(lsp, pool, t, q, [0, 1, 2], rows, 0, bits=bad)
    assert torch.equal(out[5], torch.zeros_like(out[5])) and torch.isneginf(z[5]).all()


def test_rows_of_no_sequence_give_nothing(lsp):
    pool, t, _ = case([50, 60], [2, 2], 0, nq=2, nkv=1, d=64, dtype="bf16", page=16)
    q = torch.randn(9, 2, 64, device="cuda", dtype=torch.bfloat16)
    c = lsp.make_kv_cache(*pool, *t)
    ws = torch.empty(lsp.lsp_prefix_attention_q4_workspace_bytes(c, q.dtype, 2, 2, 9), dtype=torch.uint8, device="cuda")
    out, z = torch.full_like(q, 7), torch.full((9, 2), 7.0, device="cuda")
    lsp.lsp_prefix_attention_q4(c, 0, q, ints([0, 1]), ints([2, 4, 6]), out, z, shared_len=0, scale=0.1, workspace=ws)
    torch.cuda.synchronize()
    assert not out[[0, 1, 6, 7, 8]].any() and torch.isneginf(z[[0, 1, 6, 7, 8]]).all()
    compare(oracle_cache(*pool, *t), q[2:6], [0, 1], [2, 2], out[2:6], z[2:6], scale=0.1)


@pytest.mark.parametrize("dtype", list(DT))
def test_pages_past_32_bit_offsets(lsp, dtype):
    """The last pages of pools whose pages are 72 MB apart."""
    page, d, nkv, pages, step = 128, 128, 1, 70, 72 << 20
    raw = torch.empty(2 * pages * step, dtype=torch.uint8, device="cuda")
    far = [raw[i * step:].as_strided((1, pages, nkv, page, 72), (step, 2 * step, page * 72, 72, 1)) for i in range(2)]
    near = make_pool(1, 8, nkv, page, d, torch.Generator().manual_seed(3), "cuda")
    for x, y in zip(far, near):
        x[:, -8:] = y
    table = torch.tensor([[pages - 1, pages - 5, pages - 3], [pages - 1, pages - 5, pages - 2]], dtype=torch.int32)
    lens = torch.tensor([300, 270], dtype=torch.int32)
    q = torch.randn(5, 8, d, generator=torch.Generator().manual_seed(4)).to(DT[dtype]).cuda()
    refs = torch.ones(pages, dtype=torch.int32)
    out, z = attend(lsp, far, [x.cuda() for x in (table, lens, refs)], q, [0, 1], [2, 3], 256)
    compare(oracle_cache(*near, table - (pages - 8), lens, refs[:8]), q, [0, 1], [2, 3], out, z)


@pytest.mark.parametrize("dtype", list(DT))
def test_captured_calls_follow_the_lengths_and_take_turns_with_a_workspace(lsp, dtype):
    lens, rows, shared = [300, 280], [2, 2], 256
    pool, t, q = case(lens, rows, shared, nq=8, nkv=2, d=128, dtype=dtype, page=16)
    c = lsp.make_kv_cache(*pool, *t)
    ids, start = ints([0, 1]), ints([0, 2, 4])
    ws = torch.empty(lsp.lsp_prefix_attention_q4_workspace_bytes(c, q.dtype, 8, 2, 4), dtype=torch.uint8, device="cuda")
    calls = []
    for scale in (0.1, 0.05):
        out, z = torch.empty_like(q), torch.empty(4, 8, device="cuda")
        run = lambda: lsp.lsp_prefix_attention_q4(c, 0, q, ids, start, out, z, shared_len=shared, scale=scale, workspace=ws)
        run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        calls.append((graph, out, z, scale))
    for new in ([300, 280], [290, 262], [4, 270]):
        t[1].copy_(torch.tensor(new, dtype=torch.int32))
        for graph, out, z, scale in calls:
            out.fill_(9)
            graph.replay()
        torch.cuda.synchronize()
        for graph, out, z, scale in calls:
            compare(oracle_cache(*pool, *t), q, [0, 1], rows, out, z, scale=scale)


def test_two_calls_at_once_on_streams_of_their_own(lsp):
    made = [case([5000 + 700 * i, 4800], [1, 2 + i], 4096, nq=8, nkv=2, d=128, dtype=dt, page=64, seed=i)
            for i, dt in enumerate(("bf16", "f32"))]
    want = [attend(lsp, pool, t, q, [0, 1], [1, 2 + i], 4096) for i, (pool, t, q) in enumerate(made)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    held = []
    torch.cuda.synchronize()
    for turn in range(20):
        for i, (pool, t, q) in enumerate(made):
            c = lsp.make_kv_cache(*pool, *t)
            if turn == 0:
                ws = torch.empty(lsp.lsp_prefix_attention_q4_workspace_bytes(c, q.dtype, 8, 2, q.shape[0]), dtype=torch.uint8, device="cuda")
                held.append((ints([0, 1]), ints([0, 1, 3 + i]), ws, torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")))
                torch.cuda.synchronize()
            ids, start, ws, out, z = held[i]
            lsp.lsp_prefix_attention_q4(c, 0, q, ids, start, out, z, shared_len=4096, scale=128 ** -0.5, workspace=ws, stream=streams[i])
    torch.cuda.synchronize()
    for (out, z), (_, _, _, o, y) in zip(want, held):
        assert torch.equal(out, o) and torch.equal(z, y)


@pytest.mark.parametrize("dtype", list(DT))
def test_long_context_split_over_the_whole_gpu(lsp, dtype):
    """A few rows over 20K tokens, against fp64 on the GPU."""
    from tests.q4_common import held
    lens, rows, shared = [20500, 20999], [3, 1], 20480
    pool, t, q = case(lens, rows, shared, nq=8, nkv=2, d=128, dtype=dtype, page=64)
    out, z = attend(lsp, pool, t, q, [0, 1], rows, shared)
    kk, vv = (torch.from_numpy(held(x)).cuda().double() for x in pool)
    for b, r0 in ((0, 0), (1, 3)):
        pages = t[0][b, :-(-lens[b] // 64)].long()
        k, v = (x[0, pages].transpose(1, 2).reshape(-1, 2, 128)[:lens[b]] for x in (kk, vv))
        for i in range(rows[b]):
            n = lens[b] - rows[b] + i + 1
            s = torch.einsum("hd,nhd->hn", q[r0 + i].double(), k[:n].repeat_interleave(4, 1)) * 128 ** -0.5
            w = torch.softmax(s, -1)
            want = torch.einsum("hn,nhd->hd", w, v[:n].repeat_interleave(4, 1))
            size = torch.einsum("hn,nhd->hd", w, v[:n].abs().repeat_interleave(4, 1))
            tol = (2 ** -8 + 2 ** -10) * (size + want.abs()) if dtype == "bf16" else 4e-5 * size
            assert ((out[r0 + i].double() - want).abs() <= tol).all()
            assert (z[r0 + i].double() - torch.logsumexp(s, -1)).abs().max() < 2e-5 + 2e-6 * 12


def check_by_sequence(pool, t, q, lens, rows, out, z):
    """Sequence by sequence in fp64, one KV head, nothing shared."""
    from tests.q4_common import held
    kk, vv = (torch.from_numpy(held(x)).cuda() for x in pool)
    d, page, at = q.shape[2], pool[0].shape[3], 0
    tol = (lambda size, want: (2 ** -8 + 2 ** -10) * (size + want.abs())) if q.dtype == torch.bfloat16 else (lambda size, want: 4e-5 * size)
    for b, (n, r) in enumerate(zip(lens, rows)):
        pages = t[0][b, :-(-n // page)].long()
        k, v = (x[0, pages, 0].reshape(-1, d)[:n].double() for x in (kk, vv))
        s = torch.einsum("rhd,nd->rhn", q[at:at + r].double(), k) * d ** -0.5
        seen = torch.arange(n, device="cuda")[None] <= torch.arange(n - r, n, device="cuda")[:, None]
        s = s.masked_fill(~seen[:, None], -torch.inf)
        w = torch.softmax(s, -1)
        want, size = w @ v, w @ v.abs()
        assert bool(((out[at:at + r].double() - want).abs() <= tol(size, want)).all()), b
        lse = torch.logsumexp(s, -1)
        assert bool(((z[at:at + r].double() - lse).abs() <= 2e-5 + 2e-6 * lse.abs()).all()), b
        at += r


# 64 heads on one KV head: a tile of the tensor cores has two tokens, so 1 and 2 rows are one tile, 3 and 4 two
@pytest.mark.parametrize("order", [(4, 1), (3, 2, 1), (4, 4, 1, 1), (1, 4, 1, 3, 9)])
@pytest.mark.parametrize("d,blocks", [(64, 2), (128, 3)])
def test_one_and_two_row_tiles_by_turns(lsp, order, d, blocks):
    n = 400
    rows = [order[i % len(order)] for i in range(n)]
    lens = [128 * (1 + i % blocks) + 7 + 5 * i % 113 for i in range(n)]
    pool, t, q = case(lens, rows, 0, nq=64, nkv=1, d=d, dtype="bf16", page=16)
    seqs = list(range(n))
    out, z = attend(lsp, pool, t, q, seqs, rows, 0)
    check_by_sequence(pool, t, q, lens, rows, out, z)
    for fill in (0, 0x5A):
        again, z2 = attend(lsp, pool, t, q, seqs, rows, 0, fill=fill)
        assert torch.equal(out, again) and torch.equal(z, z2)


@pytest.mark.parametrize("n", [150, 180, 480, 700, 1024])
@pytest.mark.parametrize("dtype", list(DT))
def test_batches_around_what_there_is_room_for(lsp, n, dtype):
    """The schedule of a batch lies in shared memory: more sequences leave room for fewer tiles, or for another kernel."""
    rows = [1 + i % 2 for i in range(n)]
    lens = [20 + 37 * i % 150 for i in range(n)]
    pool, t, q = case(lens, rows, 0, nq=20, nkv=1, d=128, dtype=dtype, page=32)
    out, z = attend(lsp, pool, t, q, list(range(n)), rows, 0)
    check_by_sequence(pool, t, q, lens, rows, out, z)


def test_the_workspace_of_a_call_is_enough_whatever_is_shared(lsp):
    """It is asked for before it is known how much is shared, and the kernel is chosen by that."""
    for n, q in ((1, 1), (3, 1), (16, 1), (40, 1), (4, 9), (2, 300)):
        lens, rows = [2 * 64 + 300 + i for i in range(n)], [q] * n
        pool, t, x = case(lens, rows, 128, nq=8, nkv=2, d=64, dtype="bf16", page=64)
        oc = oracle_cache(*pool, *t)
        for shared in (0, 64, 128):
            out, z = attend(lsp, pool, t, x, list(range(n)), rows, shared)
            compare(oc, x, list(range(n)), rows, out, z)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows", [[2, 1], [40, 35]])
@pytest.mark.parametrize("k_by,v_by", [(60, -120), (-110, 100)])
def test_very_large_and_very_small_values(lsp, rows, k_by, v_by, dtype):
    """Powers of two change no rounding while results are normal numbers: keys times 2^k_by under queries times
    2^-k_by, and values times 2^v_by, give the bits of what they are without them.  Values of 2^-120 give sums below
    2^-126, whose last place is 2^-149: some 300 products and four roundings of a sum lose at most 1200 times half of
    that, 2^-139.  Beside that the output is rounded once more: by half a last place, 2^-134 of a bf16 subnormal, and
    where the lost bits cross a tie by a whole one (2^-8, 2^-23 of it)."""
    lens, shared = [300, 277], 128
    pool, t, q = case(lens, rows, shared, nq=4, nkv=2, d=128, dtype=dtype, page=32, seed=5)
    want, lse = attend(lsp, pool, t, q, [0, 1], rows, shared)
    scaled = []
    for x, by in zip(pool, (k_by, v_by)):
        page, d = x.shape[3], x.shape[4] // 9 * 16
        y = x.clone().flatten(3)
        bits = y[..., page * d // 2:].view(torch.bfloat16)
        bits.copy_((bits.double() * 2.0 ** by).bfloat16())
        scaled.append(y.unflatten(-1, (page, -1)))
    out, z = attend(lsp, scaled, t, (q.double() * 2.0 ** -k_by).to(q.dtype), [0, 1], rows, shared)
    want = want.double() * 2.0 ** v_by
    off = (out.double() - want).abs()
    assert torch.equal(z, lse)
    if v_by > 0:
        assert float(off.max()) == 0
    else:
        step, least = (2 ** -8, 2 ** -134) if dtype == "bf16" else (2 ** -23, 2 ** -150)
        assert bool((off <= step * want.abs() + least + 2 ** -139).all())


@pytest.mark.parametrize("rows,shared,dtype", [(1, 0, "bf16"), (1, 4096, "bf16"), (9, 8192, "bf16"), (3, 2048, "f32")])
def test_the_same_call_gives_the_same_bits(lsp, rows, shared, dtype):
    """Long sequences through the rings of both kernels, call behind call."""
    n = 24
    lens = [shared + rows + 400 * i % 5000 for i in range(n)]
    pool, t, q = case(lens, [rows] * n, shared, nq=32, nkv=8, d=128, dtype=dtype, page=64)
    c = lsp.make_kv_cache(*pool, *t)
    ws = torch.empty(lsp.lsp_prefix_attention_q4_workspace_bytes(c, q.dtype, 32, n, n * rows), dtype=torch.uint8, device="cuda")
    ids, start = ints(range(n)), ints(range(0, n * rows + 1, rows))
    outs = []
    for _ in range(60):
        outs.append((torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")))
        lsp.lsp_prefix_attention_q4(c, 0, q, ids, start, *outs[-1], shared_len=shared, scale=128 ** -0.5, workspace=ws)
    torch.cuda.synchronize()
    for out in outs[1:]:
        assert torch.equal(out[0], outs[0][0]) and torch.equal(out[1], outs[0][1])
