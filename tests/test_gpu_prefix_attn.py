"""lsp_prefix_attention against the oracle's fp64 attention over the same pages.

Tolerances, from the arithmetic: bf16 rounds the weights (relative error at most 2^-8 each) and the
output (2^-8 of it), so an output is within 2^-8 (sum_j w_j |v_j| + |o|), plus 2^-10 of the same size
for the fp32 sums, the exponential's 2^-22 and the joining of segments.  f32: the scores' fp32 dot
products of up to 128 terms of |score| < 20 move a weight by at most about 1e-5; 4e-5 of sum_j w_j
|v_j|.  lse is fp32 in both: 2e-5 + 2e-6 |lse|.
"""
import numpy as np
import pytest
import torch

from oracle.target import cache_attention
from tests.gpu_common import lsp_lib
from tests.target_common import DT, make_cache, make_pool, oracle_cache, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


def attend(lsp, pool, t, q, seqs, rows, shared, layer=0, scale=None, lse=True, stream=None, bits=0, fill=0xFF):
    """-> (out, lse) of one call; the workspace starts as NaN patterns."""
    c = lsp.make_kv_cache(*pool, *t)
    start = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32, device="cuda")
    ids = torch.tensor(seqs, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(256, lsp.lsp_prefix_attention_workspace_bytes(c, q.shape[1], len(seqs), q.shape[0])),
                     dtype=torch.uint8, device="cuda").fill_(fill)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    z = torch.full(q.shape[:2], float("nan"), device="cuda") if lse else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    lsp.lsp_prefix_attention(c, layer, q, ids, start, out, z, shared_len=shared, scale=scale or q.shape[2] ** -0.5,
                             workspace=ws, dev_error=err, stream=stream)
    torch.cuda.synchronize()
    assert int(err.item()) == bits
    return out, z


def compare(oc, q, seqs, rows, out, z, layer=0, scale=None):
    start = np.concatenate([[0], np.cumsum(rows)]).astype(int)
    want, lse, size = cache_attention(oc, layer, up(q), seqs, start, scale or q.shape[2] ** -0.5)
    got = out.double().cpu().numpy()
    tol = ((2 ** -8 + 2 ** -10) * (size + np.abs(want)) if q.dtype == torch.bfloat16 else 4e-5 * size) + 1e-30
    assert np.isfinite(got).all()
    worst = np.max(np.abs(got - want) / tol)
    assert worst <= 1, worst
    if z is not None:
        zg = z.double().cpu().numpy()
        assert np.array_equal(np.isneginf(zg), np.isneginf(lse))
        f = np.isfinite(lse)
        assert (np.abs(zg[f] - lse[f]) <= 2e-5 + 2e-6 * np.abs(lse[f])).all()


def case(lens, rows, shared, *, nq, nkv, d, dtype, page, layers=1, order="dense", seed=0, extra=3, spare=2):
    g = torch.Generator().manual_seed(seed)
    need = shared // page + sum(-(-n // page) - min(-(-n // page), shared // page) for n in lens)
    pool = make_pool(layers, need + extra, nkv, page, d, dtype, g, order, "cuda")
    t = make_cache(lens, shared, page, pool, spare=spare, seed=seed)
    q = (torch.randn(sum(rows), nq, d, generator=g) * 1.5).to(DT[dtype]).cuda()
    return pool, [x.cuda() for x in t], q


CASES = {
    # one token a sequence, from one token of context on
    "step": dict(lens=[301, 340, 305], rows=[1, 1, 1], shared=300, nq=8, nkv=2, d=128, page=16),
    "one token": dict(lens=[1], rows=[1], shared=0, nq=2, nkv=2, d=128, page=16),
    "one request": dict(lens=[1000], rows=[3], shared=997, nq=4, nkv=1, d=64, page=64),
    # nothing shared; lengths around a page's and a block's end
    "own only": dict(lens=[1, 15, 16, 17, 64, 65, 127, 128, 129, 400], rows=[1, 2, 16, 1, 5, 4, 3, 2, 1, 7], shared=0, nq=6, nkv=2, d=128, page=16),
    # a shared part that ends inside a page, of one block, of one page
    "ragged block": dict(lens=[300, 290, 333, 289], rows=[9, 1, 17, 3], shared=283, nq=10, nkv=2, d=128, page=32),
    "one shared block": dict(lens=[130, 131, 150], rows=[2, 3, 17], shared=128, nq=8, nkv=1, d=128, page=128),
    "one shared page": dict(lens=[20, 31], rows=[4, 5], shared=19, nq=3, nkv=3, d=64, page=16),
    # more rows than a tile and than a unit, for the shared part and in one sequence
    "many rows": dict(lens=[700, 650, 620, 800], rows=[90, 40, 20, 180], shared=515, nq=4, nkv=1, d=128, page=64),
    "a long chunk": dict(lens=[600], rows=[600], shared=0, nq=2, nkv=1, d=64, page=32),
    # rows before the end of the shared tokens: they are read as each sequence's own
    "rows inside the shared part": dict(lens=[256, 300], rows=[100, 3], shared=256, nq=4, nkv=2, d=128, page=16),
    # sequences without rows, without tokens, and shorter than their rows
    "empty ones": dict(lens=[0, 40, 5, 33, 0], rows=[0, 0, 9, 2, 3], shared=0, nq=4, nkv=2, d=128, page=16),
    "heads not of eight": dict(lens=[270, 290], rows=[17, 11], shared=256, nq=35, nkv=5, d=128, page=256),
    "many heads a key head": dict(lens=[270, 290, 300], rows=[3, 1, 2], shared=260, nq=64, nkv=1, d=64, page=16),
    # several segments of one to four key blocks for every CTA, shared ones of one and two row tiles among them
    "more segments than CTAs": dict(lens=[270 + 7 * i % 391 for i in range(90)], rows=[1 + i % 2 for i in range(90)], shared=260, nq=8, nkv=8, d=64, page=16),
    "uneven segments": dict(lens=[150 + 131 * i % 700 for i in range(60)], rows=[1 + 7 * i % 21 for i in range(60)], shared=140, nq=16, nkv=4, d=128, page=32),
    "many sequences": dict(lens=[120 + i for i in range(70)], rows=[i % 3 for i in range(70)], shared=112, nq=2, nkv=1, d=64, page=16),
}


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("name", list(CASES))
def test_equals_the_oracle(lsp, name, dtype):
    kw = dict(CASES[name], dtype=dtype)
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
    pool, t, _ = case(lens, rows, shared, nq=4, nkv=2, d=64, dtype=dtype, page=16, layers=3, order="tokens")
    g = torch.Generator().manual_seed(5)
    fused = torch.randn(sum(rows), 8, 64, generator=g).to(DT[dtype]).cuda()
    q = fused[:, 2:6]                                # a slice of a q/k/v row
    seqs = [2, 0, 3, 1]
    oc = oracle_cache(*pool, *t)
    for layer, stream in ((2, None), (0, torch.cuda.Stream())):
        out, _ = attend(lsp, pool, t, q, seqs, rows, shared, layer=layer, scale=0.2, lse=False, stream=stream)
        compare(oc, q, seqs, rows, out, None, layer=layer, scale=0.2)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("page", [16, 128])
def test_what_lies_in_unused_places_is_never_seen(lsp, page, dtype):
    lens, rows, shared = [page * 3 + 5, page * 4 + 1, 7], [4, 1, 2], 0
    kw = dict(nq=8, nkv=2, d=128, dtype=dtype, page=page)
    pool, t, q = case(lens, rows, shared, **kw)
    seqs = [0, 1, 2]
    oc = oracle_cache(*pool, *t)
    used = torch.zeros(pool[0].shape[1], page, dtype=torch.bool)
    for s, n in enumerate(lens):
        for i in range(n):
            used[t[0][s, i // page], i % page] = True
    bad = torch.tensor([float("nan"), float("inf"), float("-inf"), 3e38]).to(DT[dtype])
    junk = bad[torch.randint(0, 4, pool[0].shape, generator=torch.Generator().manual_seed(1))].cuda()
    free = ~used.cuda()[None, :, None, :, None]
    for x in pool:
        x.copy_(torch.where(free, junk, x))
    out, z = attend(lsp, pool, t, q, seqs, rows, shared)
    compare(oc, q, seqs, rows, out, z)


@pytest.mark.parametrize("dtype", list(DT))
def test_large_scores_and_a_key_that_takes_all_the_weight(lsp, dtype):
    lens, rows, shared = [400, 390], [5, 3], 384
    pool, t, q = case(lens, rows, shared, nq=4, nkv=2, d=128, dtype=dtype, page=16)
    k = pool[0]
    k[0, t[0][0, 3].item(), :, 5] = q[0, ::2] * 4   # scores of several hundred, late in the first block's pages
    k[0, t[0][0, 20].item(), :, 1] = q[1, ::2] * 6  # and a larger one in a later block
    oc = oracle_cache(*pool, *t)
    want, lse, _ = cache_attention(oc, 0, up(q), [0, 1], [0, 5, 8], 128 ** -0.5)
    out, z = attend(lsp, pool, t, q, [0, 1], rows, shared)
    # scores near 1e3: their fp32 error (about 2^-23 of the sum of |terms|) moves a weight by up to 1e-3
    np.testing.assert_allclose(out.double().cpu().numpy(), want, rtol=0, atol=2 ** -7 * np.abs(want).max() + 4e-3)
    np.testing.assert_allclose(z.cpu().numpy(), lse, rtol=1e-6, atol=1e-3)


@pytest.mark.parametrize("dtype", list(DT))
def test_entries_outside_the_cache_are_reported(lsp, dtype):
    lens, rows = [50, 60, 40], [2, 3, 1]
    pool, t, q = case(lens, rows, 0, nq=4, nkv=2, d=64, dtype=dtype, page=16)
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
    ids, start = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 1], [2, 4, 6]))
    ws = torch.empty(lsp.lsp_prefix_attention_workspace_bytes(c, 2, 2, 9), dtype=torch.uint8, device="cuda")
    out, z = torch.full_like(q, 7), torch.full((9, 2), 7.0, device="cuda")
    lsp.lsp_prefix_attention(c, 0, q, ids, start, out, z, shared_len=0, scale=0.1, workspace=ws)
    torch.cuda.synchronize()
    assert not out[[0, 1, 6, 7, 8]].any() and torch.isneginf(z[[0, 1, 6, 7, 8]]).all()
    compare(oracle_cache(*pool, *t), q[2:6], [0, 1], [2, 2], out[2:6], z[2:6], scale=0.1)


@pytest.mark.parametrize("dtype", list(DT))
def test_pages_past_32_bit_offsets(lsp, dtype):
    es = 2 if dtype == "bf16" else 4
    page, d, nkv = 128, 128, 4
    pages = 2 ** 32 // (page * d * nkv * es) + 9
    k = torch.zeros(1, pages, nkv, page, d, dtype=DT[dtype], device="cuda")
    v = torch.zeros_like(k)
    g = torch.Generator().manual_seed(3)
    for x in (k, v):
        x[0, -8:] = torch.randn(8, nkv, page, d, generator=g).to(DT[dtype]).cuda()
    table = torch.tensor([[pages - 1, pages - 5, pages - 3], [pages - 1, pages - 5, pages - 2]], dtype=torch.int32)
    lens = torch.tensor([300, 270], dtype=torch.int32)
    q = torch.randn(5, 8, d, generator=g).to(DT[dtype]).cuda()
    refs = torch.ones(pages, dtype=torch.int32)
    t = [x.cuda() for x in (table, lens, refs)]
    out, z = attend(lsp, (k, v), t, q, [0, 1], [2, 3], 256)
    near = table - (pages - 8)
    oc = oracle_cache(k[:, -8:], v[:, -8:], near, lens, refs[:8])
    compare(oc, q, [0, 1], [2, 3], out, z)


def test_a_captured_call_follows_the_lengths(lsp):
    """Lengths and tables are read on the device: a captured call sees the cache as it is at replay."""
    lens, rows, shared = [300, 280], [2, 2], 256
    pool, t, q = case(lens, rows, shared, nq=8, nkv=2, d=128, dtype="bf16", page=16)
    c = lsp.make_kv_cache(*pool, *t)
    ids, start = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 1], [0, 2, 4]))
    ws = torch.empty(lsp.lsp_prefix_attention_workspace_bytes(c, 8, 2, 4), dtype=torch.uint8, device="cuda")
    out, z = torch.empty_like(q), torch.empty(4, 8, device="cuda")
    call = lambda: lsp.lsp_prefix_attention(c, 0, q, ids, start, out, z, shared_len=shared, scale=0.1, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for new in ([300, 280], [290, 262], [4, 270]):
        t[1].copy_(torch.tensor(new, dtype=torch.int32))
        out.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        compare(oracle_cache(*pool, *t), q, [0, 1], rows, out, z, scale=0.1)


def test_long_context_split_over_the_whole_gpu(lsp):
    """A few rows over 20K tokens, against fp64 on the GPU."""
    lens, rows, shared = [20500, 20999], [3, 1], 20480
    pool, t, q = case(lens, rows, shared, nq=8, nkv=2, d=128, dtype="bf16", page=64)
    out, z = attend(lsp, pool, t, q, [0, 1], rows, shared)
    for b, r0 in ((0, 0), (1, 3)):
        pages = t[0][b, :-(-lens[b] // 64)].long()
        k, v = (x[0, pages].transpose(1, 2).reshape(-1, 2, 128)[:lens[b]].double() for x in pool)
        for i in range(rows[b]):
            n = lens[b] - rows[b] + i + 1
            s = torch.einsum("hd,nhd->hn", q[r0 + i].double(), k[:n].repeat_interleave(4, 1)) * 128 ** -0.5
            w = torch.softmax(s, -1)
            want = torch.einsum("hn,nhd->hd", w, v[:n].repeat_interleave(4, 1))
            size = torch.einsum("hn,nhd->hd", w, v[:n].abs().repeat_interleave(4, 1))
            assert ((out[r0 + i].double() - want).abs() <= (2 ** -8 + 2 ** -10) * (size + want.abs())).all()
            assert (z[r0 + i].double() - torch.logsumexp(s, -1)).abs().max() < 2e-5 + 2e-6 * 12
