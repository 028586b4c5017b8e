"""lsp_prefix_attention where its distribution of work is at an edge: more shared items than CTAs (some dealt
whole, the rest cut), key ranges of several units cut in the middle, and so much work that places on the line of
what is cut take more than 32-bit arithmetic.

Tolerances: those of the other tests of this call, and for sums over some 2^11 key blocks in turn 8 sqrt(2^11)
2^-24 = 2e-5 of sum_j w_j |v_j| more (fp32 rounding errors of either sign).
"""
import pytest
import torch

from tests.gpu_common import lsp_lib
from tests.target_common import DT, make_cache, make_pool, oracle_cache
from tests.test_gpu_prefix_attn import attend, case, compare

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


CASES = {
    "more items than CTAs": dict(lens=[434 + 3 * i for i in range(40)], rows=[33] * 40, shared=400, nq=32, nkv=4, d=64, page=16),
    "more items than CTAs, d 128": dict(lens=[300 + 5 * i for i in range(24)], rows=[20 + i for i in range(24)], shared=256, nq=32, nkv=8, d=128, page=64),
    "ranges of several units": dict(lens=[2100 + 40 * i for i in range(12)], rows=[30 + i for i in range(12)], shared=2050, nq=8, nkv=2, d=128, page=32),
    "a last unit of one tile": dict(lens=[1500 + i for i in range(9)], rows=[15] * 9, shared=1400, nq=16, nkv=2, d=64, page=128),
}


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("name", list(CASES))
def test_dealt_and_cut_items(lsp, name, dtype):
    kw = dict(CASES[name], dtype=dtype)
    pool, t, q = case(**kw)
    out, z = attend(lsp, pool, t, q, list(range(len(kw["lens"]))), kw["rows"], kw["shared"])
    compare(oracle_cache(*pool, *t), q, list(range(len(kw["lens"]))), kw["rows"], out, z)
    again, z2 = attend(lsp, pool, t, q, list(range(len(kw["lens"]))), kw["rows"], kw["shared"], fill=0)
    assert torch.equal(out, again) and torch.equal(z, z2)


# rows and keys so that every shared item is on the line, and the line is longer than 2^21
@pytest.mark.parametrize("dtype,rows,shared", [("bf16", [900, 1500], 460800), ("f32", [1200, 1100], 131072)])
def test_a_line_beyond_32_bit_products(lsp, dtype, rows, shared):
    page, nkv, rep, d = 256, 8, 2 if dtype == "bf16" else 1, 64
    lens = [shared + r + 300 for r in rows]
    g = torch.Generator(device="cuda").manual_seed(3)
    need = shared // page + sum(-(-(n - shared) // page) for n in lens)
    k, v = torch.randn(2, 1, need, nkv, page, d, generator=g, device="cuda").to(DT[dtype])
    t = [x.cuda() for x in make_cache(lens, shared, page, (k, v))]
    q = (torch.randn(sum(rows), nkv * rep, d, generator=g, device="cuda") * 1.5).to(DT[dtype])
    out, z = attend(lsp, (k, v), t, q, [0, 1], rows, shared)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(z).all())
    at = [0, 1, 127, 128, 500, rows[0] - 1, rows[0], rows[0] + 513, sum(rows) - 130, sum(rows) - 1]
    for i, row in enumerate(at):
        b = int(row >= rows[0])
        n = lens[b] - rows[b] + (row - b * rows[0]) + 1
        pages = t[0][b, :-(-n // page)].long()
        for h in {(3 * i) % (nkv * rep), nkv * rep - 1}:
            kk, vv = (x[0, pages, h // rep].reshape(-1, d)[:n].double() for x in (k, v))
            s = kk @ q[row, h].double() * d ** -0.5
            w = torch.softmax(s, 0)
            want, size, lse = w @ vv, w @ vv.abs(), float(torch.logsumexp(s, 0))
            tol = (2 ** -8 + 2 ** -10) * (size + want.abs()) if dtype == "bf16" else (4e-5 + 2e-5) * size
            assert bool(((out[row, h].double() - want).abs() <= tol).all()), (row, h)
            assert abs(float(z[row, h]) - lse) <= 2e-5 + 2e-6 * abs(lse)


@pytest.mark.parametrize("dtype", list(DT))
def test_rows_of_no_sequence_beside_a_shared_prefix(lsp, dtype):
    """They are stacked with the others against the shared pages, and give 0 all the same; so does an entry
    outside the cache, and the others are not disturbed."""
    lens, rows, shared = [310, 333, 340], [5, 9, 17], 300
    pool, t, _ = case(lens, rows, shared, nq=4, nkv=2, d=64, dtype=dtype, page=16)
    total, before = 44, 6
    q = torch.randn(total, 4, 64, device="cuda").to(DT[dtype])
    c = lsp.make_kv_cache(*pool, *t)
    start = torch.tensor([6, 11, 20, 37, 40], dtype=torch.int32, device="cuda")
    ids = torch.tensor([0, 1, 2, 99], dtype=torch.int32, device="cuda")      # the last one does not exist
    ws = torch.empty(lsp.lsp_prefix_attention_workspace_bytes(c, 4, 4, total), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out, z = torch.full_like(q, 7), torch.full((total, 4), 7.0, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    lsp.lsp_prefix_attention(c, 0, q, ids, start, out, z, shared_len=shared, scale=0.125, workspace=ws, dev_error=err)
    torch.cuda.synchronize()
    assert int(err) == lsp.LSP_DEV_BAD_SEQ
    none = list(range(before)) + list(range(37, total))
    assert not out[none].any() and torch.isneginf(z[none]).all()
    compare(oracle_cache(*pool, *t), q[6:37], [0, 1, 2], rows, out[6:37], z[6:37], scale=0.125)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rise", [20.0, 45.0, 300.0, 5000.0])
@pytest.mark.parametrize("spots", [(130,), (200,), (140, 220, 400), (1, 300, 390, 511, 640, 1000)])
def test_maxima_that_rise_late(lsp, dtype, rise, spots):
    """Scores that jump by `rise` at each of `spots`, in either half of a key block, for some of the rows: weights
    relative to the maximum so far would pass every range."""
    n, d = 1100, 64
    pool, t, q = case([n, n], [3, 2], 1024, nq=4, nkv=2, d=d, dtype=dtype, page=64, seed=11)
    k = pool[0]
    q[:, :, 0] = torch.tensor([4.0, 0.0, 2.0, 0.5], device="cuda").to(q.dtype)       # which heads see the jumps, and how
    k[..., 0] = 0
    for i, pos in enumerate(spots):
        pages, slot = t[0][:, pos // 64].long(), pos % 64
        for pg in pages.tolist():
            k[0, pg, :, slot, 0] = (i + 1) * rise * 2                                # head 0: (i + 1) rise at scale 1 / 8
    out, z = attend(lsp, pool, t, q, [0, 1], [3, 2], 1024)
    compare(oracle_cache(*pool, *t), q, [0, 1], [3, 2], out, z)
