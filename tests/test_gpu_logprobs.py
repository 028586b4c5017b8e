"""lsp_logprobs against the oracle in fp64.

Tolerances, from the arithmetic (x = z / T, ulp(a) at most 2^-23 |a|).  lse = m / T + ln S: every weight 2^t has t
rounded once after a difference and a product (2^-23 |t| in all) and the exponential's 2^-22, so S is off by at most
2^-22 + 2^-23 ln-weighted |t| (the entropy's size, below 2^-22 H / ln 2), fp32 sums of some 100 terms a thread and
joins of a few levels add 2^-17 at the worst: ln S is within 1e-5 + 1e-6 H.  A log probability adds the rounding of
its own difference and quotient, 2^-22 |logprob|.  The entropy is ln S - A / S of such sums: 2e-5 (1 + H).  Tokens and
their order are compared for equality.
"""
import numpy as np
import pytest
import torch

from oracle import cache_q4
from tests.gpu_common import lsp_lib
from tests.target_common import DT, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


def ints(x):
    return torch.tensor([int(i) for i in x], dtype=torch.int32, device="cuda")


def call(lsp, z, tokens, k, temperature=1.0, bits=0, stream=None):
    rows = z.shape[0]
    out = [torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda"),
           torch.full((rows, k), 7, dtype=torch.int32, device="cuda"), torch.full((rows, k), 7.0, device="cuda")]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    lsp.lsp_logprobs(z, tokens, *out, temperature=temperature, dev_error=err, stream=stream)
    torch.cuda.synchronize()
    assert int(err.item()) == bits
    return out


def check(z, tokens, k, temperature, out):
    lp, h, top, tl = cache_q4.logprobs(up(z), tokens.tolist(), temperature, k)
    got = [x.double().cpu().numpy() for x in out]
    for a, b in zip((got[0], got[1], got[3]), (lp, h, tl)):
        assert np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(np.isneginf(a), np.isneginf(b))
    np.testing.assert_array_equal(got[2], top)
    got = [np.where(np.isfinite(x), x, 0) for x in got]          # (where they are not finite they are alike)
    lp, tl, f = np.where(np.isfinite(lp), lp, 0), np.where(np.isfinite(tl), tl, 0), np.isfinite(lp)
    size = np.where(np.isfinite(h), h, 0)
    assert (np.abs(got[0] - lp)[f] <= (1e-5 + 1e-6 * size + 2 ** -22 * np.abs(lp))[f]).all(), np.abs(got[0] - lp)[f].max()
    h, f = np.where(np.isfinite(h), h, 0), np.isfinite(h)
    assert (np.abs(got[1] - h)[f] <= (2e-5 * (1 + size))[f]).all(), np.abs(got[1] - h)[f].max()
    assert (np.abs(got[3] - tl) <= 1e-5 + 1e-6 * size[:, None] + 2 ** -22 * np.abs(tl)).all()


def logits(rows, V, dtype, seed, spread=2.5, banned=0.001):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, V, generator=g) * spread
    x[torch.rand(x.shape, generator=g) < banned] = -float("inf")
    return x.to(DT[dtype])


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,V,k,T", [(1, 1, 1, 1.0), (3, 2, 2, 0.7), (2, 7, 5, 1.0), (5, 33, 32, 2.0), (4, 1000, 20, 1.0),
                                        (7, 4097, 32, 0.5), (2, 32001, 5, 1.0), (40, 20011, 1, 1.0), (700, 5003, 8, 1.3),
                                        (1300, 1003, 3, 1.0), (3, 151936, 20, 1.0), (1, 600001, 32, 1.0), (6, 9000, 0, 1.0)])
def test_equals_the_oracle(lsp, rows, V, k, T, dtype):
    z = logits(rows, V, dtype, V + rows)
    tokens = torch.randint(0, V, (rows,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    tokens[torch.arange(rows) % 4 == 3] = -1
    z, tokens = z.cuda(), tokens.cuda()
    out = call(lsp, z, tokens, k, T)
    check(z, tokens, k, T, out)
    again = call(lsp, z, tokens, k, T)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("by", range(8))
def test_rows_that_start_and_end_anywhere(lsp, by, dtype):
    V, rows, k = 2100 + by, 3, 6
    g = torch.Generator().manual_seed(by)
    wide = (torch.randn(rows * (V + 13) + 20, generator=g) * 3).to(DT[dtype]).cuda()
    z = wide[by:].as_strided((rows, V), (V + 13, 1))
    z[:, 0] = 30.0                                   # the first and the last element are among the largest
    z[:, V - 1] = 29.0
    tokens = ints([0, V - 1, 5])
    out = call(lsp, z, tokens, k)
    check(z, tokens, k, 1.0, out)
    assert out[2][:, :2].tolist() == [[0, V - 1]] * rows


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("k", [1, 7, 32])
def test_equal_logits_go_by_their_index(lsp, k, dtype):
    V = 30000
    g = torch.Generator().manual_seed(k)
    z = torch.stack([torch.zeros(V), torch.full((V,), -5.0), torch.randint(-2, 3, (V,), generator=g).float(),
                     torch.randint(0, 2000, (V,), generator=g).float() / 100, (torch.arange(V) // 7).float() / 1000,
                     -(torch.arange(V) // 9).float() / 1000,
                     torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)]).to(DT[dtype]).cuda()
    tokens = ints([0, V - 1, 5, 6, 7, 8, 9])
    check(z, tokens, k, 1.0, call(lsp, z, tokens, k))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("k", [1, 5, 32])
def test_large_logits_crowded_into_few_places(lsp, k, dtype):
    """Rising and falling rows, and rows whose large elements all lie in the same places of every 4096 (or 8192)
    elements, far more of them than a list of candidates holds."""
    V = 151936
    ramp = torch.arange(V) / V * 20
    rows = [ramp, -ramp]
    for period in (2048, 4096):
        x = torch.zeros(V)
        few = (torch.arange(V) % period) < 32 * (4 if dtype == "f32" else 8)
        x[few] = 3 + ramp[few]
        rows += [x, x.flip(0)]
    z = torch.stack(rows).to(DT[dtype]).cuda()
    tokens = ints(range(len(rows)))
    check(z, tokens, k, 1.0, call(lsp, z, tokens, k))


@pytest.mark.parametrize("dtype", list(DT))
def test_rows_of_few_finite_logits_and_of_none(lsp, dtype):
    V, inf, nan = 5003, float("inf"), float("nan")
    z = torch.full((9, V), -inf)
    z[0, 17] = 2.0                                   # one possible token
    z[1, 4000], z[1, 3] = -1e30, -2e30
    z[3, 5], z[3, 6] = inf, 1.0
    z[4, 2000] = nan
    z[5] = torch.randn(V, generator=torch.Generator().manual_seed(0))
    z[5, 4999] = nan
    z[6] = 1e30
    z[6, 9] = 3e38
    z[7] = -3e38
    z[8, :3] = torch.tensor([1.0, 2.0, 3.0])
    z = z.to(DT[dtype]).cuda()
    tokens = ints([17, 3, 0, 6, 1, 2, 9, 8, 4])
    for k in (3, 32):
        check(z, tokens, k, 1.0, call(lsp, z, tokens, k))


@pytest.mark.parametrize("T", [1e-30, 1e-3, 1e3, 1e30])
def test_extreme_temperatures(lsp, T):
    z = logits(3, 3001, "f32", 5).cuda()
    tokens = z.argmax(-1).to(torch.int32)
    check(z, tokens, 4, T, call(lsp, z, tokens, 4, T))


def test_tokens_outside_the_vocabulary_and_missing_results(lsp):
    V = 1001
    z = logits(6, V, "f32", 9).cuda()
    tokens = ints([0, V, -1, -2, 1000, 2 ** 31 - 1])
    out = call(lsp, z, tokens, 4, bits=lsp.LSP_DEV_BAD_TOKEN)
    check(z, tokens, 4, 1.0, out)
    lp, top = torch.zeros(6, device="cuda"), torch.zeros(6, 4, dtype=torch.int32, device="cuda")
    lsp.lsp_logprobs(z, tokens, lp)
    assert torch.equal(lp, out[0])
    lsp.lsp_logprobs(z, tokens, lp, None, top)
    assert torch.equal(top, out[2])
    tl = torch.zeros(6, 4, device="cuda")
    lsp.lsp_logprobs(z, tokens, lp, None, None, tl)
    assert torch.equal(tl, out[3])
    lsp.lsp_logprobs(z[:0], tokens[:0], lp[:0])


def test_a_row_does_not_depend_on_the_others(lsp):
    """A call of few rows splits each over more CTAs than one of many; tokens agree, numbers to their tolerance."""
    z = logits(300, 32000, "bf16", 2).cuda()
    tokens = ints(range(300))
    many, one = call(lsp, z, tokens, 20), call(lsp, z[:1], tokens[:1], 20)
    assert torch.equal(many[2][:1], one[2])
    check(z[:1], tokens[:1], 20, 1.0, [x[:1] for x in many])
    check(z[:1], tokens[:1], 20, 1.0, one)


@pytest.mark.parametrize("rows,V,k", [(70001, 7, 3), (9000, 40, 32), (3000, 600, 5)])
def test_many_short_rows(lsp, rows, V, k):
    """A cluster goes through hundreds of rows, some without a token, in any run of 32."""
    g = torch.Generator().manual_seed(rows)
    z = (torch.randn(rows, V, generator=g) * 3).cuda()
    tokens = torch.randint(0, V, (rows,), generator=g, dtype=torch.int32)
    tokens[torch.rand(rows, generator=g) < 0.3] = -1
    tokens[5000:5500] = -1
    tokens = tokens.cuda()
    out = call(lsp, z, tokens, k)
    live = tokens >= 0
    lp = torch.log_softmax(z.double(), -1)
    want = lp.gather(1, tokens.clamp(min=0).long()[:, None])[:, 0]
    assert bool((out[0][~live] == -torch.inf).all()) and bool((out[1][~live] == 0).all())
    assert bool((out[2][~live] == -1).all()) and bool((out[3][~live] == -torch.inf).all())
    assert float((out[0].double() - want)[live].abs().max()) <= 3e-5
    assert float((out[1].double() + (lp.exp() * lp).sum(-1))[live].abs().max()) <= 2e-4
    order = torch.sort(z, descending=True, stable=True).indices[:, :k]
    assert torch.equal(out[2][live], order[live].int())
    assert float((out[3].double() - lp.gather(1, order))[live].abs().max()) <= 3e-5


@pytest.mark.parametrize("rows,V,dtype", [(272, 151936, "f32"), (700, 151936, "bf16"), (40, 300007, "f32")])
def test_the_same_call_gives_the_same_bits(lsp, rows, V, dtype):
    """Long rows through the ring, call behind call: no piece is lost to the copy that follows it, or taken twice."""
    z = torch.randn(rows, V, device="cuda", generator=torch.Generator("cuda").manual_seed(V)).mul_(2.5).to(DT[dtype])
    tokens = ints(range(rows))
    outs = []
    for _ in range(100):
        outs.append([torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, 5, dtype=torch.int32, device="cuda"),
                     torch.empty(rows, 5, device="cuda")])
        lsp.lsp_logprobs(z, tokens, *outs[-1])
    torch.cuda.synchronize()
    for out in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], out))
    for at in range(0, rows, 50):
        lp = torch.log_softmax(z[at:at + 50].double(), -1)
        want = lp.gather(1, tokens[at:at + 50].long()[:, None])[:, 0]
        assert float((outs[0][0][at:at + 50].double() - want).abs().max()) <= 3e-5


def test_streams_and_graphs(lsp):
    z, tokens = logits(20, 40001, "f32", 3).cuda(), ints(range(20))
    want = call(lsp, z, tokens, 6)
    side = torch.cuda.Stream()
    got = call(lsp, z, tokens, 6, stream=side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    out = [torch.empty_like(x) for x in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lsp.lsp_logprobs(z, tokens, *out)
    for seed in range(2):
        z.copy_(logits(20, 40001, "f32", 30 + seed))
        tokens.copy_(ints([-1 if i % 3 == seed else 100 * i for i in range(20)]))
        graph.replay()
        torch.cuda.synchronize()
        check(z, tokens, 6, 1.0, out)
