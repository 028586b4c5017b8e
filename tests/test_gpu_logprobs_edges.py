"""lsp_logprobs where its arithmetic has least room: near-certain tokens, logits at the limit of its faster steps,
filtered rows, rows at any address.  Tolerances: test_gpu_logprobs.py's."""
import numpy as np
import pytest
import torch

from tests.gpu_common import lsp_lib
from tests.target_common import DT
from tests.test_gpu_logprobs import call, check, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [33, 5003, 151936])
def test_log_probabilities_are_never_positive(lsp, V, dtype):
    """One logit holds nearly all of the probability: its log probability is 0 or just below."""
    rows = 300
    g = torch.Generator().manual_seed(V)
    z = torch.randn(rows, V, generator=g)
    at = torch.randint(0, V, (rows,), generator=g)
    z[torch.arange(rows), at] = 20 + 20 * torch.rand(rows, generator=g)
    z[::3] += 100 * torch.randn(len(z[::3]), 1, generator=g)
    z, tokens = z.to(DT[dtype]).cuda(), at.int().cuda()
    for T in (1.0, 0.7, 0.01):
        out = call(lsp, z, tokens, 2, T)
        assert float(out[0].max()) <= 0 and float(out[3].max()) <= 0
        check(z[:40], tokens[:40], 2, T, [x[:40] for x in out])
    z[:, :], z[:, 5] = -float("inf"), 3.0            # the only token
    out = call(lsp, z, ints([5] * rows), 2)
    assert not out[0].any() and not out[1].any() and not out[3][:, 0].any()


def frames(by):
    """Rows whose threads meet a plateau first and a larger logit in their last piece, both next to +-1e6 / c,
    c = log2(e) / T: up to there t = z c - ref, beyond it t = (z - m) c."""
    V, limit = 131072, 1e6 * np.log(2)
    z = np.zeros((24, V), np.float32)
    for r in range(24):
        low = by * limit - 6.0 + 0.0625 * 5 * r if by > 0 else by * limit - 7.0 + 0.0625 * 5 * r
        z[r] = low
        z[r].reshape(8, -1)[:, -2048::16] = np.float32(low) + np.float32(6.25)
    return torch.from_numpy(z).cuda()


@pytest.mark.parametrize("by", [1, -1])
def test_logits_on_both_sides_of_the_limit_of_the_fast_steps(lsp, by):
    z = frames(by)
    tokens = ints([0, 131071 - 15] * 12)
    check(z, tokens, 3, 1.0, call(lsp, z, tokens, 3))
    # (the same x, everything by a power of two)
    check(z / 1024, tokens, 3, 2.0 ** -10, call(lsp, z / 1024, tokens, 3, 2.0 ** -10))


def filtered(rows, V, dtype, finite, seed, lowest=False):
    """All but `finite` logits of a row are the type's way of saying never."""
    g = torch.Generator().manual_seed(seed)
    z = torch.full((rows, V), float(torch.finfo(DT[dtype]).min) if lowest else -float("inf"))
    for r in range(rows):
        at = torch.randperm(V, generator=g)[:finite]
        z[r, at] = torch.randn(finite, generator=g) * 3
    return z.to(DT[dtype])


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("lowest", [False, True])
@pytest.mark.parametrize("rows,V,finite,k", [(3, 151936, 50, 20), (3, 151936, 5, 32), (2, 151937, 1, 32), (3, 20011, 31, 32),
                                             (3, 2047, 3, 32), (400, 9001, 20, 20), (2, 33, 2, 32), (4, 600001, 900, 32)])
def test_filtered_rows(lsp, rows, V, finite, k, lowest, dtype):
    z = filtered(rows, V, dtype, finite, V + k, lowest).cuda()
    tokens = z.argmax(-1).int()
    check(z, tokens, k, 1.0, call(lsp, z, tokens, k))


@pytest.mark.parametrize("dtype", list(DT))
def test_ties_at_the_cut_in_the_head_the_tail_and_far_apart(lsp, dtype):
    """More equal logits than a list of them holds, with larger ones among them, in rows that start at any address."""
    V, k = 40013, 32
    for by in range(4):
        wide = torch.full((by + 5 * (V + 3),), -7.0)
        z = wide[by:].as_strided((5, V), (V + 3, 1))
        z[1, -300:] = 2.0                            # the ties are at the end
        z[1, 0] = 2.0
        z[2, 5::7] = 1.5                             # everywhere
        z[2, 3], z[2, V - 1] = 1.75, 9.0
        z[3, 1000:30000] = 4.0                       # in one stretch, with some larger ones
        z[3, 1500:1520] = 5.0
        z[4, ::2] = 1.0                              # larger ones in more places than alternatives
        z[4, 100:30000:311] = 2.0
        wide = wide.to(DT[dtype]).cuda()
        z = wide[by:].as_strided((5, V), (V + 3, 1))
        tokens = ints([0, V - 1, 3, 1500, 100])
        for n in (1, 17, k):
            check(z, tokens, n, 1.0, call(lsp, z, tokens, n))


def elapsed(lsp, z, tokens, k):
    out = [torch.empty(z.shape[0], device="cuda"), None, torch.empty(z.shape[0], k, dtype=torch.int32, device="cuda")]
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    best = float("inf")
    for _ in range(6):
        a.record()
        for _ in range(5):
            lsp.lsp_logprobs(z, tokens, *out)
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("dtype,k", [("bf16", 20), ("bf16", 32), ("f32", 32)])
def test_rows_of_mostly_equal_logits_take_no_multiple_of_others(lsp, dtype, k):
    """(Reading such rows again for every alternative takes bf16 12 to 45 times as long as usual; this way it is 2 to 3.)"""
    V = 151936
    g = torch.Generator("cuda").manual_seed(1)
    for rows in (64, 600):                           # parts of a row, and whole rows
        z = (torch.randn(rows, V, device="cuda", generator=g) * 2.5).to(DT[dtype])
        tokens = ints([7] * rows)
        usual = elapsed(lsp, z, tokens, k)
        keep = torch.rand(rows, V, device="cuda", generator=g) < 50 / V
        for x in (torch.where(keep, z, -float("inf")), torch.zeros_like(z),
                  torch.sort(z.float(), descending=True).values.to(DT[dtype])):        # filtered, equal, the largest side by side
            x[:, 7] = 1.0
            assert elapsed(lsp, x, tokens, k) < 6 * usual


@pytest.mark.parametrize("dtype", list(DT))
def test_a_row_at_any_address(lsp, dtype):
    """The same row at several addresses: its sums may go another way, its tokens may not."""
    V, k = 30011, 20
    g = torch.Generator().manual_seed(3)
    row = (torch.randn(V, generator=g) * 3).to(DT[dtype]).cuda()
    row[::1000] = 12.5                               # equal ones among the largest
    outs = []
    for by in range(8):
        wide = torch.zeros(V + 8, dtype=DT[dtype], device="cuda")
        wide[by:by + V] = row
        z = wide[by:by + V][None]
        outs.append(call(lsp, z, ints([4321]), k))
        check(z, ints([4321]), k, 1.0, outs[-1])
    assert all(torch.equal(o[2], outs[0][2]) for o in outs)
