"""lsp_prefix_attention where segments of one and of two row tiles follow each other in the same CTA: both streams
add up the first kind together and each its own of the second, and the barriers between them go from one kind to
the other at every step.  bf16 only (the other type has one stream); tolerances: those of the other tests of this
call.
"""
import pytest
import torch

from tests.gpu_common import lsp_lib
from tests.test_gpu_prefix_attn import attend, case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


def check(pool, t, q, lens, rows, out, z):
    """Sequence by sequence in fp64, one KV head."""
    d, page, at = q.shape[2], pool[0].shape[3], 0
    for b, (n, r) in enumerate(zip(lens, rows)):
        pages = t[0][b, :-(-n // page)].long()
        k, v = (x[0, pages, 0].reshape(-1, d)[:n].double() for x in pool)
        s = torch.einsum("rhd,nd->rhn", q[at:at + r].double(), k) * d ** -0.5
        seen = torch.arange(n, device="cuda")[None] <= torch.arange(n - r, n, device="cuda")[:, None]
        s = s.masked_fill(~seen[:, None], -torch.inf)
        w = torch.softmax(s, -1)
        want, size = w @ v, w @ v.abs()
        assert bool(((out[at:at + r].double() - want).abs() <= (2 ** -8 + 2 ** -10) * (size + want.abs())).all()), b
        lse = torch.logsumexp(s, -1)
        assert bool(((z[at:at + r].double() - lse).abs() <= 2e-5 + 2e-6 * lse.abs()).all()), b
        at += r


# 64 heads on one KV head: a tile has two tokens, so 1 and 2 rows are one tile, 3 and 4 two
@pytest.mark.parametrize("order", [(4, 1), (3, 2, 1), (4, 4, 1, 1), (1, 4, 1, 3, 9)])
@pytest.mark.parametrize("d,blocks", [(64, 2), (128, 3)])
def test_one_and_two_row_tiles_by_turns(lsp, order, d, blocks):
    n = 700
    rows = [order[i % len(order)] for i in range(n)]
    lens = [128 * (1 + i % blocks) + 7 + 5 * i % 113 for i in range(n)]
    pool, t, q = case(lens, rows, 0, nq=64, nkv=1, d=d, dtype="bf16", page=16)
    seqs = list(range(n))
    out, z = attend(lsp, pool, t, q, seqs, rows, 0)
    check(pool, t, q, lens, rows, out, z)
    for fill in (0, 0x5A):
        again, z2 = attend(lsp, pool, t, q, seqs, rows, 0, fill=fill)
        assert torch.equal(out, again) and torch.equal(z, z2)
