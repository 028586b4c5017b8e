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
