"""The oracle of the target side against something other than itself: attention over pages equals
torch's scaled_dot_product_attention over the gathered tokens, page operations keep every token's
values and every page's holders, acceptance frequencies follow the target's distribution."""
import numpy as np
import pytest
import torch

from oracle.target import PagedCache, cache_attention, verify_probs


@pytest.mark.parametrize("lens,rows", [((5, 33, 16), (1, 3, 16)), ((40, 7, 64), (2, 7, 40))])
def test_paged_attention_is_sdpa_over_the_tokens(lens, rows):
    rng = np.random.RandomState(3)
    page, nkv, rep, d = 16, 2, 3, 8
    pages = sum(-(-n // page) for n in lens)
    place = iter(rng.permutation(pages))
    table = np.full((3, 5), -1)
    for b, n in enumerate(lens):
        for i in range(-(-n // page)):
            table[b, i] = next(place)
    c = PagedCache(rng.randn(1, pages, nkv, page, d), rng.randn(1, pages, nkv, page, d), table, lens, np.ones(pages, int))
    start = np.concatenate([[0], np.cumsum(rows)])
    q = rng.randn(start[-1], nkv * rep, d)
    out, lse, _ = cache_attention(c, 0, q, [0, 1, 2], start, 0.3)
    for b, n in enumerate(lens):
        k, v = (torch.from_numpy(x).permute(1, 0, 2).repeat_interleave(rep, 0) for x in c.tokens(0, b))
        x = torch.from_numpy(q[start[b]:start[b + 1]]).permute(1, 0, 2)
        mask = torch.arange(n)[None] <= torch.arange(n - rows[b], n)[:, None]
        want = torch.nn.functional.scaled_dot_product_attention(x, k, v, attn_mask=mask, scale=0.3)
        np.testing.assert_allclose(out[start[b]:start[b + 1]], want.permute(1, 0, 2).numpy(), atol=1e-12)
        s = (x @ k.transpose(1, 2) * 0.3).masked_fill(~mask, -np.inf)
        np.testing.assert_allclose(lse[start[b]:start[b + 1]].T, torch.logsumexp(s, -1).numpy(), atol=1e-12)


def test_page_operations_keep_tokens_and_holders():
    rng = np.random.RandomState(1)
    page, pages = 4, 60
    c = PagedCache(np.zeros((2, pages, 1, page, 2)), np.zeros((2, pages, 1, page, 2)), np.full((6, 8), -1), np.zeros(6, int),
                   np.zeros(pages, int))
    told = [np.zeros((0, 1, 2)) for _ in range(6)]      # what each sequence should read, layer 1
    for step in range(200):
        op = rng.randint(4)
        s, d = rng.choice(6, 2, replace=False)
        if op == 0:
            assert not c.fork([s], [d])
            told[d] = told[s].copy()
        elif op == 1:
            a = int(rng.randint(0, 9))
            if len(told[s]) + a > 32:
                continue
            bad, short = c.reserve([s], [a])
            assert not bad and not short
            new = rng.randn(a, 1, 2)
            c.write(1, [s], [0, a], new, new)
            told[s] = np.concatenate([told[s], new])
        elif op == 2:
            n = int(rng.randint(0, 32))
            assert not c.trim([s], [n])
            told[s] = told[s][:n]
        else:
            live = c.compact()
            assert (c.refs[:live] > 0).all() and (c.refs[live:] == 0).all()
        count = np.zeros(pages, int)
        for x in range(6):
            np.testing.assert_array_equal(c.tokens(1, x)[0], told[x])
            np.testing.assert_array_equal(c.tokens(1, x)[1], told[x])
            assert (c.table[x, c.held(x):] == -1).all()
            for pg in c.table[x, :c.held(x)]:
                count[pg] += 1
        np.testing.assert_array_equal(count, c.refs)


def test_accepted_and_redrawn_tokens_follow_the_target():
    rng = np.random.RandomState(0)
    V, N = 5, 20000
    p, q = rng.dirichlet(np.ones(V), 2), rng.dirichlet(np.ones(V), 1)
    got = np.zeros(V)
    for _ in range(N):
        y = rng.choice(V, p=q[0])
        r, t = verify_probs(p, q, [y], 1, rng.rand(1), rng.exponential(size=V))
        got[y if r else t] += 1
    assert ((got - N * p[0]) ** 2 / (N * p[0])).sum() < 18.5      # chi-squared, 4 degrees, 1e-3


def test_acceptance_corners():
    e = np.ones(4)
    p = np.array([[0.5, 0.5, 0, 0], [0, 0, 0, 0]])
    assert verify_probs(p, None, [0], 1, [0.4], e) == (1, -1)          # nothing to draw from
    assert verify_probs(p, None, [0], 1, [0.6], e) == (0, 1)           # a point mass leaves the rest
    assert verify_probs(p, p[:1], [2], 1, [0.6], e) == (0, 0)          # p - q is empty: p itself, lowest index
    assert verify_probs(p, p[:1], [9], 1, [0.0], e) == (0, 0)          # a token outside is rejected
