"""The example's rounds (drafter state, paged cache, shared-prefix attention, verification) end to end.

Greedy speculative generation is lossless: every token has to be the argmax of the
target's logits after the tokens before it, recomputed densely in 64 bits.  With
fp32 storage a logit passes through 4 products a layer and the last one, each of at
most 256 terms after a normalisation: a relative error of about 16 x 2^-24 a
product, 13 of them over 3 layers, on logits below 2: under 3e-5.  TOL is 1e-4, and
the same for the keys and values of the cache, which are below 8.
"""
import os
import sys

import pytest
import torch

from paper_2609_37029_gb300 import synth
from tests.gpu_common import lsp_lib

pytestmark = pytest.mark.gpu

TOL = 1e-4
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    lsp_lib()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import target_round
    finally:
        sys.path.pop(0)
    return target_round


def dense(run, tokens):
    """(logits [n][V], k, v [L][n][nkv][d]) of a whole token list in 64 bits."""
    s, t = run.s, run.target
    n, rep = len(tokens), s.nq // s.nkv
    rms = lambda x: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    x = run.held["embed"][torch.tensor(tokens, device="cuda")].double() * s.H ** 0.5
    seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    ks, vs = [], []
    for layer in range(s.L):
        y = (rms(x) @ t.qkv[layer].double().T).view(n, -1, s.d)
        q, k, v = y.split([s.nq, s.nkv, s.nkv], 1)
        z = torch.einsum("qgrd,kgd->grqk", q.reshape(n, s.nkv, rep, s.d), k) * s.d ** -0.5
        p = torch.softmax(z.masked_fill(~seen, -torch.inf), -1)
        x = x + torch.einsum("grqk,kgd->qgrd", p, v).reshape(n, -1) @ t.back[layer].double().T
        ks.append(k)
        vs.append(v)
    return rms(x) @ run.held["lm_head"].double().T, torch.stack(ks), torch.stack(vs)


def check_run(run, prompt):
    run.check()
    s, t, page = run.s, run.target, run.target.k.shape[3]
    assert t.len.tolist()[1:] == [run.prompt + len(x) - 1 for x in run.tokens]     # the last one is not in yet
    own = sum(-(-x // page) - run.prompt // page for x in t.len.tolist())
    assert int((t.refs > 0).sum()) == run.prompt // page + own      # own: the part page of the prompt itself too
    assert t.refs.tolist() == torch.bincount(t.table[t.table >= 0].long(), minlength=t.refs.numel()).tolist()
    for b, toks in enumerate(run.tokens):
        z, k, v = dense(run, prompt.tolist() + toks[:-1])
        rows = z[run.prompt - 1:]
        got = rows.gather(1, torch.tensor(toks, device="cuda")[:, None])[:, 0]
        assert float(rows.abs().max()) < 2
        assert bool((got >= rows.amax(1) - TOL).all()), b
        n = k.shape[1]
        pages = t.table[b + 1, :-(-n // page)].long()
        for pool, want in ((t.k, k), (t.v, v)):
            have = pool[:, pages].transpose(2, 3).flatten(1, 2)[:, :n]
            assert float((have.double() - want).abs().max()) <= TOL


@pytest.mark.parametrize("prompt_len", [1, 64, 150])
def test_greedy_generation_is_lossless(example, prompt_len):
    s = synth.TINY.with_(C=3)
    g = torch.Generator().manual_seed(prompt_len)
    prompt = torch.randint(0, s.V, (prompt_len,), generator=g, dtype=torch.int32).cuda()
    rounds = 12
    first = example.Generation(s, prompt, rounds)
    try:
        for _ in range(rounds):
            first.step()
        check_run(first, prompt)
        truth = first.tokens
    finally:
        first.close()
    # proposals that are right up to a place that moves with the request and the round
    second = example.Generation(s, prompt, rounds)
    try:
        for i in range(3):
            want, y = [], torch.empty(s.C, s.B, dtype=torch.int64)
            for b in range(s.C):
                at, good = len(second.tokens[b]), min((b + i) % 4, s.B)
                nxt = (truth[b][at:at + s.B] + [0] * s.B)[:s.B]
                nxt[good] = (nxt[good] + 1) % s.V
                y[b] = torch.tensor(nxt)
                want.append(good)
            got = second.step(y.cuda())
            if all(second.tokens[b] == truth[b][:len(second.tokens[b])] for b in range(s.C)):
                assert got == want
        check_run(second, prompt)
        assert sum(map(sum, second.accepted)) > 0
    finally:
        second.close()


def test_sampled_bf16_rounds(example):
    """The example's own sizes: near-uniform distributions on both sides, so proposals pass, and not all."""
    s = synth.SMALL.with_(layer_scale=False)
    prompt = torch.randint(0, s.V, (300,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    run = example.Generation(s, prompt, 3, temperature=1.0)
    try:
        for _ in range(3):
            run.step()
        run.check()
        assert all(0 <= x < s.V for row in run.tokens for x in row)
        assert 0 < sum(map(sum, run.accepted)) < 3 * s.C * s.B
        assert run.target.len.tolist()[1:] == [300 + len(x) - 1 for x in run.tokens]
    finally:
        run.close()
