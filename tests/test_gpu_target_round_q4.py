"""The example's rounds over a cache held in 4 bits, with log probabilities and a state rebuilt from the cache.

Given the values that the cache holds, the target is an exact computation again: every greedy token has to be the
argmax of its logits, recomputed densely in 64 bits over those values, and the reported numbers theirs.  TOL: that of
the rounds over a cache of fp32 (a relative error of about 16 x 2^-24 a product, 13 of them, on logits below 2: under
3e-5); log probabilities and entropies are off by no more than twice the logits and lsp_logprobs' own 1e-5 (entropies:
2e-5 (1 + H), H below 10).
"""
import os
import sys

import pytest
import torch

from oracle import cache_q4
from paper_2609_37029_gb300 import synth
from tests.gpu_common import export_state, f64, lsp_lib, window_in_prefix_order

pytestmark = pytest.mark.gpu

TOL = 1e-4
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


@pytest.fixture(scope="module")
def example(lsp):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import target_round
    finally:
        sys.path.pop(0)
    return target_round


def dense_over_cache(run, b, tokens):
    """fp64 logits [n][V] of a token list over the keys and values that the cache holds of request b."""
    s, t = run.s, run.target
    n, rep = len(tokens), s.nq // s.nkv
    k, v = (x.double() for x in t.read(b + 1, n))
    rms = lambda x: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    x = run.held["embed"][torch.tensor(tokens, device="cuda")].double() * s.H ** 0.5
    seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    for layer in range(s.L):
        q = (rms(x) @ t.qkv[layer].double().T).view(n, -1, s.d)[:, :s.nq]
        z = torch.einsum("qgrd,kgd->grqk", q.reshape(n, s.nkv, rep, s.d), k[layer]) * s.d ** -0.5
        p = torch.softmax(z.masked_fill(~seen, -torch.inf), -1)
        x = x + torch.einsum("grqk,kgd->qgrd", p, v[layer]).reshape(n, -1) @ t.back[layer].double().T
    return rms(x) @ run.held["lm_head"].double().T


@pytest.mark.parametrize("prompt_len", [1, 64, 150])
def test_greedy_tokens_and_their_log_probabilities(lsp, example, prompt_len):
    s = synth.TINY.with_(C=3)
    prompt = torch.randint(0, s.V, (prompt_len,), generator=torch.Generator().manual_seed(prompt_len), dtype=torch.int32).cuda()
    run = example.Generation(s, prompt, 10, q4=True)
    try:
        for _ in range(10):
            run.step()
        run.check()
        for b, toks in enumerate(run.tokens):
            assert int(run.target.len[b + 1]) == prompt_len + len(toks) - 1
            z = dense_over_cache(run, b, prompt.tolist() + toks[:-1])[prompt_len - 1:]
            assert float(z.abs().max()) < 2
            got = z.gather(1, torch.tensor(toks, device="cuda")[:, None])[:, 0]
            assert bool((got >= z.amax(1) - TOL).all()), b
            lp = torch.log_softmax(z, -1)
            assert len(run.logprobs[b]) == len(toks) - 1            # (the prompt's own token was drawn from it)
            for i, (said, entropy, top, top_lp) in enumerate(run.logprobs[b], 1):
                row = lp[i]
                assert abs(said - float(row[toks[i]])) <= 2 * TOL
                assert abs(entropy + float((row.exp() * row).sum())) <= 2 * TOL + 2e-4
                assert top[0] == toks[i] and len(set(top)) == 3
                for token, x in zip(top, top_lp):
                    assert abs(x - float(row[token])) <= 2 * TOL
                assert float(row.topk(3).values[-1]) - float(row[top[-1]]) <= 2 * TOL
        # what the cache holds is a fixed point of its format
        k, v = run.target.read(1, int(run.len[0]))
        for x in (k, v):
            y = x.cpu().numpy()
            assert (cache_q4.values(y.astype("float64")) == y).all()
    finally:
        run.close()


def test_a_state_rebuilt_from_the_cache(lsp, example):
    s = synth.TINY.with_(C=3)
    prompt = torch.randint(0, s.V, (70,), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    run = example.Generation(s, prompt, 4, q4=True)
    try:
        for _ in range(4):
            run.step()
        for b in range(s.C):
            n = int(run.len[b])
            st = run.rebuild(b)
            try:
                one = s.with_(C=1)
                ex = export_state(lsp, st, one)
                assert ex["t"].tolist() == [n]
                k, v = (f64(x) for x in run.target.read(b + 1, n))
                wk, wv = (window_in_prefix_order(f64(ex[x])[0], n, s.W) for x in ("win_k", "win_v"))    # [L][nkv][rows][d]
                m = min(n, s.W)
                assert (wk == k[:, n - m:].transpose(0, 2, 1, 3)).all() and (wv == v[:, n - m:].transpose(0, 2, 1, 3)).all()
                assert (f64(ex["h"])[0] == f64(run.boundary[:, b])).all()
                # and the drafter runs on it
                y = torch.empty(1, s.B, dtype=torch.int32, device="cuda")
                block = torch.full((1, s.B), -1, dtype=torch.int32, device="cuda")
                block[:, 0] = run.committed[b]
                lsp.lsp_draft(st, block, run.weights, lsp.make_sample_params(0.0), y)
                assert lsp.lsp_get_error(st) == (lsp.LSP_OK, 0) and bool(((y >= 0) & (y < s.V)).all())
            finally:
                lsp.lsp_state_destroy(st)
        run.check()
    finally:
        run.close()


def test_sampled_bf16_rounds(example):
    s = synth.SMALL.with_(layer_scale=False)
    prompt = torch.randint(0, s.V, (300,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    run = example.Generation(s, prompt, 3, temperature=1.0, q4=True)
    try:
        for _ in range(3):
            run.step()
        run.check()
        assert all(0 <= x < s.V for row in run.tokens for x in row)
        assert run.target.len.tolist()[1:] == [300 + len(x) - 1 for x in run.tokens]
        assert [len(x) for x in run.logprobs] == [len(x) - 1 for x in run.tokens]
        assert all(x[0] <= 0 and x[1] >= 0 and x[3][0] >= x[0] - 1e-5 for row in run.logprobs for x in row)
    finally:
        run.close()
