"""Speculative generation over a paged cache: continuations of one shared prompt.

A toy target (random weights, no positional encoding: attention and a projection
back, per layer) generates C continuations of a prompt.  Each round, per request:
the drafter proposes B tokens from its fixed-size state (lsp_draft); the target
takes the committed token and the proposals as B + 1 new rows of its cache
(lsp_pages_reserve, then per layer lsp_pages_write and lsp_prefix_attention, the
prompt's pages read once for all requests); lsp_verify_probs accepts r of the
proposals and gives the next committed token; lsp_logprobs gives what a server
answers beside the tokens; lsp_pages_trim gives back the rejected rows;
lsp_view_update folds the r + 1 kept rows into the drafter's state.  The prompt
itself runs once, and lsp_pages_fork hands its pages to the requests.

With --cache q4 the cache is held in 4 bits (lsp_pages_write_q4,
lsp_prefix_attention_q4).  At the end the drafter's state of the first request is
built again from the cache (lsp_pages_read), as a server does that dropped it.

    python examples/target_round.py [--rounds 8] [--prompt 500] [--temperature 1] [--cache bf16|q4]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_37029_gb300 import lsp, synth  # noqa: E402


def whole(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Target:
    """The toy target and its paged cache: sequence 0 is the prompt, 1..C its continuations."""

    def __init__(self, s, weights, most_tokens, page=64, seed=5, q4=False):
        self.s, self.w, self.q4 = s, weights, q4
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.qkv, self.back = ([torch.randn(o, i, generator=g, device="cuda").mul_(i ** -0.5).to(s.torch_dtype)
                                for _ in range(s.L)]
                               for o, i in (((s.nq + 2 * s.nkv) * s.d, s.H), (s.H, s.nq * s.d)))
        held = -(-most_tokens // page)
        pool = (2, s.L, (s.C + 1) * held, s.nkv, page, s.d * 9 // 16 if q4 else s.d)
        self.k, self.v = torch.zeros(pool, dtype=torch.uint8 if q4 else s.torch_dtype, device="cuda")
        self.table = torch.full((s.C + 1, held), -1, dtype=torch.int32, device="cuda")
        self.len = torch.zeros(s.C + 1, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(pool[2], dtype=torch.int32, device="cuda")
        self.cache = lsp.make_kv_cache(self.k, self.v, self.table, self.len, self.refs)
        self.pages_ws = torch.empty(lsp.lsp_pages_workspace_bytes(self.cache), dtype=torch.uint8, device="cuda")
        self.error = torch.zeros(1, dtype=torch.int32, device="cuda")

    def forward(self, tokens, seqs, add, start, shared):
        """New rows (tokens [total], rows [start[i], start[i+1]) of sequence seqs[i], add[i] of them) through
        the target: k, v [L][total][nkv][d], hidden states [L][total][H] and fp32 logits [total][V]."""
        s, c, total = self.s, self.cache, tokens.numel()
        if self.q4:
            room = lsp.lsp_prefix_attention_q4_workspace_bytes(c, s.torch_dtype, s.nq, seqs.numel(), total)
            write, attend = lsp.lsp_pages_write_q4, lsp.lsp_prefix_attention_q4
        else:
            room = lsp.lsp_prefix_attention_workspace_bytes(c, s.nq, seqs.numel(), total)
            write, attend = lsp.lsp_pages_write, lsp.lsp_prefix_attention
        ws = torch.empty(room, dtype=torch.uint8, device="cuda")
        lsp.lsp_pages_reserve(c, seqs, add, self.pages_ws, self.error)
        x = self.w["embed"][tokens.long()].float() * s.H ** 0.5
        k, v, h = [], [], []
        for layer in range(s.L):
            y = (rms(x).to(s.torch_dtype) @ self.qkv[layer].T).view(total, s.nq + 2 * s.nkv, s.d)
            q, kn, vn = y.split([s.nq, s.nkv, s.nkv], dim=1)         # slices of the fused rows, no copy
            out = torch.empty(total, s.nq, s.d, dtype=s.torch_dtype, device="cuda")
            write(c, layer, seqs, start, kn, vn, self.error)
            attend(c, layer, q, seqs, start, out, shared_len=shared, scale=s.d ** -0.5, workspace=ws, dev_error=self.error)
            x = x + (out.view(total, -1) @ self.back[layer].T).float()
            k.append(kn)
            v.append(vn)
            h.append(x.to(s.torch_dtype))
        logits = (rms(x).to(s.torch_dtype) @ self.w["lm_head"].T).float()
        return torch.stack(k), torch.stack(v), torch.stack(h), logits

    def read(self, seq, tokens):
        """k, v [L][tokens][nkv][d] of a sequence's last tokens, as the cache holds them."""
        s = self.s
        k, v = torch.empty(2, s.L, tokens, s.nkv, s.d, dtype=s.torch_dtype, device="cuda")
        seqs, start = whole([seq]), whole([0, tokens])
        for layer in range(s.L):
            lsp.lsp_pages_read(self.cache, layer, seqs, start, k[layer], v[layer], self.error)
        return k, v


def rms(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)


def distribution(logits, temperature):
    """What the tests and draws run on: softmax at the temperature, all on the argmax at 0."""
    if temperature > 0:
        return torch.softmax(logits / temperature, -1)
    return torch.zeros_like(logits).scatter_(-1, logits.argmax(-1, keepdim=True), 1.0)


class Generation:
    def __init__(self, s, prompt, rounds, temperature=0.0, seed=11, q4=False):
        """prompt: int32 [P] of token ids; the cache has room for `rounds` rounds, in 4 bits with q4."""
        self.s, self.T, self.seed, self.round = s, temperature, seed, 0
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        w = synth.make_weights(s, device="cuda")
        self.weights, self.held = lsp.make_weights(w), w
        self.prompt = prompt.numel()
        self.target = t = Target(s, w, self.prompt + (rounds + 1) * (s.B + 1), q4=q4)
        self.seqs = whole(list(range(1, s.C + 1)))
        self.start = whole([i * (s.B + 1) for i in range(s.C + 1)])
        self.add = whole([s.B + 1] * s.C)
        # the prompt, once; every request then holds its pages
        one = whole([0])
        k, v, h, z = t.forward(prompt, one, whole([self.prompt]), whole([0, self.prompt]), 0)
        lsp.lsp_pages_fork(t.cache, whole([0] * s.C), self.seqs, t.error)
        # ... and a drafter state over it
        self.state = lsp.lsp_state_create(lsp.make_config(s))
        lsp.lsp_state_init(self.state, w["G"])
        rows = [x[None].expand(s.C, *x.shape).contiguous() for x in (k, v, h)]
        lsp.lsp_view_update(self.state, *rows, whole([self.prompt] * s.C))
        p = distribution(z[-1:], self.T)
        self.committed = (p / self.exponentials(s.C)).argmax(-1).to(torch.int32)
        self.len = torch.full((s.C,), self.prompt, dtype=torch.int32, device="cuda")
        self.tokens = [[int(a)] for a in self.committed]
        self.logprobs = [[] for _ in range(s.C)]                    # (log probability, entropy, top tokens, theirs) a token
        self.boundary = h[:, -1:].expand(-1, s.C, -1).clone()       # hidden states of each request's last folded row [L][C][H]
        self.accepted = []

    def exponentials(self, rows):
        return torch.empty(rows, self.s.V, device="cuda").exponential_(generator=self.gen).clamp_(min=1e-20)

    def step(self, proposals=None):
        """One round; proposals [C][B] in the place of the drafter's, if given.  Returns r of each request."""
        s, t = self.s, self.target
        y, zq = torch.empty(s.C, s.B, dtype=torch.int32, device="cuda"), torch.empty(s.C, s.B, s.V, device="cuda")
        block = torch.full((s.C, s.B), -1, dtype=torch.int32, device="cuda")
        block[:, 0] = self.committed
        lsp.lsp_draft(self.state, block, self.weights, lsp.make_sample_params(self.T, self.seed, self.round), y, zq)
        if proposals is not None:
            y = proposals.to(torch.int32).contiguous()
        rows = torch.cat([self.committed[:, None], y], 1)
        k, v, h, z = t.forward(rows.flatten(), self.seqs, self.add, self.start, self.prompt)
        p = distribution(z.view(s.C, s.B + 1, s.V), self.T)
        # greedy or foreign proposals were not drawn from a distribution
        q = distribution(zq, self.T) if self.T > 0 and proposals is None else None
        r, nxt = torch.empty_like(self.committed), torch.empty_like(self.committed)
        out = torch.empty(s.C, s.B + 1, dtype=torch.int32, device="cuda")
        u = torch.rand(s.C, s.B, generator=self.gen, device="cuda")
        lsp.lsp_verify_probs(p, q, y, u, self.exponentials(s.C), r, nxt, out_tokens=out, dev_error=t.error)
        lp, entropy, top, top_lp = self.answers(z, out)
        keep = r + 1                                                # the committed token and the accepted ones
        self.len += keep
        lsp.lsp_pages_trim(t.cache, self.seqs, self.len, t.error)
        by_request = lambda x: x.unflatten(1, (s.C, s.B + 1)).transpose(0, 1).contiguous()
        lsp.lsp_view_update(self.state, by_request(k), by_request(v), by_request(h), keep)
        self.committed, self.round = nxt, self.round + 1
        got = r.tolist()                                            # the round's result, on the host
        for b, row in enumerate(out.tolist()):
            self.tokens[b] += row[:got[b] + 1]
            at = [b * (s.B + 1) + i for i in range(got[b] + 1)]
            self.logprobs[b] += list(zip(lp[at].tolist(), entropy[at].tolist(), top[at].tolist(), top_lp[at].tolist()))
            self.boundary[:, b] = h[:, at[-1]]
        self.accepted.append(got)
        return got

    def answers(self, logits, out, k=3):
        """Log probability and entropy of every emitted token, and the k likeliest in its place (-1: none emitted)."""
        rows = logits.shape[0]
        lp, entropy, top_lp = (torch.empty(*x, device="cuda") for x in ((rows,), (rows,), (rows, k)))
        top = torch.empty(rows, k, dtype=torch.int32, device="cuda")
        lsp.lsp_logprobs(logits, out.view(-1), lp, entropy, top, top_lp, temperature=self.T or 1.0, dev_error=self.target.error)
        return lp, entropy, top, top_lp

    def rebuild(self, b):
        """A drafter state of request b alone, from what the cache holds of it."""
        s = self.s.with_(C=1)
        n = int(self.len[b])
        k, v = self.target.read(b + 1, n)
        h = torch.zeros(s.L, n, s.H, dtype=s.torch_dtype, device="cuda")
        h[:, -1] = self.boundary[:, b]                              # (all that the state takes of them)
        state = lsp.lsp_state_create(lsp.make_config(s))
        lsp.lsp_state_init(state, self.held["G"])
        lsp.lsp_view_update(state, k[None], v[None], h[None], whole([n]))
        return state

    def check(self):
        """Raises if a kernel saw something wrong in any of the rounds."""
        rc, bits = lsp.lsp_get_error(self.state)
        bits |= int(self.target.error)
        if rc != lsp.LSP_OK or bits:
            raise RuntimeError(f"device error bits {bits:#x}")

    def close(self):
        lsp.lsp_state_destroy(self.state)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--rounds", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=500)
    ap.add_argument("--temperature", type=float, default=1.0)
    ap.add_argument("--cache", choices=["bf16", "q4"], default="bf16")
    a = ap.parse_args()
    s = synth.SMALL.with_(layer_scale=False)
    prompt = torch.randint(0, s.V, (a.prompt,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    run = Generation(s, prompt, a.rounds, a.temperature, q4=a.cache == "q4")
    for i in range(a.rounds):
        print(f"round {i}: accepted {run.step()} of {s.B}")
    run.check()
    live = int((run.target.refs > 0).sum())
    said = [x[0] for row in run.logprobs for x in row]
    print(f"mean log probability of {len(said)} tokens {sum(said) / len(said):.3f}")
    lsp.lsp_state_destroy(run.rebuild(0))
    print(f"{sum(map(len, run.tokens))} tokens for {s.C} continuations of a prompt of {a.prompt}; {live} pages live")
    run.close()


if __name__ == "__main__":
    main()
