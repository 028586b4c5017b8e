"""Workloads of the target side of a drafting round, for measuring its operators.

Three groups of operators of one verification round over a paged key/value cache:

* attend   attention of the round's candidate rows over the cache, the batch's
           shared prefix read once for all requests (lsp_prefix_attention);
* pages    branching sequences off a shared prompt, reserving, writing and
           giving back pages, and compacting a fragmented pool (lsp_pages_*);
* verify   acceptance of the drafted tokens against the target's probabilities
           from given random numbers (lsp_verify_probs).

Each case is a dict of plain values.  run() takes the calls a program makes of
the library where `own` is true, and computes the same results with elementary
torch operations in 32 bits where it is false; exact() computes them in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

BF16, F32 = "bf16", "f32"


# ------------------------------------------------------------------ cases
def listed():
    return [
        # two requests that each generate one token behind a short system prompt: latency
        attend_case("attend step small", n=2, nq=8, nkv=2, shared=500, own=(1, 40), q=(1, 1), page=16),
        # one token of each of 16 requests over a 32K prompt: the cache's bytes count
        attend_case("attend step 32K", n=16, nq=32, nkv=8, shared=32768, own=(1, 500), q=(1, 1), page=64),
        # a round's block and committed token of 16 requests over a 32K prompt
        attend_case("attend round 32K", n=16, nq=32, nkv=8, shared=32768, own=(17, 1500), q=(17, 17), page=64),
        # the larger target: 32 requests with ragged blocks over a 128K prompt
        attend_case("attend round 128K", n=32, nq=40, nkv=8, shared=131072, own=(17, 2000), q=(9, 17), page=64),
        # 32-bit storage, two query heads a key head, ragged blocks, a prompt that ends inside a page
        attend_case("attend f32 ragged", n=5, nq=4, nkv=2, d=64, dtype=F32, shared=2047, own=(1, 333), q=(1, 9), page=32),
        # two continuations of one short prompt
        branch_case("branch small", parents=1, fan=2, layers=4, nkv=2, tokens=(300, 300), add=17, page=16),
        # four continuations of each of 16 prompts over all layers of a cache
        branch_case("branch large", parents=16, fan=4, layers=32, nkv=8, tokens=(1000, 4000), add=17, page=64),
        # a small pool with a few requests gone
        compact_case("compact small", pages=200, live=120, layers=4, nkv=2, page=16, seqs=12),
        # a pool two thirds full, all layers moved
        compact_case("compact large", pages=3000, live=2000, layers=8, nkv=8, page=64, seqs=64),
        # four requests, a small vocabulary of odd size
        verify_case("verify small", C=4, B=16, V=32001),
        # a round of 16 requests over the whole vocabulary
        verify_case("verify round", C=16, B=16, V=151936),
        # 64 requests with 16-bit probabilities and drafts without a distribution of their own
        verify_case("verify 64", C=64, B=16, V=151936, dtype=BF16, draft=False),
    ]


def attend_case(name, *, n, nq, nkv, shared, own, q, page, d=128, dtype=BF16, layers=2, mix=1):
    return named(name, op="attend", dtype=dtype, n=n, nq=nq, nkv=nkv, d=d, page=page, shared=shared,
                 own_lo=own[0], own_hi=own[1], q_lo=q[0], q_hi=q[1], layers=layers, mix=mix)


def branch_case(name, *, parents, fan, layers, nkv, tokens, add, page, d=128, dtype=BF16, mix=1):
    return named(name, op="branch", dtype=dtype, parents=parents, fan=fan, layers=layers, nkv=nkv, d=d,
                 lo=tokens[0], hi=tokens[1], add=add, page=page, mix=mix)


def compact_case(name, *, pages, live, layers, nkv, page, seqs, d=128, dtype=BF16):
    return named(name, op="compact", dtype=dtype, pages=pages, live=live, layers=layers, nkv=nkv, d=d, page=page, seqs=seqs)


def verify_case(name, *, C, B, V, dtype=F32, draft=True):
    return named(name, op="verify", dtype=dtype, C=C, B=B, V=V, draft=draft)


def named(name, **case):
    return {**({"name": name} if name else {}), **case}


def spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    x = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    x = max(lo, min(hi, x))
    return x + 1 if x == 3072 else x


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "branch", "compact", "verify", "verify"])
    if op == "attend":
        most = work(listed()[3])["flops"]
        while True:
            dtype = F32 if rng.random() < 0.2 else BF16
            nq, nkv = rng.choice([(4, 2), (8, 2), (32, 8), (40, 8), (8, 8), (16, 1), (6, 2), (28, 4)])
            kind = rng.random()
            q = (1, 1) if kind < 0.35 else (1, 17) if kind < 0.8 else (20, spread(rng, 40, 600))
            shared = 0 if rng.random() < 0.15 else spread(rng, 16, 131072 if dtype == BF16 else 8192)
            lo = spread(rng, 1, 64)
            case = attend_case("", n=spread(rng, 1, 48), nq=nq, nkv=nkv, d=rng.choice([64, 128]), dtype=dtype, shared=shared,
                               own=(lo, max(lo, spread(rng, 8, 8000 if shared < 4096 else 2000))), q=q,
                               page=rng.choice([16, 32, 64, 128]), layers=rng.choice([1, 2, 3]), mix=rng.randrange(1 << 20))
            if work(case)["flops"] <= (most if dtype == BF16 else most / 32):
                return case
    if op == "branch":
        while True:
            lo = spread(rng, 1, 2000)
            case = branch_case("", parents=spread(rng, 1, 24), fan=spread(rng, 1, 8), layers=spread(rng, 1, 36),
                               nkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128]), dtype=rng.choice([BF16, BF16, F32]),
                               tokens=(lo, spread(rng, lo, 5000)), add=spread(rng, 1, 200), page=rng.choice([16, 32, 64, 128]),
                               mix=rng.randrange(1 << 20))
            if branch_bytes(case) < 6e9:
                return case
    if op == "compact":
        while True:
            pages = spread(rng, 20, 20000)
            case = compact_case("", pages=pages, live=max(1, int(pages * rng.uniform(0.1, 0.95))), layers=spread(rng, 1, 36),
                                nkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128]), dtype=rng.choice([BF16, BF16, F32]),
                                page=rng.choice([16, 32, 64, 128]), seqs=spread(rng, 1, 100))
            if pool_bytes(case, pages) < 6e9:
                return case
    return verify_case("", C=spread(rng, 1, 64), B=spread(rng, 1, 16), V=spread(rng, 1000, 151936),
                       dtype=rng.choice([F32, F32, BF16]), draft=rng.random() < 0.7)


# ------------------------------------------------------------------ sizes of a case
def size_of(case):
    return 2 if case["dtype"] == BF16 else 4


def torch_type(case):
    return torch.bfloat16 if case["dtype"] == BF16 else torch.float32


def pool_bytes(case, pages):
    return 2 * case["layers"] * pages * case["nkv"] * case["page"] * case["d"] * size_of(case)


def attend_lens(case):
    """(rows, tokens past the shared ones) of each request."""
    r = random.Random(case["mix"])
    rows = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["n"])]
    return rows, [max(x, r.randint(case["own_lo"], max(case["own_lo"], case["own_hi"]))) for x in rows]


def branch_lens(case):
    r = random.Random(case["mix"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["parents"])]


def branch_pages(case):
    """Pages that the parents hold, and most that their branches can add."""
    page = case["page"]
    held = sum(-(-x // page) for x in branch_lens(case))
    return held, case["parents"] * case["fan"] * (-(-case["add"] // page) + 1)


def branch_bytes(case):
    return pool_bytes(case, sum(branch_pages(case)))


def work(case):
    es = size_of(case)
    if case["op"] == "attend":
        rows, tail = attend_lens(case)
        nq, nkv, d, shared = case["nq"], case["nkv"], case["d"], case["shared"]
        keys = shared + sum(tail)
        seen = sum(x * shared + sum(o - x + i + 1 for i in range(x)) for x, o in zip(rows, tail))
        return {"bytes": 2 * keys * nkv * d * es + 2 * sum(rows) * nq * d * es + 4 * sum(rows) * nq, "flops": 4 * seen * nq * d}
    if case["op"] == "branch":
        token = 2 * case["nkv"] * case["d"] * es
        copied = sum(x % case["page"] for x in branch_lens(case)) * case["fan"] * case["layers"] * token
        written = case["parents"] * case["fan"] * case["add"] * token
        return {"bytes": 2 * copied + 2 * written + 12 * sum(branch_pages(case)), "flops": 0}
    if case["op"] == "compact":
        moved = case["live"] * (1 - case["live"] / case["pages"])
        return {"bytes": 2 * moved * pool_bytes(case, 1) + 12 * case["pages"], "flops": 0}
    C, B, V = case["C"], case["B"], case["V"]
    return {"bytes": C * V * (4 + es * (2 if case["draft"] else 1)) + C * B * 20, "flops": 3 * C * V}


# ------------------------------------------------------------------ inputs
def generator(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g


def whole(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def new_pool(case, pages, g):
    shape = (case["layers"], pages, case["nkv"], case["page"], case["d"])
    k = torch.empty(shape, dtype=torch_type(case), device="cuda").normal_(generator=g)
    v = torch.empty(shape, dtype=torch_type(case), device="cuda").normal_(generator=g)
    return k, v


def cache_of(k, v, table, lens, refs):
    """The handle that a program keeps of its cache, beside the tensors themselves."""
    s = {"k": k, "v": v, "table": table, "len": lens, "refs": refs}
    if own:
        from paper_2609_37029_gb300 import lsp
        s["cache"] = lsp.make_kv_cache(k, v, table, lens, refs)
    return s


def prepare(case, seed):
    s = {"attend": prepare_attend, "branch": prepare_branch, "compact": prepare_compact, "verify": prepare_verify}[case["op"]](case, seed)
    return {**s, "case": case}


def prepare_attend(case, seed):
    """Sequences whose first pages are the same ones, the rest their own, at shuffled places of the pool.
    Queries share a direction that the prompt's first tokens answer to, so that some keys stand out."""
    g, n, page, d = generator(seed), case["n"], case["page"], case["d"]
    rows, tail = attend_lens(case)
    common = case["shared"] // page
    held = [-(-(case["shared"] + x) // page) for x in tail]
    need = common + sum(h - common for h in held)
    pages = need + 3
    place = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
    table = torch.full((n, max(held) + 2), -1, dtype=torch.int32)
    refs = torch.zeros(pages, dtype=torch.int32)
    at = common
    for b in range(n):
        table[b, :common] = place[:common]
        table[b, common:held[b]] = place[at:at + held[b] - common]
        at += held[b] - common
    refs[place[:need].long()] = 1
    refs[place[:common].long()] = n
    k, v = new_pool(case, pages, g)
    lean = torch.randn(case["nkv"], d, generator=g, device="cuda") * 0.5
    first = int(table[0, 0])
    k[:, first, :, :4] += (2.0 * lean).to(k.dtype)[None, :, None]
    v += 0.1
    q = torch.randn(sum(rows), case["nkv"], case["nq"] // case["nkv"], d, generator=g, device="cuda") * 1.5 + lean[None, :, None]
    start = [0]
    for x in rows:
        start.append(start[-1] + x)
    s = cache_of(k, v, table.cuda(), whole([case["shared"] + x for x in tail]), refs.cuda())
    s.update(q=q.reshape(sum(rows), case["nq"], d).to(k.dtype).contiguous(), seqs=whole(list(range(n))), start=whole(start),
             total=sum(rows), rows=max(rows), own_pages=max(held) - common, layer=case["layers"] - 1, scale=d ** -0.5)
    if own:
        from paper_2609_37029_gb300 import lsp
        nbytes = lsp.lsp_prefix_attention_workspace_bytes(s["cache"], case["nq"], n, sum(rows))
        s["workspace"] = torch.empty(max(1, nbytes), dtype=torch.uint8, device="cuda")
    return s


def prepare_branch(case, seed):
    """Parents with shuffled pages; their branches' rows of the table are empty. The branches keep all but a
    few of the rows that they add, as after a round that accepted some of its tokens."""
    g, page, n = generator(seed), case["page"], case["parents"]
    lens, (held, more) = branch_lens(case), branch_pages(case)
    kids = n * case["fan"]
    pages = held + more + 5
    place = torch.randperm(pages, generator=g, device="cuda")[:held].to(torch.int32).cpu()
    width = -(-(max(lens) + case["add"]) // page) + 1
    table, at = torch.full((n + kids, width), -1, dtype=torch.int32), 0
    for b, x in enumerate(lens):
        m = -(-x // page)
        table[b, :m] = place[at:at + m]
        at += m
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[place.long()] = 1
    k, v = new_pool(case, pages, g)
    s = cache_of(k, v, table.cuda(), whole(lens + [0] * kids), refs.cuda())
    rows = (kids * case["add"], case["nkv"], case["d"])
    drop = torch.randint(0, case["add"] + 1, (kids,), generator=g, device="cuda", dtype=torch.int32)
    s.update(src=whole([b for b in range(n) for _ in range(case["fan"])]), dst=whole(list(range(n, n + kids))),
             add=whole([case["add"]] * kids), start=whole([i * case["add"] for i in range(kids + 1)]),
             k_new=torch.randn(rows, generator=g, device="cuda").to(k.dtype), v_new=torch.randn(rows, generator=g, device="cuda").to(k.dtype),
             keep=whole([x + case["add"] for x in lens for _ in range(case["fan"])]) - drop)
    if own:
        from paper_2609_37029_gb300 import lsp
        s["workspace"] = torch.empty(lsp.lsp_pages_workspace_bytes(s["cache"]), dtype=torch.uint8, device="cuda")
    return s


def prepare_compact(case, seed):
    """A pool whose live pages lie anywhere; the sequences hold them in turn, and share a few."""
    g, pages, live, n = generator(seed), case["pages"], case["live"], case["seqs"]
    place = torch.randperm(pages, generator=g, device="cuda")[:live].to(torch.int32).cpu()
    common = min(4, live // 2)
    cuts = [common + (live - common) * b // n for b in range(n + 1)]
    table = torch.full((n, common + max(b - a for a, b in zip(cuts, cuts[1:])) + 1), -1, dtype=torch.int32)
    lens = []
    for b in range(n):
        m = cuts[b + 1] - cuts[b]
        table[b, :common] = place[:common]
        table[b, common:common + m] = place[cuts[b]:cuts[b + 1]]
        lens.append((common + m) * case["page"])
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[place.long()] = 1
    refs[place[:common].long()] = n
    k, v = new_pool(case, pages, g)
    s = cache_of(k, v, table.cuda(), whole(lens), refs.cuda())
    s.update(table0=s["table"].clone(), refs0=s["refs"].clone(), live=whole([0]))
    if own:
        from paper_2609_37029_gb300 import lsp
        s["workspace"] = torch.empty(lsp.lsp_pages_workspace_bytes(s["cache"]), dtype=torch.uint8, device="cuda")
    return s


def prepare_verify(case, seed):
    """Target distributions cut to their likelier tokens, drafts that agree with them to a degree of the request's own."""
    g, C, B, V = generator(seed), case["C"], case["B"], case["V"]
    z = torch.randn(C, B + 1, V, generator=g, device="cuda") * 3
    p = torch.softmax(z, -1)
    p = torch.where(p * V < 1.0, torch.zeros_like(p), p)
    p /= p.sum(-1, keepdim=True)
    a = 0.9 + 0.099 * torch.rand(C, 1, 1, generator=g, device="cuda")
    zq = a * z[:, :B] + torch.sqrt(1 - a * a) * 3 * torch.randn(C, B, V, generator=g, device="cuda")
    q = torch.softmax(zq, -1)
    pick = torch.empty(C, B, V, device="cuda").exponential_(generator=g)
    y = (q / pick).argmax(-1) if case["draft"] else q.argmax(-1)
    s = {"p": p.to(torch_type(case)).contiguous(), "q": q.to(torch_type(case)).contiguous() if case["draft"] else None, "y": y.to(torch.int32)}
    s.update(n=torch.randint(max(0, B - 4), B + 1, (C,), generator=g, device="cuda", dtype=torch.int32),
             u=torch.rand(C, B, generator=g, device="cuda"), e=torch.empty(C, V, device="cuda").exponential_(generator=g).clamp_(min=1e-20))
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return {"attend": own_attend, "branch": own_branch, "compact": own_compact, "verify": own_verify}[op](s)
    return {"attend": plain_attend, "branch": plain_branch, "compact": plain_compact, "verify": plain_verify}[op](s)


def own_attend(s):
    from paper_2609_37029_gb300 import lsp
    out, lse = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device="cuda")
    lsp.lsp_prefix_attention(s["cache"], s["layer"], s["q"], s["seqs"], s["start"], out, lse, shared_len=s["case"]["shared"], scale=s["scale"],
                             workspace=s["workspace"])
    return {"out": out, "lse": lse}


def own_branch(s):
    from paper_2609_37029_gb300 import lsp
    lsp.lsp_pages_fork(s["cache"], s["src"], s["dst"])
    lsp.lsp_pages_reserve(s["cache"], s["dst"], s["add"], s["workspace"])
    lsp.lsp_pages_write(s["cache"], 0, s["dst"], s["start"], s["k_new"], s["v_new"])
    lsp.lsp_pages_trim(s["cache"], s["dst"], s["keep"])
    return {x: s[x] for x in ("k", "v", "table", "len", "refs")}


def own_compact(s):
    from paper_2609_37029_gb300 import lsp
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    lsp.lsp_pages_compact(s["cache"], s["live"], s["workspace"])
    return {x: s[x] for x in ("k", "v", "table", "refs", "live")}


def own_verify(s):
    from paper_2609_37029_gb300 import lsp
    C, B = s["y"].shape
    got, token = torch.empty(C, dtype=torch.int32, device="cuda"), torch.empty(C, dtype=torch.int32, device="cuda")
    out = torch.empty(C, B + 1, dtype=torch.int32, device="cuda")
    lsp.lsp_verify_probs(s["p"], s["q"], s["y"], s["u"], s["e"], got, token, n_draft=s["n"], out_tokens=out)
    return {"accepted": got, "next": token, "tokens": out}


def plain_attend(s):
    """Scores over the shared pages and over each request's own ones, one softmax over both."""
    c, k, v = s["case"], s["k"][s["layer"]], s["v"][s["layer"]]
    nkv, rep, d, page = c["nkv"], c["nq"] // c["nkv"], c["d"], c["page"]
    common, total, n, most = c["shared"] // page, s["total"], c["n"], s["rows"]
    first = s["table"][s["seqs"][0].long(), :common].long()
    kp = k[first].permute(1, 0, 2, 3).reshape(nkv, common * page, d).float()
    vp = v[first].permute(1, 0, 2, 3).reshape(nkv, common * page, d).float()
    rest = s["table"][s["seqs"].long(), common:common + s["own_pages"]].long().clamp(min=0)
    ko = k[rest].permute(0, 2, 1, 3, 4).reshape(n, nkv, -1, d).float()
    vo = v[rest].permute(0, 2, 1, 3, 4).reshape(n, nkv, -1, d).float()
    q = s["q"].float().reshape(total, nkv, rep, d) * s["scale"]
    start, lens = s["start"].long(), s["len"][s["seqs"].long()].long()
    row = torch.arange(total, device="cuda")
    b = torch.searchsorted(start, row, right=True) - 1
    i = row - start[b]
    rows = start[1:] - start[:-1]
    pad = (start[:-1, None] + torch.arange(most, device="cuda")).clamp(max=total - 1)
    sp = torch.matmul(q.permute(1, 0, 2, 3).reshape(nkv, total * rep, d), kp.transpose(1, 2))
    so = torch.matmul(q[pad].permute(0, 2, 1, 3, 4).reshape(n, nkv, most * rep, d), ko.transpose(2, 3)).reshape(n, nkv, most, rep, -1)
    seen = (lens - rows - common * page)[:, None] + torch.arange(1, most + 1, device="cuda")
    hidden = torch.arange(so.shape[-1], device="cuda") >= seen[..., None]
    so.masked_fill_(hidden[:, None, :, None, :], -math.inf)
    so = so.permute(0, 2, 1, 3, 4)[b, i]
    sp = sp.reshape(nkv, total, rep, common * page)
    top = so.amax(-1)
    if common:
        top = torch.maximum(top, sp.amax(-1).transpose(0, 1))
    so = torch.exp(so - top[..., None])
    sp = sp.sub_(top.transpose(0, 1)[..., None]).exp_()
    norm = so.sum(-1) + sp.sum(-1).transpose(0, 1)
    wide = torch.zeros(n, most, nkv, rep, so.shape[-1], device="cuda")
    wide[b, i] = so
    out = torch.matmul(wide.permute(0, 2, 1, 3, 4).reshape(n, nkv, most * rep, -1), vo).reshape(n, nkv, most, rep, d).permute(0, 2, 1, 3, 4)[b, i]
    out = out + torch.matmul(sp.reshape(nkv, total * rep, common * page), vp).reshape(nkv, total, rep, d).transpose(0, 1)
    out = out / norm[..., None]
    return {"out": out.reshape(total, c["nq"], d).to(s["q"].dtype), "lse": (top + torch.log(norm)).reshape(total, c["nq"])}


def plain_branch(s):
    """Fork, reserve with copies of shared last pages, write and trim, by indexing."""
    c, table, lens, refs, src, dst = s["case"], s["table"], s["len"], s["refs"], s["src"].long(), s["dst"].long()
    page, column = c["page"], torch.arange(table.shape[1], device="cuda")
    one = torch.ones((), dtype=torch.int32, device="cuda")
    # fork: the branches let go of what they hold and hold their parents' pages
    old, new = table[dst], table[src]
    refs.scatter_add_(0, old.clamp(min=0).flatten().long(), -(old >= 0).int().flatten())
    refs.scatter_add_(0, new.clamp(min=0).flatten().long(), (new >= 0).int().flatten())
    table[dst] = new
    lens[dst] = lens[src]
    # reserve: the k-th page that is asked for is the k-th lowest free one
    have = lens[dst]
    before, after = (have + page - 1) // page, (have + s["add"] + page - 1) // page
    last = table[dst, (before - 1).clamp(min=0).long()]
    part = (have % page != 0) & (s["add"] > 0)
    same = (last[:, None] == last[None, :]) & part[:, None] & part[None, :]
    earlier = torch.tril(same, -1).sum(-1)
    copy = part & (earlier < refs[last.long()] - 1)
    need = after - before + copy.int()
    free = torch.cumsum((refs == 0).int(), 0)
    base = torch.cumsum(need, 0) - need
    most = -(-c["add"] // page) + 1
    at = torch.arange(most, device="cuda")
    page_of = torch.searchsorted(free, base[:, None] + at + 1).int()
    taken = at < need[:, None]
    refs.scatter_add_(0, page_of.clamp(max=refs.numel() - 1).flatten().long(), taken.int().flatten())
    refs.scatter_add_(0, last.long(), -copy.int())
    to = torch.where(copy, page_of[:, 0], last).long()
    used = torch.arange(page, device="cuda") < (have % page)[:, None]
    for pool in (s["k"], s["v"]):
        pool[:, to] = torch.where((used & copy[:, None])[None, :, None, :, None], pool[:, last.long()], pool[:, to])
    where = (before - copy.int())[:, None] + at
    where = torch.where(taken, where, table.shape[1] - 1).long()
    rows = table[dst]
    keep = rows[:, -1:].clone()
    rows.scatter_(1, where, torch.where(taken, page_of, keep.expand_as(page_of)))
    table[dst] = rows
    lens[dst] = have + s["add"]
    # write: the new rows are the last ones of each branch
    kid = torch.arange(dst.numel(), device="cuda").repeat_interleave(c["add"])
    spot = (have[kid] + torch.arange(c["add"], device="cuda").repeat(dst.numel())).long()
    pages = table[dst[kid], spot // page].long()
    s["k"][0][pages, :, spot % page] = s["k_new"]
    s["v"][0][pages, :, spot % page] = s["v_new"]
    # trim: pages past the kept tokens are let go
    rows = table[dst]
    gone = (column >= ((s["keep"] + page - 1) // page)[:, None]) & (rows >= 0)
    refs.scatter_add_(0, rows.clamp(min=0).flatten().long(), -(gone * one).flatten())
    table[dst] = torch.where(gone, -one, rows)
    lens[dst] = torch.minimum(lens[dst], s["keep"])
    return {x: s[x] for x in ("k", "v", "table", "len", "refs")}


def plain_compact(s):
    """The k-th live page past the first `live` ones goes to the k-th free place among them."""
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    table, refs = s["table"], s["refs"]
    live = refs > 0
    count = live.sum()
    at = torch.arange(refs.numel(), device="cuda")
    hole, mover = torch.nonzero(~live & (at < count)).flatten(), torch.nonzero(live & (at >= count)).flatten()
    s["k"][:, hole] = s["k"][:, mover]
    s["v"][:, hole] = s["v"][:, mover]
    at[mover] = hole
    table.copy_(torch.where(table >= 0, at[table.clamp(min=0).long()].int(), table))
    refs[hole] = refs[mover]
    refs[mover] = 0
    s["live"].copy_(count)
    return {x: s[x] for x in ("k", "v", "table", "refs", "live")}


def plain_verify(s):
    p, q, y, n = s["p"], s["q"], s["y"].long(), s["n"]
    C, B = y.shape
    V, at = p.shape[-1], torch.arange(C, device="cuda")
    py = p[:, :B].gather(-1, y[..., None])[..., 0].float()
    qy = q.gather(-1, y[..., None])[..., 0].float() if q is not None else torch.ones_like(py)
    ok = (s["u"] * qy < py) & (torch.arange(B, device="cuda") < n[:, None])
    r = torch.cumprod(ok.int(), -1).sum(-1)
    pr, last = p[at, r].float(), r.clamp(max=B - 1)
    qr = q[at, last].float() if q is not None else (torch.arange(V, device="cuda") == y[at, last][:, None]).float()
    w = torch.where((r < n)[:, None], (pr - qr).clamp(min=0), pr)
    w = torch.where((w > 0).any(-1, keepdim=True), w, pr)
    score = torch.where(w > 0, w / s["e"], torch.full_like(w, -1.0))
    top = score.amax(-1, keepdim=True)
    token = torch.where(score == top, torch.arange(V, device="cuda"), V).amin(-1)
    token = torch.where(top[:, 0] < 0, -torch.ones_like(token), token)
    spot = torch.arange(B + 1, device="cuda")
    drafted = torch.cat([y, y[:, :1]], 1)
    out = torch.where(spot < r[:, None], drafted, torch.where(spot == r[:, None], token[:, None], -torch.ones_like(drafted)))
    return {"accepted": r.int(), "next": token.int(), "tokens": out.int()}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    if case["op"] == "attend":
        return exact_attend(prepare_plainly(case, seed))
    if case["op"] == "verify":
        return exact_verify(prepare_plainly(case, seed))
    return None     # the page operators move values and count: nothing is rounded


def prepare_plainly(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def exact_attend(s):
    """Request by request and head by head: softmax(scale q K^T) V over the tokens that a row sees."""
    c, start = s["case"], s["start"].tolist()
    k, v, page, rep = s["k"][s["layer"]], s["v"][s["layer"]], c["page"], c["nq"] // c["nkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    for b, length in enumerate(s["len"].tolist()):
        pages = s["table"][b, :-(-length // page)].long()
        rows = slice(start[b], start[b + 1])
        m = start[b + 1] - start[b]
        seen = torch.arange(length, device="cuda")[None] <= torch.arange(length - m, length, device="cuda")[:, None]
        for g in range(c["nkv"]):
            heads = slice(g * rep, (g + 1) * rep)
            kk = k[pages, g].reshape(-1, c["d"])[:length].double()
            vv = v[pages, g].reshape(-1, c["d"])[:length].double()
            x = s["q"][rows, heads].double().reshape(m * rep, -1) @ kk.T * s["scale"]
            x = x.reshape(m, rep, length).masked_fill(~seen[:, None], -math.inf)
            z = torch.logsumexp(x, -1)
            lse[rows, heads] = z
            out[rows, heads] = (torch.exp(x - z[..., None]).reshape(m * rep, length) @ vv).reshape(m, rep, -1)
    return {"out": out, "lse": lse}


def exact_verify(s):
    p, y, u = s["p"].double().cpu().numpy(), s["y"].cpu().numpy(), s["u"].double().cpu().numpy()
    q = s["q"].double().cpu().numpy() if s["q"] is not None else None
    e, n = s["e"].double().cpu().numpy(), s["n"].cpu().numpy()
    C, B = y.shape
    got, token, out = np.zeros(C, np.int32), np.zeros(C, np.int32), np.full((C, B + 1), -1, np.int32)
    for b in range(C):
        r = 0
        while r < n[b] and u[b, r] * (q[b, r, y[b, r]] if q is not None else 1.0) < p[b, r, y[b, r]]:
            r += 1
        w = p[b, r].copy()
        if r < n[b]:
            if q is None:
                w[y[b, r]] = 0.0
            else:
                w = np.maximum(w - q[b, r], 0.0)
            w = w if w.any() else p[b, r]
        got[b], token[b] = r, int(np.argmax(w / e[b])) if w.any() else -1
        out[b, :r], out[b, r] = y[b, :r], token[b]
    return {"accepted": got, "next": token, "tokens": out}
