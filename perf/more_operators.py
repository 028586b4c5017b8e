"""Workloads of a target's side that keeps its cache in 4 bits and reports probabilities, for measuring its operators.

* attend    attention of the newest rows over a paged cache held in 4 bits, the
            batch's shared prefix read once for all (lsp_prefix_attention_q4);
* write     quantising new rows into the cache and reading them back
            (lsp_pages_write_q4, lsp_pages_read);
* read      reading whole sequences back into dense rows (lsp_pages_read);
* logprobs  log probabilities of given tokens, entropies and the likeliest
            alternatives of each row of logits (lsp_logprobs).

A value x of a group of 32 dims is held as c s: s, the group's scale, is the least
number of five significant bits with 7 s >= max |x|, and c the whole number
nearest x / s (ties to even).  A head of a page is one block of bytes: the codes
c + 8 of all its slots, then their scales in bfloat16.  Element 8 w + 2 k + h of a
group is at bits 16 h + 4 k of its 32-bit word w.

Each case is a dict of plain values.  run() takes the calls a program makes of
the library where `own` is true, and computes the same results with elementary
torch operations where it is false; exact() computes them in 64 bits.
"""
import math
import random

import torch

own = False

BF16, F32 = "bf16", "f32"
GROUP = 32


# ------------------------------------------------------------------ cases
def listed():
    return [
        # two requests that each generate one token behind a short system prompt: latency
        attend_case("attend step small", n=2, nq=8, nkv=2, shared=500, own=(1, 40), q=(1, 1), page=16),
        # one token of each of 16 requests over a 32K prompt
        attend_case("attend step 32K", n=16, nq=32, nkv=8, shared=32768, own=(1, 500), q=(1, 1), page=64),
        # one token of each of 32 requests with conversations of their own, nothing shared: every byte of the cache
        attend_case("attend step own", n=32, nq=32, nkv=8, shared=0, own=(500, 16000), q=(1, 1), page=64),
        # a round's block and committed token of 16 requests over a 32K prompt: the products count
        attend_case("attend round 32K", n=16, nq=32, nkv=8, shared=32768, own=(17, 1500), q=(17, 17), page=64),
        # 32-bit rows, two query heads a key head, ragged blocks, a prompt that ends inside a page
        attend_case("attend f32 ragged", n=5, nq=4, nkv=2, d=64, dtype=F32, shared=2047, own=(1, 333), q=(1, 9), page=32),
        # a round's new rows in one layer: 16 requests of a block and the committed token
        move_case("write round", op="write", n=16, nkv=8, tokens=(17, 17), page=64),
        # the rows of a batch of prompts in one layer
        move_case("write prompts", op="write", n=8, nkv=8, tokens=(1500, 9000), page=64),
        # a few short sequences of odd lengths, 32-bit rows
        move_case("read small", op="read", n=3, nkv=2, d=64, dtype=F32, tokens=(1, 300), page=16),
        # what a drafter's prefill takes of one layer: whole prompts
        move_case("read prompts", op="read", n=8, nkv=8, tokens=(1500, 9000), page=64),
        # four emitted tokens, a small vocabulary of odd size
        logprobs_case("logprobs small", rows=4, V=32001, k=5),
        # every position of a round of 16 requests, some of whose tokens were not emitted
        logprobs_case("logprobs round", rows=272, V=151936, k=20, skip=0.3),
        # the candidates of 64 requests with 16-bit logits
        logprobs_case("logprobs 64", rows=1088, V=151936, k=5, dtype=BF16),
    ]


def attend_case(name, *, n, nq, nkv, shared, own, q, page, d=128, dtype=BF16, layers=2, mix=1):
    return named(name, op="attend", dtype=dtype, n=n, nq=nq, nkv=nkv, d=d, page=page, shared=shared,
                 own_lo=own[0], own_hi=own[1], q_lo=q[0], q_hi=q[1], layers=layers, mix=mix)


def move_case(name, *, op, n, nkv, tokens, page, d=128, dtype=BF16, layers=2, mix=1):
    return named(name, op=op, dtype=dtype, n=n, nkv=nkv, d=d, lo=tokens[0], hi=tokens[1], page=page, layers=layers, mix=mix)


def logprobs_case(name, *, rows, V, k, dtype=F32, skip=0.0, temperature=1.0, mix=1):
    return named(name, op="logprobs", dtype=dtype, rows=rows, V=V, k=k, skip=skip, temperature=temperature, mix=mix)


def named(name, **case):
    return {**({"name": name} if name else {}), **case}


def spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "write", "read", "logprobs", "logprobs"])
    most = {case["name"]: work(case) for case in listed()}
    if op == "attend":
        while True:
            dtype = F32 if rng.random() < 0.2 else BF16
            nq, nkv = rng.choice([(4, 2), (8, 2), (32, 8), (40, 8), (8, 8), (16, 1), (6, 2), (28, 4)])
            kind = rng.random()
            q = (1, 1) if kind < 0.45 else (1, 17) if kind < 0.85 else (20, spread(rng, 40, 600))
            shared = 0 if rng.random() < 0.25 else spread(rng, 16, 131072 if dtype == BF16 else 8192)
            lo = spread(rng, 1, 500)
            case = attend_case("", n=spread(rng, 1, 48), nq=nq, nkv=nkv, d=rng.choice([64, 128]), dtype=dtype, shared=shared,
                               own=(lo, max(lo, spread(rng, 8, 16000 if shared < 4096 else 2000))), q=q,
                               page=rng.choice([16, 32, 64, 128, 256]), layers=rng.choice([1, 2, 3]), mix=rng.randrange(1 << 20))
            w = work(case)
            if w["flops"] <= most["attend round 32K"]["flops"] / (1 if dtype == BF16 else 32) and w["bytes"] <= most["attend step own"]["bytes"]:
                return case
    if op in ("write", "read"):
        while True:
            lo = spread(rng, 1, 2000)
            case = move_case("", op=op, n=spread(rng, 1, 64), nkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128]),
                             dtype=rng.choice([BF16, BF16, F32]), tokens=(lo, spread(rng, lo, 9000)),
                             page=rng.choice([16, 32, 64, 128, 256]), layers=rng.choice([1, 2, 3]), mix=rng.randrange(1 << 20))
            if work(case)["bytes"] <= most[op + " prompts"]["bytes"]:
                return case
    while True:
        case = logprobs_case("", rows=spread(rng, 1, 1088), V=spread(rng, 1000, 151936), k=rng.choice([0, 1, 5, 20, 32]),
                             dtype=rng.choice([F32, BF16]), skip=rng.choice([0.0, 0.0, 0.4]), temperature=rng.choice([1.0, 1.0, 0.7]),
                             mix=rng.randrange(1 << 20))
        if work(case)["bytes"] <= most["logprobs 64"]["bytes"]:
            return case


# ------------------------------------------------------------------ sizes of a case
def size_of(case):
    return 2 if case["dtype"] == BF16 else 4


def torch_type(case):
    return torch.bfloat16 if case["dtype"] == BF16 else torch.float32


def attend_lens(case):
    """(rows, tokens past the shared ones) of each request."""
    r = random.Random(case["mix"])
    rows = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["n"])]
    return rows, [max(x, r.randint(case["own_lo"], max(case["own_lo"], case["own_hi"]))) for x in rows]


def move_lens(case):
    r = random.Random(case["mix"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["n"])]


def emitted(case):
    """Which rows of logits have a token."""
    r = random.Random(case["mix"])
    return [r.random() >= case["skip"] for _ in range(case["rows"])]


def work(case):
    es = size_of(case)
    if case["op"] == "attend":
        rows, tail = attend_lens(case)
        nq, nkv, d, shared = case["nq"], case["nkv"], case["d"], case["shared"]
        keys = shared + sum(tail)
        seen = sum(x * shared + sum(o - x + i + 1 for i in range(x)) for x, o in zip(rows, tail))
        return {"bytes": 2 * keys * nkv * d * 9 // 16 + 2 * sum(rows) * nq * d * es + 4 * sum(rows) * nq, "flops": 4 * seen * nq * d}
    if case["op"] in ("write", "read"):
        values = 2 * sum(move_lens(case)) * case["nkv"] * case["d"]
        return {"bytes": values * (2 if case["op"] == "write" else 1) * (16 * es + 9) // 16, "flops": values * (4 if case["op"] == "write" else 1)}
    live = sum(emitted(case))
    return {"bytes": live * case["V"] * es + case["rows"] * (12 + 8 * case["k"]), "flops": 5 * live * case["V"]}


# ------------------------------------------------------------------ the held form
def scale_of(x):
    """Scales [..., d / 32, 1] of rows x [..., d] in fp32."""
    a = x.unflatten(-1, (-1, GROUP)).abs().amax(-1, keepdim=True)
    bits = (a / torch.full_like(a, 7.0)).view(torch.int32) & ~0x7FFFF
    low = bits.view(torch.float32)
    return torch.where(7 * low < a, (bits + 0x80000).view(torch.float32), low)


def codes_of(x, s):
    """Whole numbers -7..7 of rows x [..., d]; 64 bits, so that no quotient moves across a border."""
    y = x.unflatten(-1, (-1, GROUP))
    return torch.where(s > 0, torch.round(y.double() / s.double()), torch.zeros((), dtype=torch.float64, device=x.device)).to(torch.int32)


def pack(x):
    """(codes [..., d / 2] uint8, scales [..., d / 32] bfloat16) of rows x [..., d]."""
    s = scale_of(x.float())
    c = (codes_of(x.float(), s) + 8).flatten(-2).unflatten(-1, (-1, 4, 2)).transpose(-1, -2)      # [..., words, h, k]
    c = c.unflatten(-1, (2, 2))
    return (c[..., 0] | c[..., 1] << 4).to(torch.uint8).flatten(-3), s[..., 0].to(torch.bfloat16)


def unpack(codes, scales):
    """Rows [..., d] in fp32."""
    b = codes.unflatten(-1, (-1, 2, 2)).to(torch.int32)                                           # [..., words, h, byte]
    c = torch.stack([b & 15, b >> 4], -1).flatten(-2).transpose(-1, -2).flatten(-3) - 8
    return (c.unflatten(-1, (-1, GROUP)) * scales.float()[..., None]).flatten(-2)


def parts(pool):
    """(codes [layers][pages][nkv][page][d / 2], scales [...][d / 32]) as views of a pool's bytes."""
    page, held = pool.shape[3:]
    d = held * 16 // 9
    block = pool.flatten(3)
    return block[..., :page * d // 2].unflatten(-1, (page, -1)), block[..., page * d // 2:].view(torch.bfloat16).unflatten(-1, (page, -1))


# ------------------------------------------------------------------ inputs
def generator(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g


def whole(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def new_pool(case, pages, g, lean=None):
    """Pools of quantised normal values: k, v [layers][pages][nkv][page][9 d / 16] bytes.  lean: (page, direction)
    of keys that lie the same way."""
    shape = (case["layers"], pages, case["nkv"], case["page"], case["d"])
    pools = []
    for i in range(2):
        pool = torch.empty(shape[:-1] + (case["d"] * 9 // 16,), dtype=torch.uint8, device="cuda")
        codes, scales = parts(pool)
        for layer in range(case["layers"]):
            for at in range(0, pages, 512):
                x = torch.randn((min(512, pages - at),) + shape[2:], generator=g, device="cuda") + (0.1 if i else 0.0)
                if i == 0 and lean is not None and at <= lean[0] < at + 512:
                    x[lean[0] - at, :, :4] += 2.0 * lean[1][:, None]
                codes[layer, at:at + 512], scales[layer, at:at + 512] = pack(x)
        pools.append(pool)
    return pools


def cache_of(k, v, table, lens, refs):
    """The handle that a program keeps of its cache, beside the tensors themselves."""
    s = {"k": k, "v": v, "table": table, "len": lens, "refs": refs}
    if own:
        from paper_2609_37029_gb300 import lsp
        s["cache"] = lsp.make_kv_cache(k, v, table, lens, refs)
    return s


def starts(rows):
    at = [0]
    for x in rows:
        at.append(at[-1] + x)
    return at


def prepare(case, seed):
    make = {"attend": prepare_attend, "write": prepare_move, "read": prepare_move, "logprobs": prepare_logprobs}[case["op"]]
    return {**make(case, seed), "case": case}


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
    lean = torch.randn(case["nkv"], d, generator=g, device="cuda") * 0.5
    k, v = new_pool(case, pages, g, (int(table[0, 0]), lean))
    q = torch.randn(sum(rows), case["nkv"], case["nq"] // case["nkv"], d, generator=g, device="cuda") * 1.5 + lean[None, :, None]
    s = cache_of(k, v, table.cuda(), whole([case["shared"] + x for x in tail]), refs.cuda())
    s.update(q=q.reshape(sum(rows), case["nq"], d).to(torch_type(case)).contiguous(), seqs=whole(list(range(n))), start=whole(starts(rows)),
             total=sum(rows), rows=max(rows), own_pages=max(held) - common, layer=case["layers"] - 1, scale=d ** -0.5)
    if own:
        from paper_2609_37029_gb300 import lsp
        nbytes = lsp.lsp_prefix_attention_q4_workspace_bytes(s["cache"], s["q"].dtype, case["nq"], n, sum(rows))
        s["workspace"] = torch.empty(max(1, nbytes), dtype=torch.uint8, device="cuda")
    return s


def prepare_move(case, seed):
    """Sequences with shuffled pages that end in the rows concerned: all of their tokens to be read, or room behind
    some earlier ones for what is to be written.  Keys and values of a few dims are larger, as keys' are."""
    g, n, page = generator(seed), case["n"], case["page"]
    rows = move_lens(case)
    before = [0] * n if case["op"] == "read" else [(37 * b) % 200 for b in range(n)]
    held = [-(-(x + y) // page) for x, y in zip(before, rows)]
    pages = sum(held) + 3
    place = torch.randperm(pages, generator=g, device="cuda")[:sum(held)].to(torch.int32).cpu()
    table, refs, at = torch.full((n, max(held) + 1), -1, dtype=torch.int32), torch.zeros(pages, dtype=torch.int32), 0
    for b in range(n):
        table[b, :held[b]] = place[at:at + held[b]]
        at += held[b]
    refs[place.long()] = 1
    k, v = new_pool(case, pages, g)
    s = cache_of(k, v, table.cuda(), whole([x + y for x, y in zip(before, rows)]), refs.cuda())
    total, size = sum(rows), torch.exp(torch.randn(case["nkv"], case["d"], generator=g, device="cuda"))
    s.update(seqs=whole(list(range(n))), start=whole(starts(rows)), total=total, layer=case["layers"] - 1)
    if case["op"] == "write":
        shape = (total, case["nkv"], case["d"])
        s.update({x: (torch.randn(shape, generator=g, device="cuda") * size).to(torch_type(case)) for x in ("k_new", "v_new")})
    return s


def prepare_logprobs(case, seed):
    """Logits with a long flat tail and a few likely tokens, some banned; tokens that were drawn from them."""
    g, rows, V = generator(seed), case["rows"], case["V"]
    z = torch.empty(rows, V, dtype=torch_type(case), device="cuda")
    token = torch.empty(rows, dtype=torch.int32, device="cuda")
    for at in range(0, rows, 64):
        x = torch.randn(min(64, rows - at), V, generator=g, device="cuda") * 2.5
        x[torch.rand(x.shape, generator=g, device="cuda") < 0.001] = -math.inf
        z[at:at + 64] = x
        token[at:at + 64] = (z[at:at + 64].float() - torch.empty_like(x).exponential_(generator=g).log()).argmax(-1)
    gone = torch.tensor([not x for x in emitted(case)], device="cuda")
    return {"z": z, "token": torch.where(gone, -torch.ones_like(token), token)}


# ------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return {"attend": own_attend, "write": own_write, "read": own_read, "logprobs": own_logprobs}[op](s)
    return {"attend": plain_attend, "write": plain_write, "read": plain_read, "logprobs": plain_logprobs}[op](s)


def own_attend(s):
    from paper_2609_37029_gb300 import lsp
    out, lse = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device="cuda")
    lsp.lsp_prefix_attention_q4(s["cache"], s["layer"], s["q"], s["seqs"], s["start"], out, lse, shared_len=s["case"]["shared"],
                                scale=s["scale"], workspace=s["workspace"])
    return {"out": out, "lse": lse}


def new_rows(s):
    shape = (s["total"], s["case"]["nkv"], s["case"]["d"])
    return [torch.empty(shape, dtype=torch_type(s["case"]), device="cuda") for _ in range(2)]


def own_write(s):
    from paper_2609_37029_gb300 import lsp
    k, v = new_rows(s)
    lsp.lsp_pages_write_q4(s["cache"], s["layer"], s["seqs"], s["start"], s["k_new"], s["v_new"])
    lsp.lsp_pages_read(s["cache"], s["layer"], s["seqs"], s["start"], k, v)
    return {"k": k, "v": v}


def own_read(s):
    from paper_2609_37029_gb300 import lsp
    k, v = new_rows(s)
    lsp.lsp_pages_read(s["cache"], s["layer"], s["seqs"], s["start"], k, v)
    return {"k": k, "v": v}


def own_logprobs(s):
    from paper_2609_37029_gb300 import lsp
    rows, k = s["case"]["rows"], s["case"]["k"]
    logprob, entropy = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    top, top_logprob = torch.empty(rows, k, dtype=torch.int32, device="cuda"), torch.empty(rows, k, device="cuda")
    lsp.lsp_logprobs(s["z"], s["token"], logprob, entropy, top, top_logprob, temperature=s["case"]["temperature"])
    return {"logprob": logprob, "entropy": entropy, "top": top, "top_logprob": top_logprob}


def plain_attend(s):
    """Scores over the shared pages and over each request's own ones, one softmax over both."""
    c = s["case"]
    (kc, ks), (vc, vs) = parts(s["k"]), parts(s["v"])
    kc, ks, vc, vs = (x[s["layer"]] for x in (kc, ks, vc, vs))
    nkv, rep, d, page = c["nkv"], c["nq"] // c["nkv"], c["d"], c["page"]
    common, total, n, most = c["shared"] // page, s["total"], c["n"], s["rows"]
    first = s["table"][s["seqs"][0].long(), :common].long()
    kp = unpack(kc[first], ks[first]).permute(1, 0, 2, 3).reshape(nkv, common * page, d)
    vp = unpack(vc[first], vs[first]).permute(1, 0, 2, 3).reshape(nkv, common * page, d)
    rest = s["table"][s["seqs"].long(), common:common + s["own_pages"]].long().clamp(min=0)
    ko = unpack(kc[rest], ks[rest]).permute(0, 2, 1, 3, 4).reshape(n, nkv, -1, d)
    vo = unpack(vc[rest], vs[rest]).permute(0, 2, 1, 3, 4).reshape(n, nkv, -1, d)
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


def places(s):
    """(page, slot) of each row: an entry's rows are the last tokens of its sequence."""
    row, start, page = torch.arange(s["total"], device="cuda"), s["start"].long(), s["case"]["page"]
    b = torch.searchsorted(start, row, right=True) - 1
    seq = s["seqs"].long()[b]
    spot = s["len"].long()[seq] - start[b + 1] + row
    return s["table"][seq, spot // page].long(), spot % page


def plain_write(s):
    page, slot = places(s)
    for pool, new in ((s["k"], s["k_new"]), (s["v"], s["v_new"])):
        codes, scales = parts(pool)
        codes[s["layer"]][page, :, slot], scales[s["layer"]][page, :, slot] = pack(new)
    return plain_read(s)


def plain_read(s):
    page, slot = places(s)
    rows = []
    for pool in (s["k"], s["v"]):
        codes, scales = parts(pool)
        rows.append(unpack(codes[s["layer"]][page, :, slot], scales[s["layer"]][page, :, slot]).to(torch_type(s["case"])))
    return {"k": rows[0], "v": rows[1]}


def plain_logprobs(s):
    """Rows without a token: -inf, 0 and no alternatives."""
    c, V, k = s["case"], s["case"]["V"], s["case"]["k"]
    live = s["token"] >= 0
    z = s["z"].float() / c["temperature"]
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    norm = e.sum(-1, keepdim=True)
    lse = top + torch.log(norm)
    logp = z - lse
    entropy = -torch.where(e > 0, e / norm * logp, torch.zeros_like(e)).sum(-1)
    logprob = logp.gather(-1, s["token"].clamp(min=0).long()[:, None])[:, 0]
    column, tokens, values, left = torch.arange(V, device="cuda"), [], [], s["z"].float()
    for _ in range(k):                                  # ties go to the lowest index
        best = left.amax(-1, keepdim=True)
        at = torch.where(left == best, column, V).amin(-1)
        tokens.append(torch.where(live, at, -torch.ones_like(at)))
        values.append(torch.where(live, logp.gather(-1, at[:, None])[:, 0], torch.full_like(entropy, -math.inf)))
        left = left.scatter(-1, at[:, None], -math.inf)
    none = torch.empty(c["rows"], 0, device="cuda")
    return {"logprob": torch.where(live, logprob, torch.full_like(logprob, -math.inf)), "entropy": torch.where(live, entropy, torch.zeros_like(entropy)),
            "top": torch.stack(tokens, -1).int() if k else none.int(), "top_logprob": torch.stack(values, -1) if k else none}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare_plainly(case, seed)
    return {"attend": exact_attend, "write": exact_write, "read": exact_read, "logprobs": exact_logprobs}[case["op"]](s)


def prepare_plainly(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def held_values(pool, layer, pages, head, d):
    """[tokens][d] in 64 bits of a head of some pages, from the definition of the bytes."""
    page = pool.shape[3]
    block = pool[layer, pages, head].reshape(len(pages), -1)
    words = block[:, :page * d // 2].reshape(-1, d // 8, 4).to(torch.int64)
    word = sum(words[..., i] << (8 * i) for i in range(4))
    c = torch.stack([(word >> (16 * (e & 1) + 4 * (e >> 1))) & 15 for e in range(8)], -1).reshape(-1, d // GROUP, GROUP) - 8
    raw = block[:, page * d // 2:].reshape(-1, d // GROUP, 2).to(torch.int64)
    scale = ((raw[..., 0] | raw[..., 1] << 8) << 16).to(torch.int32).view(torch.float32).double()
    return (c.double() * scale[..., None]).reshape(-1, d)


def exact_attend(s):
    """Request by request and head by head: softmax(scale q K^T) V over the tokens that a row sees."""
    c, start = s["case"], s["start"].tolist()
    page, rep, d = c["page"], c["nq"] // c["nkv"], c["d"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    for b, length in enumerate(s["len"].tolist()):
        pages = s["table"][b, :-(-length // page)].long()
        rows = slice(start[b], start[b + 1])
        m = start[b + 1] - start[b]
        seen = torch.arange(length, device="cuda")[None] <= torch.arange(length - m, length, device="cuda")[:, None]
        for g in range(c["nkv"]):
            heads = slice(g * rep, (g + 1) * rep)
            kk, vv = (held_values(s[x], s["layer"], pages, g, d)[:length] for x in ("k", "v"))
            x = s["q"][rows, heads].double().reshape(m * rep, -1) @ kk.T * s["scale"]
            x = x.reshape(m, rep, length).masked_fill(~seen[:, None], -math.inf)
            z = torch.logsumexp(x, -1)
            lse[rows, heads] = z
            out[rows, heads] = (torch.exp(x - z[..., None]).reshape(m * rep, length) @ vv).reshape(m, rep, -1)
    return {"out": out, "lse": lse}


def exact_write(s):
    """The scale by its binary exponent and 16 steps of its mantissa, the code by its distance to the scale's multiples."""
    rows = {}
    for x in ("k", "v"):
        y = s[x + "_new"].double().reshape(s["total"], -1, GROUP)
        a = y.abs().amax(-1, keepdim=True)
        mantissa, exponent = torch.frexp(a / 7)             # mantissa in [1/2, 1): 16 / 32 .. 31 / 32
        unit = ((exponent.to(torch.int64) - 5 + 1023) << 52).view(torch.float64)
        scale = torch.ceil(mantissa * 32) * unit
        scale = torch.where(7 * (scale - unit) >= a, scale - unit, scale)
        low = torch.floor(y / scale)
        rest = y - low * scale
        up = (rest > scale / 2) | ((rest == scale / 2) & (low % 2 != 0))
        rows[x] = torch.where(a > 0, (low + up) * scale, torch.zeros_like(y)).reshape(s[x + "_new"].shape)
    return rows


def exact_read(s):
    c, rows = s["case"], {x: [] for x in ("k", "v")}
    for b, length in enumerate(s["len"].tolist()):
        pages = s["table"][b, :-(-length // c["page"])].long()
        for x in rows:
            rows[x].append(torch.stack([held_values(s[x], s["layer"], pages, g, c["d"])[:length] for g in range(c["nkv"])], 1))
    return {x: torch.cat(y) for x, y in rows.items()}


def exact_logprobs(s):
    c, k = s["case"], s["case"]["k"]
    logprob = torch.full((c["rows"],), -math.inf, dtype=torch.float64, device="cuda")
    entropy = torch.zeros_like(logprob)
    top = torch.full((c["rows"], k), -1, dtype=torch.int32, device="cuda")
    top_logprob = torch.full((c["rows"], k), -math.inf, dtype=torch.float64, device="cuda")
    for r, token in enumerate(s["token"].tolist()):
        if token < 0:
            continue
        z = s["z"][r].double() / c["temperature"]
        logp = z - torch.logsumexp(z, -1)
        logprob[r] = logp[token]
        entropy[r] = torch.special.entr(torch.exp(logp)).sum()
        at = torch.sort(s["z"][r].float(), descending=True, stable=True).indices[:k]
        top[r], top_logprob[r] = at.int(), logp[at]
    return {"logprob": logprob, "entropy": entropy, "top": top, "top_logprob": top_logprob}
