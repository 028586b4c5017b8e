"""lsp_prefix_attention behind calls that change what it reads: lengths, tables and row ranges are those of the
calls before it on the stream, however closely they follow one another.  Tolerances: those of the other tests of
this call."""
import pytest
import torch

from tests.gpu_common import lsp_lib
from tests.target_common import oracle_cache
from tests.test_gpu_prefix_attn import case, compare

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


# one row a sequence (several warps share an output row), and several (a warp has several heads)
@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("dtype,rows", [("bf16", 1), ("bf16", 20), ("f32", 1), ("f32", 20)])
def test_lengths_of_the_call_before(lsp, dtype, rows, graph):
    n, shared, page, steps = 9, 300, 16, 12
    lens = [700 + 11 * i for i in range(n)]
    pool, t, q = case(lens, [rows] * n, shared, nq=8, nkv=2, d=64, dtype=dtype, page=page)
    c = lsp.make_kv_cache(*pool, *t)
    ids = torch.arange(n, dtype=torch.int32, device="cuda")
    start = (torch.arange(n + 1, device="cuda") * rows).to(torch.int32)
    ws = torch.empty(lsp.lsp_prefix_attention_workspace_bytes(c, 8, n, n * rows), dtype=torch.uint8, device="cuda")
    # every step cuts the sequences to other lengths, some of them not at all
    new = [[x - 37 * (k + 1) + 5 * ((i + k) % 3) if (i + k) % 4 else x for i, x in enumerate(lens)] for k in range(steps)]
    for k in range(1, steps):
        new[k] = [min(a, b) for a, b in zip(new[k - 1], new[k])]
    cuts = torch.tensor(new, dtype=torch.int32, device="cuda")
    outs = [(torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")) for _ in range(steps)]
    keep = [x.clone() for x in t]

    def calls():
        for x, y in zip(t, keep):
            x.copy_(y)
        for k in range(steps):
            lsp.lsp_pages_trim(c, ids, cuts[k])
            lsp.lsp_prefix_attention(c, 0, q, ids, start, *outs[k], shared_len=shared, scale=0.125, workspace=ws)

    calls()
    torch.cuda.synchronize()
    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            calls()
        for out, z in outs:
            out.fill_(9), z.fill_(9)
        for _ in range(3):
            g.replay()
        torch.cuda.synchronize()
    for k in (0, 1, 5, steps - 1):
        oc = oracle_cache(*pool, keep[0], torch.tensor(new[k]), keep[2])
        compare(oc, q, list(range(n)), [rows] * n, *outs[k], scale=0.125)
    assert t[1].tolist() == new[-1]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_row_ranges_and_sequences_of_the_call_before(lsp, dtype):
    """start and seqs change between two calls, by copies on the stream."""
    lens = [400, 333, 290, 511]
    pool, t, q = case(lens, [3] * 4, 256, nq=4, nkv=2, d=128, dtype=dtype, page=32)
    c = lsp.make_kv_cache(*pool, *t)
    ws = torch.empty(lsp.lsp_prefix_attention_workspace_bytes(c, 4, 4, 12), dtype=torch.uint8, device="cuda")
    ids, start = (torch.zeros(x, dtype=torch.int32, device="cuda") for x in (4, 5))
    plans = [([0, 1, 2, 3], [3, 3, 3, 3]), ([3, 0, 2, 1], [1, 5, 0, 6]), ([2, 99, 1, 0], [4, 2, 4, 2]), ([1, 3, 0, 2], [9, 1, 1, 1])] * 4
    dev = [tuple(torch.tensor(x, dtype=torch.int32, device="cuda") for x in (s, [sum(r[:i]) for i in range(5)])) for s, r in plans]
    outs = [(torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")) for _ in plans]
    torch.cuda.synchronize()
    for (s, r), o in zip(dev, outs):
        ids.copy_(s)
        start.copy_(r)
        lsp.lsp_prefix_attention(c, 0, q, ids, start, *o, shared_len=256, scale=0.1, workspace=ws)
    torch.cuda.synchronize()
    oc = oracle_cache(*pool, *t)
    for (s, r), o in zip(plans, outs):
        compare(oc, q, s, r, *o, scale=0.1)
