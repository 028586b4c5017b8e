"""lsp_verify_probs against the oracle.  The acceptance products, the residual and the scores are
single fp32 operations, so every token and length has to be equal, ties and empty rows among them."""
import numpy as np
import pytest
import torch

from oracle.target import verify_probs
from tests.gpu_common import lsp_lib

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


def probs(C, B, V, rng, agree=0.9):
    z = rng.randn(C, B + 1, V) * 3
    zq = agree * z[:, :B] + np.sqrt(1 - agree ** 2) * 3 * rng.randn(C, B, V)

    def soft(x):
        e = np.exp(x - x.max(-1, keepdims=True))
        return e / e.sum(-1, keepdims=True)
    p = soft(z)
    p[p * V < 0.7] = 0                                  # as a filter of unlikely tokens leaves them
    return p.astype(np.float32), soft(zq).astype(np.float32) if B else np.zeros((C, 0, V), np.float32)


def check(lsp, p, q, y, n, u, e, bits=0):
    """p, q: CUDA tensors (q may be None); y, n, u, e: numpy."""
    C, B = y.shape
    dev = lambda x, t: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to("cuda", t)
    acc, tok = (torch.full((C,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    out = torch.full((C, B + 1), -7, dtype=torch.int32, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    lsp.lsp_verify_probs(p, q, dev(y, torch.int32), dev(u, torch.float32), dev(e, torch.float32), acc, tok,
                         n_draft=dev(n, torch.int32), out_tokens=out, dev_error=err)
    torch.cuda.synchronize()
    pn, qn = p.float().cpu().numpy(), None if q is None else q.float().cpu().numpy()
    for b in range(C):
        m = B if n is None else min(max(int(n[b]), 0), B)
        r, t = verify_probs(pn[b], None if qn is None else qn[b], y[b], m, u[b], e[b])
        assert (int(acc[b]), int(tok[b])) == (r, t), b
        assert out[b].tolist() == list(y[b, :r]) + [t] + [-1] * (B - r), b
    assert int(err.item()) == bits
    return acc.cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("C,B,V", [(1, 1, 1), (3, 4, 7), (2, 0, 50), (5, 16, 1000), (1, 40, 4096), (7, 5, 32001), (40, 3, 513)])
def test_equals_the_oracle(lsp, C, B, V, draft, dtype):
    rng = np.random.RandomState(C * 1000 + B + V)
    p, q = probs(C, B, V, rng, 0.99)
    y = rng.randint(0, V, (C, B))
    for b in range(C):
        for i in range(B):
            y[b, i] = rng.choice(V, p=q[b, i].astype(np.float64) / q[b, i].astype(np.float64).sum()) if draft else p[b, i].argmax()
    n = rng.randint(0, B + 1, C)
    u, e = rng.rand(C, B).astype(np.float32), rng.exponential(size=(C, V)).astype(np.float32)
    p, q = (torch.from_numpy(x).cuda().to(dtype) for x in (p, q))
    check(lsp, p, q if draft else None, y, n, u, e)
    check(lsp, p, q if draft else None, y, None, u, e)


def test_whole_vocabulary_and_every_outcome(lsp):
    rng = np.random.RandomState(3)
    C, B, V = 16, 16, 151936
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(C, B + 1, V, generator=g, device="cuda") * 3
    p = torch.softmax(z, -1)
    q = torch.softmax(z[:, :B] + 0.2 * torch.randn(C, B, V, generator=g, device="cuda"), -1)
    y = (q / torch.empty_like(q).exponential_(generator=g)).argmax(-1).cpu().numpy()
    got = check(lsp, p, q, y, None, rng.rand(C, B) * 0.99, rng.exponential(size=(C, V)))
    assert len(set(got.tolist())) > 3                   # rejections at several places


@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 0), (8, 0), (8, 1)])
def test_padded_rows_and_odd_addresses(lsp, pad, shift):
    rng = np.random.RandomState(pad + shift)
    C, B, V = 3, 4, 1001 if pad == 3 else 1000
    p, q = probs(C, B, V, rng)
    y = rng.randint(0, V, (C, B))
    wide = []
    for x in (p, q):
        flat = torch.full((x.shape[0] * x.shape[1] * (V + pad) + shift,), float("nan"), device="cuda")
        w = flat[shift:].view(x.shape[0], x.shape[1], V + pad)[..., :V]
        w.copy_(torch.from_numpy(x))
        wide.append(w)
    check(lsp, *wide, y, None, rng.rand(C, B), rng.exponential(size=(C, V)))


def test_ties_empty_rows_and_bad_tokens(lsp):
    C, B, V = 6, 2, 4000
    p, q = np.zeros((C, B + 1, V), np.float32), np.zeros((C, B, V), np.float32)
    y, u, e = np.zeros((C, B), int), np.full((C, B), 0.5, np.float32), np.ones((C, V), np.float32)
    p[0, 0, [3, 900, 3999]] = 0.25                      # rejected at once; a tie: the lowest
    p[0, 0, 0], q[0, 0, 0] = 0.0, 1.0
    p[1, :, 7], q[1, :, 7], q[1, :, 0] = 1.0, 2.0, 1.0  # nothing left of p - q: drawn from p
    y[2] = [V, 5]                                       # a token outside
    p[2, 0, 10] = 1.0
    p[3, :, 0], q[3, :, 0] = 1.0, 1.0                   # accepted throughout, then p is empty
    p[3, 2] = 0.0
    p[4] = np.nan                                       # no weight is above 0
    p[5, 0, 1:3] = [0.5, 0.25]
    e[5, 1:3] = [np.inf, 1.0]                           # a variate of infinity never wins
    y[5] = 9
    q[5, 0, 9] = 1.0
    p, q = torch.from_numpy(p).cuda(), torch.from_numpy(q).cuda()
    check(lsp, p, q, y, None, u, e, lsp.LSP_DEV_BAD_TOKEN)
    check(lsp, p, q, np.abs(y) % V, np.array([0, 1, 2, -1, 3, 1]), u, e, lsp.LSP_DEV_BAD_DELTA)


def test_runs_twice_alike_in_a_graph_and_on_a_side_stream(lsp):
    rng = np.random.RandomState(11)
    C, B, V = 9, 8, 5000
    p, q = (torch.from_numpy(x).cuda() for x in probs(C, B, V, rng, 0.995))
    y = torch.from_numpy(rng.randint(0, V, (C, B)).astype(np.int32)).cuda()
    u, e = torch.from_numpy(rng.rand(C, B).astype(np.float32)).cuda(), torch.from_numpy(rng.exponential(size=(C, V)).astype(np.float32)).cuda()
    res = [torch.zeros(2, C, dtype=torch.int32, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    lsp.lsp_verify_probs(p, q, y, u, e, res[0][0], res[0][1])
    side = torch.cuda.Stream()
    lsp.lsp_verify_probs(p, q, y, u, e, res[1][0], res[1][1], stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lsp.lsp_verify_probs(p, q, y, u, e, res[2][0], res[2][1])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(res[0], res[1]) and torch.equal(res[0], res[2])
