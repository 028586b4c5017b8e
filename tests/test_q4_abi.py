"""Refusals of the calls over a cache held in 4 bits and of lsp_logprobs: by the library, of bare addresses and sizes,
and by the binding, of tensors (no GPU needed: nothing is launched)."""
import pytest
import torch

from tests.test_target_abi import cache as plain_cache
from tests.test_target_binding import ints, no_gpu, refused


@pytest.fixture(scope="module")
def lsp():
    from paper_2609_37029_gb300 import build
    build.build()
    from paper_2609_37029_gb300 import lsp as mod
    return mod


def cache(lsp, **kw):
    c = plain_cache(lsp)
    c.dtype = lsp.LSP_DTYPE_Q4
    c.s_slot, c.s_head, c.s_page, c.s_layer = 72, 72 * 64, 144 * 64, 144 * 64 * 100
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def test_the_cache(lsp):
    f = lsp._f["lsp_pages_fork"]
    assert lsp.lsp_pages_workspace_bytes(cache(lsp)) == lsp.lsp_pages_workspace_bytes(plain_cache(lsp)) > 0
    assert f(cache(lsp), 16, 16, 0, None, None) == lsp.LSP_OK
    for kw in (dict(s_slot=64), dict(s_slot=128), dict(s_head=72 * 64 - 16), dict(s_head=72 * 64 + 8), dict(s_page=72 * 63), dict(s_layer=2 ** 40),
               dict(s_page=-144 * 64), dict(d=32), dict(page=8), dict(page=48)):
        c = cache(lsp, **kw)
        assert f(c, 16, 16, 1, None, None) == lsp.LSP_ERR_SHAPE, kw
        assert lsp.lsp_pages_workspace_bytes(c) == 0
        assert lsp._f["lsp_prefix_attention_q4_workspace_bytes"](c, 0, 4, 1, 1) == 0
    # an axis of one has no stride; any order of the others
    assert f(cache(lsp, layers=1, nkv=1, s_layer=3, s_head=5), 16, 16, 0, None, None) == lsp.LSP_OK
    assert f(cache(lsp, s_page=72 * 64, s_head=72 * 64 * 100), 16, 16, 0, None, None) == lsp.LSP_OK
    assert f(cache(lsp, k=0x1008), 16, 16, 1, None, None) == lsp.LSP_ERR_ARG
    assert f(cache(lsp, dtype=3), 16, 16, 1, None, None) == lsp.LSP_ERR_ARG


def test_each_kind_of_cache_has_its_calls(lsp):
    A, q4, bf16, bf16_cache = lsp.LSP_ERR_ARG, cache(lsp), 0, plain_cache(lsp)
    assert lsp._f["lsp_pages_write"](q4, 0, 16, 16, 1, 0x7000, 0x8000, 256, 5, None, None) == A
    assert lsp._f["lsp_pages_write_q4"](bf16_cache, 0, 16, 16, 1, 0x7000, 0x8000, bf16, 256, 5, None, None) == A
    attend = [0, 0x7000, 1024, 8, 16, 16, 2, 6, 10, 0.1, 0x8000, None, 0x9000, 1 << 40, None, None]
    assert lsp._f["lsp_prefix_attention"](q4, *attend) == A
    assert lsp._f["lsp_prefix_attention_q4"](bf16_cache, *attend[:2], bf16, *attend[2:]) == A
    assert lsp.lsp_prefix_attention_workspace_bytes(q4, 4, 1, 1) == 0
    assert lsp._f["lsp_prefix_attention_q4_workspace_bytes"](bf16_cache, bf16, 4, 1, 1) == 0
    assert lsp._f["lsp_prefix_attention_q4_workspace_bytes"](q4, lsp.LSP_DTYPE_Q4, 4, 1, 1) == 0
    assert lsp._f["lsp_prefix_attention_q4_workspace_bytes"](None, bf16, 4, 1, 1) == 0
    # reading: the cache's own type, or either of a cache in 4 bits
    read = [0, 16, 16, 1, 0x7000, 0x8000]
    assert lsp._f["lsp_pages_read"](bf16_cache, *read, lsp.LSP_DTYPE_F32, 256, 5, None, None) == A
    assert lsp._f["lsp_pages_read"](q4, *read, lsp.LSP_DTYPE_Q4, 256, 5, None, None) == A


@pytest.mark.parametrize("name", ["lsp_pages_write_q4", "lsp_pages_read"])
def test_rows(lsp, name):
    A, S = lsp.LSP_ERR_ARG, lsp.LSP_ERR_SHAPE
    base = dict(cache=cache(lsp), layer=0, seqs=16, start=16, n=1, k=0x7000, v=0x8000, dtype=1, stride=256, total=5, err=None, stream=None)

    def call(**kw):
        return lsp._f[name](*{**base, **kw}.values())
    for kw in (dict(cache=None), dict(layer=2), dict(layer=-1), dict(seqs=None), dict(start=None), dict(n=-1), dict(total=-1), dict(k=None),
               dict(v=None), dict(k=0x7008), dict(v=0x8004), dict(dtype=7), dict(seqs=18), dict(start=17), dict(err=0x9001)):
        assert call(**kw) == A, kw
    for kw in (dict(stride=255), dict(stride=258), dict(total=2 ** 28 + 1), dict(stride=2 ** 40)):
        assert call(**kw) == S, kw
    assert call(total=0, k=None, v=None) == lsp.LSP_OK
    assert call(n=0) == lsp.LSP_OK


def test_attention(lsp):
    A, S = lsp.LSP_ERR_ARG, lsp.LSP_ERR_SHAPE
    base = dict(cache=cache(lsp), layer=0, q=0x7000, dtype=0, q_stride=1024, nq=8, seqs=16, start=16, n=2, total=6, shared_len=10,
                scale=0.1, out=0x8000, lse=None, ws=0x9000, nbytes=1 << 40, err=None, stream=None)

    def call(**kw):
        return lsp._f["lsp_prefix_attention_q4"](*{**base, **kw}.values())
    for kw in (dict(cache=None), dict(layer=-1), dict(layer=2), dict(q=None), dict(out=None), dict(seqs=None), dict(start=None),
               dict(n=0), dict(total=-1), dict(nq=0), dict(shared_len=-1), dict(scale=0.0), dict(scale=-1.0), dict(dtype=2), dict(dtype=-1),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(q=0x7008), dict(out=0x8004), dict(ws=None), dict(ws=0x9010),
               dict(lse=0x9002), dict(seqs=17), dict(start=18), dict(err=0x9003)):
        assert call(**kw) == A, kw
    for kw in (dict(nq=7), dict(nq=2 * 65), dict(n=1025), dict(q_stride=1000), dict(q_stride=1028), dict(total=2 ** 28),
               dict(dtype=1, q_stride=1026)):
        assert call(**kw) == S, kw
    assert call(total=0) == lsp.LSP_OK


def test_logprobs(lsp):
    A, S = lsp.LSP_ERR_ARG, lsp.LSP_ERR_SHAPE
    base = dict(z=0x1000, dtype=1, tokens=0x2000, rows=3, V=100, ld=100, T=1.0, k=5, logprob=0x3000, entropy=0x4000, top=0x5000, tl=0x6000,
                err=None, stream=None)

    def call(**kw):
        return lsp._f["lsp_logprobs"](*{**base, **kw}.values())
    for kw in (dict(z=None), dict(tokens=None), dict(logprob=None), dict(dtype=2), dict(rows=-1), dict(k=-1), dict(T=0.0), dict(T=-1.0),
               dict(T=float("nan")), dict(T=float("inf")), dict(T=1e-38), dict(T=1e38), dict(z=0x1002), dict(dtype=0, z=0x1001), dict(tokens=0x2002),
               dict(logprob=0x3001), dict(entropy=0x4002), dict(top=0x5001), dict(tl=0x6002), dict(err=0x7001)):
        assert call(**kw) == A, kw
    for kw in (dict(V=0), dict(V=2 ** 26 + 1, ld=2 ** 31), dict(ld=99), dict(k=33), dict(V=4, ld=4), dict(rows=2 ** 27 + 1), dict(ld=2 ** 40)):
        assert call(**kw) == S, kw
    assert call(rows=0, z=None) == lsp.LSP_OK


# ------------------------------------------------------------------ the binding
def tensors(lsp, layers=2, pages=5, nkv=2, page=16, d=64):
    k = torch.zeros(layers, pages, nkv, page, d * 9 // 16, dtype=torch.uint8)
    return k, torch.zeros_like(k), ints(4, 7), ints(4), ints(pages)


def held_cache(lsp, **kw):
    held = tensors(lsp, **kw)
    c = lsp.make_kv_cache(*held)
    c.held = held
    return c


def test_the_binding_takes_a_cache_of_bytes(lsp):
    k, v, *rest = tensors(lsp, d=128, page=32)
    c = lsp.make_kv_cache(k, v, *rest)
    assert (c.layers, c.pages, c.nkv, c.page, c.d, c.dtype) == (2, 5, 2, 32, 128, lsp.LSP_DTYPE_Q4)
    assert (c.s_layer, c.s_page, c.s_head, c.s_slot) == (72 * 32 * 10, 72 * 32 * 2, 72 * 32, 72)
    both = torch.zeros(5, 2, 2, 2, 32, 72, dtype=torch.uint8)            # pages, pools, heads, layers
    a, b = (both[:, i].permute(2, 0, 1, 3, 4) for i in range(2))
    c = lsp.make_kv_cache(a, b, *rest)
    assert (c.s_layer, c.s_page, c.s_head) == (72 * 32, 72 * 32 * 8, 72 * 32 * 2)
    for bad in (torch.zeros(2, 5, 2, 32, 70, dtype=torch.uint8), torch.zeros(2, 5, 2, 32, 80, dtype=torch.uint8)[..., :72],
                k.to(torch.int8), k.transpose(2, 3)):
        with pytest.raises(ValueError):
            lsp.make_kv_cache(bad, bad, *rest)
    assert lsp.lsp_prefix_attention_q4_workspace_bytes(plain_cache(lsp), torch.bfloat16, 4, 1, 1) == 0
    with pytest.raises(ValueError):
        lsp.lsp_prefix_attention_q4_workspace_bytes(c, torch.float16, 4, 1, 1)


@no_gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name,k,v", [("lsp_pages_write_q4", "k_new", "v_new"), ("lsp_pages_read", "k_out", "v_out")])
def test_rows_of_the_binding(lsp, name, k, v, dtype):
    other = torch.float32 if dtype == torch.bfloat16 else torch.bfloat16
    rows = torch.zeros(6, 2, 64, dtype=dtype)
    base = {"cache": held_cache(lsp), "layer": 5, "seqs": ints(3), "start": ints(4), k: rows, v: rows.clone(), "dev_error": ints(1),
            "stream": 0}                             # (there is no layer 5: the library refuses it)
    plain = plain_cache(lsp, nkv=2, d=64, dtype=1 if dtype == torch.bfloat16 else 0)
    refused(lsp, getattr(lsp, name), base, [
        ("4 bits" if "write" in name else "cache's type", dict(cache=plain)),
        ("one type", {v: rows.to(other)}),
        ("bfloat16 or float32", {k: rows.half(), v: rows.half()}),
        ("same strides", {v: rows[:4]}),
        ("same strides", {k: rows[..., :32], v: rows[..., :32]}),
        ("same strides", {k: rows.flatten(1), v: rows.flatten(1)}),
        ("same strides", {k: torch.zeros(6, 3, 64, dtype=dtype), v: torch.zeros(6, 3, 64, dtype=dtype)}),
        ("seqs", dict(seqs=ints(3).long())),
        ("seqs", dict(start=ints(3))),
        ("seqs", dict(start=ints(8)[::2])),
        ("dev_error", dict(dev_error=ints(0))),
    ])
    fused = torch.zeros(6, 8, 64, dtype=dtype)
    refused(lsp, getattr(lsp, name), {**base, k: fused[:, 2:4], v: fused[:, 4:6], "dev_error": None}, [])


@no_gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_of_the_binding(lsp, dtype):
    other = torch.float32 if dtype == torch.bfloat16 else torch.bfloat16
    q = torch.zeros(6, 4, 64, dtype=dtype)
    base = dict(cache=held_cache(lsp), layer=0, q=q, seqs=ints(3), start=ints(4), out=torch.zeros_like(q), lse=torch.zeros(6, 4), shared_len=0,
                scale=1.0, workspace=torch.zeros(1 << 10, dtype=torch.uint8), dev_error=ints(1), stream=0)
    refused(lsp, lsp.lsp_prefix_attention_q4, base, [
        ("4 bits", dict(cache=plain_cache(lsp, nkv=2, d=64))),
        ("one type", dict(out=q.to(other))),
        ("bfloat16 or float32", dict(q=q.half(), out=q.half())),
        ("dense within", dict(q=q[..., :32], out=q[..., :32])),
        ("dense within", dict(q=q.flatten(1), out=q.flatten(1))),
        ("dense within", dict(out=q[:5])),
        ("seqs", dict(seqs=ints(3).long())),
        ("seqs", dict(start=ints(3))),
        ("lse", dict(lse=torch.zeros(6, 4, dtype=torch.float64))),
        ("lse", dict(lse=torch.zeros(5, 4))),
        ("workspace", dict(workspace=torch.zeros(1 << 11, dtype=torch.uint8)[::2])),
        ("dev_error", dict(dev_error=torch.zeros(1, dtype=torch.uint8))),
    ])
    # a cache in 4 bits has no use for the calls of the others
    with pytest.raises(ValueError, match="cache's type"):
        lsp.lsp_prefix_attention(**base)
    with pytest.raises(ValueError, match="cache's type"):
        rows = torch.zeros(6, 2, 64, dtype=dtype)
        lsp.lsp_pages_write(base["cache"], 0, ints(3), ints(4), rows, rows)


@no_gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logprobs_of_the_binding(lsp, dtype):
    z = torch.zeros(6, 100, dtype=dtype)
    base = dict(logits=z, tokens=ints(6), logprob=torch.zeros(6), entropy=torch.zeros(6), top=ints(6, 5), top_logprob=torch.zeros(6, 5),
                temperature=1.0, dev_error=ints(1), stream=0)
    refused(lsp, lsp.lsp_logprobs, base, [
        ("bfloat16 or float32", dict(logits=z.half())),
        ("logits", dict(logits=z[0])),
        ("logits", dict(logits=z.T.contiguous().T)),
        ("logits", dict(logits=z[:1].expand(6, 100))),
        ("tokens", dict(tokens=ints(6).long())),
        ("tokens", dict(tokens=ints(5))),
        ("tokens", dict(tokens=ints(12)[::2])),
        ("tokens", dict(logprob=torch.zeros(6).double())),
        ("tokens", dict(logprob=torch.zeros(7))),
        ("tokens", dict(entropy=torch.zeros(6).half())),
        ("top", dict(top=ints(6, 5).long())),
        ("top", dict(top=ints(30))),
        ("top", dict(top=ints(6, 10)[:, :5])),
        ("top", dict(top_logprob=torch.zeros(5, 5))),
        ("one shape", dict(top_logprob=torch.zeros(6, 4))),
        ("dev_error", dict(dev_error=ints(0))),
    ])
    wide = torch.zeros(6, 130, dtype=dtype)[:, 3:103]
    for kw in (dict(logits=wide), dict(entropy=None, top=None, top_logprob=None, dev_error=None), dict(top=None), dict(top_logprob=None)):
        refused(lsp, lsp.lsp_logprobs, {**base, **kw}, [])


def test_attention_scales(lsp):
    """Scores of eighths of the values have a factor of 8 log2(e) scale, which must be a number."""
    def call(scale):
        return lsp._f["lsp_prefix_attention_q4"](cache(lsp), 0, 0x7000, 0, 1024, 8, 16, 16, 2, 6, 10, scale, 0x8000, None, 0x9000, 0, None, None)
    for scale in (1.5 * 2.0 ** 120, 2.0 ** 125, 3e38):
        assert call(scale) == lsp.LSP_ERR_ARG
