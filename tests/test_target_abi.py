"""Refusals of the target-side calls that the host makes (no GPU needed: nothing is launched)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lsp():
    from paper_2609_37029_gb300 import build
    build.build()
    from paper_2609_37029_gb300 import lsp as mod
    return mod


def cache(lsp, **kw):
    c = lsp.lsp_kv_cache()
    c.k, c.v, c.table, c.len, c.refs = 0x1000, 0x2000, 0x3000, 0x4000, 0x5000
    c.layers, c.pages, c.page, c.nkv, c.d, c.seqs, c.max_pages = 2, 100, 64, 2, 128, 4, 30
    c.dtype = lsp.LSP_DTYPE_BF16
    c.s_slot, c.s_head, c.s_page, c.s_layer = 128, 128 * 64, 128 * 128, 128 * 128 * 100
    for n, v in kw.items():
        setattr(c, n, v)
    return c


SHAPES = [dict(page=48), dict(page=8), dict(page=512), dict(d=96), dict(d=32), dict(layers=0), dict(pages=0), dict(pages=2 ** 20 + 1),
          dict(nkv=0), dict(seqs=0), dict(max_pages=0), dict(seqs=2 ** 16, max_pages=2 ** 15), dict(page=256, max_pages=2 ** 23),
          dict(s_slot=4), dict(s_head=130), dict(s_page=-128), dict(s_layer=2 ** 40)]


@pytest.mark.parametrize("kw", SHAPES, ids=str)
def test_unsupported_caches(lsp, kw):
    c = cache(lsp, **kw)
    assert lsp.lsp_pages_workspace_bytes(c) == 0
    assert lsp.lsp_prefix_attention_workspace_bytes(c, 4, 1, 1) == 0
    assert lsp._f["lsp_pages_fork"](c, 16, 16, 1, None, None) == lsp.LSP_ERR_SHAPE


def test_page_calls(lsp):
    f, A, S = lsp._f, lsp.LSP_ERR_ARG, lsp.LSP_ERR_SHAPE
    c = cache(lsp)
    need = lsp.lsp_pages_workspace_bytes(c)
    assert need > 0
    assert f["lsp_pages_fork"](None, 16, 16, 1, None, None) == A
    for missing in ("k", "v", "table", "len", "refs"):
        assert f["lsp_pages_trim"](cache(lsp, **{missing: None}), 16, 16, 1, None, None) == A
    assert f["lsp_pages_trim"](cache(lsp, k=0x1008), 16, 16, 1, None, None) == A
    assert f["lsp_pages_trim"](cache(lsp, dtype=5), 16, 16, 1, None, None) == A
    for name in ("lsp_pages_fork", "lsp_pages_trim"):
        assert f[name](c, None, 16, 1, None, None) == A
        assert f[name](c, 16, None, 1, None, None) == A
        assert f[name](c, 16, 16, -1, None, None) == A
        assert f[name](c, 16, 16, 1025, None, None) == S
        assert f[name](c, 16, 16, 0, None, None) == lsp.LSP_OK
    assert f["lsp_pages_reserve"](c, 16, 16, 1, None, need, None, None) == A
    assert f["lsp_pages_reserve"](c, 16, 16, 1, 0x6000, need - 1, None, None) == A
    assert f["lsp_pages_reserve"](c, 16, 16, 1, 0x6004, need, None, None) == A
    assert f["lsp_pages_reserve"](c, 16, 16, 1025, 0x6000, need, None, None) == S
    assert f["lsp_pages_compact"](c, None, 0x6000, need - 1, None) == A
    w = f["lsp_pages_write"]
    assert w(c, 2, 16, 16, 1, 0x7000, 0x8000, 256, 5, None, None) == A          # no such layer
    assert w(c, 0, 16, 16, 1, 0x7002, 0x8000, 256, 5, None, None) == A
    assert w(c, 0, 16, 16, 1, None, 0x8000, 256, 5, None, None) == A
    assert w(c, 0, 16, 16, 1, 0x7000, 0x8000, 255, 5, None, None) == S          # rows overlap
    assert w(c, 0, 16, 16, 1, 0x7000, 0x8000, 260, 5, None, None) == S          # not 16-byte rows
    assert w(c, 0, 16, 16, 1, None, None, 256, 0, None, None) == lsp.LSP_OK


def test_attention_calls(lsp):
    A, S = lsp.LSP_ERR_ARG, lsp.LSP_ERR_SHAPE
    base = dict(cache=cache(lsp), layer=0, q=0x7000, q_stride=1024, nq=8, seqs=16, start=16, n=2, total=6, shared_len=10,
                scale=0.1, out=0x8000, lse=None, ws=0x9000, nbytes=1 << 40, err=None, stream=None)

    def call(**kw):
        return lsp._f["lsp_prefix_attention"](*{**base, **kw}.values())
    for kw in (dict(cache=None), dict(layer=-1), dict(layer=2), dict(q=None), dict(out=None), dict(seqs=None), dict(start=None),
               dict(n=0), dict(total=-1), dict(nq=0), dict(shared_len=-1), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(q=0x7008), dict(out=0x8004), dict(ws=None), dict(ws=0x9010)):
        assert call(**kw) == A, kw
    for kw in (dict(nq=7), dict(nq=2 * 65), dict(n=1025), dict(q_stride=1000), dict(q_stride=1028), dict(total=2 ** 28)):
        assert call(**kw) == S, kw
    assert call(total=0) == lsp.LSP_OK


def test_verify_calls(lsp):
    A, S = lsp.LSP_ERR_ARG, lsp.LSP_ERR_SHAPE
    base = dict(p=0x1000, q=0x2000, dtype=lsp.LSP_DTYPE_F32, y=0x3000, n=None, u=0x4000, e=0x5000, C=2, B=3, V=100, lt=100, ld=100,
                acc=0x6000, tok=0x7000, out=None, err=None, stream=None)

    def call(**kw):
        return lsp._f["lsp_verify_probs"](*{**base, **kw}.values())
    for kw in (dict(p=None), dict(y=None), dict(u=None), dict(e=None), dict(acc=None), dict(tok=None), dict(dtype=7), dict(p=0x1002),
               dict(q=0x2002), dict(e=0x5002)):
        assert call(**kw) == A, kw
    for kw in (dict(C=0), dict(B=-1), dict(B=1025), dict(V=0), dict(lt=99), dict(ld=99), dict(V=2 ** 30 + 1, lt=2 ** 31, ld=2 ** 31)):
        assert call(**kw) == S, kw


def test_the_struct_is_the_header_s(lsp):
    assert ctypes.sizeof(lsp.lsp_kv_cache) == 5 * 8 + 4 * 8 + 8 * 4


def test_the_binding_takes_strides_and_refuses_other_tensors(lsp):
    import torch
    k = torch.zeros(5, 2, 16, 3, 64, dtype=torch.bfloat16).permute(1, 0, 3, 2, 4)       # slots outside the heads
    table, lens, refs = torch.zeros(4, 7, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), torch.zeros(5, dtype=torch.int32)
    c = lsp.make_kv_cache(k, k, table, lens, refs)
    assert (c.layers, c.pages, c.nkv, c.page, c.d, c.seqs, c.max_pages) == (2, 5, 3, 16, 64, 4, 7)
    assert (c.s_layer, c.s_page, c.s_head, c.s_slot) == (16 * 192, 2 * 16 * 192, 64, 192)
    for bad in ((k.half(), k.half(), table, lens, refs), (k, k[:1], table, lens, refs), (k, k, table.long(), lens, refs),
                (k, k, table, lens[:2], refs), (k, k, table, lens, refs[:2]), (k.transpose(3, 4), k.transpose(3, 4), table, lens, refs)):
        with pytest.raises(ValueError):
            lsp.make_kv_cache(*bad)
    q = torch.zeros(3, 6, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lsp.lsp_prefix_attention(c, 0, q.transpose(0, 1), lens, lens, q, shared_len=0, scale=1.0, workspace=q)
    with pytest.raises(ValueError):
        lsp.lsp_pages_write(c, 0, lens, lens, q, q)                                     # six heads, the cache has three
    p = torch.zeros(2, 4, 10)
    with pytest.raises(ValueError):
        lsp.lsp_verify_probs(p, p, lens.view(2, 2), p, p, lens, lens)
