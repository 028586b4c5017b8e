"""Lists, results and error words of the target-side calls that do not start at a word's address are refused on the
host (no GPU needed: nothing is launched)."""
import pytest

from tests.test_target_abi import cache


@pytest.fixture(scope="module")
def lsp():
    from paper_2609_37029_gb300 import build
    build.build()
    from paper_2609_37029_gb300 import lsp as mod
    return mod


def each(call, lsp, names, base):
    for name in names:
        for by in (1, 2, 3):
            assert call(**{**base, name: 0x9000 + by}) == lsp.LSP_ERR_ARG, (name, by)


def test_page_calls(lsp):
    c = cache(lsp)
    need = lsp.lsp_pages_workspace_bytes(c)
    for name in ("lsp_pages_fork", "lsp_pages_trim"):
        each(lambda a, b, err: lsp._f[name](c, a, b, 1, err, None), lsp, ["a", "b", "err"], dict(a=16, b=16, err=None))
    each(lambda a, b, err: lsp._f["lsp_pages_reserve"](c, a, b, 1, 0x6000, need, err, None), lsp, ["a", "b", "err"],
         dict(a=16, b=16, err=None))
    each(lambda live: lsp._f["lsp_pages_compact"](c, live, 0x6000, need, None), lsp, ["live"], dict(live=None))
    each(lambda a, b, err: lsp._f["lsp_pages_write"](c, 0, a, b, 1, 0x7000, 0x8000, 256, 5, err, None), lsp, ["a", "b", "err"],
         dict(a=16, b=16, err=None))
    for name in ("table", "len", "refs"):
        assert lsp._f["lsp_pages_trim"](cache(lsp, **{name: 0x3002}), 16, 16, 1, None, None) == lsp.LSP_ERR_ARG


def test_attention(lsp):
    each(lambda seqs, start, lse, err: lsp._f["lsp_prefix_attention"](
        cache(lsp), 0, 0x7000, 1024, 8, seqs, start, 2, 6, 10, 0.1, 0x8000, lse, 0x9000, 1 << 40, err, None),
        lsp, ["seqs", "start", "lse", "err"], dict(seqs=16, start=16, lse=None, err=None))


def test_verification(lsp):
    base = dict(y=0x3000, n=None, u=0x4000, e=0x5000, acc=0x6000, tok=0x7000, out=None, err=None)
    each(lambda y, n, u, e, acc, tok, out, err: lsp._f["lsp_verify_probs"](
        0x1000, 0x2000, lsp.LSP_DTYPE_F32, y, n, u, e, 2, 3, 100, 100, 100, acc, tok, out, err, None), lsp, list(base), base)
