"""What the Python binding of the target-side calls refuses: the library gets bare addresses, so a tensor of another
type, length or layout than it takes would be read, or written, past its end.  Nothing is launched (no GPU): a call
that is in order gets as far as the library, which has no device here, or refuses it for a reason of its own."""
import pytest
import torch


@pytest.fixture(scope="module")
def lsp():
    from paper_2609_37029_gb300 import build
    build.build()
    from paper_2609_37029_gb300 import lsp as mod
    return mod


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def cache(lsp, dtype):
    k = torch.zeros(2, 5, 2, 16, 64, dtype=dtype)
    held = [k, torch.zeros_like(k), ints(4, 7), ints(4), ints(5)]
    c = lsp.make_kv_cache(*held)
    c.held = held
    return c


def refused(lsp, call, base, changes):
    """Every change of `base` raises ValueError with its own text; `base` itself gets to the library."""
    with pytest.raises(lsp.LspError):                # (no device)
        call(**base)
    for text, kw in changes:
        with pytest.raises(ValueError, match=text):
            call(**{**base, **kw})


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls that are in order would run")
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention(lsp, dtype):
    other = torch.float32 if dtype == torch.bfloat16 else torch.bfloat16
    c = cache(lsp, dtype)
    q = torch.zeros(6, 4, 64, dtype=dtype)
    base = dict(cache=c, layer=0, q=q, seqs=ints(3), start=ints(4), out=torch.zeros_like(q), lse=torch.zeros(6, 4), shared_len=0,
                scale=1.0, workspace=torch.zeros(1 << 10, dtype=torch.uint8), dev_error=ints(1), stream=0)
    refused(lsp, lsp.lsp_prefix_attention, base, [
        ("cache's type", dict(q=q.to(other), out=q.to(other))),
        ("cache's type", dict(out=q.to(other))),
        ("bfloat16 or float32", dict(q=q.half(), out=q.half())),
        ("dense within", dict(q=q[..., :32], out=q[..., :32])),
        ("dense within", dict(out=q[:5])),
        ("seqs", dict(seqs=ints(3).long())),
        ("seqs", dict(seqs=ints(6)[::2])),
        ("seqs", dict(start=ints(4).long())),
        ("seqs", dict(start=ints(3))),
        ("seqs", dict(start=ints(8)[::2])),
        ("lse", dict(lse=torch.zeros(6, 4, dtype=torch.float64))),
        ("lse", dict(lse=torch.zeros(6, 4, dtype=torch.bfloat16))),
        ("lse", dict(lse=torch.zeros(5, 4))),
        ("lse", dict(lse=torch.zeros(4, 6).T)),
        ("workspace", dict(workspace=torch.zeros(1 << 11, dtype=torch.uint8)[::2])),
        ("dev_error", dict(dev_error=torch.zeros(1, dtype=torch.uint8))),
        ("dev_error", dict(dev_error=ints(0))),
    ])
    # rows of a fused projection, no sums of exponentials, no error word: in order too
    wide = torch.zeros(6, 8, 64, dtype=dtype)
    refused(lsp, lsp.lsp_prefix_attention, {**base, "q": wide[:, 2:6], "lse": None, "dev_error": None}, [])


no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="the calls that are in order would run")


@no_gpu
@pytest.mark.parametrize("name", ["lsp_pages_fork", "lsp_pages_trim", "lsp_pages_reserve"])
def test_page_lists(lsp, name):
    a, b = ("src", "dst") if name == "lsp_pages_fork" else ("seqs", "new_len" if name == "lsp_pages_trim" else "add")
    base = {"cache": cache(lsp, torch.float32), a: ints(3), b: ints(3), "dev_error": ints(1), "stream": 0}
    changes = [(None, {b: ints(2)}), (None, {b: ints(4)}), (None, {a: ints(2)}), (None, {a: ints(3).long()}),
               (None, {b: ints(3).long()}), (None, {b: torch.zeros(3)}), (None, {a: ints(6)[::2]}), (None, {b: ints(6)[::2]})]
    changes = [("lists", kw) for _, kw in changes] + [("dev_error", dict(dev_error=torch.zeros(3, dtype=torch.uint8)))]
    if name == "lsp_pages_reserve":
        base["workspace"] = torch.zeros(1 << 16, dtype=torch.uint8)
        changes.append(("workspace", dict(workspace=torch.zeros(1 << 17, dtype=torch.uint8)[::2])))
    refused(lsp, getattr(lsp, name), base, changes)


@no_gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_page_writes(lsp, dtype):
    other = torch.float32 if dtype == torch.bfloat16 else torch.bfloat16
    rows = torch.zeros(6, 2, 64, dtype=dtype)
    base = dict(cache=cache(lsp, dtype), layer=5, seqs=ints(3), start=ints(4), k_new=rows, v_new=rows.clone(), dev_error=ints(1),
                stream=0)                            # (there is no layer 5: the library refuses it)
    refused(lsp, lsp.lsp_pages_write, base, [
        ("cache's type", dict(k_new=rows.to(other), v_new=rows.to(other))),
        ("cache's type", dict(v_new=rows.to(other))),
        ("bfloat16 or float32", dict(k_new=rows.half(), v_new=rows.half())),
        ("same strides", dict(v_new=rows[:4])),
        ("same strides", dict(k_new=rows[..., :32], v_new=rows[..., :32])),
        ("seqs", dict(seqs=ints(3).long())),
        ("seqs", dict(start=ints(3))),
        ("seqs", dict(start=ints(5))),
        ("seqs", dict(start=ints(4).long())),
        ("dev_error", dict(dev_error=ints(0))),
    ])


@no_gpu
def test_compaction(lsp):
    base = dict(cache=cache(lsp, torch.float32), live=ints(1), workspace=torch.zeros(1 << 16, dtype=torch.uint8), stream=0)
    refused(lsp, lsp.lsp_pages_compact, base, [
        ("live", dict(live=ints(0))),
        ("live", dict(live=torch.zeros(1, dtype=torch.uint8))),
        ("live", dict(live=torch.zeros(1))),
        ("workspace", dict(workspace=torch.zeros(1 << 17, dtype=torch.uint8)[::2])),
    ])


@no_gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_verification(lsp, dtype):
    C, B, V = 3, 4, 10
    f32 = lambda *x: torch.zeros(*x)
    base = dict(target_probs=torch.zeros(C, B + 1, V, dtype=dtype), draft_probs=torch.zeros(C, B, V, dtype=dtype), draft_tokens=ints(C, B),
                u=f32(C, B), e=f32(C, V), accepted_len=ints(C), next_token=ints(C), n_draft=ints(C), out_tokens=ints(C, B + 1),
                dev_error=ints(1), stream=0)
    changes = [("one type", dict(draft_probs=torch.zeros(C, B, V, dtype=torch.float16))),
               ("evenly spaced", dict(draft_probs=torch.zeros(C, B - 1, V, dtype=dtype)))]
    changes += [("contiguous float32", kw) for kw in (
        dict(u=f32(C, B).double()), dict(u=f32(C, B).half()), dict(u=f32(C, B - 1)), dict(u=f32(C, B + 1)[:, :B]), dict(u=f32(B, C).T),
        dict(e=f32(C, V).bfloat16()), dict(e=f32(V)), dict(e=f32(C, 2 * V)[:, :V]), dict(e=f32(V).expand(C, V)))]
    changes += [("contiguous int32", kw) for kw in (
        dict(draft_tokens=ints(C, B).long()), dict(draft_tokens=ints(C, B + 1)[:, :B]), dict(accepted_len=ints(C).long()),
        dict(accepted_len=ints(C - 1)), dict(next_token=ints(C).long()), dict(next_token=ints(2 * C)[::2]), dict(n_draft=ints(C + 1)),
        dict(n_draft=f32(C)), dict(out_tokens=ints(C, B)), dict(out_tokens=ints(C, B + 1).long()))]
    changes += [("dev_error", dict(dev_error=torch.zeros(4, dtype=torch.uint8)))]
    refused(lsp, lsp.lsp_verify_probs, base, changes)
    for kw in (dict(draft_probs=None), dict(n_draft=None, out_tokens=None, dev_error=None),
               dict(target_probs=torch.zeros(C, B + 1, V + 6, dtype=dtype)[..., :V])):
        refused(lsp, lsp.lsp_verify_probs, {**base, **kw}, [])
    # no candidates at all
    none = dict(target_probs=torch.zeros(C, 1, V, dtype=dtype), draft_probs=None, draft_tokens=ints(C, 0), u=f32(C, 0), out_tokens=ints(C, 1))
    refused(lsp, lsp.lsp_verify_probs, {**base, **none}, [])


@no_gpu
def test_the_stride_of_an_axis_of_one_may_be_anything(lsp):
    """One head, one row, one layer, one page: dense however torch counts the steps along them."""
    def odd(t, **steps):
        stride = list(t.stride())
        for axis, step in steps.items():
            assert t.shape[int(axis[1:])] == 1
            stride[int(axis[1:])] = step
        return t.as_strided(t.shape, stride)
    k = torch.zeros(1, 1, 1, 16, 64)
    c = lsp.make_kv_cache(odd(k, a0=7), odd(k, a1=3, a2=1), ints(4, 7), ints(4), ints(1))
    q = torch.zeros(6, 1, 64)
    lists = dict(seqs=ints(3), start=ints(4), stream=0)
    for x in (odd(q, a1=1), odd(q, a1=12345), q.transpose(0, 1).contiguous().transpose(0, 1)):
        refused(lsp, lsp.lsp_prefix_attention, dict(cache=c, layer=0, q=x, out=torch.zeros_like(q), shared_len=0, scale=1.0,
                                                    workspace=torch.zeros(64, dtype=torch.uint8), **lists), [])
        refused(lsp, lsp.lsp_pages_write, dict(cache=c, layer=5, k_new=x, v_new=q, **lists), [])
    one = torch.zeros(1, 1, 64)
    refused(lsp, lsp.lsp_pages_write, dict(cache=c, layer=5, k_new=odd(one, a0=1), v_new=odd(one, a0=500, a1=9), **lists), [])
    # but not of any other
    two = torch.zeros(1, 2, 1, 16, 64)
    with pytest.raises(ValueError):
        lsp.make_kv_cache(two, torch.zeros(1, 4, 1, 16, 64)[:, ::2], ints(4, 7), ints(4), ints(2))
    wide = torch.zeros(6, 1, 128)[..., :64]
    refused(lsp, lsp.lsp_pages_write, dict(cache=c, layer=5, k_new=wide, v_new=wide, **lists), [
        ("same strides", dict(v_new=q)), ("same strides", dict(v_new=torch.zeros(6, 1, 128)[..., ::2]))])
