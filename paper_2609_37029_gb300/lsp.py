"""Python binding of liblsp (include/lsp.h): argument marshalling only.

Every function here has the name of the C entry point it calls and does no
computation of its own: tensors are passed as raw device pointers, structs are
mirrored with ctypes, and a non-zero status raises LspError.  The library must
have been built (paper_2609_37029_gb300.build); importing this module without
it fails loudly -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import (POINTER, Structure, c_char_p, c_float, c_int, c_int64, c_size_t, c_uint32,
                    c_uint64, c_void_p)

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "liblsp.so")

LSP_MAX_DRAFT_LAYERS = 16
LSP_OK, LSP_ERR_ARG, LSP_ERR_SHAPE, LSP_ERR_CUDA = 0, -1, -2, -3
LSP_ERR_TIMEOUT, LSP_ERR_STATE, LSP_ERR_NOMEM, LSP_ERR_UNSUPPORTED = -4, -5, -6, -7
LSP_DEV_TIMEOUT, LSP_DEV_BAD_TOKEN, LSP_DEV_BAD_DELTA = 1, 2, 4
LSP_DEV_BAD_SEQ, LSP_DEV_NO_PAGE = 8, 16
LSP_NO_BOUNDARY = 1
LSP_DTYPE_BF16, LSP_DTYPE_F32, LSP_DTYPE_Q4 = 0, 1, 2

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_37029_gb300.build`"
                      " (the CUDA library is required; there is no CPU path)")
_lib = ctypes.CDLL(LIB_PATH)


class lsp_config(Structure):
    _fields_ = [(n, c_int) for n in "C B L D H nq nkv d F V W R rc dtype".split()] + [
        ("layer_map", c_int * LSP_MAX_DRAFT_LAYERS), ("rope_theta", c_float), ("rms_eps", c_float),
        ("flags", c_uint32)]


class lsp_target_feats(Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("h", c_void_p), ("rows", c_int), ("h_rows", c_int)]


_LAYER_FIELDS = ["in_norm", "wq", "wk", "wv", "q_norm", "k_norm", "wo", "post_norm", "w_gate",
                 "w_up", "w_down"]
_TOP_FIELDS = ["embed", "final_norm", "lm_head", "fuse", "pos", "mask_emb", "Ec", "Wc"]


class lsp_layer_weights(Structure):
    _fields_ = [(n, c_void_p) for n in _LAYER_FIELDS]


class lsp_weights(Structure):
    _fields_ = [(n, c_void_p) for n in _TOP_FIELDS] + [
        ("layer", lsp_layer_weights * LSP_MAX_DRAFT_LAYERS)]


class lsp_sample_params(Structure):
    _fields_ = [("temperature", c_float), ("round", c_uint32), ("seed", c_uint64)]


class lsp_kv_cache(Structure):
    _fields_ = [(n, c_void_p) for n in "k v table len refs".split()] + [
        (n, c_int64) for n in "s_layer s_page s_head s_slot".split()] + [
        (n, c_int) for n in "layers pages page nkv d dtype seqs max_pages".split()]


class LspError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lsp_status_string(status)} ({status})")


def _sig(name, res, *args):
    f = getattr(_lib, name)
    f.restype = res
    f.argtypes = list(args)
    return f


_f = {
    "lsp_status_string": _sig("lsp_status_string", c_char_p, c_int),
    "lsp_state_bytes": _sig("lsp_state_bytes", c_size_t, POINTER(lsp_config)),
    "lsp_config_check": _sig("lsp_config_check", c_int, POINTER(lsp_config)),
    "lsp_state_create": _sig("lsp_state_create", c_int, POINTER(lsp_config), POINTER(c_void_p)),
    "lsp_state_destroy": _sig("lsp_state_destroy", None, c_void_p),
    "lsp_state_init": _sig("lsp_state_init", c_int, c_void_p, c_void_p, c_void_p),
    "lsp_view_update": _sig("lsp_view_update", c_int, c_void_p, POINTER(lsp_target_feats), c_void_p,
                            c_void_p),
    "lsp_prefill": _sig("lsp_prefill", c_int, c_void_p, c_int, POINTER(lsp_target_feats), c_void_p),
    "lsp_verify": _sig("lsp_verify", c_int, c_void_p, c_void_p, c_void_p, c_void_p,
                       POINTER(lsp_sample_params), c_void_p, c_void_p, c_void_p),
    "lsp_draft": _sig("lsp_draft", c_int, c_void_p, c_void_p, POINTER(lsp_weights),
                      POINTER(lsp_sample_params), c_void_p, c_void_p, c_void_p),
    "lsp_sample": _sig("lsp_sample", c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                       POINTER(lsp_sample_params), c_void_p, c_void_p, c_void_p),
    "lsp_sample_noalloc": _sig("lsp_sample_noalloc", c_int, c_void_p, c_void_p, c_void_p, c_void_p,
                               c_int, c_int, c_int, c_int, c_int, POINTER(lsp_sample_params),
                               c_void_p, c_void_p, c_void_p, c_void_p),
    "lsp_linear_workspace_bytes": _sig("lsp_linear_workspace_bytes", c_size_t, c_int, c_int, c_int),
    "lsp_gemm_plan_info": _sig("lsp_gemm_plan_info", c_int, c_int, c_int, c_int, c_int, c_int, c_int,
                               POINTER(c_int), POINTER(c_int), POINTER(c_int)),
    "lsp_linear": _sig("lsp_linear", c_int, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int,
                       c_int, c_void_p, c_size_t, c_void_p),
    "lsp_philox_words": _sig("lsp_philox_words", c_int, c_uint64, c_uint32, c_uint32, c_uint32,
                             c_void_p, c_int, c_void_p),
    "lsp_get_error": _sig("lsp_get_error", c_int, c_void_p, POINTER(c_uint32), c_int, c_void_p),
    "lsp_stage_count": _sig("lsp_stage_count", c_int, c_void_p),
    "lsp_round_launches": _sig("lsp_round_launches", c_int, c_void_p),
    "lsp_stage_name": _sig("lsp_stage_name", c_char_p, c_void_p, c_int),
    "lsp_set_stage_events": _sig("lsp_set_stage_events", c_int, c_void_p, POINTER(c_void_p), c_int),
    "lsp_state_export": _sig("lsp_state_export", c_int, c_void_p, c_void_p, c_size_t, c_void_p),
    "lsp_state_import": _sig("lsp_state_import", c_int, c_void_p, c_void_p, c_size_t, c_void_p),
    "lsp_pages_workspace_bytes": _sig("lsp_pages_workspace_bytes", c_size_t, POINTER(lsp_kv_cache)),
    "lsp_pages_fork": _sig("lsp_pages_fork", c_int, POINTER(lsp_kv_cache), c_void_p, c_void_p, c_int,
                           c_void_p, c_void_p),
    "lsp_pages_reserve": _sig("lsp_pages_reserve", c_int, POINTER(lsp_kv_cache), c_void_p, c_void_p,
                              c_int, c_void_p, c_size_t, c_void_p, c_void_p),
    "lsp_pages_write": _sig("lsp_pages_write", c_int, POINTER(lsp_kv_cache), c_int, c_void_p, c_void_p,
                            c_int, c_void_p, c_void_p, c_int64, c_int, c_void_p, c_void_p),
    "lsp_pages_trim": _sig("lsp_pages_trim", c_int, POINTER(lsp_kv_cache), c_void_p, c_void_p, c_int,
                           c_void_p, c_void_p),
    "lsp_pages_compact": _sig("lsp_pages_compact", c_int, POINTER(lsp_kv_cache), c_void_p, c_void_p,
                              c_size_t, c_void_p),
    "lsp_prefix_attention_workspace_bytes": _sig("lsp_prefix_attention_workspace_bytes", c_size_t,
                                                 POINTER(lsp_kv_cache), c_int, c_int, c_int),
    "lsp_prefix_attention": _sig("lsp_prefix_attention", c_int, POINTER(lsp_kv_cache), c_int, c_void_p,
                                 c_int64, c_int, c_void_p, c_void_p, c_int, c_int, c_int, c_float,
                                 c_void_p, c_void_p, c_void_p, c_size_t, c_void_p, c_void_p),
    "lsp_pages_write_q4": _sig("lsp_pages_write_q4", c_int, POINTER(lsp_kv_cache), c_int, c_void_p, c_void_p,
                               c_int, c_void_p, c_void_p, c_int, c_int64, c_int, c_void_p, c_void_p),
    "lsp_pages_read": _sig("lsp_pages_read", c_int, POINTER(lsp_kv_cache), c_int, c_void_p, c_void_p,
                           c_int, c_void_p, c_void_p, c_int, c_int64, c_int, c_void_p, c_void_p),
    "lsp_prefix_attention_q4_workspace_bytes": _sig("lsp_prefix_attention_q4_workspace_bytes", c_size_t,
                                                    POINTER(lsp_kv_cache), c_int, c_int, c_int, c_int),
    "lsp_prefix_attention_q4": _sig("lsp_prefix_attention_q4", c_int, POINTER(lsp_kv_cache), c_int, c_void_p,
                                    c_int, c_int64, c_int, c_void_p, c_void_p, c_int, c_int, c_int, c_float,
                                    c_void_p, c_void_p, c_void_p, c_size_t, c_void_p, c_void_p),
    "lsp_logprobs": _sig("lsp_logprobs", c_int, c_void_p, c_int, c_void_p, c_int, c_int, c_int64, c_float,
                         c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p),
    "lsp_verify_probs": _sig("lsp_verify_probs", c_int, c_void_p, c_void_p, c_int, c_void_p, c_void_p,
                             c_void_p, c_void_p, c_int, c_int, c_int, c_int64, c_int64, c_void_p,
                             c_void_p, c_void_p, c_void_p, c_void_p),
}


_pages_workspace_bytes, _pages_fork, _pages_reserve = (
    _f[n] for n in ("lsp_pages_workspace_bytes", "lsp_pages_fork", "lsp_pages_reserve"))
_pages_write, _pages_trim, _pages_compact = (_f[n] for n in ("lsp_pages_write", "lsp_pages_trim", "lsp_pages_compact"))
_prefix_attention_workspace_bytes, _prefix_attention, _verify_probs = (
    _f[n] for n in ("lsp_prefix_attention_workspace_bytes", "lsp_prefix_attention", "lsp_verify_probs"))
_pages_write_q4, _pages_read, _prefix_attention_q4_workspace_bytes, _prefix_attention_q4, _logprobs = (
    _f[n] for n in ("lsp_pages_write_q4", "lsp_pages_read", "lsp_prefix_attention_q4_workspace_bytes",
                    "lsp_prefix_attention_q4", "lsp_logprobs"))


def _ptr(x):
    """Device/host address of a tensor (or an int address, or None)."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


_raw_stream = None


def _stream(stream):
    global _raw_stream
    if stream is None:
        if _raw_stream is None:
            import torch
            torch.cuda.current_stream()                 # initialises CUDA where nothing has yet
            get, dev = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
            _raw_stream = lambda: get(dev())            # current_stream().cuda_stream without a Stream object
        return _raw_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(rc, where):
    if rc != LSP_OK:
        raise LspError(rc, where)


# ------------------------------------------------------------------ struct builders
def make_config(shape) -> lsp_config:
    """lsp_config from any object with the shape fields (e.g. synth.LspShape)."""
    c = lsp_config()
    for n in "C B L D H nq nkv d F V W R rc".split():
        setattr(c, n, int(getattr(shape, n)))
    c.dtype = LSP_DTYPE_BF16 if shape.dtype == "bf16" else LSP_DTYPE_F32
    lm = list(getattr(shape, "layer_map", ()) or ())
    for j in range(LSP_MAX_DRAFT_LAYERS):
        c.layer_map[j] = int(lm[j]) if j < len(lm) else -1
    c.rope_theta = float(shape.rope_theta)
    c.rms_eps = float(shape.rms_eps)
    c.flags = LSP_NO_BOUNDARY if getattr(shape, "no_boundary", False) else 0
    return c


def make_weights(w: dict) -> lsp_weights:
    """lsp_weights of device pointers from a dict of tensors (synth.make_weights layout)."""
    s = lsp_weights()
    for n in _TOP_FIELDS:
        setattr(s, n, _ptr(w[n]))
    for j, lw in enumerate(w["layers"]):
        for n in _LAYER_FIELDS:
            setattr(s.layer[j], n, _ptr(lw[n]))
    return s


def make_kv_cache(k, v, table, lens, refs) -> lsp_kv_cache:
    """lsp_kv_cache of device pointers: k, v [layers][pages][nkv][page][d] in any order of the first
    four axes (their strides are taken), int32 table [seqs][max_pages], lens [seqs], refs [pages].
    A cache held in 4 bits: uint8 k, v [layers][pages][nkv][page][9 d / 16], the last two axes dense (a
    head's block of codes and scales, see LSP_DTYPE_Q4 in the header) and the others in any order.
    The struct holds addresses only: the caller keeps the tensors."""
    import torch
    apart = any(a != b for a, b, n in zip(k.stride(), v.stride(), k.shape) if n > 1)
    if k.shape != v.shape or apart or k.dtype != v.dtype or k.dim() != 5 or k.stride(4) != 1:
        raise ValueError("k and v: the same 5-D shape, type and strides, the last axis dense")
    for t in (table, lens, refs):
        if t.dtype != torch.int32 or not t.is_contiguous():
            raise ValueError("table, lens and refs: contiguous int32")
    if table.dim() != 2 or lens.numel() != table.shape[0] or refs.numel() != k.shape[1]:
        raise ValueError("table [seqs][max_pages], lens [seqs], refs [pages]")
    c = lsp_kv_cache()
    c.k, c.v, c.table, c.len, c.refs = (t.data_ptr() for t in (k, v, table, lens, refs))
    c.s_layer, c.s_page, c.s_head, c.s_slot = k.stride()[:4]
    c.layers, c.pages, c.nkv, c.page, c.d = k.shape
    if k.dtype == torch.uint8:
        if k.stride(3) != k.shape[4] or k.shape[4] % 9:
            raise ValueError("k and v of a cache in 4 bits: [page][9 d / 16] dense")
        c.d, c.dtype = k.shape[4] // 9 * 16, LSP_DTYPE_Q4
    else:
        c.dtype = _dtype_code(k.dtype)
    c.seqs, c.max_pages = table.shape
    return c


def make_sample_params(temperature=0.0, seed=0, rnd=0) -> lsp_sample_params:
    return lsp_sample_params(float(temperature), int(rnd) & 0xFFFFFFFF, int(seed) & (2 ** 64 - 1))


# ------------------------------------------------------------------ entry points
def lsp_status_string(status: int) -> str:
    return _f["lsp_status_string"](status).decode()


def lsp_config_check(cfg: lsp_config) -> int:
    return _f["lsp_config_check"](ctypes.byref(cfg))


def lsp_state_bytes(cfg: lsp_config) -> int:
    return _f["lsp_state_bytes"](ctypes.byref(cfg))


def lsp_state_create(cfg: lsp_config) -> int:
    h = c_void_p()
    _check(_f["lsp_state_create"](ctypes.byref(cfg), ctypes.byref(h)), "lsp_state_create")
    return h.value


def lsp_state_destroy(st) -> None:
    _f["lsp_state_destroy"](st)


def lsp_state_init(st, G, stream=None) -> None:
    _check(_f["lsp_state_init"](st, _ptr(G), _stream(stream)), "lsp_state_init")


def lsp_view_update(st, k, v, h, accepted_len, rows=None, stream=None, h_rows=0) -> None:
    """h_rows = 1: h is [C][L][1][H], the hidden state of each request's last new row only."""
    f = lsp_target_feats(_ptr(k), _ptr(v), _ptr(h), int(rows if rows is not None else k.shape[2]), int(h_rows))
    _check(_f["lsp_view_update"](st, ctypes.byref(f), _ptr(accepted_len), _stream(stream)),
           "lsp_view_update")


def lsp_prefill(st, b, k, v, h, rows=None, stream=None, h_rows=0) -> None:
    """k, v: [L][t][nkv][d], h: [L][t][H] of request b's whole prefix ([L][1][H], the last
    row only, with h_rows = 1)."""
    f = lsp_target_feats(_ptr(k), _ptr(v), _ptr(h), int(rows if rows is not None else k.shape[1]),
                         int(h_rows))
    _check(_f["lsp_prefill"](st, int(b), ctypes.byref(f), _stream(stream)), "lsp_prefill")


def lsp_verify(st, target_logits, draft_logits, draft_tokens, sp: lsp_sample_params, accepted_len,
               next_token, stream=None) -> None:
    _check(_f["lsp_verify"](st, _ptr(target_logits), _ptr(draft_logits), _ptr(draft_tokens),
                            ctypes.byref(sp), _ptr(accepted_len), _ptr(next_token), _stream(stream)),
           "lsp_verify")


def lsp_draft(st, block_tokens, weights: lsp_weights, sp: lsp_sample_params, out_tokens,
              out_logits=None, stream=None) -> None:
    _check(_f["lsp_draft"](st, _ptr(block_tokens), ctypes.byref(weights), ctypes.byref(sp),
                           _ptr(out_tokens), _ptr(out_logits), _stream(stream)), "lsp_draft")


def lsp_sample(st, base_logits, prev_token, Ec, Wc, sp: lsp_sample_params, out_tokens,
               out_logits=None, stream=None) -> None:
    _check(_f["lsp_sample"](st, _ptr(base_logits), _ptr(prev_token), _ptr(Ec), _ptr(Wc),
                            ctypes.byref(sp), _ptr(out_tokens), _ptr(out_logits), _stream(stream)),
           "lsp_sample")


def lsp_sample_noalloc(base_logits, prev_token, Ec, Wc, dtype, C, B, V, rc,
                       sp: lsp_sample_params, out_tokens, out_logits=None, dev_error=None,
                       stream=None) -> None:
    _check(_f["lsp_sample_noalloc"](_ptr(base_logits), _ptr(prev_token), _ptr(Ec), _ptr(Wc), dtype,
                                    C, B, V, rc, ctypes.byref(sp), _ptr(out_tokens),
                                    _ptr(out_logits), _ptr(dev_error), _stream(stream)),
           "lsp_sample_noalloc")


def lsp_linear_workspace_bytes(M: int, N: int, splits: int) -> int:
    return _f["lsp_linear_workspace_bytes"](M, N, splits)


def lsp_gemm_plan_info(dtype, M, N, K, swiglu, num_sms):
    """(splits, token groups, token rows per group) of the projection GEMM's plan (host only)."""
    s, g, r = c_int(0), c_int(0), c_int(0)
    _check(_f["lsp_gemm_plan_info"](dtype, M, N, K, int(bool(swiglu)), num_sms, ctypes.byref(s),
                                    ctypes.byref(g), ctypes.byref(r)), "lsp_gemm_plan_info")
    return s.value, g.value, r.value


def lsp_linear(X, W, Y, M, N, K, dtype, splits=1, workspace=None, workspace_bytes=0,
               stream=None) -> None:
    _check(_f["lsp_linear"](_ptr(X), _ptr(W), _ptr(Y), M, N, K, dtype, splits, _ptr(workspace),
                            workspace_bytes, _stream(stream)), "lsp_linear")


def lsp_philox_words(seed, rnd, b, i, out, count, stream=None) -> None:
    _check(_f["lsp_philox_words"](int(seed) & (2 ** 64 - 1), int(rnd), int(b), int(i), _ptr(out),
                                  int(count), _stream(stream)), "lsp_philox_words")


def lsp_get_error(st, clear=True, stream=None):
    """(status, LSP_DEV_* bits) of the state's device error word."""
    bits = c_uint32(0)
    rc = _f["lsp_get_error"](st, ctypes.byref(bits), 1 if clear else 0, _stream(stream))
    return rc, bits.value


def lsp_round_launches(st) -> int:
    return _f["lsp_round_launches"](st)


def lsp_stage_count(st) -> int:
    return _f["lsp_stage_count"](st)


def lsp_stage_name(st, k: int) -> str:
    r = _f["lsp_stage_name"](st, k)
    return r.decode() if r else ""


def lsp_set_stage_events(st, events) -> None:
    """events: a list of torch.cuda.Event(enable_timing=True) (or raw handles); [] turns it off."""
    handles = [e.cuda_event if hasattr(e, "cuda_event") else int(e) for e in events]
    for e in events:
        if hasattr(e, "cuda_event") and e.cuda_event == 0:
            raise ValueError("create each torch.cuda.Event before passing it (record it once)")
    arr = (c_void_p * max(1, len(handles)))(*handles)
    _check(_f["lsp_set_stage_events"](st, arr, len(handles)), "lsp_set_stage_events")


def lsp_state_export(st, host_buf, stream=None) -> None:
    _check(_f["lsp_state_export"](st, _ptr(host_buf), host_buf.numel() * host_buf.element_size(),
                                  _stream(stream)), "lsp_state_export")


def lsp_state_import(st, host_buf, stream=None) -> None:
    _check(_f["lsp_state_import"](st, _ptr(host_buf), host_buf.numel() * host_buf.element_size(),
                                  _stream(stream)), "lsp_state_import")


# The calls below are made once a layer or a round, with kernels of a few microseconds behind them: their
# tensors' addresses are taken in place, and what does not change from call to call is looked up once.
_codes: dict = {}
_int32 = _float32 = None


def _types() -> None:
    global _int32, _float32
    import torch
    _int32, _float32 = torch.int32, torch.float32
    _codes.update({torch.bfloat16: LSP_DTYPE_BF16, torch.float32: LSP_DTYPE_F32})


def _dtype_code(dtype) -> int:
    """LSP_DTYPE_* of a torch type (ValueError for any but bfloat16 and float32)."""
    if not _codes:
        _types()
    if dtype not in _codes:
        raise ValueError("bfloat16 or float32 tensors")
    return _codes[dtype]


def _opt(x):
    return None if x is None else x.data_ptr()


def _dense(t, dtype, n) -> bool:
    """n elements of this type, without gaps: what a bare address stands for."""
    return t.dtype == dtype and t.numel() == n and t.is_contiguous()


def _word(dev_error):
    if dev_error is None:
        return None
    if dev_error.element_size() != 4 or dev_error.numel() < 1:
        raise ValueError("dev_error: a 32-bit word")
    return dev_error.data_ptr()


def _room(workspace):
    """(address, bytes) of a workspace."""
    if not workspace.is_contiguous():
        raise ValueError("workspace: a contiguous tensor")
    return workspace.data_ptr(), workspace.nbytes


def lsp_pages_workspace_bytes(cache: lsp_kv_cache) -> int:
    return _pages_workspace_bytes(cache)


def _entries(a, b) -> int:
    """The entries of a page call: two int32 lists of one length."""
    if not _codes:
        _types()
    n = a.numel()
    if not _dense(a, _int32, n) or not _dense(b, _int32, n):
        raise ValueError("an entry's lists: contiguous int32 of one length")
    return n


def lsp_pages_fork(cache: lsp_kv_cache, src, dst, dev_error=None, stream=None) -> None:
    n = _entries(src, dst)
    _check(_pages_fork(cache, src.data_ptr(), dst.data_ptr(), n, _word(dev_error), _stream(stream)), "lsp_pages_fork")


def lsp_pages_reserve(cache: lsp_kv_cache, seqs, add, workspace, dev_error=None, stream=None) -> None:
    n = _entries(seqs, add)
    _check(_pages_reserve(cache, seqs.data_ptr(), add.data_ptr(), n, *_room(workspace), _word(dev_error),
                          _stream(stream)), "lsp_pages_reserve")


def _rows(cache, k, v, seqs, start):
    """Keys and values of rows that a call moves into or out of a cache: (type, elements between rows, rows, entries)."""
    shape, stride, other, d, n = k.shape, k.stride(), v.stride(), cache.d, seqs.numel()
    # (the stride along an axis of one is never used, and may be anything)
    if (len(shape) != 3 or shape != v.shape or shape[1] != cache.nkv or shape[2] != d or stride[2] != 1 or other[2] != 1
            or shape[1] > 1 and (stride[1] != d or other[1] != d) or shape[0] > 1 and stride[0] != other[0]):
        raise ValueError("keys and values: [total][nkv][d] of the same strides, dense within a row")
    code = _dtype_code(k.dtype)
    if v.dtype != k.dtype:
        raise ValueError("keys and values: one type, the cache's type")
    if not _dense(seqs, _int32, n) or not _dense(start, _int32, n + 1):
        raise ValueError("seqs [n] and start [n + 1]: contiguous int32")
    return code, stride[0], shape[0], n


def lsp_pages_write_q4(cache: lsp_kv_cache, layer, seqs, start, k_new, v_new, dev_error=None, stream=None) -> None:
    """lsp_pages_write into a cache held in 4 bits: bfloat16 or float32 k_new, v_new [total][nkv][d]."""
    code, step, total, n = _rows(cache, k_new, v_new, seqs, start)
    if cache.dtype != LSP_DTYPE_Q4:
        raise ValueError("a cache held in 4 bits")
    _check(_pages_write_q4(cache, layer, seqs.data_ptr(), start.data_ptr(), n, k_new.data_ptr(), v_new.data_ptr(), code,
                           step, total, _word(dev_error), _stream(stream)), "lsp_pages_write_q4")


def lsp_pages_read(cache: lsp_kv_cache, layer, seqs, start, k_out, v_out, dev_error=None, stream=None) -> None:
    """k_out, v_out: [total][nkv][d] of the cache's type (bfloat16 or float32 for a cache held in 4 bits), dense
    within a row, the same stride between rows; rows [start[i], start[i + 1]) get the last tokens of sequence seqs[i]."""
    code, step, total, n = _rows(cache, k_out, v_out, seqs, start)
    if cache.dtype != code and cache.dtype != LSP_DTYPE_Q4:
        raise ValueError("k_out and v_out: the cache's type")
    _check(_pages_read(cache, layer, seqs.data_ptr(), start.data_ptr(), n, k_out.data_ptr(), v_out.data_ptr(), code, step,
                       total, _word(dev_error), _stream(stream)), "lsp_pages_read")


def lsp_pages_write(cache: lsp_kv_cache, layer, seqs, start, k_new, v_new, dev_error=None, stream=None) -> None:
    """k_new, v_new: [total][nkv][d] of the cache's type, dense within a row, the same stride between rows; seqs
    [n], start [n + 1] int32."""
    code, step, total, n = _rows(cache, k_new, v_new, seqs, start)
    if cache.dtype != code:
        raise ValueError("k_new and v_new: the cache's type")
    _check(_pages_write(cache, layer, seqs.data_ptr(), start.data_ptr(), n, k_new.data_ptr(), v_new.data_ptr(),
                        step, total, _word(dev_error), _stream(stream)), "lsp_pages_write")


def lsp_pages_trim(cache: lsp_kv_cache, seqs, new_len, dev_error=None, stream=None) -> None:
    n = _entries(seqs, new_len)
    _check(_pages_trim(cache, seqs.data_ptr(), new_len.data_ptr(), n, _word(dev_error), _stream(stream)),
           "lsp_pages_trim")


def lsp_pages_compact(cache: lsp_kv_cache, live, workspace, stream=None) -> None:
    """live: int32 [1] that receives the number of live pages, or None."""
    if not _codes:
        _types()
    if live is not None and not _dense(live, _int32, 1):
        raise ValueError("live: one int32")
    _check(_pages_compact(cache, _opt(live), *_room(workspace), _stream(stream)), "lsp_pages_compact")


def lsp_prefix_attention_workspace_bytes(cache: lsp_kv_cache, nq: int, n: int, total: int) -> int:
    return _prefix_attention_workspace_bytes(cache, nq, n, total)


def lsp_prefix_attention_q4_workspace_bytes(cache: lsp_kv_cache, dtype, nq: int, n: int, total: int) -> int:
    """dtype: of the rows, torch.bfloat16 or torch.float32."""
    return _prefix_attention_q4_workspace_bytes(cache, _dtype_code(dtype), nq, n, total)


def _attention_rows(cache, q, seqs, start, out, lse):
    """Arguments that both attention calls take: (type, elements between rows, rows, heads, entries)."""
    shape, stride, d, n = q.shape, q.stride(), cache.d, seqs.numel()
    if (len(shape) != 3 or stride[1] != d and shape[1] > 1 or stride[2] != 1 or shape[2] != d or out.shape != shape
            or not out.is_contiguous()):
        raise ValueError("q: [total][nq][d], dense within a row; out: the same shape, contiguous")
    code = _dtype_code(q.dtype)
    if out.dtype != q.dtype:
        raise ValueError("q and out: one type, the cache's type")
    if not _dense(seqs, _int32, n) or not _dense(start, _int32, n + 1):
        raise ValueError("seqs [n] and start [n + 1]: contiguous int32")
    if lse is not None and not _dense(lse, _float32, shape[0] * shape[1]):
        raise ValueError("lse: contiguous float32 [total][nq]")
    return code, stride[0], shape[0], shape[1], n


def lsp_prefix_attention(cache: lsp_kv_cache, layer, q, seqs, start, out, lse=None, *, shared_len, scale,
                         workspace, dev_error=None, stream=None) -> None:
    """q: [total][nq][d] of the cache's type, dense within a row (a slice of a fused q/k/v row will do); out:
    the same, dense; seqs [n], start [n + 1] int32; lse: float32 [total][nq] or None."""
    code, step, total, nq, n = _attention_rows(cache, q, seqs, start, out, lse)
    if code != cache.dtype:
        raise ValueError("q and out: the cache's type")
    _check(_prefix_attention(cache, layer, q.data_ptr(), step, nq, seqs.data_ptr(), start.data_ptr(), n, total,
                             shared_len, scale, out.data_ptr(), _opt(lse), *_room(workspace),
                             _word(dev_error), _stream(stream)), "lsp_prefix_attention")


def lsp_prefix_attention_q4(cache: lsp_kv_cache, layer, q, seqs, start, out, lse=None, *, shared_len, scale,
                            workspace, dev_error=None, stream=None) -> None:
    """lsp_prefix_attention over a cache held in 4 bits: q and out bfloat16 or float32."""
    code, step, total, nq, n = _attention_rows(cache, q, seqs, start, out, lse)
    if cache.dtype != LSP_DTYPE_Q4:
        raise ValueError("a cache held in 4 bits")
    _check(_prefix_attention_q4(cache, layer, q.data_ptr(), code, step, nq, seqs.data_ptr(), start.data_ptr(), n, total,
                                shared_len, scale, out.data_ptr(), _opt(lse), *_room(workspace),
                                _word(dev_error), _stream(stream)), "lsp_prefix_attention_q4")


def _row_stride(t, C, rows, V):
    """Elements between the rows of t [C][rows][V], evenly spaced."""
    stride = t.stride()
    ld = stride[1] if rows > 1 else stride[0] if C > 1 else max(V, stride[1])
    if t.shape != (C, rows, V) or (V > 1 and stride[2] != 1) or (C > 1 and stride[0] != rows * ld):
        raise ValueError("target_probs [C][B+1][V] and draft_probs [C][B][V], rows evenly spaced")
    return ld


def lsp_verify_probs(target_probs, draft_probs, draft_tokens, u, e, accepted_len, next_token, n_draft=None,
                     out_tokens=None, dev_error=None, stream=None) -> None:
    """target_probs [C][B+1][V], draft_probs [C][B][V] (or None) of one type, bfloat16 or float32; the
    stride between their rows may exceed V.  Contiguous: int32 draft_tokens [C][B], n_draft [C], accepted_len
    [C], next_token [C] and out_tokens [C][B+1], float32 u [C][B] and e [C][V]."""
    C, B = draft_tokens.shape
    V, dtype = target_probs.shape[2], target_probs.dtype
    code, ld_q, drafted = _dtype_code(dtype), 0, None
    ld_t = _row_stride(target_probs, C, B + 1, V)
    if draft_probs is not None and B > 0:
        if draft_probs.dtype != dtype:
            raise ValueError("target_probs and draft_probs: one type")
        ld_q, drafted = _row_stride(draft_probs, C, B, V), draft_probs.data_ptr()
    if not _dense(u, _float32, C * B) or not _dense(e, _float32, C * V):
        raise ValueError("u [C][B] and e [C][V]: contiguous float32")
    if (not _dense(draft_tokens, _int32, C * B) or not _dense(accepted_len, _int32, C) or not _dense(next_token, _int32, C)
            or n_draft is not None and not _dense(n_draft, _int32, C)
            or out_tokens is not None and not _dense(out_tokens, _int32, C * (B + 1))):
        raise ValueError("draft_tokens, n_draft, accepted_len, next_token and out_tokens: contiguous int32 of their sizes")
    _check(_verify_probs(target_probs.data_ptr(), drafted, code, draft_tokens.data_ptr(), _opt(n_draft),
                         u.data_ptr(), e.data_ptr(), C, B, V, ld_t, ld_q, accepted_len.data_ptr(),
                         next_token.data_ptr(), _opt(out_tokens), _word(dev_error), _stream(stream)),
           "lsp_verify_probs")


def lsp_logprobs(logits, tokens, logprob, entropy=None, top=None, top_logprob=None, *, temperature=1.0, dev_error=None,
                 stream=None) -> None:
    """logits [rows][V] bfloat16 or float32, dense within a row (which may be followed by anything).
    Contiguous: int32 tokens [rows] (-1: none) and top [rows][k], float32 logprob and entropy [rows], top_logprob
    [rows][k]; all but logprob may be None."""
    if logits.dim() != 2:
        raise ValueError("logits: [rows][V]")
    rows, V = logits.shape
    stride, k = logits.stride(), 0
    code = _dtype_code(logits.dtype)
    if V > 1 and stride[1] != 1 or rows > 1 and stride[0] < V:
        raise ValueError("logits: [rows][V], dense within a row")
    if not _dense(tokens, _int32, rows) or not _dense(logprob, _float32, rows) or entropy is not None and not _dense(entropy, _float32, rows):
        raise ValueError("tokens [rows]: contiguous int32; logprob and entropy [rows]: contiguous float32")
    for t, dtype in ((top, _int32), (top_logprob, _float32)):
        if t is not None:
            if t.dim() != 2 or not _dense(t, dtype, rows * t.shape[1]):
                raise ValueError("top: contiguous int32 [rows][k]; top_logprob: contiguous float32 [rows][k]")
            k = t.shape[1]
    if top is not None and top_logprob is not None and top.shape != top_logprob.shape:
        raise ValueError("top and top_logprob: one shape")
    _check(_logprobs(logits.data_ptr(), code, tokens.data_ptr(), rows, V, stride[0] if rows > 1 else V, temperature, k,
                     logprob.data_ptr(), _opt(entropy), _opt(top), _opt(top_logprob), _word(dev_error), _stream(stream)),
           "lsp_logprobs")


EXPORTED = sorted(_f)
