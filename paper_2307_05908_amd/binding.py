"""ctypes binding of libppd (include/ppd.h, include/ppd_measure.h, include/ppd_layers.h): argument marshalling only.

Every step of the decode path runs in the HIP kernels behind the C ABI; this
module turns torch device tensors into the pointer tables the library takes
and mirrors its entry points under the same names.  There is no CPU fallback:
if the library cannot be loaded, importing the symbols raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct
from typing import Dict, List, NamedTuple, Optional

import numpy as np

from . import build as _build

PPD_MAX_K = 8
KERNEL_CLASSES = ("embed", "gemm_qkv", "attn", "attn_merge", "gemm_o", "gemm_ffn_in", "gemm_ffn_out",
                  "head", "select", "commit", "phase")
_LAYER_FIELDS = ("ln1_g", "ln1_b", "wq", "wk", "wv", "wo", "bq", "bk", "bv", "bo",
                 "ln2_g", "ln2_b", "w_in", "w_up", "w_out", "b_in", "b_out")
# order of the per-layer members in ppd_weights
_W_LAYER_ORDER = ("ln1_g", "ln1_b", "wq", "wk", "wv", "wo", "bq", "bk", "bv", "bo",
                  "ln2_g", "ln2_b", "w_in", "w_up", "w_out", "b_in", "b_out")


class ModelDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("n_layers", "d_model", "n_heads", "head_dim", "d_ff", "vocab", "max_ctx",
                 "norm", "act", "pos", "has_bias", "wdtype")] + \
               [("norm_eps", ctypes.c_float), ("rope_theta", ctypes.c_float), ("eos_id", ctypes.c_int32)]


class Weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("tok_emb", "pos_emb", "lnf_g", "lnf_b", "lm_head", "early_head")] + \
               [(n, ctypes.POINTER(ctypes.c_void_p)) for n in _W_LAYER_ORDER]


class StepInfo(ctypes.Structure):
    _fields_ = [("token", ctypes.c_int32), ("matched", ctypes.c_int32), ("match_idx", ctypes.c_int32),
                ("cand", ctypes.c_int32 * PPD_MAX_K)]


class Stats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint64) for n in
                ("rounds", "matches", "runs", "main_layer_rows", "branch_layer_rows", "plain_steps",
                 "weight_bytes", "kv_bytes")]


class PagedCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + \
               [(n, ctypes.c_int64) for n in ("k_page", "k_pos", "k_head", "v_page", "v_pos", "v_head")] + \
               [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "n_kv_heads", "head_dim", "dtype")]


class PagedBatch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q_start", "kv_len", "pages")] + [("pages_stride", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("max_pages", "n_seqs", "n_tokens")]


class Rows(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class PageTable(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("pages_stride", ctypes.c_int64), ("free_pages", ctypes.c_void_p)] + \
               [(n, ctypes.c_int32) for n in ("max_pages", "n_pages", "page_size", "n_seqs")]


class PagedCacheFp4(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_scales", "v_scales")] + \
               [(n, ctypes.c_int64) for n in ("k_page", "k_pos", "k_head", "v_page", "v_pos", "v_head",
                                              "ks_page", "ks_pos", "ks_head", "vs_page", "vs_pos", "vs_head")] + \
               [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "n_kv_heads", "head_dim", "dtype")]


class LogitRules(ctypes.Structure):
    _fields_ = [("history", ctypes.c_void_p), ("history_stride", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in ("history_len", "prompt_len", "repetition", "presence", "frequency", "bias_start", "bias_ids", "bias", "mask")] + \
               [("mask_stride", ctypes.c_int64), ("mask_row", ctypes.c_void_p), ("n_bias", ctypes.c_int32), ("n_masks", ctypes.c_int32)]


EXPORTS = ("ppd_create", "ppd_reset", "ppd_prefill", "ppd_step", "plain_greedy_step", "ppd_get_logits",
           "ppd_get_early_logits", "ppd_get_stats", "ppd_set_profiling", "ppd_set_graphs", "ppd_set_sampling", "ppd_get_kernel_time",
           "ppd_time_ffn_in", "ppd_get_chain_rounds", "ppd_set_chain_wait", "ppd_stream_read_probe", "ppd_early_topk", "ppd_early_topk_noalloc", "ppd_destroy",
           "ppd_strerror", "ppd_last_hip_error",
           "ppd_paged_append", "ppd_paged_attention", "ppd_paged_attention_workspace", "ppd_verify_drafts", "ppd_verify_drafts_workspace",
           "ppd_paged_plan", "ppd_adjust_logits")
# (those with a digit in their names)
FP4_EXPORTS = ("ppd_paged_append_fp4", "ppd_paged_attention_fp4", "ppd_paged_attention_fp4_workspace")

_lib = None


def load_library() -> ctypes.CDLL:
    """Load libppd.so (built in-tree).  Raises if it is missing and cannot be built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB_PATH):
        _build.build(True)
    # torch ships its own HIP runtime (same soname).  Import it first so that libppd binds to the
    # runtime that owns the caller's tensors and streams; loaded the other way round the process
    # would hold two HIP runtimes and device pointers of one would be unknown to the other.
    import torch  # noqa: F401
    lib = ctypes.CDLL(_build.LIB_PATH)
    vp, ci = ctypes.c_void_p, ctypes.c_int
    lib.ppd_create.argtypes = [ctypes.POINTER(ModelDims), ctypes.POINTER(Weights), ci, ci, vp, ctypes.POINTER(vp)]
    lib.ppd_reset.argtypes = [vp]
    lib.ppd_prefill.argtypes = [vp, vp, ci]
    lib.ppd_step.argtypes = [vp, vp, ci, ctypes.POINTER(StepInfo)]
    lib.plain_greedy_step.argtypes = [vp, vp]
    lib.ppd_get_logits.argtypes = [vp, vp]
    lib.ppd_get_early_logits.argtypes = [vp, vp]
    lib.ppd_get_stats.argtypes = [vp, ctypes.POINTER(Stats)]
    lib.ppd_set_profiling.argtypes = [vp, ci]
    lib.ppd_set_graphs.argtypes = [vp, ci]
    lib.ppd_set_sampling.argtypes = [vp, ci, ci, ctypes.c_double, ctypes.c_uint64]
    lib.ppd_get_kernel_time.argtypes = [vp, ci, ci, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_uint64)]
    lib.ppd_time_ffn_in.argtypes = [vp, ci, ci, ctypes.POINTER(ctypes.c_double)]
    lib.ppd_get_chain_rounds.argtypes = [vp, ctypes.POINTER(ctypes.c_uint64), ctypes.POINTER(ctypes.c_uint64)]
    lib.ppd_set_chain_wait.argtypes = [vp, ci]
    lib.ppd_stream_read_probe.argtypes = [vp, ctypes.c_uint64, ci, ctypes.POINTER(ctypes.c_double)]
    lib.ppd_early_topk.argtypes = [ci, ci, ci, ctypes.c_float, ci, vp, vp, vp, vp, ci, vp, vp, vp, vp]
    lib.ppd_early_topk_noalloc.argtypes = lib.ppd_early_topk.argtypes
    cp, bp, rp = ctypes.POINTER(PagedCache), ctypes.POINTER(PagedBatch), ctypes.POINTER(Rows)
    cl, cu, cf = ctypes.c_int64, ctypes.c_uint64, ctypes.c_float
    lib.ppd_paged_append.argtypes = [cp, bp, ci, rp, rp, rp, rp, vp, vp, cf, ci, cf, vp]
    lib.ppd_paged_attention.argtypes = [cp, bp, ci, rp, rp, vp, cf, ci, vp, cu, vp]
    lib.ppd_paged_attention_workspace.argtypes = [cp, bp, ci, ctypes.POINTER(cu)]
    lib.ppd_verify_drafts.argtypes = [ci, ci, ci, ci, vp, vp, vp, cl, vp, cl, vp, vp, vp, vp, vp, cu, vp]
    lib.ppd_verify_drafts_workspace.argtypes = [ci, ci, ci, ci, ctypes.POINTER(cu)]
    tp, fp, lp = ctypes.POINTER(PageTable), ctypes.POINTER(PagedCacheFp4), ctypes.POINTER(LogitRules)
    lib.ppd_paged_plan.argtypes = [tp, vp, vp, vp, vp, vp, ci, vp, vp, vp, vp, vp, vp, vp]
    lib.ppd_paged_append_fp4.argtypes = [fp, bp, ci, rp, rp, rp, rp, rp, rp, vp, vp, cf, ci, cf, vp]
    lib.ppd_paged_attention_fp4.argtypes = [fp, bp, ci, rp, rp, vp, cf, ci, vp, cu, vp]
    lib.ppd_paged_attention_fp4_workspace.argtypes = [fp, bp, ci, ctypes.POINTER(cu)]
    lib.ppd_adjust_logits.argtypes = [ci, ci, ci, ci, vp, vp, vp, cl, vp, cl, lp, vp]
    lib.ppd_destroy.argtypes = [vp]
    lib.ppd_destroy.restype = None
    lib.ppd_strerror.argtypes = [ci]
    lib.ppd_strerror.restype = ctypes.c_char_p
    lib.ppd_last_hip_error.argtypes = [vp]
    _lib = lib
    return lib


class PPDError(RuntimeError):
    def __init__(self, code: int, what: str, hip: int = 0):
        msg = load_library().ppd_strerror(code).decode()
        super().__init__(f"{what}: {msg} (code {code}" + (f", hipError {hip})" if hip else ")"))
        self.code = code


def upload_model(model, device="cuda:0") -> Dict[str, object]:
    """Copy a host model (``cfg``, ``g``, ``layers`` of numpy arrays; bf16 as uint16 bits) to the GPU.
    Returns {name: tensor or list of tensors}; torch is used for device memory only."""
    import torch

    def up(a):
        if a is None:
            return None
        t = torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a)
        t = t.to(device)
        return t.view(torch.bfloat16) if a.dtype == np.uint16 else t

    dev = {k: up(v) for k, v in model.g.items()}
    for f in _LAYER_FIELDS:
        dev[f] = [up(a) for a in model.layers[f]]
    return dev


def ppd_stream_read_probe(dev_tensor, iters: int = 5) -> float:
    """GB/s of a plain streaming read of a device tensor (measurement aid of the library)."""
    nbytes = dev_tensor.numel() * dev_tensor.element_size()
    out = ctypes.c_double(0.0)
    rc = load_library().ppd_stream_read_probe(dev_tensor.data_ptr(), nbytes, iters, ctypes.byref(out))
    if rc != 0:
        raise PPDError(rc, "ppd_stream_read_probe", load_library().ppd_last_hip_error(None))
    return float(out.value)


def _early_topk_call(fn_name, h, norm_g, norm_b, head, k, norm, norm_eps, want_logits, stream):
    import torch
    lib = load_library()
    vocab, d_model = head.shape
    wdtype = 0 if head.dtype == torch.float32 else 1
    ids = torch.empty(k, dtype=torch.int32, device=h.device)
    vals = torch.empty(k, dtype=torch.float32, device=h.device)
    logits = torch.empty(vocab, dtype=torch.float32, device=h.device) if want_logits else None
    st = stream if stream is not None else torch.cuda.current_stream()
    rc = getattr(lib, fn_name)(d_model, vocab, int(norm), float(norm_eps), wdtype, norm_g.data_ptr(),
                               None if norm_b is None else norm_b.data_ptr(), head.data_ptr(), h.data_ptr(), int(k),
                               ids.data_ptr(), vals.data_ptr(), None if logits is None else logits.data_ptr(),
                               ctypes.c_void_p(st.cuda_stream))
    if rc != 0:
        raise PPDError(rc, fn_name, lib.ppd_last_hip_error(None))
    return ids, vals, logits


def ppd_early_topk(h, norm_g, norm_b, head, k, norm, norm_eps=1e-5, want_logits=False, stream=None):
    """Stand-alone early prediction on device tensors: (ids int32[k], logits of those float[k], all logits or None).
    h: float32 [d_model]; norm_g / norm_b / head: float32 or bfloat16 tensors of the model's weight type."""
    return _early_topk_call("ppd_early_topk", h, norm_g, norm_b, head, k, norm, norm_eps, want_logits, stream)


def ppd_early_topk_noalloc(h, norm_g, norm_b, head, k, norm, norm_eps=1e-5, want_logits=False, stream=None):
    """The same through the entry point that allocates nothing (fixed scratch array in the library; asynchronous:
    the outputs are complete once the stream's work has run).  The output tensors are the caller's, made here."""
    return _early_topk_call("ppd_early_topk_noalloc", h, norm_g, norm_b, head, k, norm, norm_eps, want_logits, stream)


# ---- operators on paged keys and values (include/ppd_layers.h)
# A call's host side is most of its time where there is little to do, so the structs go over as packed bytes (the layouts of PagedCache,
# PagedBatch and Rows) and each check is made once.
_PACK_CACHE, _PACK_BATCH, _PACK_ROWS = struct.Struct("@QQ6q5i4x").pack, struct.Struct("@3Qq3i4x").pack, struct.Struct("@Q2q").pack
_fast = None


def _layers():
    """torch, the type codes, and the library's functions as they are called here."""
    global _fast
    if _fast is None:
        import torch
        lib = load_library()
        vp, ci, cl, cu, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float

        def fn(name, *argtypes):
            f = lib._FuncPtr((name, lib))
            f.argtypes = argtypes
            return f

        _fast = (torch, {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream,
                 fn("ppd_paged_append", vp, vp, ci, vp, vp, vp, vp, vp, vp, cf, ci, cf, vp),
                 fn("ppd_paged_attention", vp, vp, ci, vp, vp, vp, cf, ci, vp, cu, vp),
                 fn("ppd_verify_drafts", ci, ci, ci, ci, vp, vp, vp, cl, vp, cl, vp, vp, vp, vp, vp, cu, vp))
    return _fast


def _on_device(first, others, stream, call):
    """call() with the tensors' GPU as the current one, on `stream`, which is where it allocates too.  Tensors that another stream than the
    current one reads or writes are not given away before that stream is done with them."""
    torch = _layers()[0]
    dev = first.device
    if dev.type != "cuda":
        raise ValueError("tensors on a GPU")
    with torch.cuda.device(dev):
        if stream is None or stream == torch.cuda.current_stream():
            return call()
        if stream.device != dev:
            raise ValueError("the stream is another GPU's")
        for t in (first, *others):
            if t is not None:
                t.record_stream(stream)
        with torch.cuda.stream(stream):
            return call()


def _same_gpu(dev, *tensors):
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("all tensors on one GPU")


def _scratch(workspace):
    """(address, bytes): those that lie in a row."""
    if workspace is None:
        return None, 0
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return workspace.data_ptr(), workspace.nbytes


def _paged_batch(i32, pages, q_start, kv_len, n_tokens):
    """(batch as bytes, entries of a row of the table, sequences)."""
    if pages.dtype is not i32 or q_start.dtype is not i32 or kv_len.dtype is not i32:
        raise ValueError("pages, q_start, kv_len: int32")
    n, table = kv_len.numel(), pages.shape
    if len(table) != 2 or table[0] != n or q_start.numel() != n + 1:
        raise ValueError("pages [n_seqs, max_pages], q_start [n_seqs + 1], kv_len [n_seqs]")
    most, (p0, p1) = table[1], pages.stride()
    if not (q_start.is_contiguous() and kv_len.is_contiguous()) or (p1 != 1 and most > 1):
        raise ValueError("q_start, kv_len and the rows of pages must be contiguous")
    return _PACK_BATCH(q_start.data_ptr(), kv_len.data_ptr(), pages.data_ptr(), p0, most, n, n_tokens), most, n


def _paged_args(k_cache, v_cache, pages, q_start, kv_len, n_tokens):
    """(cache, batch) as bytes, and the sizes that a workspace depends on."""
    torch, codes = _layers()[:2]
    shape, dtype, i32 = k_cache.shape, k_cache.dtype, torch.int32
    if len(shape) != 4 or v_cache.shape != shape or dtype not in codes or v_cache.dtype is not dtype:
        raise ValueError("k_cache, v_cache: [n_pages, page_size, n_kv_heads, head_dim], both float32, bfloat16 or float16")
    n_pages, size, kv_heads, head_dim = shape
    k0, k1, k2, k3 = k_cache.stride()
    v0, v1, v2, v3 = v_cache.stride()
    if k3 != 1 or v3 != 1:
        raise ValueError("k_cache, v_cache: head_dim must be contiguous")
    code = codes[dtype]
    batch, most, n = _paged_batch(i32, pages, q_start, kv_len, n_tokens)
    return (_PACK_CACHE(k_cache.data_ptr(), v_cache.data_ptr(), k0, k1, k2, v0, v1, v2, n_pages, size, kv_heads, head_dim, code), batch,
            (n_pages, size, kv_heads, head_dim, code, most, n, n_tokens))


def _rows(t, dtype, head_dim, what, n_tokens, heads=None):
    """The rows as bytes, and their heads."""
    shape = t.shape
    if len(shape) == 3:
        n, h, d = shape
        if n == n_tokens and d == head_dim and t.dtype is dtype and (heads is None or h == heads):
            s0, s1, s2 = t.stride()
            if s2 != 1:
                raise ValueError(what + ": head_dim must be contiguous")
            return _PACK_ROWS(t.data_ptr(), s0, s1), h
    raise ValueError(what + ": [n_tokens, heads, head_dim] of the cache's type")


def ppd_paged_append(k_cache, v_cache, pages, q_start, kv_len, q, k, v, q_gain=None, k_gain=None, norm_eps=1e-5, rotary_dim=0,
                     rope_theta=10000.0, q_out=None, stream=None):
    """Queries and keys of a ragged batch normalised per head (where a gain is given) and rotated, keys and values written to their
    pages.  q [n_tokens, n_heads, head_dim] (None: keys and values only), k and v [n_tokens, n_kv_heads, head_dim].  Returns q_out
    (made here if not given, without contents where a row belongs to no sequence; may be q itself).  Asynchronous."""
    torch, _, device, raw_stream, append, _, _ = _layers()
    dev = k_cache.get_device()
    if stream is not None or dev < 0 or dev != device():
        return _on_device(k_cache, (v_cache, pages, q_start, kv_len, q, k, v, q_gain, k_gain, q_out), stream, lambda: ppd_paged_append(
            k_cache, v_cache, pages, q_start, kv_len, q, k, v, q_gain, k_gain, norm_eps, rotary_dim, rope_theta, q_out))
    _same_gpu(dev, v_cache, pages, q_start, kv_len, q, k, v, q_gain, k_gain, q_out)
    n = k.shape[0]
    cache, batch, sizes = _paged_args(k_cache, v_cache, pages, q_start, kv_len, n)
    dtype, kv_heads, head_dim = k_cache.dtype, sizes[2], sizes[3]
    kr, vr = _rows(k, dtype, head_dim, "k", n, kv_heads)[0], _rows(v, dtype, head_dim, "v", n, kv_heads)[0]
    qr, outr, heads = None, None, 0
    if q is not None:
        qr, heads = _rows(q, dtype, head_dim, "q", n)
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        outr = _rows(q_out, dtype, head_dim, "q_out", n, heads)[0]
    for g in (q_gain, k_gain):
        if g is not None and (g.dtype is not dtype or g.numel() != head_dim or not g.is_contiguous()):
            raise ValueError("gains: [head_dim] of the cache's type")
    rc = append(cache, batch, heads, qr, outr, kr, vr, None if q_gain is None else q_gain.data_ptr(), None if k_gain is None else k_gain.data_ptr(),
                norm_eps, rotary_dim, rope_theta, raw_stream(dev))
    if rc != 0:
        raise PPDError(rc, "ppd_paged_append", load_library().ppd_last_hip_error(None))
    return q_out if q is not None else None


@functools.lru_cache(maxsize=4096)
def _attention_workspace(sizes, heads):
    """Bytes that ppd_paged_attention_workspace gives for these sizes (0 where it refuses: the call itself will)."""
    pages, size, kv_heads, head_dim, code, max_pages, seqs, tokens = sizes
    c = PagedCache(4096, 4096, 0, 0, 0, 0, 0, 0, pages, size, kv_heads, head_dim, code)
    b = PagedBatch(4096, 4096, 4096, max_pages, max_pages, seqs, tokens)
    need = ctypes.c_uint64()
    return need.value if load_library().ppd_paged_attention_workspace(c, b, heads, need) == 0 else 0


def ppd_paged_attention(q, k_cache, v_cache, pages, q_start, kv_len, scale=None, window=0, out=None, want_lse=False, workspace=None, stream=None):
    """Attention of a ragged batch's new tokens over their sequences' pages: (out [n_tokens, n_heads, head_dim], lse float32
    [n_tokens, n_heads] or None).  scale None: 1 / sqrt(head_dim).  out, and workspace (a uint8 tensor), are made here if not given; rows
    of no sequence keep what out holds (a new one holds nothing there).  Asynchronous."""
    torch, _, device, raw_stream, _, attention, _ = _layers()
    dev = k_cache.get_device()
    if stream is not None or dev < 0 or dev != device():
        return _on_device(k_cache, (q, v_cache, pages, q_start, kv_len, out, workspace), stream, lambda: ppd_paged_attention(
            q, k_cache, v_cache, pages, q_start, kv_len, scale, window, out, want_lse, workspace))
    _same_gpu(dev, q, v_cache, pages, q_start, kv_len, out, workspace)
    n = q.shape[0]
    cache, batch, sizes = _paged_args(k_cache, v_cache, pages, q_start, kv_len, n)
    dtype, head_dim = k_cache.dtype, sizes[3]
    qr, heads = _rows(q, dtype, head_dim, "q", n)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    outr = _rows(out, dtype, head_dim, "out", n, heads)[0]
    lse = torch.empty((n, heads), dtype=torch.float32, device=q.device) if want_lse else None
    if workspace is None:
        need = _attention_workspace(sizes, heads)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    rc = attention(cache, batch, heads, qr, outr, None if lse is None else lse.data_ptr(), head_dim ** -0.5 if scale is None else scale, window,
                   *_scratch(workspace), raw_stream(dev))
    if rc != 0:
        raise PPDError(rc, "ppd_paged_attention", load_library().ppd_last_hip_error(None))
    return out, lse


@functools.lru_cache(maxsize=4096)
def _verify_workspace(seqs, rows, vocab, code):
    need = ctypes.c_uint64()
    return need.value if load_library().ppd_verify_drafts_workspace(seqs, rows, vocab, code, need) == 0 else 0


def ppd_verify_drafts(target_logits, ids, row_start, uniform, draft_logits=None, temperature=None, tokens=None, accepted=None, workspace=None,
                      stream=None):
    """Drafted tokens against the target model's logits: (tokens int32 [n_rows], accepted int32 [n_seqs]).  target_logits and
    draft_logits [n_rows, vocab], ids int32 [n_rows], row_start int32 [n_seqs + 1], uniform float32 [n_rows, 2], temperature float32
    [n_seqs] (0: arg max).  tokens, accepted and workspace (a uint8 tensor) are made here if not given.  Asynchronous."""
    torch, codes, device, raw_stream, _, _, verify = _layers()
    z, d = target_logits, draft_logits
    dev = z.get_device()
    if stream is not None or dev < 0 or dev != device():
        return _on_device(z, (ids, row_start, uniform, d, temperature, tokens, accepted, workspace), stream, lambda: ppd_verify_drafts(
            z, ids, row_start, uniform, d, temperature, tokens, accepted, workspace))
    _same_gpu(dev, ids, row_start, uniform, d, temperature, tokens, accepted, workspace)
    i32, f32 = torch.int32, torch.float32
    if z.dim() != 2 or z.dtype not in codes or (z.shape[1] > 1 and z.stride(1) != 1):
        raise ValueError("target_logits: [n_rows, vocab], vocab contiguous, float32, bfloat16 or float16")
    n, vocab = z.shape
    if d is not None and (d.shape != z.shape or d.dtype != z.dtype or (vocab > 1 and d.stride(1) != 1)):
        raise ValueError("draft_logits: as target_logits")
    seqs = row_start.numel() - 1
    if ids.dtype != i32 or ids.numel() != n or row_start.dtype != i32 or seqs < 1:
        raise ValueError("ids int32 [n_rows], row_start int32 [n_seqs + 1]")
    if uniform.dtype != f32 or uniform.numel() != 2 * n or (temperature is not None and (temperature.dtype != f32 or temperature.numel() != seqs)):
        raise ValueError("uniform float32 [n_rows, 2], temperature float32 [n_seqs]")
    if tokens is None:
        tokens = torch.empty(n, dtype=i32, device=z.device)
    if accepted is None:
        accepted = torch.empty(seqs, dtype=i32, device=z.device)
    if tokens.dtype != i32 or tokens.numel() != n or accepted.dtype != i32 or accepted.numel() != seqs:
        raise ValueError("tokens int32 [n_rows], accepted int32 [n_seqs]")
    if not all(x is None or x.is_contiguous() for x in (ids, row_start, uniform, temperature, tokens, accepted)):
        raise ValueError("all but the logits must be contiguous")
    code = codes[z.dtype]
    if workspace is None:
        need = _verify_workspace(seqs, n, vocab, code)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=z.device)
    rc = verify(seqs, n, vocab, code, row_start.data_ptr(), ids.data_ptr(), z.data_ptr(), z.stride(0) if n > 1 else vocab,
                None if d is None else d.data_ptr(), 0 if d is None else d.stride(0) if n > 1 else vocab,
                None if temperature is None else temperature.data_ptr(), uniform.data_ptr(), tokens.data_ptr(), accepted.data_ptr(),
                *_scratch(workspace), raw_stream(dev))
    if rc != 0:
        raise PPDError(rc, "ppd_verify_drafts", load_library().ppd_last_hip_error(None))
    return tokens, accepted


# ---- a step's batch, pages of 4-bit numbers, logits as requests want them
_PACK_TABLE, _PACK_CACHE_FP4 = struct.Struct("@QqQ4i").pack, struct.Struct("@4Q12q5i4x").pack
_PACK_RULES = struct.Struct("@Qq9QqQ2i").pack
_step_fns = None


def _step():
    """torch, the type codes, and the library's functions as they are called here."""
    global _step_fns
    if _step_fns is None:
        torch, codes, device, raw_stream = _layers()[:4]
        lib = load_library()
        vp, ci, cl, cu, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float

        def fn(name, *argtypes):
            f = lib._FuncPtr((name, lib))
            f.argtypes = argtypes
            return f

        _step_fns = (torch, codes, device, raw_stream,
                     fn("ppd_paged_plan", vp, vp, vp, vp, vp, vp, ci, vp, vp, vp, vp, vp, vp, vp),
                     fn("ppd_paged_append_fp4", vp, vp, ci, vp, vp, vp, vp, vp, vp, vp, vp, cf, ci, cf, vp),
                     fn("ppd_paged_attention_fp4", vp, vp, ci, vp, vp, vp, cf, ci, vp, cu, vp),
                     fn("ppd_adjust_logits", ci, ci, ci, ci, vp, vp, vp, cl, vp, cl, vp, vp))
    return _step_fns


def _ptr(t):
    return None if t is None else t.data_ptr()


class Plan(NamedTuple):
    """What ppd_paged_plan gives: q_start, kv_len and granted are a batch for the operators on pages; row_seq, positions and slots are None
    where they were not asked for."""
    q_start: object
    kv_len: object
    granted: object
    counters: object
    row_seq: object
    positions: object
    slots: object


def ppd_paged_plan(pages, free_pages, counters, held, wanted, page_size, n_rows, kept=None, want_rows=True, q_start=None, kv_len=None, granted=None,
                   counters_out=None, row_seq=None, positions=None, slots=None, stream=None):
    """A step's batch from what each sequence holds, keeps and wants: pages int32 [n_seqs, max_pages] and free_pages int32 [n_pages] are changed
    in place, counters int64 [2], held, wanted and kept (None: all stays) int32 [n_seqs], n_rows the rows of the batch's tensors.  Returns
    a Plan; its tensors are made here if not given (kv_len may be held, counters_out counters), row_seq, positions and slots only with want_rows.
    Asynchronous."""
    torch, _, device, raw_stream, plan, _, _, _ = _step()
    dev = pages.get_device()
    given = (q_start, kv_len, granted, counters_out, row_seq, positions, slots)
    if stream is not None or dev < 0 or dev != device():
        return _on_device(pages, (free_pages, counters, held, wanted, kept, *given), stream, lambda: ppd_paged_plan(
            pages, free_pages, counters, held, wanted, page_size, n_rows, kept, want_rows, *given))
    _same_gpu(dev, free_pages, counters, held, wanted, kept, *given)
    i32, i64 = torch.int32, torch.int64
    n = held.numel()
    table = pages.shape
    if pages.dtype is not i32 or len(table) != 2 or table[0] != n or (table[1] > 1 and pages.stride(1) != 1) or free_pages.dtype is not i32 or free_pages.dim() != 1:
        raise ValueError("pages int32 [n_seqs, max_pages], its rows contiguous, free_pages int32 [n_pages]")
    if held.dtype is not i32 or wanted.dtype is not i32 or wanted.numel() != n or (kept is not None and (kept.dtype is not i32 or kept.numel() != n)):
        raise ValueError("held, wanted, kept: int32 [n_seqs]")
    if counters.dtype is not i64 or counters.numel() != 2:
        raise ValueError("counters: int64 [2]")
    if q_start is kv_len is granted is counters_out is row_seq is positions is slots is None:      # (two allocations for all of them)
        sizes32, sizes64 = ((n + 1, n, n, n_rows, n_rows), (2, n_rows)) if want_rows else ((n + 1, n, n), (2,))
        made32 = torch.empty(sum(sizes32), dtype=i32, device=pages.device).split_with_sizes(sizes32)
        made64 = torch.empty(sum(sizes64), dtype=i64, device=pages.device).split_with_sizes(sizes64)
        made = (*made32[:3], made64[0], *made32[3:], made64[1]) if want_rows else (*made32, made64[0], None, None, None)
    else:
        made = []
        for t, size, dtype, make, name in ((q_start, n + 1, i32, True, "q_start"), (kv_len, n, i32, True, "kv_len"), (granted, n, i32, True, "granted"),
                                           (counters_out, 2, i64, True, "counters_out"), (row_seq, n_rows, i32, want_rows, "row_seq"),
                                           (positions, n_rows, i32, want_rows, "positions"), (slots, n_rows, i64, want_rows, "slots")):
            if t is None and make:
                t = torch.empty(size, dtype=dtype, device=pages.device)
            elif t is not None and (t.dtype is not dtype or t.numel() != size or not t.is_contiguous()):
                raise ValueError(f"{name}: {dtype}, {size} numbers in a row")
            made.append(t)
    if not (free_pages.is_contiguous() and counters.is_contiguous() and held.is_contiguous() and wanted.is_contiguous() and (kept is None or kept.is_contiguous())):
        raise ValueError("all but pages must be contiguous")
    rc = plan(_PACK_TABLE(pages.data_ptr(), pages.stride(0), free_pages.data_ptr(), table[1], free_pages.numel(), page_size, n), counters.data_ptr(), _ptr(made[3]),
              held.data_ptr(), _ptr(kept), wanted.data_ptr(), n_rows, _ptr(made[0]), _ptr(made[1]), _ptr(made[2]), *(_ptr(t) for t in made[4:]), raw_stream(dev))
    if rc != 0:
        raise PPDError(rc, "ppd_paged_plan", load_library().ppd_last_hip_error(None))
    return Plan._make(made)


def _rows_made(out, like, dtype, head_dim, what, n_tokens, heads):
    """`out`, made here as one piece if not given, and its rows as bytes."""
    if out is None:
        out = like.new_empty((n_tokens, heads, head_dim))
        return out, _PACK_ROWS(out.data_ptr(), heads * head_dim, head_dim)
    return out, _rows(out, dtype, head_dim, what, n_tokens, heads)[0]


def _paged_args_fp4(k_codes, k_scales, v_codes, v_scales, pages, q_start, kv_len, dtype, n_tokens):
    """(cache, batch) as bytes, and the sizes that a workspace depends on."""
    torch, codes = _step()[:2]
    u8 = torch.uint8
    if dtype not in codes:
        raise ValueError("rows of float32, bfloat16 or float16")
    shape = k_codes.shape
    if len(shape) != 4 or v_codes.shape != shape or k_codes.dtype is not u8 or v_codes.dtype is not u8:
        raise ValueError("k_codes, v_codes: uint8 [n_pages, page_size, n_kv_heads, head_dim / 2]")
    n_pages, size, kv_heads, half = shape
    if k_scales.shape != (n_pages, size, kv_heads, half // 16) or v_scales.shape != k_scales.shape or k_scales.dtype is not u8 or v_scales.dtype is not u8:
        raise ValueError("k_scales, v_scales: uint8 [n_pages, page_size, n_kv_heads, head_dim / 32]")
    k0, k1, k2, k3 = k_codes.stride()
    v0, v1, v2, v3 = v_codes.stride()
    x0, x1, x2, x3 = k_scales.stride()
    y0, y1, y2, y3 = v_scales.stride()
    if not k3 == v3 == x3 == y3 == 1:
        raise ValueError("codes and scales of a row must be contiguous")
    batch, most, n = _paged_batch(torch.int32, pages, q_start, kv_len, n_tokens)
    code, head_dim = codes[dtype], 2 * half
    return (_PACK_CACHE_FP4(k_codes.data_ptr(), v_codes.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(), k0, k1, k2, v0, v1, v2, x0, x1, x2, y0, y1, y2,
                            n_pages, size, kv_heads, head_dim, code), batch, (n_pages, size, kv_heads, head_dim, code, most, n, n_tokens))


def ppd_paged_append_fp4(k_codes, k_scales, v_codes, v_scales, pages, q_start, kv_len, q, k, v, q_gain=None, k_gain=None, norm_eps=1e-5, rotary_dim=0,
                         rope_theta=10000.0, q_out=None, k_out=None, v_out=None, want_values=False, stream=None):
    """ppd_paged_append into pages of 4-bit numbers: codes uint8 [n_pages, page_size, n_kv_heads, head_dim / 2], scales uint8 [..., head_dim / 32].
    Returns (q_out, k_out, v_out); with want_values k_out and v_out, the keys and values as the pages have them now, are made here if not given (otherwise
    they are None if not given).  Asynchronous."""
    torch, _, device, raw_stream, _, append, _, _ = _step()
    dev = k_codes.get_device()
    if stream is not None or dev < 0 or dev != device():
        return _on_device(k_codes, (k_scales, v_codes, v_scales, pages, q_start, kv_len, q, k, v, q_gain, k_gain, q_out, k_out, v_out), stream,
                          lambda: ppd_paged_append_fp4(k_codes, k_scales, v_codes, v_scales, pages, q_start, kv_len, q, k, v, q_gain, k_gain, norm_eps,
                                                       rotary_dim, rope_theta, q_out, k_out, v_out, want_values))
    _same_gpu(dev, k_scales, v_codes, v_scales, pages, q_start, kv_len, q, k, v, q_gain, k_gain, q_out, k_out, v_out)
    n, dtype = k.shape[0], k.dtype
    cache, batch, sizes = _paged_args_fp4(k_codes, k_scales, v_codes, v_scales, pages, q_start, kv_len, dtype, n)
    kv_heads, head_dim = sizes[2], sizes[3]
    kr, vr = _rows(k, dtype, head_dim, "k", n, kv_heads)[0], _rows(v, dtype, head_dim, "v", n, kv_heads)[0]
    qr, outr, heads = None, None, 0
    if q is not None:
        qr, heads = _rows(q, dtype, head_dim, "q", n)
        q_out, outr = _rows_made(q_out, q, dtype, head_dim, "q_out", n, heads)
    kor = vor = None
    if want_values or k_out is not None:
        k_out, kor = _rows_made(k_out, k, dtype, head_dim, "k_out", n, kv_heads)
    if want_values or v_out is not None:
        v_out, vor = _rows_made(v_out, v, dtype, head_dim, "v_out", n, kv_heads)
    for g in (q_gain, k_gain):
        if g is not None and (g.dtype is not dtype or g.numel() != head_dim or not g.is_contiguous()):
            raise ValueError("gains: [head_dim] of the rows' type")
    rc = append(cache, batch, heads, qr, outr, kr, vr, kor, vor, _ptr(q_gain), _ptr(k_gain), norm_eps, rotary_dim, rope_theta, raw_stream(dev))
    if rc != 0:
        raise PPDError(rc, "ppd_paged_append_fp4", load_library().ppd_last_hip_error(None))
    return q_out if q is not None else None, k_out, v_out


@functools.lru_cache(maxsize=4096)
def _attention_fp4_workspace(sizes, heads):
    """Bytes that ppd_paged_attention_fp4_workspace gives for these sizes (0 where it refuses: the call itself will)."""
    pages, size, kv_heads, head_dim, code, max_pages, seqs, tokens = sizes
    c = PagedCacheFp4(4096, 4096, 4096, 4096, *[0] * 12, pages, size, kv_heads, head_dim, code)
    b = PagedBatch(4096, 4096, 4096, max_pages, max_pages, seqs, tokens)
    need = ctypes.c_uint64()
    return need.value if load_library().ppd_paged_attention_fp4_workspace(c, b, heads, need) == 0 else 0


def ppd_paged_attention_fp4(q, k_codes, k_scales, v_codes, v_scales, pages, q_start, kv_len, scale=None, window=0, out=None, want_lse=False, workspace=None,
                            stream=None):
    """ppd_paged_attention over pages of 4-bit numbers (see ppd_paged_append_fp4): (out [n_tokens, n_heads, head_dim] of q's type, lse float32
    [n_tokens, n_heads] or None).  Asynchronous."""
    torch, _, device, raw_stream, _, _, attention, _ = _step()
    dev = k_codes.get_device()
    if stream is not None or dev < 0 or dev != device():
        return _on_device(k_codes, (q, k_scales, v_codes, v_scales, pages, q_start, kv_len, out, workspace), stream, lambda: ppd_paged_attention_fp4(
            q, k_codes, k_scales, v_codes, v_scales, pages, q_start, kv_len, scale, window, out, want_lse, workspace))
    _same_gpu(dev, q, k_scales, v_codes, v_scales, pages, q_start, kv_len, out, workspace)
    n, dtype = q.shape[0], q.dtype
    cache, batch, sizes = _paged_args_fp4(k_codes, k_scales, v_codes, v_scales, pages, q_start, kv_len, dtype, n)
    head_dim = sizes[3]
    qr, heads = _rows(q, dtype, head_dim, "q", n)
    out, outr = _rows_made(out, q, dtype, head_dim, "out", n, heads)
    lse = torch.empty((n, heads), dtype=torch.float32, device=q.device) if want_lse else None
    if workspace is None:
        need = _attention_fp4_workspace(sizes, heads)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    rc = attention(cache, batch, heads, qr, outr, _ptr(lse), head_dim ** -0.5 if scale is None else scale, window, *_scratch(workspace), raw_stream(dev))
    if rc != 0:
        raise PPDError(rc, "ppd_paged_attention_fp4", load_library().ppd_last_hip_error(None))
    return out, lse


def ppd_adjust_logits(logits, row_start, ids=None, history=None, history_len=None, prompt_len=None, repetition=None, presence=None, frequency=None,
                      bias_start=None, bias_ids=None, bias=None, mask=None, mask_row=None, out=None, stream=None):
    """Penalties for tokens that a text has, biases and masks on logits [n_rows, vocab]; returns out, made here if not given (may be logits).
    row_start int32 [n_seqs + 1], ids int32 [n_rows]; history int32 [n_seqs, most], history_len and prompt_len int32 [n_seqs]; repetition, presence and
    frequency float32 [n_seqs]; bias_start int32 [n_seqs + 1], bias_ids int32 and bias float32 [n_bias]; mask int32 [n_masks, at least vocab / 32] with a
    bit for every token that is allowed, mask_row int32 [n_rows].  Asynchronous."""
    torch, codes, device, raw_stream, _, _, _, adjust = _step()
    z = logits
    dev = z.get_device()
    others = (row_start, ids, history, history_len, prompt_len, repetition, presence, frequency, bias_start, bias_ids, bias, mask, mask_row, out)
    if stream is not None or dev < 0 or dev != device():
        return _on_device(z, others, stream, lambda: ppd_adjust_logits(z, *others))
    _same_gpu(dev, *others)
    i32, f32 = torch.int32, torch.float32
    if z.dim() != 2 or z.dtype not in codes or (z.shape[1] > 1 and z.stride(1) != 1):
        raise ValueError("logits: [n_rows, vocab], vocab contiguous, float32, bfloat16 or float16")
    n, vocab = z.shape
    if out is None:
        out = torch.empty_like(z, memory_format=torch.contiguous_format)
    elif out.shape != z.shape or out.dtype is not z.dtype or (vocab > 1 and out.stride(1) != 1):
        raise ValueError("out: as logits")
    seqs = row_start.numel() - 1
    if row_start.dtype is not i32 or seqs < 1 or (ids is not None and (ids.dtype is not i32 or ids.numel() != n)):
        raise ValueError("row_start int32 [n_seqs + 1], ids int32 [n_rows]")
    for t, dtype in ((history_len, i32), (prompt_len, i32), (repetition, f32), (presence, f32), (frequency, f32)):
        if t is not None and (t.dtype is not dtype or t.numel() != seqs):
            raise ValueError("history_len, prompt_len int32 [n_seqs], repetition, presence, frequency float32 [n_seqs]")
    if (history is None) != (history_len is None) or (bias is None) != (bias_ids is None) or (bias is None) != (bias_start is None) or (mask is None) != (mask_row is None):
        raise ValueError("history with history_len, bias with bias_start and bias_ids, mask with mask_row")
    most = many = masks = words = 0
    if history is not None:
        if history.dtype is not i32 or history.dim() != 2 or history.shape[0] != seqs:
            raise ValueError("history int32 [n_seqs, most]")
        most = history.shape[1]
    if bias is not None:
        many = bias.numel()
        if bias.dtype is not f32 or bias_ids.dtype is not i32 or bias_ids.numel() != many or bias_start.dtype is not i32 or bias_start.numel() != seqs + 1:
            raise ValueError("bias_start int32 [n_seqs + 1], bias_ids int32 [n_bias], bias float32 [n_bias]")
    if mask is not None:
        if mask.dtype is not i32 or mask.dim() != 2 or mask.shape[1] < (vocab + 31) // 32 or mask_row.dtype is not i32 or mask_row.numel() != n:
            raise ValueError("mask int32 [n_masks, at least vocab / 32], mask_row int32 [n_rows]")
        masks, words = mask.shape
    if not all(t is None or t.is_contiguous() for t in others[:-1]):
        raise ValueError("all but the logits must be contiguous")
    if most == 0:                                           # (nothing in them: as if they were not given)
        history = history_len = None
    if many == 0:
        bias_start = bias_ids = bias = None
    if masks == 0:
        mask = mask_row = None
    rules = _PACK_RULES(_ptr(history) or 0, most, *(_ptr(t) or 0 for t in (history_len, prompt_len, repetition, presence, frequency, bias_start, bias_ids, bias, mask)),
                        words, _ptr(mask_row) or 0, many, masks)
    rc = adjust(seqs, n, vocab, codes[z.dtype], row_start.data_ptr(), _ptr(ids), z.data_ptr(), z.stride(0) if n > 1 else vocab, out.data_ptr(),
                out.stride(0) if n > 1 else vocab, rules, raw_stream(dev))
    if rc != 0:
        raise PPDError(rc, "ppd_adjust_logits", load_library().ppd_last_hip_error(None))
    return out


class PPD:
    """One decoding context.  ``dev`` is what ``upload_model`` returned (kept alive here)."""

    def __init__(self, cfg, dev: Dict[str, object], k: Optional[int] = None, exit_layer: Optional[int] = None,
                 eos_id: int = -1, early_head=None, stream=None):
        import torch
        lib = load_library()
        self.cfg, self.dev = cfg, dev
        self.k = cfg.k if k is None else k
        self.exit_layer = cfg.exit_layer if exit_layer is None else exit_layer
        d = ModelDims(cfg.n_layers, cfg.d_model, cfg.n_heads, cfg.head_dim, cfg.d_ff, cfg.vocab, cfg.max_ctx,
                      cfg.norm, cfg.act, cfg.pos, cfg.has_bias, cfg.wdtype, cfg.norm_eps, cfg.rope_theta, eos_id)
        w = Weights()

        def ptr(t):
            return None if t is None else t.data_ptr()

        for n in ("tok_emb", "pos_emb", "lnf_g", "lnf_b", "lm_head"):
            setattr(w, n, ptr(dev.get(n)))
        self._early = early_head
        w.early_head = ptr(early_head)
        self._tabs = []
        for f in _W_LAYER_ORDER:
            tab = (ctypes.c_void_p * cfg.n_layers)(*[ptr(t) for t in dev[f]])
            self._tabs.append(tab)
            setattr(w, f, tab)
        self._stream = stream if stream is not None else torch.cuda.current_stream()
        h = ctypes.c_void_p()
        rc = lib.ppd_create(ctypes.byref(d), ctypes.byref(w), self.k, self.exit_layer,
                            ctypes.c_void_p(self._stream.cuda_stream), ctypes.byref(h))
        if rc != 0:
            raise PPDError(rc, "ppd_create", lib.ppd_last_hip_error(None))
        self._h = h
        self._tok = np.zeros(4, dtype=np.int32)
        self._logits = np.zeros(cfg.vocab, dtype=np.float32)
        # looked up once: the step calls are made thousands of times per second
        self._tok_ptr = self._tok.ctypes.data
        self._fn_step, self._fn_plain = lib.ppd_step, lib.plain_greedy_step

    def _chk(self, rc: int, what: str) -> int:
        if rc < 0:
            raise PPDError(rc, what, load_library().ppd_last_hip_error(self._h))
        return rc

    def close(self):
        if getattr(self, "_h", None):
            load_library().ppd_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def ppd_reset(self):
        self._chk(load_library().ppd_reset(self._h), "ppd_reset")

    def ppd_prefill(self, prompt):
        p = np.ascontiguousarray(prompt, dtype=np.int32)
        self._chk(load_library().ppd_prefill(self._h, p.ctypes.data, len(p)), "ppd_prefill")

    def ppd_step(self, want_info: bool = True):
        """One round.  Returns (token or None after EOS, StepInfo or None)."""
        info = StepInfo() if want_info else None
        n = self._fn_step(self._h, self._tok_ptr, 1, ctypes.byref(info) if want_info else None)
        if n < 0:
            self._chk(n, "ppd_step")
        return (int(self._tok[0]) if n == 1 else None), info

    def plain_greedy_step(self):
        n = self._fn_plain(self._h, self._tok_ptr)
        if n < 0:
            self._chk(n, "plain_greedy_step")
        return int(self._tok[0]) if n == 1 else None

    def ppd_get_logits(self) -> np.ndarray:
        self._chk(load_library().ppd_get_logits(self._h, self._logits.ctypes.data), "ppd_get_logits")
        return self._logits.copy()

    def ppd_get_early_logits(self) -> np.ndarray:
        self._chk(load_library().ppd_get_early_logits(self._h, self._logits.ctypes.data), "ppd_get_early_logits")
        return self._logits.copy()

    def ppd_get_stats(self) -> Dict[str, int]:
        s = Stats()
        self._chk(load_library().ppd_get_stats(self._h, ctypes.byref(s)), "ppd_get_stats")
        return {n: int(getattr(s, n)) for n, _ in Stats._fields_}

    def ppd_set_profiling(self, level: int):
        self._chk(load_library().ppd_set_profiling(self._h, int(level)), "ppd_set_profiling")

    def ppd_set_graphs(self, on: bool):
        self._chk(load_library().ppd_set_graphs(self._h, int(on)), "ppd_set_graphs")

    def ppd_set_sampling(self, mode: int, top_k: int = 0, top_p: float = 1.0, seed: int = 0):
        """Final prediction by arg max (0), top-k sampling (1) or top-p sampling (2)."""
        self._chk(load_library().ppd_set_sampling(self._h, int(mode), int(top_k), float(top_p), int(seed)), "ppd_set_sampling")

    def ppd_time_ffn_in(self, reps: int = 64, groups: int = 1) -> float:
        """Average milliseconds per FFN-in GEMM launch in a back-to-back burst (invalidates the sequence);
        groups = 2: the two-group launch of a pipelined step."""
        out = ctypes.c_double(0.0)
        self._chk(load_library().ppd_time_ffn_in(self._h, reps, groups, ctypes.byref(out)), "ppd_time_ffn_in")
        return float(out.value)

    def ppd_get_chain_rounds(self):
        """(rounds whose main token went through its layers in one launch, rounds that were run again)."""
        n, again = ctypes.c_uint64(), ctypes.c_uint64()
        self._chk(load_library().ppd_get_chain_rounds(self._h, ctypes.byref(n), ctypes.byref(again)), "ppd_get_chain_rounds")
        return int(n.value), int(again.value)

    def ppd_set_chain_wait(self, ticks: int = 0):
        self._chk(load_library().ppd_set_chain_wait(self._h, int(ticks)), "ppd_set_chain_wait")

    def ppd_get_kernel_time(self) -> Dict[str, Dict[str, float]]:
        out = {}
        ms, n = ctypes.c_double(), ctypes.c_uint64()
        for groups in (1, 2):
            for i, name in enumerate(KERNEL_CLASSES):
                self._chk(load_library().ppd_get_kernel_time(self._h, i, groups, ctypes.byref(ms), ctypes.byref(n)),
                          "ppd_get_kernel_time")
                if n.value:
                    out[f"{name}.g{groups}"] = {"ms": ms.value, "launches": int(n.value)}
        return out
