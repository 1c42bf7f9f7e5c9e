"""MoE verification pass of EcoSpec (arXiv 2607.12696) on MI355X / gfx950.

Thin ctypes binding of ``libecospec_moe.so`` (declared in
``include/ecospec_moe.h``).  The functions carry the C names and only
marshal arguments: PyTorch supplies device memory and the current HIP
stream, and every step of the pass runs in the library's HIP kernels.  If
the library has not been built, importing the functions that need it raises
``ImportError``; there is no fallback.

    moe_route_topk(logits, k, score)            -> (topk_idx, topk_w)
    moe_route_topk_hidden(x, w_router, k, score) -> (topk_idx, topk_w)
    moe_route_topk_grouped(logits, bias, k, n_group, topk_group, scale) -> (topk_idx, topk_w)
    moe_expert_union(topk_idx, E)               -> Routing
    moe_verify_workspace_size(weights, T, k)    -> bytes
    moe_pack_weights(fmt, w, s)                 -> (w_packed, s_packed)   once per model load
    moe_pack_gate_up / moe_pack_down            -> the paired layouts pack_layer uses by default
    moe_verify_layer(x, weights, routing)       -> y   (weights packed)
    moe_select_tree(parent, P, pred, E, budget) -> (selected, marginal_cost)
    moe_route_union(logits, k, score)           -> Routing   (route + union in one call)
    moe_verify_step(x, logits, weights, k, score) = moe_route_union + moe_verify_layer

and the rest of a layer's verification step:

    moe_add_rmsnorm(x, weight, eps, residual, qfmt) -> (sum, y, q, scales)
    moe_latent_attn(q, kv_new, token_offsets, pages, block_table, cache_len, r, scale, mask) -> (o, lse)
    moe_latent_prompt(q, k, k_rope, v, q_offsets, kv_offsets, scale)   -> (o, lse)
    moe_cache_append(k_new, v_new, token_offsets, k, v, k_scale, v_scale, block_table, cache_len)
    moe_cache_attn(q, k_new, v_new, token_offsets, k, v, k_scale, v_scale, block_table, cache_len, scale, mask) -> (o, lse)

and the two ends of a decoding step:

    moe_pages_update(cache_len, token_offsets, block_table, free_pages, n_free, page, N, keep_len) -> PageUpdate
    moe_latent_append(kv_new, pages, slots, rows)
    moe_grouped_prompt(q, k, v, q_offsets, kv_offsets, scale)           -> (o, lse)
    moe_token_logprobs(logits, tokens, k, scale)                        -> TokenLogprobs
"""
from __future__ import annotations

import ctypes as C
import functools
import os
import threading
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libecospec_moe.so")

MOE_OK, MOE_ERR_INVALID_ARG, MOE_ERR_UNSUPPORTED, MOE_ERR_WORKSPACE, MOE_ERR_HIP = range(5)
MOE_SCORE_SOFTMAX, MOE_SCORE_SIGMOID = 0, 1
MOE_W_BF16, MOE_W_FP8_E4M3_B128, MOE_W_MXFP4 = 0, 1, 2
MOE_SEL_COST_RATIO, MOE_SEL_CONFIDENCE, MOE_SEL_GLOBAL_COST, MOE_SEL_COST_DIFF = 0, 1, 2, 3
MOE_ACT_SWIGLU, MOE_ACT_SWIGLU_OAI = 0, 1
MOE_ACTQ_BF16, MOE_ACTQ_MXFP8 = 0, 1
MOE_Q_NONE, MOE_Q_FP8_GROUP, MOE_Q_MXFP8, MOE_Q_FP8_ROW = 0, 1, 2, 3
MOE_F32, MOE_BF16 = 0, 1

EXPORTED = ("moe_route_topk", "moe_route_union", "moe_route_topk_grouped", "moe_router_workspace_size", "moe_route_topk_hidden", "moe_expert_union", "moe_verify_workspace_size", "moe_verify_layer",
            "moe_verify_layer_timed", "moe_packed_size", "moe_pack_weights", "moe_pack_gate_up", "moe_pack_down",
            "moe_select_tree", "moe_status_string", "moe_last_error", "moe_verify_layer_noalloc",
            "moe_add_rmsnorm", "moe_latent_attn_workspace_size", "moe_latent_attn", "moe_latent_prompt",
            "moe_cache_append", "moe_cache_append_slots", "moe_cache_attn_workspace_size", "moe_cache_attn",
            "moe_pages_update", "moe_latent_append", "moe_grouped_prompt_workspace_size", "moe_grouped_prompt",
            "moe_token_logprobs_workspace_size", "moe_token_logprobs")


class MoeError(RuntimeError):
    def __init__(self, fn: str, status: int, detail: str = ""):
        self.status = status
        super().__init__(f"{fn}: status {status} ({_status_string(status)}){': ' + detail if detail else ''}")


class moe_weights_t(C.Structure):
    _fields_ = [("fmt", C.c_int), ("d", C.c_int), ("d_ff", C.c_int), ("E", C.c_int)] + [
        (n, C.c_void_p) for n in ("w_gate", "w_up", "w_down", "s_gate", "s_up", "s_down", "sh_gate", "sh_up",
                                  "sh_down", "sh_s_gate", "sh_s_up", "sh_s_down")] + [
        ("act", C.c_int), ("alpha", C.c_float), ("limit", C.c_float),
        ("b_gate", C.c_void_p), ("b_up", C.c_void_p), ("b_down", C.c_void_p), ("act_fmt", C.c_int),
        ("down_paired", C.c_int)]


class moe_routing_t(C.Structure):
    _fields_ = [("T", C.c_int), ("k", C.c_int), ("E", C.c_int)] + [
        (n, C.c_void_p) for n in ("topk_idx", "topk_w", "counts", "union_ids", "n_unique", "offsets", "perm")]


class moe_drafts_t(C.Structure):
    _fields_ = [("N", C.c_int), ("B", C.c_int), ("token_offsets", C.c_void_p), ("mask", C.c_void_p)]


class moe_latent_cache_t(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("r", "p", "n_pages", "page", "max_blocks")] + [
        (n, C.c_void_p) for n in ("pages", "block_table", "cache_len")]


class moe_prompt_t(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("N", "M", "B", "H", "dn", "p", "dv", "max_tokens")] + [
        (n, C.c_void_p) for n in ("q_offsets", "kv_offsets", "q", "k", "k_rope", "v")] + [
        (n, C.c_int64) for n in ("k_stride", "k_head", "v_stride", "v_head")] + [("scale", C.c_float)]


class moe_cache_t(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("Hkv", "D", "n_pages", "page", "max_blocks")] + [
        (n, C.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "block_table", "cache_len")]


class moe_page_pool_t(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("B", "n_pages", "page", "max_blocks")] + [
        (n, C.c_void_p) for n in ("block_table", "cache_len", "free_pages", "n_free")]


class moe_grouped_prompt_t(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("N", "M", "B", "H", "Hkv", "D", "max_tokens")] + [
        (n, C.c_void_p) for n in ("q_offsets", "kv_offsets", "q", "k", "v")] + [
        (n, C.c_int64) for n in ("q_stride", "q_head", "k_stride", "k_head", "v_stride", "v_head")] + [("scale", C.c_float)]


_lock = threading.Lock()
_lib = None


def lib() -> C.CDLL:
    """The loaded library; raises ImportError if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_12696_amd.build`")
            L = C.CDLL(LIB_PATH)
            p, i = C.c_void_p, C.c_int
            L.moe_route_topk.argtypes = [p, i, i, i, i, p, p, p]
            L.moe_route_union.argtypes = [p, i, i, i, i, p, p, p, p, p, p, p, p]
            L.moe_route_topk_grouped.argtypes = [p, p, i, i, i, i, i, C.c_float, p, p, p]
            L.moe_router_workspace_size.argtypes = [i, i, i, C.POINTER(C.c_size_t)]
            L.moe_route_topk_hidden.argtypes = [p, p, i, i, i, i, i, p, p, p, p, C.c_size_t, p]
            L.moe_expert_union.argtypes = [p, i, i, i, p, p, p, p, p, p]
            L.moe_verify_workspace_size.argtypes = [C.POINTER(moe_weights_t), i, i, C.POINTER(C.c_size_t)]
            L.moe_verify_layer.argtypes = [p, C.POINTER(moe_weights_t), C.POINTER(moe_routing_t), p, p, C.c_size_t, p]
            L.moe_verify_layer_noalloc.argtypes = [p, C.POINTER(moe_weights_t), C.POINTER(moe_routing_t), p, p]
            L.moe_verify_layer_timed.argtypes = [p, C.POINTER(moe_weights_t), C.POINTER(moe_routing_t), p, p,
                                                 C.c_size_t, p, C.POINTER(C.c_void_p)]
            L.moe_packed_size.argtypes = [i, i, i, i, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
            L.moe_pack_weights.argtypes = [i, i, i, i, p, p, p, p, p]
            L.moe_pack_gate_up.argtypes = [i, i, i, i, p, p, p, p, p, p, p, p]
            L.moe_pack_down.argtypes = [i, i, i, i, p, p, p, p, p]
            L.moe_select_tree.argtypes = [i, p, p, i, i, p, i, p, i, C.c_double, C.c_double, i, p, p, p]
            st = C.POINTER
            L.moe_add_rmsnorm.argtypes = [p, p, p, i, i, C.c_float, i, p, p, p, p, p]
            L.moe_latent_attn_workspace_size.argtypes = [st(moe_latent_cache_t), i, i, i, st(C.c_size_t)]
            L.moe_latent_attn.argtypes = [st(moe_latent_cache_t), st(moe_drafts_t), p, p, i, C.c_float, p, p, p,
                                          C.c_size_t, p]
            L.moe_latent_prompt.argtypes = [st(moe_prompt_t), p, p, p]
            L.moe_cache_append.argtypes = [st(moe_cache_t), p, p, i, p, i, i, p, i, p]
            L.moe_cache_append_slots.argtypes = [st(moe_cache_t), p, p, i, p, i, i, p, i, p, p]
            L.moe_cache_attn_workspace_size.argtypes = [st(moe_cache_t), i, i, i, st(C.c_size_t)]
            L.moe_cache_attn.argtypes = [st(moe_cache_t), st(moe_drafts_t), p, p, p, i, C.c_float, p, p, p, C.c_size_t, p]
            L.moe_pages_update.argtypes = [st(moe_page_pool_t), p, p, i, p, p, p, p, p, p]
            L.moe_latent_append.argtypes = [p, i, i, i, i, p, i, p, i, p, p]
            L.moe_grouped_prompt_workspace_size.argtypes = [i, st(C.c_size_t)]
            L.moe_grouped_prompt.argtypes = [st(moe_grouped_prompt_t), p, p, p, C.c_size_t, p]
            L.moe_token_logprobs_workspace_size.argtypes = [i, st(C.c_size_t)]
            L.moe_token_logprobs.argtypes = [p, i, C.c_int64, i, i, C.c_float, p, i, i, p, p, p, p, p, p, C.c_size_t, p]
            L.moe_status_string.argtypes = [i]
            L.moe_status_string.restype = C.c_char_p
            L.moe_last_error.restype = C.c_char_p
            for f in ("moe_route_topk", "moe_route_union", "moe_route_topk_grouped", "moe_router_workspace_size", "moe_route_topk_hidden", "moe_expert_union", "moe_verify_workspace_size", "moe_verify_layer",
                      "moe_verify_layer_noalloc", "moe_verify_layer_timed", "moe_packed_size", "moe_pack_weights", "moe_pack_gate_up",
                      "moe_pack_down", "moe_select_tree", "moe_add_rmsnorm", "moe_latent_attn_workspace_size",
                      "moe_latent_attn", "moe_latent_prompt", "moe_cache_append", "moe_cache_append_slots",
                      "moe_cache_attn_workspace_size", "moe_cache_attn", "moe_pages_update", "moe_latent_append", "moe_grouped_prompt_workspace_size",
                      "moe_grouped_prompt", "moe_token_logprobs_workspace_size", "moe_token_logprobs"):
                getattr(L, f).restype = i
            _lib = L
    return _lib


def _status_string(s: int) -> str:
    try:
        return lib().moe_status_string(s).decode()
    except ImportError:
        return "library not loaded"


def _check(fn: str, status: int):
    if status != MOE_OK:
        detail = lib().moe_last_error().decode() if status == MOE_ERR_HIP else ""
        raise MoeError(fn, status, detail)


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


# The host side of a call is on the critical path of the smallest passes (a GPT-OSS step of one token runs 28 us on
# the GPU; its Python took 24 us, with 12 us of launches 36 us a step).  So the stream is read as a raw handle
# (0.1 us; torch.cuda.current_stream builds a Stream object, 1.9 us), the C structs are built by one constructor call,
# and a routing's integer arrays come from one allocation.

_raw_stream = None  # device index -> handle of its current stream


def _stream(t) -> int:
    """Handle of the current stream of t's device (t is a device tensor)."""
    global _raw_stream
    if _raw_stream is None:
        torch = _torch()
        # Not part of torch's public interface: a torch without it takes the public way.
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)
    return _raw_stream(t.get_device())


def _dev_ptr(t, what: str) -> int:
    if t is None:
        return 0
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


# --------------------------------------------------------------------------- routing

def moe_route_topk(logits, k: int, score: int, topk_idx=None, topk_w=None):
    """Router top-k of fp32 logits [T, E] on the device -> (int32 [T, k], fp32 [T, k])."""
    torch = _torch()
    T, E = logits.shape
    if logits.dtype != torch.float32:
        raise ValueError("logits must be float32")
    if topk_idx is None:
        topk_idx = torch.empty(T, k, dtype=torch.int32, device=logits.device)
    if topk_w is None:
        topk_w = torch.empty(T, k, dtype=torch.float32, device=logits.device)
    _check("moe_route_topk", lib().moe_route_topk(_dev_ptr(logits, "logits"), T, E, k, score,
                                                    _dev_ptr(topk_idx, "topk_idx"), _dev_ptr(topk_w, "topk_w"),
                                                    _stream(logits)))
    return topk_idx, topk_w


def moe_route_topk_grouped(logits, bias, k: int, n_group: int, topk_group: int, scale: float, topk_idx=None,
                           topk_w=None):
    """Group-limited sigmoid routing (correction bias [E] or None, routed scaling `scale`) of fp32
    logits [T, E] on the device -> (int32 [T, k], fp32 [T, k])."""
    torch = _torch()
    T, E = logits.shape
    if logits.dtype != torch.float32 or (bias is not None and (bias.dtype != torch.float32 or bias.numel() != E)):
        raise ValueError("logits [T, E] and bias [E] must be float32")
    if topk_idx is None:
        topk_idx = torch.empty(T, k, dtype=torch.int32, device=logits.device)
    if topk_w is None:
        topk_w = torch.empty(T, k, dtype=torch.float32, device=logits.device)
    _check("moe_route_topk_grouped", lib().moe_route_topk_grouped(
        _dev_ptr(logits, "logits"), _dev_ptr(bias, "bias"), T, E, k, n_group, topk_group, scale,
        _dev_ptr(topk_idx, "topk_idx"), _dev_ptr(topk_w, "topk_w"), _stream(logits)))
    return topk_idx, topk_w


def moe_router_workspace_size(T: int, d: int, E: int) -> int:
    n = C.c_size_t(0)
    _check("moe_router_workspace_size", lib().moe_router_workspace_size(T, d, E, C.byref(n)))
    return n.value


def moe_route_topk_hidden(x, w_router, k: int, score: int, logits=None, workspace=None, topk_idx=None, topk_w=None):
    """Router logits x . W_r^T (bf16 x [T, d], bf16 W_r [E, d]) and their top-k on the device
    -> (int32 [T, k], fp32 [T, k]); the fp32 logits land in `logits` [T, E] when it is given."""
    torch = _torch()
    T, d = x.shape
    E, d2 = w_router.shape
    if d2 != d:
        raise ValueError("x and w_router disagree on d")
    if x.dtype != torch.bfloat16 or w_router.dtype != torch.bfloat16:
        raise ValueError("x and w_router must be bfloat16")
    if logits is not None and (logits.dtype != torch.float32 or tuple(logits.shape) != (T, E)):
        raise ValueError("logits must be float32 [T, E]")
    if topk_idx is None:
        topk_idx = torch.empty(T, k, dtype=torch.int32, device=x.device)
    if topk_w is None:
        topk_w = torch.empty(T, k, dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = torch.empty(moe_router_workspace_size(T, d, E), dtype=torch.uint8, device=x.device)
    _check("moe_route_topk_hidden", lib().moe_route_topk_hidden(
        _dev_ptr(x, "x"), _dev_ptr(w_router, "w_router"), T, d, E, k, score, _dev_ptr(topk_idx, "topk_idx"),
        _dev_ptr(topk_w, "topk_w"), _dev_ptr(logits, "logits"), _dev_ptr(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), _stream(x)))
    return topk_idx, topk_w


@dataclass
class Routing:
    """Device routing of T tokens: the outputs of moe_route_topk and moe_expert_union.  moe_verify_layer
    reads topk_idx / topk_w and writes the union and grouping arrays itself."""
    T: int
    k: int
    E: int
    topk_idx: object
    topk_w: object
    counts: object
    union_ids: object
    n_unique: object
    offsets: object
    perm: object

    def c_struct(self) -> moe_routing_t:
        return moe_routing_t(self.T, self.k, self.E, _dev_ptr(self.topk_idx, "topk_idx"), _dev_ptr(self.topk_w, "topk_w"),
                             _dev_ptr(self.counts, "counts"), _dev_ptr(self.union_ids, "union_ids"),
                             _dev_ptr(self.n_unique, "n_unique"), _dev_ptr(self.offsets, "offsets"),
                             _dev_ptr(self.perm, "perm"))


def _union_arrays(S: int, E: int, device):
    """Empty int32 counts [E], union_ids [E], n_unique [1], offsets [E + 1], perm [S], from one allocation."""
    torch = _torch()
    return torch.empty(3 * E + 2 + S, dtype=torch.int32, device=device).split((E, E, 1, E + 1, S))


def moe_expert_union(topk_idx, E: int, topk_w=None, out: Routing | None = None) -> Routing:
    """Expert union, counts, offsets and stable grouping of topk_idx [T, k] on the device."""
    T, k = topk_idx.shape
    dev = topk_idx.device
    if out is None:
        out = Routing(T, k, E, topk_idx, topk_w, *_union_arrays(T * k, E, dev))
    _check("moe_expert_union", lib().moe_expert_union(
        _dev_ptr(topk_idx, "topk_idx"), T, k, E, _dev_ptr(out.counts, "counts"), _dev_ptr(out.union_ids, "union_ids"),
        _dev_ptr(out.n_unique, "n_unique"), _dev_ptr(out.offsets, "offsets"), _dev_ptr(out.perm, "perm"),
        _stream(topk_idx)))
    return out


def routing_for(topk_idx, topk_w, E: int) -> Routing:
    """A Routing around a top-k (moe_route_topk's output) with empty union and grouping arrays, which
    moe_verify_layer fills."""
    T, k = topk_idx.shape
    return Routing(T, k, E, topk_idx, topk_w, *_union_arrays(T * k, E, topk_idx.device))


def moe_route_union(logits, k: int, score: int, out: Routing | None = None) -> Routing:
    """moe_route_topk + moe_expert_union of fp32 logits [T, E] in one call."""
    torch = _torch()
    T, E = logits.shape
    if logits.dtype != torch.float32:
        raise ValueError("logits must be float32")
    dev = logits.device
    if out is None:
        out = Routing(T, k, E, torch.empty(T, k, dtype=torch.int32, device=dev),
                      torch.empty(T, k, dtype=torch.float32, device=dev), *_union_arrays(T * k, E, dev))
    _check("moe_route_union", lib().moe_route_union(
        _dev_ptr(logits, "logits"), T, E, k, score, _dev_ptr(out.topk_idx, "topk_idx"), _dev_ptr(out.topk_w, "topk_w"),
        _dev_ptr(out.counts, "counts"), _dev_ptr(out.union_ids, "union_ids"), _dev_ptr(out.n_unique, "n_unique"),
        _dev_ptr(out.offsets, "offsets"), _dev_ptr(out.perm, "perm"), _stream(logits)))
    return out


# --------------------------------------------------------------------------- weight packing

def moe_packed_size(fmt: int, E: int, N: int, K: int) -> tuple[int, int]:
    wb, sb = C.c_size_t(), C.c_size_t()
    _check("moe_packed_size", lib().moe_packed_size(fmt, E, N, K, C.byref(wb), C.byref(sb)))
    return wb.value, sb.value


def moe_pack_weights(fmt: int, w, s=None):
    """Pack stacked device weights w [E, N, K(/2)] (+ scales) into the streaming layout.

    Returns (w_packed, s_packed) as flat uint8 device tensors (s_packed None for bf16).
    """
    torch = _torch()
    E, N = w.shape[0], w.shape[1]
    K = w.shape[2] * (2 if fmt == MOE_W_MXFP4 else 1)
    wb, sb = moe_packed_size(fmt, E, N, K)
    wp = torch.empty(wb, dtype=torch.uint8, device=w.device)
    sp = torch.empty(sb, dtype=torch.uint8, device=w.device) if sb else None
    _check("moe_pack_weights", lib().moe_pack_weights(fmt, E, N, K, _dev_ptr(w, "w"), _dev_ptr(s, "s"),
                                                        _dev_ptr(wp, "w_packed"), _dev_ptr(sp, "s_packed"),
                                                        _stream(w)))
    return wp, sp


def moe_pack_gate_up(fmt: int, w_gate, w_up, s_gate=None, s_up=None):
    """Pack stacked device W_gate and W_up [E, N, K(/2)] (+ scales) as one pair.

    Returns (w_packed, s_gate_packed, s_up_packed); the scales are None for bf16.
    """
    torch = _torch()
    E, N = w_gate.shape[0], w_gate.shape[1]
    K = w_gate.shape[2] * (2 if fmt == MOE_W_MXFP4 else 1)
    wb, sb = moe_packed_size(fmt, E, N, K)
    wp = torch.empty(2 * wb, dtype=torch.uint8, device=w_gate.device)
    sgp = torch.empty(sb, dtype=torch.uint8, device=w_gate.device) if sb else None
    sup = torch.empty(sb, dtype=torch.uint8, device=w_gate.device) if sb else None
    _check("moe_pack_gate_up", lib().moe_pack_gate_up(
        fmt, E, N, K, _dev_ptr(w_gate, "w_gate"), _dev_ptr(s_gate, "s_gate"), _dev_ptr(w_up, "w_up"),
        _dev_ptr(s_up, "s_up"), _dev_ptr(wp, "w_packed"), _dev_ptr(sgp, "s_gate_packed"), _dev_ptr(sup, "s_up_packed"),
        _stream(w_gate)))
    return wp, sgp, sup


def moe_pack_down(fmt: int, w, s=None):
    """Pack stacked device W_down [E, N, K(/2)] (+ scales) with each wavefront's two row tiles
    interleaved.  Returns (w_packed, s_packed) like moe_pack_weights."""
    torch = _torch()
    E, N = w.shape[0], w.shape[1]
    K = w.shape[2] * (2 if fmt == MOE_W_MXFP4 else 1)
    wb, sb = moe_packed_size(fmt, E, N, K)
    wp = torch.empty(wb, dtype=torch.uint8, device=w.device)
    sp = torch.empty(sb, dtype=torch.uint8, device=w.device) if sb else None
    _check("moe_pack_down", lib().moe_pack_down(fmt, E, N, K, _dev_ptr(w, "w"), _dev_ptr(s, "s"),
                                                  _dev_ptr(wp, "w_packed"), _dev_ptr(sp, "s_packed"), _stream(w)))
    return wp, sp


def pack_layer(layer: dict, pair: bool = True, down_pair: bool = True) -> dict:
    """A layer dict (interchange layout, device tensors) with every matrix packed; with `pair`,
    W_gate and W_up as one pair (moe_pack_gate_up; the dict then has no "up" / "sh_up" entry);
    with `down_pair`, W_down by moe_pack_down (the dict then has down_paired = 1)."""
    out = {k: layer[k] for k in ("fmt", "d", "d_ff", "act", "alpha", "limit", "b_gate", "b_up", "b_down", "act_fmt")
           if k in layer}
    if down_pair:
        out["down_paired"] = 1
    out["E"] = int(layer.get("E", layer["gate"].shape[0]))
    fmt = int(layer["fmt"])
    for prefix in ("", "sh_"):
        names = ("gate", "up", "down")
        if pair and layer.get(prefix + "gate") is not None and layer.get(prefix + "up") is not None:
            wp, sgp, sup = moe_pack_gate_up(fmt, layer[prefix + "gate"], layer[prefix + "up"],
                                            layer.get(prefix + "s_gate"), layer.get(prefix + "s_up"))
            out[prefix + "gate"] = wp
            if sgp is not None:
                out[prefix + "s_gate"], out[prefix + "s_up"] = sgp, sup
            names = ("down",)
        for name in names:
            if layer.get(prefix + name) is None:
                continue
            pack = moe_pack_down if name == "down" and down_pair else moe_pack_weights
            wp, sp = pack(fmt, layer[prefix + name], layer.get(prefix + "s_" + name))
            out[prefix + name] = wp
            if sp is not None:
                out[prefix + "s_" + name] = sp
    return out


# --------------------------------------------------------------------------- verify layer

_WEIGHT_KEYS = tuple(pre + n for n in ("gate", "up", "down") for pre in ("", "s_", "sh_", "sh_s_"))


def weights_struct(w: dict) -> moe_weights_t:
    """moe_weights_t for a layer dict (keys fmt, d, d_ff, E, gate, up, down, optional s_*, sh_*,
    fp32 biases b_gate / b_up [E, d_ff] and b_down [E, d], act / alpha / limit, and act_fmt)."""
    get, f32 = w.get, _torch().float32
    bias = []
    for name in ("b_gate", "b_up", "b_down"):
        b = get(name)
        if b is not None and b.dtype != f32:
            raise ValueError(f"{name} must be float32")
        bias.append(_dev_ptr(b, name))
    E = int(w["E"]) if "E" in w else int(w["gate"].shape[0])
    p = {n: _dev_ptr(get(n), n) for n in _WEIGHT_KEYS}
    return moe_weights_t(
        int(w["fmt"]), int(w["d"]), int(w["d_ff"]), E, p["gate"], p["up"], p["down"], p["s_gate"], p["s_up"], p["s_down"],
        p["sh_gate"], p["sh_up"], p["sh_down"], p["sh_s_gate"], p["sh_s_up"], p["sh_s_down"], int(get("act", MOE_ACT_SWIGLU)),
        float(get("alpha", 1.702)), float(get("limit", 7.0)), *bias, int(get("act_fmt", MOE_ACTQ_BF16)),
        int(get("down_paired", 0)))


def moe_verify_workspace_size(weights: dict, T: int, k: int) -> int:
    n = C.c_size_t()
    ws = weights_struct(weights)
    _check("moe_verify_workspace_size", lib().moe_verify_workspace_size(C.byref(ws), T, k, C.byref(n)))
    return n.value


def moe_verify_layer(x, weights: dict, routing: Routing, y=None, workspace=None):
    """y [T, d] bf16 = the MoE layer over the routed tokens x [T, d] bf16."""
    torch = _torch()
    T, d = x.shape
    if x.dtype != torch.bfloat16:
        raise ValueError("x must be bfloat16")
    if y is None:
        y = torch.empty_like(x)
    if workspace is None:
        workspace = torch.empty(moe_verify_workspace_size(weights, T, routing.k), dtype=torch.uint8, device=x.device)
    ws = weights_struct(weights)
    rs = routing.c_struct()
    _check("moe_verify_layer", lib().moe_verify_layer(
        _dev_ptr(x, "x"), C.byref(ws), C.byref(rs), _dev_ptr(y, "y"), _dev_ptr(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), _stream(x)))
    return y


def moe_verify_layer_noalloc(x, weights: dict, routing: Routing, y=None):
    """moe_verify_layer on the library's fixed per-GPU scratch (no workspace argument, nothing allocated
    by the library)."""
    torch = _torch()
    if x.dtype != torch.bfloat16:
        raise ValueError("x must be bfloat16")
    if y is None:
        y = torch.empty_like(x)
    ws = weights_struct(weights)
    rs = routing.c_struct()
    status = lib().moe_verify_layer_noalloc(_dev_ptr(x, "x"), C.byref(ws), C.byref(rs), _dev_ptr(y, "y"), _stream(x))
    if status == MOE_ERR_WORKSPACE:
        raise MoeError("moe_verify_layer_noalloc", status, lib().moe_last_error().decode())
    _check("moe_verify_layer_noalloc", status)
    return y


def moe_verify_layer_timed(x, weights: dict, routing: Routing, y, workspace, events):
    """moe_verify_layer that also records 5 torch.cuda.Event marks on the current stream:
    before the gate/up expert kernel (MX activations: before the quantisation of x), after it,
    before the down expert kernel, after it, after the combine kernel."""
    if len(events) != 5:
        raise ValueError("moe_verify_layer_timed takes 5 events")
    arr = (C.c_void_p * 5)(*[e.cuda_event if e is not None else None for e in events])
    ws = weights_struct(weights)
    rs = routing.c_struct()
    _check("moe_verify_layer_timed", lib().moe_verify_layer_timed(
        _dev_ptr(x, "x"), C.byref(ws), C.byref(rs), _dev_ptr(y, "y"), _dev_ptr(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), _stream(x), arr))
    return y


def moe_verify_step(x, logits, weights: dict, k: int, score: int, workspace=None, y=None):
    """Route (top-k), then verify one layer, which builds the union and grouping itself: the whole hot
    path on the device.  Returns y and the routing, its union arrays filled by the verification."""
    idx, w = moe_route_topk(logits, k, score)
    r = routing_for(idx, w, logits.shape[1])
    return moe_verify_layer(x, weights, r, y=y, workspace=workspace), r


# --------------------------------------------------------------------------- norm

def moe_add_rmsnorm(x, weight, eps: float, residual=None, qfmt: int = MOE_Q_NONE, want_y: bool = True, want_sum: bool = True,
                    sum=None, y=None, q=None, scales=None):
    """Residual addition and RMS norm of bf16 rows x [T, d] -> (sum, y, q, scales).

    sum = bf16(x + residual), y = bf16 norm, q (e4m3fn codes, uint8 [T, d]) and scales the norm in 8 bits by `qfmt`;
    what is not wanted is None.  Outputs given are written in place (sum may be x or residual, y may be x)."""
    torch = _torch()
    T, d = x.shape
    bf16, u8 = torch.bfloat16, torch.uint8
    if x.dtype != bf16 or weight.dtype != bf16 or weight.numel() != d:
        raise ValueError("x [T, d] and weight [d] must be bfloat16")
    if residual is not None and (residual.dtype != bf16 or residual.shape != x.shape):
        raise ValueError("residual must be bfloat16 [T, d]")
    for t, what in ((sum, "sum"), (y, "y")):
        if t is not None and (t.dtype != bf16 or t.shape != x.shape):
            raise ValueError(f"{what} must be bfloat16 [T, d]")
    if sum is None and want_sum:
        sum = torch.empty_like(x)
    if y is None and want_y:
        y = torch.empty_like(x)
    if qfmt != MOE_Q_NONE:
        if qfmt == MOE_Q_MXFP8:
            groups, stype = d // 32, u8
        else:
            groups, stype = (1 if qfmt == MOE_Q_FP8_ROW else (d + 127) // 128), torch.float32
        if q is None:
            q = torch.empty(T, d, dtype=u8, device=x.device)
        if scales is None:
            scales = torch.empty(T, groups, dtype=stype, device=x.device)
        if q.dtype != u8 or q.shape != x.shape or scales.dtype != stype or tuple(scales.shape) != (T, groups):
            raise ValueError("q must be uint8 [T, d] and scales of the format's type and shape")
    _check("moe_add_rmsnorm", lib().moe_add_rmsnorm(
        _dev_ptr(x, "x"), _dev_ptr(residual, "residual"), _dev_ptr(weight, "weight"), T, d, eps, qfmt,
        _dev_ptr(sum, "sum"), _dev_ptr(y, "y"), _dev_ptr(q, "q"), _dev_ptr(scales, "scales"), _stream(x)))
    return sum, y, q, scales


# --------------------------------------------------------------------------- attention

# One function to a check: with ten tensors a call, the calls between them were a third of its host time.

def _typed_ptr(t, dtype, what: str, shape) -> int:
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{what} must be {str(dtype).removeprefix('torch.')} {list(shape)}")
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


def _one_device(t, *others) -> None:
    """All tensors that are given are on t's device: a call runs there."""
    device = t.get_device()
    for o in others:
        if o is not None and o.get_device() != device:
            raise ValueError("the tensors of a call must be on one device")


@functools.cache
def _several_devices() -> bool:
    return _torch().cuda.device_count() > 1


def _enqueue(name: str, fn, t, *args) -> None:
    """fn(*args, stream) on the current stream of t's device.  A default stream's handle is null and means the current device's."""
    stream = _stream(t)
    if not stream and _several_devices():
        cuda, device = _torch().cuda, t.get_device()
        if cuda.current_device() != device:
            with cuda.device(device):
                return _check(name, fn(*args, stream))
    _check(name, fn(*args, stream))


def _int32_ptr(t, what: str, *shape) -> int:
    return _typed_ptr(t, _torch().int32, what, shape)


def _bf16_ptr(t, what: str, *shape) -> int:
    return _typed_ptr(t, _torch().bfloat16, what, shape)


def _drafts(N: int, token_offsets, mask) -> moe_drafts_t:
    """moe_drafts_t of N tokens; mask: int64 (or uint64) [N], its bit patterns, or None."""
    B = token_offsets.shape[0] - 1
    if mask is not None and (mask.element_size() != 8 or mask.is_floating_point() or tuple(mask.shape) != (N,)):
        raise ValueError("mask must be int64 or uint64 [N]")
    return moe_drafts_t(N, B, _int32_ptr(token_offsets, "token_offsets", B + 1), _dev_ptr(mask, "mask"))


def _attn_outputs(q, width: int, o, lse):
    torch = _torch()
    N, H = q.shape[0], q.shape[1]
    if o is None:
        o = torch.empty(N, H, width, dtype=torch.bfloat16, device=q.device)
    if lse is None:
        lse = torch.empty(N, H, dtype=torch.float32, device=q.device)
    if lse.dtype != torch.float32 or tuple(lse.shape) != (N, H):
        raise ValueError("lse must be float32 [N, H]")
    return o, lse, _bf16_ptr(o, "o", N, H, width), _dev_ptr(lse, "lse")


def _scratch(workspace, size_fn, name: str, cache, N: int, B: int, H: int, device):
    if workspace is None:
        n = C.c_size_t()
        _check(name, size_fn(C.byref(cache), N, B, H, C.byref(n)))
        workspace = _torch().empty(n.value, dtype=_torch().uint8, device=device)
    return workspace, workspace.numel() * workspace.element_size()


def _latent_cache(pages, block_table, cache_len, B: int, r: int) -> moe_latent_cache_t:
    n_pages, page, width = pages.shape
    blocks = block_table.shape[1]
    return moe_latent_cache_t(r, width - r, n_pages, page, blocks, _bf16_ptr(pages, "pages", n_pages, page, width),
                              _int32_ptr(block_table, "block_table", B, blocks), _int32_ptr(cache_len, "cache_len", B))


def moe_latent_attn_workspace_size(pages, block_table, cache_len, r: int, N: int, H: int) -> int:
    B, n = block_table.shape[0], C.c_size_t()
    c = _latent_cache(pages, block_table, cache_len, B, r)
    _check("moe_latent_attn_workspace_size", lib().moe_latent_attn_workspace_size(C.byref(c), N, B, H, C.byref(n)))
    return n.value


def moe_latent_attn(q, kv_new, token_offsets, pages, block_table, cache_len, r: int, scale: float, mask=None, o=None,
                    lse=None, workspace=None):
    """Latent attention in the absorbed form of the draft tokens of B sequences -> (o [N, H, r] bf16, lse [N, H] fp32).

    q [N, H, r + p] and kv_new [N, r + p] bf16; pages [n_pages, page, r + p] bf16, block_table [B, blocks] and
    cache_len [B] int32; token_offsets [B + 1] int32; mask int64 [N], bit j for the j-th draft of the sequence (None:
    causal).  All on the device; nothing is read back."""
    N, H, width = q.shape
    d = _drafts(N, token_offsets, mask)
    c = _latent_cache(pages, block_table, cache_len, d.B, r)
    o, lse, op, lp = _attn_outputs(q, r, o, lse)
    L = lib()
    workspace, nbytes = _scratch(workspace, L.moe_latent_attn_workspace_size, "moe_latent_attn_workspace_size", c, N, d.B, H,
                                 q.device)
    _check("moe_latent_attn", L.moe_latent_attn(
        C.byref(c), C.byref(d), _bf16_ptr(q, "q", N, H, c.r + c.p), _bf16_ptr(kv_new, "kv_new", N, c.r + c.p), H, scale, op, lp,
        _dev_ptr(workspace, "workspace"), nbytes, _stream(q)))
    return o, lse


def _strided_ptr(t, what: str, M: int, H: int) -> tuple[int, int, int, int]:
    """Pointer, head width, token stride and head stride of bf16 [M, H, width] with contiguous heads."""
    shape, stride = t.shape, t.stride()
    if not t.is_cuda or t.dtype is not _torch().bfloat16 or len(shape) != 3 or shape[0] != M or shape[1] != H or stride[2] != 1:
        raise ValueError(f"{what} must be bfloat16 [{M}, {H}, width] on the device, contiguous along its last axis")
    return t.data_ptr(), shape[2], stride[0], stride[1]


def moe_latent_prompt(q, k, k_rope, v, q_offsets, kv_offsets, scale: float, max_tokens: int | None = None, o=None, lse=None):
    """Latent attention in the expanded form, causal, of the prompts of B sequences -> (o [N, H, dv] bf16, lse [N, H] fp32).

    q [N, H, dn + p], k [M, H, dn], k_rope [M, p], v [M, H, dv] bf16 (k and v may be strided views of one expansion);
    q_offsets, kv_offsets [B + 1] int32.  A sequence's queries are the last of its keys' tokens.  max_tokens: at least
    the most queries of a sequence (None: N)."""
    N, H, dq = q.shape
    M, p = k_rope.shape
    B = q_offsets.shape[0] - 1
    kp, dn, ks, kh = _strided_ptr(k, "k", M, H)
    vp, dv, vs, vh = _strided_ptr(v, "v", M, H)
    o, lse, op, lp = _attn_outputs(q, dv, o, lse)
    a = moe_prompt_t(N, M, B, H, dn, p, dv, N if max_tokens is None else max_tokens,
                     _int32_ptr(q_offsets, "q_offsets", B + 1), _int32_ptr(kv_offsets, "kv_offsets", B + 1),
                     _bf16_ptr(q, "q", N, H, dn + p), kp, _bf16_ptr(k_rope, "k_rope", M, p), vp, ks, kh, vs, vh, scale)
    _check("moe_latent_prompt", lib().moe_latent_prompt(C.byref(a), op, lp, _stream(q)))
    return o, lse


def _cache(k, v, k_scale, v_scale, block_table, cache_len, B: int) -> moe_cache_t:
    torch = _torch()
    n_pages, heads, page, D = k.shape
    for t, what, dtype, shape in ((k, "k", torch.uint8, (n_pages, heads, page, D)), (v, "v", torch.uint8, (n_pages, heads, D, page)),
                                  (k_scale, "k_scale", torch.float32, (n_pages, heads)),
                                  (v_scale, "v_scale", torch.float32, (n_pages, heads))):
        if t.dtype != dtype or t.shape != shape:
            raise ValueError(f"{what} must be {dtype} {list(shape)}")
    blocks = block_table.shape[1]
    return moe_cache_t(heads, D, n_pages, page, blocks, _dev_ptr(k, "k"), _dev_ptr(v, "v"), _dev_ptr(k_scale, "k_scale"),
                       _dev_ptr(v_scale, "v_scale"), _int32_ptr(block_table, "block_table", B, blocks),
                       _int32_ptr(cache_len, "cache_len", B))


def moe_cache_append(k_new, v_new, token_offsets, k, v, k_scale, v_scale, block_table, cache_len, rows=None,
                     max_tokens: int | None = None, slots=None) -> None:
    """New tokens into the 8-bit cache, in place: sequence b's, entries token_offsets[b] .. token_offsets[b + 1] - 1 of
    `rows` (indices into k_new, v_new [n_rows, Hkv, D] bf16; None: the entries themselves), at positions cache_len[b] on.
    k [n_pages, Hkv, page, D] and v [n_pages, Hkv, D, page] uint8 codes, k_scale, v_scale [n_pages, Hkv] fp32.
    cache_len is not changed.  max_tokens: at least the most new tokens of a sequence (None: all).
    slots: int64 [N] of a moe_pages_update, for which the entries go there instead and cache_len is not read: a refused
    sequence gets nothing, and what follows fewer kept tokens than cached ones follows those."""
    B = token_offsets.shape[0] - 1
    c = _cache(k, v, k_scale, v_scale, block_table, cache_len, B)
    n_rows = k_new.shape[0]
    N = n_rows if rows is None else rows.shape[0]
    args = (C.byref(c), _bf16_ptr(k_new, "k_new", n_rows, c.Hkv, c.D), _bf16_ptr(v_new, "v_new", n_rows, c.Hkv, c.D), n_rows,
            None if rows is None else _int32_ptr(rows, "rows", N), N, B, _int32_ptr(token_offsets, "token_offsets", B + 1),
            N if max_tokens is None else max_tokens)
    if slots is None:
        _check("moe_cache_append", lib().moe_cache_append(*args, _stream(k_new)))
    else:
        slots = _typed_ptr(slots, _torch().int64, "slots", (N,))
        _check("moe_cache_append_slots", lib().moe_cache_append_slots(*args, slots, _stream(k_new)))


def moe_cache_attn_workspace_size(k, v, k_scale, v_scale, block_table, cache_len, N: int, H: int) -> int:
    B, n = block_table.shape[0], C.c_size_t()
    c = _cache(k, v, k_scale, v_scale, block_table, cache_len, B)
    _check("moe_cache_attn_workspace_size", lib().moe_cache_attn_workspace_size(C.byref(c), N, B, H, C.byref(n)))
    return n.value


def moe_cache_attn(q, k_new, v_new, token_offsets, k, v, k_scale, v_scale, block_table, cache_len, scale: float, mask=None,
                   o=None, lse=None, workspace=None):
    """Grouped-query attention of draft tokens over the 8-bit cache and each other -> (o [N, H, D] bf16, lse [N, H] fp32).

    q [N, H, D], k_new, v_new [N, Hkv, D] bf16; the cache as for moe_cache_append; mask as for moe_latent_attn."""
    N, H, D = q.shape
    d = _drafts(N, token_offsets, mask)
    c = _cache(k, v, k_scale, v_scale, block_table, cache_len, d.B)
    o, lse, op, lp = _attn_outputs(q, D, o, lse)
    L = lib()
    workspace, nbytes = _scratch(workspace, L.moe_cache_attn_workspace_size, "moe_cache_attn_workspace_size", c, N, d.B, H,
                                 q.device)
    _check("moe_cache_attn", L.moe_cache_attn(
        C.byref(c), C.byref(d), _bf16_ptr(q, "q", N, H, c.D), _bf16_ptr(k_new, "k_new", N, c.Hkv, c.D),
        _bf16_ptr(v_new, "v_new", N, c.Hkv, c.D), H, scale, op, lp, _dev_ptr(workspace, "workspace"), nbytes, _stream(q)))
    return o, lse


# --------------------------------------------------------------------------- the two ends of a decoding step

@dataclass
class PageUpdate:
    """Counts after a moe_pages_update, and where the new tokens go."""
    new_len: object    # int32 [B]
    n_free: object     # int32 [1]
    refused: object    # int32 [1]: sequences that got nothing
    slots: object      # int64 [N]: row among all pages' rows, -1: none
    positions: object  # int32 [N], -1: none


def moe_pages_update(cache_len, token_offsets, block_table, free_pages, n_free, page: int, N: int, keep_len=None,
                     out: PageUpdate | None = None) -> PageUpdate:
    """Pages for what a step changes: sequence b keeps its first keep_len[b] tokens (None: all) and gets
    token_offsets[b + 1] - token_offsets[b] new ones; pages that it no longer needs go to the free ones, those that it needs
    are taken from there.

    cache_len, keep_len [B], token_offsets [B + 1], n_free [1] int32; block_table [B, blocks] and free_pages [n_pages] int32
    are updated in place.  N: entries of slots and positions, at least the new tokens.  The counts are not changed: the new
    ones are new_len and n_free of the result, whose tensors are those of `out` where it is given (slots and positions may be
    None there)."""
    torch = _torch()
    i32, ptr = torch.int32, _typed_ptr
    B, blocks = block_table.shape
    n_pages, dev = free_pages.shape[0], block_table.device
    per, one, tokens = (B,), (1,), (N,)
    if out is None:
        ints, slots = torch.empty(B + 2 + N, dtype=i32, device=dev), torch.empty(N, dtype=torch.int64, device=dev)
        parts, at = ints.split_with_sizes((B, 1, 1, N)), ints.data_ptr()
        out = PageUpdate(parts[0], parts[1], parts[2], slots, parts[3])
        to = at, at + 4 * B, at + 4 * B + 4, slots.data_ptr(), at + 4 * B + 8
    else:
        to = [None if t is None else ptr(t, kind, what, of) for t, kind, what, of in (
            (out.new_len, i32, "new_len", per), (out.n_free, i32, "n_free", one), (out.refused, i32, "refused", one),
            (out.slots, torch.int64, "slots", tokens), (out.positions, i32, "positions", tokens))]
        _one_device(block_table, out.new_len, out.n_free, out.refused, out.slots, out.positions)
    _one_device(block_table, cache_len, free_pages, n_free, keep_len, token_offsets)
    pool = moe_page_pool_t(B, n_pages, page, blocks, ptr(block_table, i32, "block_table", (B, blocks)),
                           ptr(cache_len, i32, "cache_len", per), ptr(free_pages, i32, "free_pages", (n_pages,)),
                           ptr(n_free, i32, "n_free", one))
    _enqueue("moe_pages_update", lib().moe_pages_update, block_table,
             C.byref(pool), None if keep_len is None else ptr(keep_len, i32, "keep_len", per),
             ptr(token_offsets, i32, "token_offsets", (B + 1,)), N, *to)
    return out


def moe_latent_append(kv_new, pages, slots, rows=None) -> None:
    """New rows into the latent cache, in place: row slots[i] of the pages becomes row rows[i] (None: i) of kv_new
    [n_rows, r + p] bf16; slots int64 [N] (entries outside the pages, as -1, are dropped), rows int32 [N]; pages
    [n_pages, page, r + p] bf16."""
    torch = _torch()
    n_pages, page, width = pages.shape
    n_rows = kv_new.shape[0]
    N, = slots.shape
    _one_device(pages, kv_new, slots, rows)
    ptr = _typed_ptr
    _enqueue("moe_latent_append", lib().moe_latent_append, pages,
             ptr(pages, torch.bfloat16, "pages", (n_pages, page, width)), n_pages, page, width - 64, 64,
             ptr(kv_new, torch.bfloat16, "kv_new", (n_rows, width)), n_rows,
             None if rows is None else ptr(rows, torch.int32, "rows", (N,)), N, ptr(slots, torch.int64, "slots", (N,)))


@functools.cache
def moe_grouped_prompt_workspace_size(D: int) -> int:
    n = C.c_size_t()
    _check("moe_grouped_prompt_workspace_size", lib().moe_grouped_prompt_workspace_size(D, C.byref(n)))
    return n.value


def moe_grouped_prompt(q, k, v, q_offsets, kv_offsets, scale: float, max_tokens: int | None = None, o=None, lse=None,
                       workspace=None):
    """Grouped-query attention, causal, of the prompts of B sequences -> (o [N, H, D] bf16, lse [N, H] fp32).

    q [N, H, D], k, v [M, Hkv, D] bf16 (strided views of a projection's output, contiguous along D); q_offsets, kv_offsets
    [B + 1] int32.  A sequence's queries are the last of its keys' tokens.  max_tokens: at least the most queries of a
    sequence.  None stands for N: right, but with several sequences most workgroups are then empty, long keys are not cut into
    chunks, and B * H * N may pass the limit of 2^30."""
    torch = _torch()
    N, H = q.shape[:2]
    M, Hkv = k.shape[:2]
    B = q_offsets.shape[0] - 1
    qp, D, qs, qh = _strided_ptr(q, "q", N, H)
    kp, dk, ks, kh = _strided_ptr(k, "k", M, Hkv)
    vp, dv, vs, vh = _strided_ptr(v, "v", M, Hkv)
    if dk != D or dv != D:
        raise ValueError("q, k and v must have heads of one width")
    o, lse, op, lp = _attn_outputs(q, D, o, lse)
    if workspace is None:
        workspace = torch.empty(moe_grouped_prompt_workspace_size(D), dtype=torch.uint8, device=q.device)
    off = (B + 1,)
    _one_device(q, k, v, q_offsets, kv_offsets, o, lse, workspace)
    a = moe_grouped_prompt_t(N, M, B, H, Hkv, D, N if max_tokens is None else max_tokens,
                             _typed_ptr(q_offsets, torch.int32, "q_offsets", off),
                             _typed_ptr(kv_offsets, torch.int32, "kv_offsets", off), qp, kp, vp, qs, qh, ks, kh, vs, vh, scale)
    _enqueue("moe_grouped_prompt", lib().moe_grouped_prompt, q, C.byref(a), op, lp, _dev_ptr(workspace, "workspace"),
             workspace.numel() * workspace.element_size())
    return o, lse


@dataclass
class TokenLogprobs:
    """What moe_token_logprobs gives; what was not asked for is None."""
    logprob: object      # fp32 [N, M] (or [N], as the tokens)
    lse: object          # fp32 [N]
    entropy: object      # fp32 [N]
    top_idx: object      # int32 [N, k]
    top_logprob: object  # fp32 [N, k]


@functools.lru_cache(256)
def moe_token_logprobs_workspace_size(N: int) -> int:
    n = C.c_size_t()
    _check("moe_token_logprobs_workspace_size", lib().moe_token_logprobs_workspace_size(N, C.byref(n)))
    return n.value


def moe_token_logprobs(logits, tokens=None, k: int = 0, scale: float = 1.0, out: TokenLogprobs | None = None,
                       workspace=None) -> TokenLogprobs:
    """Log probabilities of given tokens, log-sum, entropy and the k best alternatives of rows of logits [N, V].

    logits bf16 or fp32, contiguous along V (rows may be strided); tokens int32 [N, M] or [N], entries outside [0, V) unused
    (-inf), or None; k: alternatives, largest logit first, equal ones by lower index; scale: the inverse temperature.
    out: tensors to write to (those that are None are not computed, but for what tokens and k ask for)."""
    torch = _torch()
    f32, i32, ptr = torch.float32, torch.int32, _typed_ptr
    if logits.dim() != 2 or logits.stride(1) != 1 and logits.shape[1] != 1:
        raise ValueError("logits must be [N, V], contiguous along V")
    N, V = logits.shape
    dtype, dev, stride = logits.dtype, logits.device, logits.stride(0)
    if not logits.is_cuda or dtype is not torch.bfloat16 and dtype is not f32:
        raise ValueError("logits must be bfloat16 or float32, on the device")
    if N == 1:
        stride = max(stride, V)
    M, shape = 0, None
    if tokens is not None:
        shape = tokens.shape
        if len(shape) not in (1, 2) or shape[0] != N:
            raise ValueError("tokens must be int32 [N] or [N, M]")
        M = shape[1] if len(shape) == 2 else 1
    if out is None:
        sizes = N * M, N, N, N * k, N * k
        flat = torch.empty(N * (2 + M + 2 * k), dtype=f32, device=dev)
        (given, lse, entropy, idx, top), at = flat.split_with_sizes(sizes), flat.data_ptr()
        out = TokenLogprobs(given.view(shape) if M else None, lse, entropy, idx.view(i32).view(N, k) if k else None,
                            top.view(N, k) if k else None)
        at1, at2, at3 = at + 4 * N * M, at + 4 * N * (M + 1), at + 4 * N * (M + 2)
        to = at if M else None, at1, at2, at3 if k else None, at3 + 4 * N * k if k else None
    else:
        if (out.logprob is None) != (not M) or (out.top_idx is None) != (not k):
            raise ValueError("out.logprob goes with tokens, out.top_idx with k")
        to = [None if t is None else ptr(t, kind, what, of) for t, kind, what, of in (
            (out.logprob, f32, "logprob", shape), (out.lse, f32, "lse", (N,)), (out.entropy, f32, "entropy", (N,)),
            (out.top_idx, i32, "top_idx", (N, k)), (out.top_logprob, f32, "top_logprob", (N, k)))]
    if workspace is None:
        workspace = torch.empty(moe_token_logprobs_workspace_size(N), dtype=torch.uint8, device=dev)
    _one_device(logits, tokens, workspace, out.logprob, out.lse, out.entropy, out.top_idx, out.top_logprob)
    _enqueue("moe_token_logprobs", lib().moe_token_logprobs, logits,
             logits.data_ptr(), MOE_F32 if dtype is f32 else MOE_BF16, stride, N, V, scale,
             ptr(tokens, i32, "tokens", shape) if M else None, M, k, *to, _dev_ptr(workspace, "workspace"),
             workspace.numel() * workspace.element_size())
    return out


# --------------------------------------------------------------------------- selector (host)

def moe_select_tree(parent, P, pred, E: int, budget: int, eps: float = 0.1, lam: float = 0.0,
                    mode: int = MOE_SEL_COST_RATIO, B0=None):
    """Cost-aware draft selection (Algorithm 1) on the host -> (selected, marginal_cost) int32 arrays."""
    par = np.ascontiguousarray(parent, np.int32)
    Pa = np.ascontiguousarray(P, np.float64)
    pr = np.ascontiguousarray(pred, np.int32)
    n, L, K = pr.shape
    sel = np.zeros(max(budget, 1), np.int32)
    cost = np.zeros(max(budget, 1), np.int32)
    nsel = np.zeros(1, np.int32)
    b0 = None if B0 is None else np.ascontiguousarray(B0, np.uint64)
    _check("moe_select_tree", lib().moe_select_tree(
        n, par.ctypes.data, Pa.ctypes.data, L, K, pr.ctypes.data, E, None if b0 is None else b0.ctypes.data,
        budget, eps, lam, mode, sel.ctypes.data, cost.ctypes.data, nsel.ctypes.data))
    m = int(nsel[0])
    return sel[:m].copy(), cost[:m].copy()
