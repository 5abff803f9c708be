"""Thin ctypes binding of libspecverify.so (include/spec_verify.h).

Argument marshalling only: every step of the verification path runs inside the
library's HIP kernels.  PyTorch is used for device memory and the current stream.
There is no CPU fallback; importing works without the library, calling does not.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspecverify.so")

SPEC_OK = 0
SPEC_BF16, SPEC_F32 = 0, 1
SPEC_FUSE_ARGMAX, SPEC_FUSE_MIXTURE = 0, 1
SPEC_Q_LOGITS, SPEC_Q_PROBS = 0, 1

EXPORTS = [
    "spec_verify_attn_workspace_size", "spec_verify_attn",
    "spec_fuse_drafts_workspace_size", "spec_fuse_drafts", "spec_fuse_drafts_tuned",
    "spec_accept_workspace_size", "spec_accept", "spec_accept_tuned",
    "spec_describe_attn_plan", "spec_describe_accept_plan",
    "spec_accept_noalloc", "spec_accept_noalloc_max_workspace",
    "spec_accept_greedy_workspace_size", "spec_accept_greedy",
    "spec_routing_scores", "spec_adaptive_speculation", "spec_compact_kv",
    "spec_row_stats_size", "spec_lm_head_workspace_size", "spec_lm_head", "spec_accept_prestats",
    "spec_describe_lm_head_plan",
    "spec_append_kv", "spec_append_kv_quant", "spec_verify_attn_quant_workspace_size", "spec_verify_attn_quant",
    "spec_describe_attn_quant_plan", "spec_compact_kv_quant",
    "spec_append_latent", "spec_absorb_latent", "spec_verify_attn_latent_workspace_size", "spec_verify_attn_latent",
    "spec_describe_attn_latent_plan", "spec_expand_latent", "spec_compact_latent",
    "spec_strerror", "spec_abi_version",
]


class SpecAttnDesc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("total_q", ctypes.c_int32),
        ("max_q_per_req", ctypes.c_int32), ("max_pages_per_req", ctypes.c_int32),
        ("total_kv_tokens_hint", ctypes.c_int64), ("scale", ctypes.c_float), ("out_dtype", ctypes.c_int32),
    ]


class SpecAppendDesc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("total_q", ctypes.c_int32),
        ("max_q_per_req", ctypes.c_int32), ("max_pages_per_req", ctypes.c_int32), ("num_pages", ctypes.c_int32),
        ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("rotary_scale", ctypes.c_float),
    ]


class SpecLatentDesc(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in (
        "batch", "num_heads", "latent_dim", "rope_dim", "nope_dim", "value_dim", "page_size", "total_q", "max_q_per_req", "max_pages_per_req",
        "num_pages", "interleaved", "out_dtype")] + [("rotary_scale", ctypes.c_float), ("norm_eps", ctypes.c_float), ("scale", ctypes.c_float)]


class SpecAcceptTuning(ctypes.Structure):
    """Explicit launch choices of spec_accept_tuned (0 / negative = the library's choice)."""
    _fields_ = [("path", ctypes.c_int32), ("levels", ctypes.c_int32), ("slices", ctypes.c_int32),
                ("patience", ctypes.c_int32), ("helpers", ctypes.c_int32)]

    def __init__(self, path=0, levels=0, slices=0, patience=-1, helpers=-1):
        super().__init__(path, levels, slices, patience, helpers)


class SpecError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed: {status} ({strerror(status)})")


_lib = None


def lib() -> ctypes.CDLL:
    """Load the HIP library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
        L.spec_strerror.restype = ctypes.c_char_p
        L.spec_strerror.argtypes = [i32]
        L.spec_abi_version.restype = i32
        L.spec_verify_attn_workspace_size.restype = sz
        L.spec_verify_attn_workspace_size.argtypes = [ctypes.POINTER(SpecAttnDesc)]
        L.spec_verify_attn.restype = i32
        L.spec_verify_attn.argtypes = [ctypes.POINTER(SpecAttnDesc)] + [vp] * 10 + [sz, vp]
        L.spec_fuse_drafts_workspace_size.restype = sz
        L.spec_fuse_drafts_workspace_size.argtypes = [i32] * 5
        L.spec_fuse_drafts.restype = i32
        L.spec_fuse_drafts.argtypes = [i32] * 4 + [vp] * 4 + [i32, f32, i32] + [vp] * 5 + [sz, vp]
        L.spec_fuse_drafts_tuned.restype = i32
        L.spec_fuse_drafts_tuned.argtypes = [i32] + L.spec_fuse_drafts.argtypes
        L.spec_accept_workspace_size.restype = sz
        L.spec_accept_workspace_size.argtypes = [i32] * 4
        L.spec_accept_greedy_workspace_size.restype = sz
        L.spec_accept_greedy_workspace_size.argtypes = [i32] * 3
        L.spec_accept_greedy.restype = i32
        L.spec_accept_greedy.argtypes = [i32] * 4 + [vp] * 4 + [i32, vp, vp, i32, vp, vp, vp, sz, vp]
        L.spec_routing_scores.restype = i32
        L.spec_routing_scores.argtypes = [i32] * 5 + [vp] * 5 + [i32, vp, i32, vp, vp]
        L.spec_adaptive_speculation.restype = i32
        L.spec_adaptive_speculation.argtypes = [i32, vp, vp, ctypes.c_int64, vp, vp, vp]
        L.spec_compact_kv.restype = i32
        L.spec_compact_kv.argtypes = [i32] * 5 + [vp] * 9
        L.spec_accept.restype = i32
        L.spec_accept.argtypes = ([i32] * 5 + [vp] * 4 + [i32, vp, i32, i32, vp, f32] + [vp] * 4 + [i32]
                                  + [vp] * 3 + [sz, vp])
        L.spec_accept_prestats.restype = i32
        L.spec_accept_prestats.argtypes = L.spec_accept.argtypes
        L.spec_accept_tuned.restype = i32
        L.spec_accept_tuned.argtypes = [ctypes.POINTER(SpecAcceptTuning)] + L.spec_accept.argtypes
        L.spec_accept_noalloc.restype = i32
        L.spec_accept_noalloc.argtypes = L.spec_accept.argtypes[:-3] + [vp]
        L.spec_accept_noalloc_max_workspace.restype = sz
        L.spec_accept_noalloc_max_workspace.argtypes = []
        L.spec_describe_attn_plan.restype = i32
        L.spec_describe_attn_plan.argtypes = [ctypes.POINTER(SpecAttnDesc), ctypes.c_char_p, sz]
        L.spec_describe_accept_plan.restype = i32
        L.spec_describe_accept_plan.argtypes = [ctypes.POINTER(SpecAcceptTuning)] + [i32] * 8 + [ctypes.c_char_p, sz]
        L.spec_row_stats_size.restype = sz
        L.spec_row_stats_size.argtypes = [i32, i32]
        L.spec_lm_head_workspace_size.restype = sz
        L.spec_lm_head_workspace_size.argtypes = [i32, i32, i32]
        L.spec_describe_lm_head_plan.restype = i32
        L.spec_describe_lm_head_plan.argtypes = [i32] * 3 + [ctypes.c_char_p, sz]
        L.spec_lm_head.restype = i32
        L.spec_lm_head.argtypes = [i32, i32, i32, vp, vp, f32, vp, vp, vp, sz, vp]
        i64 = ctypes.c_int64
        rows = [ctypes.POINTER(SpecAppendDesc), vp, i64, vp, i64, vp, i64]
        L.spec_append_kv.restype = i32
        L.spec_append_kv.argtypes = rows + [vp] * 10
        L.spec_append_kv_quant.restype = i32
        L.spec_append_kv_quant.argtypes = rows + [vp] * 12
        L.spec_verify_attn_quant_workspace_size.restype = sz
        L.spec_verify_attn_quant_workspace_size.argtypes = [ctypes.POINTER(SpecAttnDesc)]
        L.spec_verify_attn_quant.restype = i32
        L.spec_verify_attn_quant.argtypes = [ctypes.POINTER(SpecAttnDesc), i32] + [vp] * 12 + [sz, vp]
        L.spec_describe_attn_quant_plan.restype = i32
        L.spec_describe_attn_quant_plan.argtypes = [ctypes.POINTER(SpecAttnDesc), ctypes.c_char_p, sz]
        L.spec_compact_kv_quant.restype = i32
        L.spec_compact_kv_quant.argtypes = [i32] * 6 + [vp] * 11
        latent = ctypes.POINTER(SpecLatentDesc)
        L.spec_append_latent.restype = i32
        L.spec_append_latent.argtypes = [latent, vp, i64, vp, i64] + [vp] * 9
        L.spec_absorb_latent.restype = i32
        L.spec_absorb_latent.argtypes = [latent, vp, i64, vp, i64] + [vp] * 7
        L.spec_verify_attn_latent_workspace_size.restype = sz
        L.spec_verify_attn_latent_workspace_size.argtypes = [latent]
        L.spec_verify_attn_latent.restype = i32
        L.spec_verify_attn_latent.argtypes = [latent] + [vp] * 9 + [sz, vp]
        L.spec_describe_attn_latent_plan.restype = i32
        L.spec_describe_attn_latent_plan.argtypes = [latent, ctypes.c_char_p, sz]
        L.spec_expand_latent.restype = i32
        L.spec_expand_latent.argtypes = [latent, vp, vp, i64] + [vp] * 3
        L.spec_compact_latent.restype = i32
        L.spec_compact_latent.argtypes = [i32] * 5 + [vp] * 8
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().spec_strerror(int(status)).decode()


def _ptr(t) -> Optional[int]:
    # plain integers (None: NULL): the argument types make pointers of them without an object per argument
    if t is None:
        return None
    assert t.is_contiguous(), "tensors handed to the library must be contiguous"
    return t.data_ptr()


_raw_stream = None


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    # The handle itself: the object that torch.cuda.current_stream() builds around it costs 2.7 us, a third of a whole call
    # (1 request x 4 drafts x 1000 classes, two calls a step, bound by the host: 18.6 -> 13.6 us).
    global _raw_stream
    import torch
    if _raw_stream is None:
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _raw_stream = raw if raw is not None else lambda device: torch.cuda.current_stream(device).cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return SPEC_BF16
    if t.dtype == torch.float32:
        return SPEC_F32
    raise TypeError(f"unsupported tensor dtype {t.dtype}")


def make_attn_desc(batch, num_q_heads, num_kv_heads, head_dim, total_q, max_q_per_req, max_pages_per_req,
                   total_kv_tokens_hint=0, scale=0.0, out_dtype=SPEC_BF16, page_size=16) -> SpecAttnDesc:
    return SpecAttnDesc(batch, num_q_heads, num_kv_heads, head_dim, page_size, total_q, max_q_per_req,
                        max_pages_per_req, total_kv_tokens_hint, scale, out_dtype)


def spec_verify_attn_workspace_size(desc: SpecAttnDesc) -> int:
    return int(lib().spec_verify_attn_workspace_size(ctypes.byref(desc)))


def spec_verify_attn(desc: SpecAttnDesc, q, k_pool, v_pool, block_table, ctx_len, q_offsets, parent, out,
                     lse=None, workspace=None, stream=None) -> None:
    """Device tensors: q/k_pool/v_pool bf16, block_table/ctx_len/q_offsets/parent int32, out bf16 or
    fp32, lse fp32 or None, workspace uint8 of at least spec_verify_attn_workspace_size(desc) bytes."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().spec_verify_attn(ctypes.byref(desc), _ptr(q), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
                                _ptr(ctx_len), _ptr(q_offsets), _ptr(parent), _ptr(out), _ptr(lse),
                                _ptr(workspace), ws_bytes, _stream(stream))
    if rc != SPEC_OK:
        raise SpecError("spec_verify_attn", rc)


def spec_fuse_drafts_workspace_size(B, k_max, N, V, mode) -> int:
    return int(lib().spec_fuse_drafts_workspace_size(B, k_max, N, V, mode))


def spec_fuse_drafts(k_len, conf, draft_tokens, draft_logits, temperature, mode, fused_token, winner, q_row,
                     fused_probs=None, workspace=None, stream=None, V: Optional[int] = None) -> None:
    """conf/draft_tokens [B,k_max,N]; draft_logits [B*k_max*N, V] or None (ARGMAX)."""
    B, k_max, N = conf.shape
    if draft_logits is not None:
        V = draft_logits.shape[1]
        ldt = _dtype_code(draft_logits)
    else:
        V, ldt = (V or 0), SPEC_BF16
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().spec_fuse_drafts(B, k_max, N, V, _ptr(k_len), _ptr(conf), _ptr(draft_tokens), _ptr(draft_logits),
                                ldt, float(temperature), int(mode), _ptr(fused_token), _ptr(winner), _ptr(q_row),
                                _ptr(fused_probs), _ptr(workspace), ws_bytes, _stream(stream))
    if rc != SPEC_OK:
        raise SpecError("spec_fuse_drafts", rc)


def spec_fuse_drafts_tuned(patience, k_len, conf, draft_tokens, draft_logits, temperature, mode, fused_token, winner, q_row,
                           fused_probs=None, workspace=None, stream=None) -> None:
    """spec_fuse_drafts with logits and an explicit number of polls in the one-launch averaging."""
    B, k_max, N = conf.shape
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().spec_fuse_drafts_tuned(int(patience), B, k_max, N, draft_logits.shape[1], _ptr(k_len), _ptr(conf), _ptr(draft_tokens),
                                      _ptr(draft_logits), _dtype_code(draft_logits), float(temperature), int(mode), _ptr(fused_token),
                                      _ptr(winner), _ptr(q_row), _ptr(fused_probs), _ptr(workspace), ws_bytes, _stream(stream))
    if rc != SPEC_OK:
        raise SpecError("spec_fuse_drafts_tuned", rc)


def spec_accept_workspace_size(B, total_nodes, n_q_rows, V) -> int:
    return int(lib().spec_accept_workspace_size(B, total_nodes, n_q_rows, V))


def spec_accept(B, total_nodes, max_nodes_per_req, node_offsets, parent, draft_tokens, target_logits, draft_q,
                q_kind, q_row, temperature, u_accept, u_resample, accept_len, out_tokens, stop_node=None,
                dbg_ratio=None, workspace=None, stream=None) -> None:
    """target_logits [total_nodes+B, V], draft_q [n_q_rows, V] (bf16 or fp32 device tensors);
    out_tokens [B, out_stride] int32."""
    V = target_logits.shape[1]
    n_q_rows = 0 if draft_q is None else draft_q.shape[0]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().spec_accept(B, V, total_nodes, n_q_rows, max_nodes_per_req, _ptr(node_offsets), _ptr(parent),
                           _ptr(draft_tokens), _ptr(target_logits), _dtype_code(target_logits), _ptr(draft_q),
                           SPEC_BF16 if draft_q is None else _dtype_code(draft_q), int(q_kind), _ptr(q_row),
                           float(temperature), _ptr(u_accept), _ptr(u_resample), _ptr(accept_len),
                           _ptr(out_tokens), out_tokens.shape[1], _ptr(stop_node), _ptr(dbg_ratio),
                           _ptr(workspace), ws_bytes, _stream(stream))
    if rc != SPEC_OK:
        raise SpecError("spec_accept", rc)


def spec_accept_tuned(tuning, B, total_nodes, max_nodes_per_req, node_offsets, parent, draft_tokens, target_logits,
                      draft_q, q_kind, q_row, temperature, u_accept, u_resample, accept_len, out_tokens,
                      stop_node=None, dbg_ratio=None, workspace=None, stream=None) -> None:
    """spec_accept with explicit launch choices (a SpecAcceptTuning or None)."""
    V = target_logits.shape[1]
    n_q_rows = 0 if draft_q is None else draft_q.shape[0]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().spec_accept_tuned(None if tuning is None else ctypes.byref(tuning), B, V, total_nodes, n_q_rows,
                                 max_nodes_per_req, _ptr(node_offsets), _ptr(parent), _ptr(draft_tokens),
                                 _ptr(target_logits), _dtype_code(target_logits), _ptr(draft_q),
                                 SPEC_BF16 if draft_q is None else _dtype_code(draft_q), int(q_kind), _ptr(q_row),
                                 float(temperature), _ptr(u_accept), _ptr(u_resample), _ptr(accept_len),
                                 _ptr(out_tokens), out_tokens.shape[1], _ptr(stop_node), _ptr(dbg_ratio),
                                 _ptr(workspace), ws_bytes, _stream(stream))
    if rc != SPEC_OK:
        raise SpecError("spec_accept_tuned", rc)


def spec_accept_noalloc(B, total_nodes, max_nodes_per_req, node_offsets, parent, draft_tokens, target_logits,
                        draft_q, q_kind, q_row, temperature, u_accept, u_resample, accept_len, out_tokens,
                        stop_node=None, dbg_ratio=None, stream=None) -> None:
    """spec_accept on the library's built-in scratch array: no workspace argument, no allocation."""
    V = target_logits.shape[1]
    n_q_rows = 0 if draft_q is None else draft_q.shape[0]
    rc = lib().spec_accept_noalloc(B, V, total_nodes, n_q_rows, max_nodes_per_req, _ptr(node_offsets), _ptr(parent),
                                   _ptr(draft_tokens), _ptr(target_logits), _dtype_code(target_logits), _ptr(draft_q),
                                   SPEC_BF16 if draft_q is None else _dtype_code(draft_q), int(q_kind), _ptr(q_row),
                                   float(temperature), _ptr(u_accept), _ptr(u_resample), _ptr(accept_len),
                                   _ptr(out_tokens), out_tokens.shape[1], _ptr(stop_node), _ptr(dbg_ratio),
                                   _stream(stream))
    if rc != SPEC_OK:
        raise SpecError("spec_accept_noalloc", rc)


def spec_describe_attn_plan(desc: SpecAttnDesc) -> str:
    buf = ctypes.create_string_buffer(512)
    rc = lib().spec_describe_attn_plan(ctypes.byref(desc), buf, 512)
    if rc != SPEC_OK:
        raise SpecError("spec_describe_attn_plan", rc)
    return buf.value.decode()


def spec_describe_accept_plan(B, V, total_nodes, max_nodes_per_req, is_tree, target_dtype=SPEC_BF16, q_dtype=SPEC_BF16,
                              q_kind=SPEC_Q_LOGITS, tuning=None) -> str:
    buf = ctypes.create_string_buffer(512)
    rc = lib().spec_describe_accept_plan(None if tuning is None else ctypes.byref(tuning), B, V, total_nodes,
                                         max_nodes_per_req, int(bool(is_tree)), target_dtype, q_dtype, q_kind, buf, 512)
    if rc != SPEC_OK:
        raise SpecError("spec_describe_accept_plan", rc)
    return buf.value.decode()


def spec_describe_lm_head_plan(rows, d_model, V) -> str:
    buf = ctypes.create_string_buffer(256)
    rc = lib().spec_describe_lm_head_plan(rows, d_model, V, buf, 256)
    if rc != SPEC_OK:
        raise SpecError("spec_describe_lm_head_plan", rc)
    return buf.value.decode()


def spec_accept_prestats(B, total_nodes, max_nodes_per_req, node_offsets, parent, draft_tokens, target_logits,
                         draft_q, q_kind, q_row, temperature, u_accept, u_resample, accept_len, out_tokens,
                         stop_node=None, dbg_ratio=None, workspace=None, stream=None) -> None:
    """spec_accept whose workspace already starts with the target rows' statistics (from spec_lm_head)."""
    V = target_logits.shape[1]
    n_q_rows = 0 if draft_q is None else draft_q.shape[0]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().spec_accept_prestats(B, V, total_nodes, n_q_rows, max_nodes_per_req, _ptr(node_offsets),
                                    _ptr(parent), _ptr(draft_tokens), _ptr(target_logits),
                                    _dtype_code(target_logits), _ptr(draft_q),
                                    SPEC_BF16 if draft_q is None else _dtype_code(draft_q), int(q_kind),
                                    _ptr(q_row), float(temperature), _ptr(u_accept), _ptr(u_resample),
                                    _ptr(accept_len), _ptr(out_tokens), out_tokens.shape[1], _ptr(stop_node),
                                    _ptr(dbg_ratio), _ptr(workspace), ws_bytes, _stream(stream))
    if rc != SPEC_OK:
        raise SpecError("spec_accept_prestats", rc)


def spec_row_stats_size(rows, V) -> int:
    return int(lib().spec_row_stats_size(rows, V))


def spec_lm_head_workspace_size(rows, d_model, V) -> int:
    return int(lib().spec_lm_head_workspace_size(rows, d_model, V))


def spec_lm_head(hidden, weight, temperature, logits, target_stats, workspace, stream=None) -> None:
    """hidden [rows, d_model], weight [V, d_model], logits [rows, V]: bf16 device tensors; target_stats:
    device tensor of at least spec_row_stats_size(rows, V) bytes (normally the accept workspace)."""
    rows, d_model = hidden.shape
    V = weight.shape[0]
    assert weight.shape[1] == d_model and tuple(logits.shape) == (rows, V)
    assert target_stats.numel() * target_stats.element_size() >= spec_row_stats_size(rows, V)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().spec_lm_head(rows, d_model, V, _ptr(hidden), _ptr(weight), float(temperature), _ptr(logits),
                            _ptr(target_stats), _ptr(workspace), ws_bytes, _stream(stream))
    if rc != SPEC_OK:
        raise SpecError("spec_lm_head", rc)


def spec_accept_greedy_workspace_size(B, total_nodes, V) -> int:
    return int(lib().spec_accept_greedy_workspace_size(B, total_nodes, V))


def spec_accept_greedy(B, total_nodes, max_nodes_per_req, node_offsets, parent, draft_tokens, target_logits,
                       accept_len, out_tokens, stop_node=None, row_argmax=None, workspace=None, stream=None) -> None:
    """target_logits [total_nodes+B, V] (bf16 or fp32 device tensor); out_tokens [B, out_stride] int32."""
    V = target_logits.shape[1]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().spec_accept_greedy(B, V, total_nodes, max_nodes_per_req, _ptr(node_offsets), _ptr(parent),
                                  _ptr(draft_tokens), _ptr(target_logits), _dtype_code(target_logits),
                                  _ptr(accept_len), _ptr(out_tokens), out_tokens.shape[1], _ptr(stop_node),
                                  _ptr(row_argmax), _ptr(workspace), ws_bytes, _stream(stream))
    if rc != SPEC_OK:
        raise SpecError("spec_accept_greedy", rc)


def spec_routing_scores(k_len, conf, draft_tokens, accept_len, out_tokens, embedding, scores, stream=None) -> None:
    """conf, draft_tokens [B, k_max, N]; out_tokens [B, out_stride] int32; embedding [V, E] (bf16 or fp32);
    scores [B, N] fp32 (device tensors)."""
    B, k_max, N = conf.shape
    V, E = embedding.shape
    rc = lib().spec_routing_scores(B, k_max, N, V, E, _ptr(k_len), _ptr(conf), _ptr(draft_tokens), _ptr(accept_len),
                                   _ptr(out_tokens), out_tokens.shape[1], _ptr(embedding), _dtype_code(embedding),
                                   _ptr(scores), _stream(stream))
    if rc != SPEC_OK:
        raise SpecError("spec_routing_scores", rc)


def spec_adaptive_speculation(gamma_in, gamma_max_total, gamma_out, in_batch=None, total_out=None, stream=None) -> None:
    """gamma_in, gamma_out [R] int32, in_batch [R] int32 or None, total_out [1] int64 or None (device tensors)."""
    rc = lib().spec_adaptive_speculation(gamma_in.shape[0], _ptr(gamma_in), _ptr(in_batch), int(gamma_max_total),
                                         _ptr(gamma_out), _ptr(total_out), _stream(stream))
    if rc != SPEC_OK:
        raise SpecError("spec_adaptive_speculation", rc)


def spec_compact_kv(k_pool, v_pool, block_table, ctx_len, q_offsets, parent, stop_node, new_len=None, stream=None) -> None:
    """Pools [num_pages, Hkv, 16, D] bf16 device tensors (modified in place); the rest int32 device tensors."""
    _, Hkv, page, D = k_pool.shape
    rc = lib().spec_compact_kv(ctx_len.shape[0], Hkv, D, page, block_table.shape[1], _ptr(k_pool), _ptr(v_pool),
                               _ptr(block_table), _ptr(ctx_len), _ptr(q_offsets), _ptr(parent), _ptr(stop_node),
                               _ptr(new_len), _stream(stream))
    if rc != SPEC_OK:
        raise SpecError("spec_compact_kv", rc)


# ---- keys and values into the cache, and the 8-bit cache ----
def make_append_desc(batch, num_q_heads, num_kv_heads, head_dim, total_q, max_q_per_req, max_pages_per_req, num_pages,
                     rotary_dim=0, interleaved=False, rotary_scale=0.0, page_size=16) -> SpecAppendDesc:
    return SpecAppendDesc(batch, num_q_heads, num_kv_heads, head_dim, page_size, total_q, max_q_per_req, max_pages_per_req,
                          num_pages, rotary_dim, int(interleaved), rotary_scale)


_types = None


def _tensor_types():
    # looked up once: an import statement and three attributes of torch cost 0.4 us a call
    global _types
    if _types is None:
        import torch
        _types = (torch.int32, torch.float32, torch.bfloat16)
    return _types


def _tensor(t, dtype, entries, at, what):
    """The pointer of a contiguous tensor of that type, of at least so many entries, on device `at` (None: NULL).  The calls follow the descriptor: another
    type would be read as this one's bits, and a smaller tensor, or one of another device, beyond its end."""
    if t is None:
        return None
    if t.dtype is dtype and t.is_contiguous() and t.numel() >= entries and t.get_device() == at:
        return t.data_ptr()
    if t.dtype is not dtype:
        raise TypeError(f"{what}: {dtype} expected, not {t.dtype}")
    if not t.is_contiguous():
        raise AssertionError("tensors handed to the library must be contiguous")
    if t.numel() < entries:
        raise ValueError(f"{what}: {entries} entries expected, not {t.numel()}")
    raise ValueError(f"{what} lies on {t.device}, the cache does not")


def _places(batch, width, tokens, at, i32, block_table, ctx_len, q_offsets, parent):
    """Pointers of what says where a batch's tokens lie; the block table has rows of `width` pages (of one request, or flat: as many at least)."""
    try:                                              # (_tensor four times over costs 0.4 us more)
        if (block_table.dtype is i32 and ctx_len.dtype is i32 and q_offsets.dtype is i32
                and block_table.shape == (batch, width) and ctx_len.numel() >= batch and q_offsets.numel() > batch
                and block_table.is_contiguous() and ctx_len.is_contiguous() and q_offsets.is_contiguous()
                and block_table.get_device() == at and ctx_len.get_device() == at and q_offsets.get_device() == at
                and (parent is None or (parent.dtype is i32 and parent.numel() >= tokens and parent.is_contiguous() and parent.get_device() == at))):
            return block_table.data_ptr(), ctx_len.data_ptr(), q_offsets.data_ptr(), None if parent is None else parent.data_ptr()
    except AttributeError:                            # (None, which the library refuses itself)
        pass
    if block_table is not None and batch > 1 and block_table.dim() == 2 and block_table.shape[1] != width:
        raise ValueError(f"block_table: rows of {width} pages expected, not of {block_table.shape[1]}")
    return (_tensor(block_table, i32, batch * width, at, "block_table"), _tensor(ctx_len, i32, batch, at, "ctx_len"),
            _tensor(q_offsets, i32, batch and batch + 1, at, "q_offsets"), _tensor(parent, i32, tokens, at, "parent"))


_current_device = None


def _stream_beside(stream, at) -> int:
    """The stream's handle (None: the current one) for a call on tensors of device `at`."""
    global _current_device
    if at < 0:
        raise ValueError("the cache has to lie on a GPU device")
    if stream is not None:
        on, handle = stream.device_index, stream.cuda_stream
    else:
        if _current_device is None:
            import torch
            _stream(None)                             # (the tensors exist: nothing is left to initialise)
            _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        on = _current_device()
        handle = _raw_stream(on)
    if on != at:
        raise ValueError(f"the cache lies on device {at}, the stream belongs to device {on}")
    return handle


def _rows(t, heads, head_dim, rows, at, bf16, what):
    """(pointer, elements between tokens) of a [tokens, heads, head_dim] bf16 tensor whose tokens may lie apart."""
    if t is None:
        return None, 0
    if t.dtype is not bf16:
        raise TypeError(f"{what}: torch.bfloat16 expected, not {t.dtype}")
    apart, head, one = t.stride()                     # (ValueError for another number of dimensions)
    if t.shape != (rows, heads, head_dim) or one != 1 or (heads > 1 and head != head_dim):
        raise ValueError(f"{what}: [{rows}, {heads}, {head_dim}] with contiguous heads expected")
    if t.get_device() != at:
        raise ValueError(f"{what} lies on {t.device}, the cache does not")
    return t.data_ptr(), apart if rows > 1 else heads * head_dim


def _quant_pools(k_pool, v_pool, k_scale, v_scale, at, f32, desc=None):
    """Pointers of an 8-bit cache: k_pool [num_pages, Hkv, D / 16, 16, 16] and v_pool [num_pages, Hkv, D, 16] of torch.float8_e4m3fn
    or torch.uint8, scales [num_pages, Hkv] float32."""
    if k_pool.element_size() != 1 or v_pool.element_size() != 1:
        raise TypeError("the pools of the 8-bit cache have one byte per entry")
    pages, heads, dim, page = v_pool.shape
    scales = (pages, heads)
    if k_pool.shape != (pages, heads, dim // 16, page, 16) or k_scale.shape != scales or v_scale.shape != scales:
        raise ValueError("k_pool [num_pages, Hkv, D / 16, 16, 16], v_pool [num_pages, Hkv, D, 16] and scales [num_pages, Hkv] expected")
    if desc is not None and (heads != desc.num_kv_heads or dim != desc.head_dim):
        raise ValueError(f"a cache of {heads} heads of {dim} dimensions, the descriptor has {desc.num_kv_heads} of {desc.head_dim}")
    if k_scale.dtype is not f32 or v_scale.dtype is not f32:
        raise TypeError("k_scale, v_scale: torch.float32 expected")
    if not (k_pool.is_contiguous() and v_pool.is_contiguous() and k_scale.is_contiguous() and v_scale.is_contiguous()):
        raise AssertionError("tensors handed to the library must be contiguous")
    if not (v_pool.get_device() == at and k_scale.get_device() == at and v_scale.get_device() == at):
        raise ValueError("the pools and scales of a cache have to lie on one device")
    return k_pool.data_ptr(), v_pool.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr()


def _append(fn, desc, types, q, k, v, inv_freq, pools, block_table, ctx_len, q_offsets, parent, q_out, positions, stream, at):
    i32, f32, bf16 = types
    Hq, D, total, Hkv = desc.num_q_heads, desc.head_dim, desc.total_q, desc.num_kv_heads
    qp, qs = _rows(q, Hq, D, total, at, bf16, "q")
    kp, ks = _rows(k, Hkv, D, total, at, bf16, "k")
    vp, vs = _rows(v, Hkv, D, total, at, bf16, "v")
    rc = fn(desc, qp, qs, kp, ks, vp, vs, _tensor(inv_freq, f32, desc.rotary_dim // 2, at, "inv_freq"),
            _tensor(positions, i32, total, at, "positions"), *pools,
            *_places(desc.batch, desc.max_pages_per_req, total, at, i32, block_table, ctx_len, q_offsets, parent),
            _tensor(q_out, bf16, total * Hq * D, at, "q_out"), _stream_beside(stream, at))
    if rc != SPEC_OK:
        raise SpecError(fn.__name__, rc)


def spec_append_kv(desc: SpecAppendDesc, q, k, v, inv_freq, k_pool, v_pool, block_table, ctx_len, q_offsets, parent, q_out,
                   positions=None, stream=None) -> None:
    """Device tensors: q [total_q, Hq, D], k and v [total_q, Hkv, D] bf16 (tokens may lie apart, as slices of one projection do),
    inv_freq [rotary_dim / 2] float32, pools [num_pages, Hkv, 16, D] bf16 (modified), the rest int32; q_out [total_q, Hq, D] bf16."""
    types = _tensor_types()
    want = (desc.num_pages, desc.num_kv_heads, desc.page_size, desc.head_dim)
    if k_pool.shape != want or v_pool.shape != want:
        raise ValueError(f"pools of {want} expected, as in the descriptor")
    bf16, at = types[2], k_pool.get_device()
    if (k_pool.dtype is bf16 and v_pool.dtype is bf16 and k_pool.is_contiguous() and v_pool.is_contiguous() and v_pool.get_device() == at):
        pools = (k_pool.data_ptr(), v_pool.data_ptr())
    else:
        pools = (_tensor(k_pool, bf16, 0, at, "k_pool"), _tensor(v_pool, bf16, 0, at, "v_pool"))
    _append(lib().spec_append_kv, desc, types, q, k, v, inv_freq, pools, block_table, ctx_len, q_offsets, parent, q_out, positions, stream, at)


def spec_append_kv_quant(desc: SpecAppendDesc, q, k, v, inv_freq, k_pool, v_pool, k_scale, v_scale, block_table, ctx_len, q_offsets,
                         parent, q_out, positions=None, stream=None) -> None:
    """spec_append_kv into an 8-bit cache (pools and scales modified)."""
    if k_pool.shape[0] != desc.num_pages:
        raise ValueError(f"pools of {desc.num_pages} pages expected, as in the descriptor")
    types, at = _tensor_types(), k_pool.get_device()
    _append(lib().spec_append_kv_quant, desc, types, q, k, v, inv_freq, _quant_pools(k_pool, v_pool, k_scale, v_scale, at, types[1], desc),
            block_table, ctx_len, q_offsets, parent, q_out, positions, stream, at)


def spec_verify_attn_quant_workspace_size(desc: SpecAttnDesc) -> int:
    return int(lib().spec_verify_attn_quant_workspace_size(ctypes.byref(desc)))


def spec_verify_attn_quant(desc: SpecAttnDesc, q, k_pool, v_pool, k_scale, v_scale, block_table, ctx_len, q_offsets, parent, out,
                           lse=None, workspace=None, stream=None) -> None:
    """spec_verify_attn over an 8-bit cache; workspace of at least spec_verify_attn_quant_workspace_size(desc) bytes."""
    i32, f32, bf16 = _tensor_types()
    at, total = k_pool.get_device(), desc.total_q
    rows = total * desc.num_q_heads
    entries = rows * desc.head_dim
    ws_bytes = 0
    if workspace is not None:
        ws_bytes = workspace.nbytes
        if workspace.get_device() != at:
            raise ValueError(f"workspace lies on {workspace.device}, the cache does not")
    rc = lib().spec_verify_attn_quant(desc, k_pool.shape[0], _tensor(q, bf16, entries, at, "q"),
                                      *_quant_pools(k_pool, v_pool, k_scale, v_scale, at, f32, desc),
                                      *_places(desc.batch, desc.max_pages_per_req, total, at, i32, block_table, ctx_len, q_offsets, parent),
                                      _tensor(out, f32 if desc.out_dtype == SPEC_F32 else bf16, entries, at, "out"),
                                      _tensor(lse, f32, rows, at, "lse"), _ptr(workspace), ws_bytes, _stream_beside(stream, at))
    if rc != SPEC_OK:
        raise SpecError("spec_verify_attn_quant", rc)


def spec_describe_attn_quant_plan(desc: SpecAttnDesc) -> str:
    buf = ctypes.create_string_buffer(256)
    rc = lib().spec_describe_attn_quant_plan(ctypes.byref(desc), buf, 256)
    if rc != SPEC_OK:
        raise SpecError("spec_describe_attn_quant_plan", rc)
    return buf.value.decode()


def spec_compact_kv_quant(k_pool, v_pool, k_scale, v_scale, block_table, ctx_len, q_offsets, parent, stop_node, new_len=None,
                          stream=None) -> None:
    """spec_compact_kv over an 8-bit cache (pools and scales modified in place); the rest int32 device tensors.  parent, if given, has an entry for
    every token up to the last of q_offsets, whose value only the device knows."""
    (i32, f32, _), at = _tensor_types(), k_pool.get_device()
    pools = _quant_pools(k_pool, v_pool, k_scale, v_scale, at, f32)
    pages, heads, dim, page = v_pool.shape
    B, width = ctx_len.shape[0], block_table.shape[1]
    rc = lib().spec_compact_kv_quant(B, heads, dim, page, width, pages, *pools,
                                     *_places(B, width, 0, at, i32, block_table, ctx_len, q_offsets, parent),
                                     _tensor(stop_node, i32, B, at, "stop_node"), _tensor(new_len, i32, B, at, "new_len"),
                                     _stream_beside(stream, at))
    if rc != SPEC_OK:
        raise SpecError("spec_compact_kv_quant", rc)


# ---- the cache of latents ----
def make_latent_desc(batch, num_heads, latent_dim, rope_dim, nope_dim, value_dim, total_q, max_q_per_req, max_pages_per_req, num_pages,
                     interleaved=False, rotary_scale=0.0, norm_eps=0.0, scale=0.0, out_dtype=SPEC_BF16, page_size=16) -> SpecLatentDesc:
    return SpecLatentDesc(batch, num_heads, latent_dim, rope_dim, nope_dim, value_dim, page_size, total_q, max_q_per_req, max_pages_per_req,
                          num_pages, int(interleaved), out_dtype, rotary_scale, norm_eps, scale)


def _flat_rows(t, width, rows, at, bf16, what):
    """(pointer, elements between rows) of a [rows, width] bf16 tensor whose rows may lie apart."""
    if t is None:
        return None, 0
    if t.dtype is not bf16:
        raise TypeError(f"{what}: torch.bfloat16 expected, not {t.dtype}")
    apart, one = t.stride()                           # (ValueError for another number of dimensions)
    if t.shape != (rows, width) or one != 1:
        raise ValueError(f"{what}: [{rows}, {width}] with contiguous rows expected")
    if t.get_device() != at:
        raise ValueError(f"{what} lies on {t.device}, the call's other tensors do not")
    return t.data_ptr(), apart if rows > 1 else width


def _head_weight(t, heads, rows, width, at, bf16, what):
    """(pointer, elements between heads) of a [heads, rows, width] bf16 weight whose heads may lie apart."""
    if t is None:
        return None, 0
    if t.dtype is not bf16:
        raise TypeError(f"{what}: torch.bfloat16 expected, not {t.dtype}")
    apart, row, one = t.stride()
    if t.shape != (heads, rows, width) or one != 1 or row != width:
        raise ValueError(f"{what}: [{heads}, {rows}, {width}] with contiguous heads expected")
    if t.get_device() != at:
        raise ValueError(f"{what} lies on {t.device}, the call's other tensors do not")
    return t.data_ptr(), apart if heads > 1 else rows * width


def _latent_pool(desc, pool, bf16):
    """(pointer, device) of a cache of latents [num_pages, 16, latent_dim + rope_dim] bf16."""
    want = (desc.num_pages, desc.page_size, desc.latent_dim + desc.rope_dim)
    if pool.shape != want:
        raise ValueError(f"a pool of {want} expected, as in the descriptor")
    at = pool.get_device()
    return _tensor(pool, bf16, 0, at, "pool"), at


def spec_append_latent(desc: SpecLatentDesc, latent, key, norm_weight, inv_freq, pool, block_table, ctx_len, q_offsets, parent, positions=None,
                       stream=None) -> None:
    """Device tensors: latent [total_q, latent_dim] and key [total_q, rope_dim] bf16 (rows may lie apart, as slices of one projection do), norm_weight
    [latent_dim] bf16 or None, inv_freq [rope_dim / 2] float32, pool [num_pages, 16, latent_dim + rope_dim] bf16 (modified), the rest int32."""
    i32, f32, bf16 = _tensor_types()
    C, R, total = desc.latent_dim, desc.rope_dim, desc.total_q
    to, at = _latent_pool(desc, pool, bf16)
    rc = lib().spec_append_latent(desc, *_flat_rows(latent, C, total, at, bf16, "latent"), *_flat_rows(key, R, total, at, bf16, "key"),
                                  _tensor(norm_weight, bf16, C, at, "norm_weight"), _tensor(inv_freq, f32, R // 2, at, "inv_freq"),
                                  _tensor(positions, i32, total, at, "positions"), to,
                                  *_places(desc.batch, desc.max_pages_per_req, total, at, i32, block_table, ctx_len, q_offsets, parent),
                                  _stream_beside(stream, at))
    if rc != SPEC_OK:
        raise SpecError("spec_append_latent", rc)


def spec_absorb_latent(desc: SpecLatentDesc, q, w_key, inv_freq, ctx_len, q_offsets, parent, q_out, positions=None, stream=None) -> None:
    """q [total_q, num_heads, nope_dim + rope_dim] bf16 (tokens may lie apart), w_key [num_heads, nope_dim, latent_dim] bf16 (heads may lie apart, as the
    slice of one weight's do); q_out [total_q, num_heads, latent_dim + rope_dim] bf16."""
    i32, f32, bf16 = _tensor_types()
    H, C, R, N, total, at = desc.num_heads, desc.latent_dim, desc.rope_dim, desc.nope_dim, desc.total_q, q_out.get_device()
    rc = lib().spec_absorb_latent(desc, *_rows(q, H, N + R, total, at, bf16, "q"), *_head_weight(w_key, H, N, C, at, bf16, "w_key"),
                                  _tensor(inv_freq, f32, R // 2, at, "inv_freq"), _tensor(positions, i32, total, at, "positions"),
                                  _tensor(ctx_len, i32, desc.batch, at, "ctx_len"), _tensor(q_offsets, i32, desc.batch and desc.batch + 1, at, "q_offsets"),
                                  _tensor(parent, i32, total, at, "parent"), _tensor(q_out, bf16, total * H * (C + R), at, "q_out"),
                                  _stream_beside(stream, at))
    if rc != SPEC_OK:
        raise SpecError("spec_absorb_latent", rc)


def spec_verify_attn_latent_workspace_size(desc: SpecLatentDesc) -> int:
    return int(lib().spec_verify_attn_latent_workspace_size(ctypes.byref(desc)))


def spec_verify_attn_latent(desc: SpecLatentDesc, q, pool, block_table, ctx_len, q_offsets, parent, out, lse=None, workspace=None, stream=None) -> None:
    """q [total_q, num_heads, latent_dim + rope_dim] bf16, pool [num_pages, 16, latent_dim + rope_dim] bf16, out [total_q, num_heads, latent_dim] of the
    descriptor's type, lse [total_q, num_heads] float32 or None; workspace of at least spec_verify_attn_latent_workspace_size(desc) bytes."""
    i32, f32, bf16 = _tensor_types()
    held, at = _latent_pool(desc, pool, bf16)
    rows = desc.total_q * desc.num_heads
    ws_bytes = 0
    if workspace is not None:
        ws_bytes = workspace.nbytes
        if workspace.get_device() != at:
            raise ValueError(f"workspace lies on {workspace.device}, the cache does not")
    rc = lib().spec_verify_attn_latent(desc, _tensor(q, bf16, rows * (desc.latent_dim + desc.rope_dim), at, "q"), held,
                                       *_places(desc.batch, desc.max_pages_per_req, desc.total_q, at, i32, block_table, ctx_len, q_offsets, parent),
                                       _tensor(out, f32 if desc.out_dtype == SPEC_F32 else bf16, rows * desc.latent_dim, at, "out"),
                                       _tensor(lse, f32, rows, at, "lse"), _ptr(workspace), ws_bytes, _stream_beside(stream, at))
    if rc != SPEC_OK:
        raise SpecError("spec_verify_attn_latent", rc)


def spec_describe_attn_latent_plan(desc: SpecLatentDesc) -> str:
    buf = ctypes.create_string_buffer(256)
    rc = lib().spec_describe_attn_latent_plan(ctypes.byref(desc), buf, 256)
    if rc != SPEC_OK:
        raise SpecError("spec_describe_attn_latent_plan", rc)
    return buf.value.decode()


def spec_expand_latent(desc: SpecLatentDesc, x, w_value, q_offsets, out, stream=None) -> None:
    """x [total_q, num_heads, latent_dim] bf16, w_value [num_heads, value_dim, latent_dim] bf16 (heads may lie apart); out [total_q, num_heads, value_dim]
    bf16."""
    i32, _, bf16 = _tensor_types()
    H, C, V, total, at = desc.num_heads, desc.latent_dim, desc.value_dim, desc.total_q, out.get_device()
    rc = lib().spec_expand_latent(desc, _tensor(x, bf16, total * H * C, at, "x"), *_head_weight(w_value, H, V, C, at, bf16, "w_value"),
                                  _tensor(q_offsets, i32, desc.batch and desc.batch + 1, at, "q_offsets"), _tensor(out, bf16, total * H * V, at, "out"),
                                  _stream_beside(stream, at))
    if rc != SPEC_OK:
        raise SpecError("spec_expand_latent", rc)


def spec_compact_latent(pool, block_table, ctx_len, q_offsets, parent, stop_node, new_len=None, stream=None) -> None:
    """spec_compact_kv over a cache of latents [num_pages, 16, width] bf16 (modified in place); the rest int32 device tensors.  parent, if given, has an
    entry for every token up to the last of q_offsets, whose value only the device knows."""
    (i32, _, bf16), at = _tensor_types(), pool.get_device()
    pages, page, wide = pool.shape
    B, width = ctx_len.shape[0], block_table.shape[1]
    rc = lib().spec_compact_latent(B, wide, page, width, pages, _tensor(pool, bf16, 0, at, "pool"),
                                   *_places(B, width, 0, at, i32, block_table, ctx_len, q_offsets, parent),
                                   _tensor(stop_node, i32, B, at, "stop_node"), _tensor(new_len, i32, B, at, "new_len"), _stream_beside(stream, at))
    if rc != SPEC_OK:
        raise SpecError("spec_compact_latent", rc)
