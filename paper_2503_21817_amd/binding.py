"""ctypes binding of libskipffn.so - argument marshalling only.

Every function here has the name of the C entry point it calls
(include/skipffn.h) and does no arithmetic: PyTorch tensors provide device
memory and the current HIP stream, nothing else.  A missing library or a
non-zero status raises; there is no fallback path.
"""

from __future__ import annotations

import ctypes
import os
from ctypes import (POINTER, addressof, c_char_p, c_double, c_float, c_int, c_int32, c_int64,
                    c_size_t, c_uint32, c_void_p)

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libskipffn.so")

FLAG_DW_FP32 = 0x1
FLAG_DW_ACCUMULATE = 0x2
FLAG_NO_RESIDUAL = 0x4
FLAG_BALANCED_SPLIT = 0x8
FLAG_VALIDATE_IDX = 0x10
FLAG_QK_NORM = 0x20
FLAG_ROPE_PAIRS = 0x40

OK, EINVAL, ESHAPE, EWORKSPACE, EHIP, EUNSUPPORTED, EIDX = range(7)

# every symbol include/skipffn.h declares: (restype, argtypes)
_SIGNATURES = {
    "skipffn_compact_workspace_bytes": (c_size_t, [c_int64]),
    "skipffn_compact": (c_int, [c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p,
                                c_size_t, c_void_p]),
    "skipffn_compact_static_max_tokens": (c_int64, []),
    "skipffn_compact_static": (c_int, [c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p]),
    "skipffn_validate_idx": (c_int, [c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p]),
    "skipffn_saved_bytes": (c_size_t, [c_int64, c_int64, c_int64]),
    "skipffn_forward_workspace_bytes": (c_size_t, [c_int64, c_int64, c_int64, c_int]),
    "skipffn_forward": (c_int, [c_int64, c_int64, c_int64, c_float, c_void_p, c_void_p,
                                c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p,
                                c_void_p, c_void_p, c_void_p, c_size_t, c_uint32, c_void_p]),
    "skipffn_backward_workspace_bytes": (c_size_t, [c_int64, c_int64, c_int64]),
    "skipffn_backward": (c_int, [c_int64, c_int64, c_int64, c_float, c_void_p, c_void_p,
                                 c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p,
                                 c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                 c_size_t, c_uint32, c_void_p]),
    "skipffn_gather_rows": (c_int, [c_void_p, c_void_p, c_int64, c_int64, c_void_p, c_int64,
                                    c_void_p, c_void_p]),
    "skipffn_kv_compact": (c_int, [c_void_p, c_void_p, c_int64, c_int64, c_int64, c_int64, c_int64,
                                   c_void_p, c_int64, c_void_p, c_void_p]),
    "skipffn_summary_saved_bytes": (c_size_t, [c_int64, c_int64, c_int64]),
    "skipffn_summary_workspace_bytes": (c_size_t, [c_int64, c_int64, c_int64]),
    "skipffn_summary_forward": (c_int, [c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_int64, c_int64,
                                        c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "skipffn_summary_backward": (c_int, [c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_int64, c_int64,
                                         c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                         c_size_t, c_uint32, c_void_p]),
    "skipffn_select_retained": (c_int, [c_void_p, c_void_p, c_void_p, c_int64, c_int64, c_int64, c_int64,
                                        c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_void_p]),
    "skipffn_token_merge_workspace_bytes": (c_size_t, [c_int64, c_int64, c_int64]),
    "skipffn_token_merge": (c_int, [c_void_p, POINTER(c_int32), c_int64, c_int64, c_int64, c_void_p, c_void_p,
                                    c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "skipffn_token_merge_backward": (c_int, [c_void_p, POINTER(c_int32), c_int64, c_int64, c_int64, c_void_p,
                                             c_void_p, c_void_p]),
    "skipffn_attn_saved_bytes": (c_size_t, [c_int64, c_int64]),
    "skipffn_attn_forward_workspace_bytes": (c_size_t, [c_int64] * 6),
    "skipffn_attn_forward": (c_int, [c_int64] * 6 + [c_void_p] * 4 + [c_void_p, c_void_p, c_int, c_float, c_void_p, c_void_p,
                                                                           c_size_t, c_void_p]),
    "skipffn_attn_backward_workspace_bytes": (c_size_t, [c_int64] * 6),
    "skipffn_attn_backward": (c_int, [c_int64] * 6 + [c_void_p] * 5 + [c_void_p, c_void_p, c_int, c_float, c_void_p] +
                              [c_void_p] * 3 + [c_void_p, c_size_t, c_void_p]),
    "skipffn_attn_decode_workspace_bytes": (c_size_t, [c_int64] * 7),
    "skipffn_attn_decode": (c_int, [c_int64] * 7 + [c_void_p] * 3 + [c_void_p] * 2 + [c_void_p] * 2 + [c_int64] * 2 +
                            [c_void_p, c_void_p, c_float, c_void_p, c_size_t, c_void_p]),
    "skipffn_attn_decode_weights_workspace_bytes": (c_size_t, [c_int64] * 8),
    "skipffn_attn_decode_weights": (c_int, [c_int64] * 7 + [c_void_p] * 3 + [c_void_p] * 2 + [c_void_p] * 2 + [c_int64] * 2 +
                                    [c_void_p, c_void_p, c_float, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_int64, c_void_p, c_size_t,
                                     c_uint32, c_void_p]),
    "skipffn_attn_key_weights_workspace_bytes": (c_size_t, [c_int64] * 7),
    "skipffn_attn_key_weights": (c_int, [c_int64] * 6 + [c_void_p] * 4 + [c_int, c_float, c_void_p, c_int64, c_void_p, c_int64, c_void_p,
                                                                        c_size_t, c_uint32, c_void_p]),
    "skipffn_kv_evict": (c_int, [c_int64] * 5 + [c_int] + [c_void_p] * 2 + [c_int64] * 2 + [c_void_p] + [c_int64] * 2 + [c_void_p, c_int64, c_void_p] +
                         [c_int64] * 2 + [c_void_p] * 2 + [c_int64] * 2 + [c_void_p] + [c_int64] * 2 + [c_void_p] + [c_int64] * 2 + [c_void_p] * 2),
    "skipffn_qk_rope_forward": (c_int, [c_int64] * 6 + [c_void_p] * 3 + [c_void_p] * 3 + [c_void_p] * 2 + [c_float, c_void_p, c_int64] +
                                [c_void_p] * 3 + [c_uint32, c_void_p]),
    "skipffn_qk_rope_backward_workspace_bytes": (c_size_t, [c_int64] * 4),
    "skipffn_qk_rope_backward": (c_int, [c_int64] * 6 + [c_void_p] * 4 + [c_void_p] * 3 + [c_void_p] * 2 + [c_float] + [c_void_p] * 4 +
                                 [c_void_p, c_size_t, c_uint32, c_void_p]),
    "skipffn_probe_mfma": (c_int, [c_int64, c_int64, c_int, c_void_p, c_void_p, c_void_p]),
    "skipffn_saved_layout": (c_int, [c_int64, c_int64, c_int64, POINTER(c_size_t)]),
    "skipffn_status_string": (c_char_p, [c_int]),
    "skipffn_last_hip_error": (c_int, []),
    "skipffn_version": (c_int, []),
    "skipffn_profile_begin": (c_int, []),
    "skipffn_profile_end": (c_int, [POINTER(c_char_p), POINTER(c_double), POINTER(c_int64), c_int]),
}

_lib = None


class SkipFFNError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().skipffn_status_string(status).decode()
        if status == EHIP:
            msg += f" (hipError {lib().skipffn_last_hip_error()})"
        super().__init__(f"{where}: status {status}: {msg}")


def lib() -> ctypes.CDLL:
    """Load the C-ABI library (built by paper_2503_21817_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2503_21817_amd.build` "
                "(there is no CPU or PyTorch fallback for the Skip-FFN path)")
        l = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype = res
            fn.argtypes = args
        _lib = l
    return _lib


def exported_symbols():
    return sorted(_SIGNATURES)


def _check(status: int, where: str):
    if status != OK:
        raise SkipFFNError(status, where)


def _ptr(t):
    return None if t is None else c_void_p(t.data_ptr())


def _stream(device=None):
    # the handle that torch.cuda.current_stream().cuda_stream wraps, without the objects around it: 0.3 us for 2
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if device is None else device)


def _rargs(R, num_retained):
    """(R, num_retained pointer): R is a host int, or None to use the device count."""
    if R is None:
        if num_retained is None:
            raise ValueError("pass R or num_retained")
        return -1, _ptr(num_retained)
    return int(R), _ptr(num_retained)


# --------------------------------------------------------------------------------------
def skipffn_compact_workspace_bytes(T: int) -> int:
    return lib().skipffn_compact_workspace_bytes(T)


def skipffn_compact(skip_mask, idx, num_retained, pos=None, workspace=None):
    """skip_mask u8 [T] -> idx i32 [T] (first R entries), num_retained i32 [1], pos i32 [T]."""
    T = skip_mask.numel()
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().skipffn_compact(_ptr(skip_mask), T, _ptr(idx), _ptr(num_retained), _ptr(pos),
                                 _ptr(workspace), ws_bytes, _stream()), "skipffn_compact")


def skipffn_compact_static_max_tokens() -> int:
    return lib().skipffn_compact_static_max_tokens()


def skipffn_compact_static(skip_mask, idx, num_retained, pos=None):
    """skipffn_compact without a workspace: the library's own per-GPU scratch is used."""
    T = skip_mask.numel()
    _check(lib().skipffn_compact_static(_ptr(skip_mask), T, _ptr(idx), _ptr(num_retained), _ptr(pos), _stream()),
           "skipffn_compact_static")


def skipffn_validate_idx(idx, R, T, status, *, num_retained=None):
    """status i32 [2] on the device: {0 ok / 1 bad, first offending position}; asynchronous."""
    Rv, nr = _rargs(R, num_retained)
    _check(lib().skipffn_validate_idx(_ptr(idx), Rv, nr, T, _ptr(status), _stream()), "skipffn_validate_idx")


def skipffn_saved_bytes(R_max, C, I) -> int:
    return lib().skipffn_saved_bytes(R_max, C, I)


def skipffn_forward_workspace_bytes(R_max, C, I, has_saved) -> int:
    return lib().skipffn_forward_workspace_bytes(R_max, C, I, int(bool(has_saved)))


def skipffn_backward_workspace_bytes(R_max, C, I) -> int:
    return lib().skipffn_backward_workspace_bytes(R_max, C, I)


def skipffn_saved_layout(R_max, C, I):
    arr = (c_size_t * 8)()
    _check(lib().skipffn_saved_layout(R_max, C, I, arr), "skipffn_saved_layout")
    return list(arr)


def skipffn_forward(hidden, out, idx, R, w_gate, w_up, w_down, *, eps=1e-5, rms_gain=None,
                    num_retained=None, saved=None, workspace=None, flags=0):
    T, C = hidden.shape
    I = w_gate.shape[0]
    Rv, nr = _rargs(R, num_retained)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().skipffn_forward(T, C, I, eps, _ptr(hidden), _ptr(out), _ptr(idx), Rv, nr,
                                 _ptr(rms_gain), _ptr(w_gate), _ptr(w_up), _ptr(w_down),
                                 _ptr(saved), _ptr(workspace), ws_bytes, flags, _stream()),
           "skipffn_forward")


def skipffn_backward(grad_out, grad_hidden, idx, R, w_gate, w_up, w_down, saved, dw_gate, dw_up,
                     dw_down, *, eps=1e-5, rms_gain=None, num_retained=None, workspace=None,
                     flags=0, d_rms_gain=None):
    T, C = grad_out.shape
    I = w_gate.shape[0]
    Rv, nr = _rargs(R, num_retained)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().skipffn_backward(T, C, I, eps, _ptr(grad_out), _ptr(grad_hidden), _ptr(idx), Rv,
                                  nr, _ptr(rms_gain), _ptr(w_gate), _ptr(w_up), _ptr(w_down),
                                  _ptr(saved), _ptr(dw_gate), _ptr(dw_up), _ptr(dw_down),
                                  _ptr(d_rms_gain), _ptr(workspace), ws_bytes, flags, _stream()),
           "skipffn_backward")


def skipffn_gather_rows(src, dst, idx, R, *, num_retained=None):
    T = src.shape[0]
    row_bytes = (src.numel() // max(T, 1)) * src.element_size()
    Rv, nr = _rargs(R, num_retained)
    _check(lib().skipffn_gather_rows(_ptr(src), _ptr(dst), T, row_bytes, _ptr(idx), Rv, nr,
                                     _stream()), "skipffn_gather_rows")


def skipffn_kv_compact(src, dst, idx, R, *, num_retained=None):
    """src [..., T, D] -> dst [..., R_cap, D] (same leading dims, any R_cap >= R): every
    leading index is one slab.  Both tensors are contiguous."""
    T, D = src.shape[-2], src.shape[-1]
    n_slabs = src.numel() // max(T * D, 1)
    row_bytes = D * src.element_size()
    Rv, nr = _rargs(R, num_retained)
    _check(lib().skipffn_kv_compact(_ptr(src), _ptr(dst), n_slabs, T, row_bytes, T * row_bytes,
                                    dst.shape[-2] * row_bytes, _ptr(idx), Rv, nr, _stream()),
           "skipffn_kv_compact")


def skipffn_summary_saved_bytes(n_tok, S, C) -> int:
    return lib().skipffn_summary_saved_bytes(n_tok, S, C)


def skipffn_summary_workspace_bytes(n_tok, S, C) -> int:
    return lib().skipffn_summary_workspace_bytes(n_tok, S, C)


def _nbytes(t):
    return 0 if t is None else t.numel() * t.element_size()


def skipffn_summary_forward(hidden, tok, seg, w, out, *, saved=None, workspace=None):
    """hidden bf16 [T, C]; tok i32 [n_tok]; seg i32 [S + 1]; w bf16 [C]; out bf16 [S, C]."""
    T, C = hidden.shape
    _check(lib().skipffn_summary_forward(T, C, _ptr(hidden), _ptr(tok), _ptr(seg), tok.numel(),
                                         seg.numel() - 1, _ptr(w), _ptr(out), _ptr(saved),
                                         _ptr(workspace), _nbytes(workspace), _stream()),
           "skipffn_summary_forward")


def skipffn_summary_backward(hidden, tok, seg, w, saved, grad_out, grad_hidden, dw, *, workspace=None,
                             flags=0):
    T, C = hidden.shape
    _check(lib().skipffn_summary_backward(T, C, _ptr(hidden), _ptr(tok), _ptr(seg), tok.numel(),
                                          seg.numel() - 1, _ptr(w), _ptr(saved), _ptr(grad_out),
                                          _ptr(grad_hidden), _ptr(dw), _ptr(workspace),
                                          _nbytes(workspace), flags, _stream()),
           "skipffn_summary_backward")


def skipffn_select_retained(features, cls, seq_off, n_keep, mask, sim, *, token_pos=None, skip_mask=None):
    """features bf16 [n_feat, Cv]; cls bf16 [B, Cv]; seq_off i32 [B + 1]; n_keep: int, or an
    i32 [B] device tensor; mask u8 [n_feat]; sim f32 [n_feat]."""
    n_feat, Cv = features.shape
    nb = seq_off.numel() - 1
    if isinstance(n_keep, torch.Tensor):
        nk, nkd = 0, _ptr(n_keep)
    else:
        nk, nkd = int(n_keep), None
    T = 0 if skip_mask is None else skip_mask.numel()
    _check(lib().skipffn_select_retained(_ptr(features), _ptr(cls), _ptr(seq_off), n_feat, nb, Cv, nk, nkd,
                                         _ptr(mask), _ptr(sim), _ptr(token_pos), _ptr(skip_mask), T,
                                         _stream()), "skipffn_select_retained")


def skipffn_token_merge_workspace_bytes(n_tok, n_max, C) -> int:
    return lib().skipffn_token_merge_workspace_bytes(n_tok, n_max, C)


def skipffn_token_merge(x, seg, k, out, kept_idx, assign, avg_sim, *, workspace=None):
    """x bf16 [n_tok, C]; seg: host sequence of S + 1 offsets; out bf16 [S, k, C];
    kept_idx i32 [S, k]; assign i32 [n_tok]; avg_sim f32 [n_tok]."""
    seg = [int(v) for v in seg]
    arr = (c_int32 * len(seg))(*seg)
    _check(lib().skipffn_token_merge(_ptr(x), arr, len(seg) - 1, x.shape[1], int(k), _ptr(out),
                                     _ptr(kept_idx), _ptr(assign), _ptr(avg_sim), _ptr(workspace),
                                     _nbytes(workspace), _stream()), "skipffn_token_merge")


def skipffn_token_merge_backward(grad_out, seg, assign, grad_x):
    """grad_out bf16 [S, k, C]; seg: host sequence of S + 1 offsets; assign i32 [n_tok] from the
    forward call; grad_x bf16 [n_tok, C]."""
    seg = [int(v) for v in seg]
    arr = (c_int32 * len(seg))(*seg)
    _check(lib().skipffn_token_merge_backward(_ptr(grad_out), arr, len(seg) - 1, grad_out.shape[2],
                                              grad_out.shape[1], _ptr(assign), _ptr(grad_x), _stream()),
           "skipffn_token_merge_backward")


def _device(t, where):
    """The device of the call's tensors, which has to be the current one: its stream is what the library works on."""
    d = t.get_device()
    if d < 0 or d != torch.cuda.current_device():
        raise ValueError(f"{where}: tensors on the current GPU are wanted")
    return d


_HEADS = [c_int64 * (3 * n) for n in range(9)]


def _heads(where, device, *tensors):
    """What the library takes as skipffn_heads of tensors [..., tokens, heads, columns] whose columns lie together: the array that
    holds them, and the address of each."""
    v = []
    for t, shape in tensors:
        *_, st, sh, sc = t.stride()
        if sc != 1 and t.numel() == 0:                   # its strides say nothing
            st, sh, sc = shape[-2] * shape[-1], shape[-1], 1
        if t.shape != shape or t.dtype is not torch.bfloat16 or t.get_device() != device or (sc != 1 and shape[-1] > 1):
            raise ValueError(f"{where}: a bfloat16 tensor {tuple(shape)} on the device of the call, with contiguous columns, is wanted")
        # a stride that nothing is apart by is whatever the tensor was cut from
        v += (t.data_ptr(), st if shape[-3] > 1 else 0, sh if shape[-2] > 1 else 0)
    a = _HEADS[len(tensors)](*v)
    at = addressof(a)
    return a, range(at, at + 24 * len(tensors), 24)


def _ints(t, n, where, device):
    """Address of a contiguous int32 tensor of n values on the device."""
    if t.dtype != torch.int32 or t.numel() != n or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{where}: a contiguous int32 tensor of {n} values on the device of the call is wanted")
    return t.data_ptr()


def _buffer(t, least, where, device):
    """(address, bytes) of a workspace or a saved buffer, or of none."""
    if t is None:
        return None, 0
    n = t.numel() * t.element_size()
    if n < least or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{where}: a contiguous buffer of at least {least} bytes on the device of the call is wanted")
    return t.data_ptr(), n


def skipffn_attn_saved_bytes(Tq, Hq) -> int:
    return lib().skipffn_attn_saved_bytes(Tq, Hq)


def skipffn_attn_forward_workspace_bytes(Tq, Tk, n_seq, Hq, Hkv, D) -> int:
    return lib().skipffn_attn_forward_workspace_bytes(Tq, Tk, n_seq, Hq, Hkv, D)


def skipffn_attn_backward_workspace_bytes(Tq, Tk, n_seq, Hq, Hkv, D) -> int:
    return lib().skipffn_attn_backward_workspace_bytes(Tq, Tk, n_seq, Hq, Hkv, D)


def skipffn_attn_forward(q, k, v, out, seg_q, seg_k=None, *, causal=True, scale=None, saved=None, workspace=None):
    """q, out bf16 [Tq, Hq, D]; k, v bf16 [Tk, Hkv, D] (any token and head strides); seg_q, seg_k i32 [n_seq + 1].
    scale: None is 1 / sqrt(D)."""
    where = "skipffn_attn_forward"
    dev = _device(q, where)
    (Tq, Hq, D), (Tk, Hkv, _) = q.shape, k.shape
    kv = (Tk, Hkv, D)
    hold, (hq, hk, hv, ho) = _heads(where, dev, (q, q.shape), (k, kv), (v, kv), (out, q.shape))
    n1 = seg_q.numel()
    ws, ws_bytes = _buffer(workspace, 0, where, dev)
    sv = None if saved is None else _buffer(saved, Tq * Hq * 4, where, dev)[0]
    _check(lib().skipffn_attn_forward(Tq, Tk, n1 - 1, Hq, Hkv, D, hq, hk, hv, ho, _ints(seg_q, n1, where, dev),
                                      None if seg_k is None else _ints(seg_k, n1, where, dev), 1 if causal else 0,
                                      D ** -0.5 if scale is None else scale, sv, ws, ws_bytes, _stream(dev)), where)


def skipffn_attn_backward(q, k, v, out, grad_out, seg_q, seg_k, saved, grad_q, grad_k, grad_v, *, causal=True, scale=None,
                          workspace=None):
    """out and saved from the forward call with the same q, k, v, seg_q, seg_k, causal and scale; grad_out and grad_q as q,
    grad_k and grad_v as k."""
    where = "skipffn_attn_backward"
    dev = _device(q, where)
    (Tq, Hq, D), (Tk, Hkv, _) = q.shape, k.shape
    qs, kv = q.shape, (Tk, Hkv, D)
    hold, (hq, hk, hv, ho, hg, gq, gk, gv) = _heads(where, dev, (q, qs), (k, kv), (v, kv), (out, qs), (grad_out, qs), (grad_q, qs),
                                                    (grad_k, kv), (grad_v, kv))
    n1 = seg_q.numel()
    ws, ws_bytes = _buffer(workspace, 0, where, dev)
    _check(lib().skipffn_attn_backward(Tq, Tk, n1 - 1, Hq, Hkv, D, hq, hk, hv, ho, hg, _ints(seg_q, n1, where, dev),
                                       None if seg_k is None else _ints(seg_k, n1, where, dev), 1 if causal else 0,
                                       D ** -0.5 if scale is None else scale, _buffer(saved, Tq * Hq * 4, where, dev)[0], gq, gk, gv,
                                       ws, ws_bytes, _stream(dev)), where)


def skipffn_attn_decode_workspace_bytes(n_seq, n_groups, Hq, Hkv, D, Tp, suffix_capacity) -> int:
    return lib().skipffn_attn_decode_workspace_bytes(n_seq, n_groups, Hq, Hkv, D, Tp, suffix_capacity)


def _decode(where, q, prefix_k, prefix_v, prefix_seg, group_off, suffix_k, suffix_v, suffix_len, out, scale, workspace):
    """The library's arguments of skipffn_attn_decode, and what has to live until the call.  Flat: what it returns is a call's latency (single tokens are bound by
    the host)."""
    dev = _device(q, where)
    qs = n_seq, Hq, D = q.shape
    bare, alone = prefix_k is None, suffix_k is None
    if bare and alone:
        raise ValueError(f"{where}: a prefix or own rows are wanted")
    if bare != (prefix_v is None) or bare != (prefix_seg is None) or bare != (group_off is None) or \
            alone != (suffix_v is None) or alone != (suffix_len is None):
        raise ValueError(f"{where}: a prefix, or own rows, come with all that belongs to them")
    Hkv = (suffix_k if bare else prefix_k).shape[-2]
    Tp = n_groups = cap = seq_k = seq_v = 0
    seg = off = lens = pk = pv = sk = sv = None
    given = [(q, qs), (out, qs)]
    if not bare:
        Tp, n_groups = prefix_k.shape[0], group_off.numel() - 1
        seg, off = _ints(prefix_seg, n_groups + 1, where, dev), _ints(group_off, n_groups + 1, where, dev)
        given += [(prefix_k, (Tp, Hkv, D)), (prefix_v, (Tp, Hkv, D))]
    if not alone and n_seq > 0:
        cap = suffix_k.shape[1]
        lens = _ints(suffix_len, n_seq, where, dev)
        if n_seq > 1:
            seq_k, seq_v = suffix_k.stride(0), suffix_v.stride(0)
        own = (n_seq, cap, Hkv, D)
        given += [(suffix_k, own), (suffix_v, own)]
    hold, at = _heads(where, dev, *given)
    if not bare:
        pk, pv = at[2], at[3]
    if lens is not None:
        sk, sv = at[-2], at[-1]
    ws, ws_bytes = _buffer(workspace, 0, where, dev)
    return (n_seq, n_groups, Hq, Hkv, D, Tp, cap, at[0], pk, pv, seg, off, sk, sv, seq_k, seq_v, lens, at[1],
            D ** -0.5 if scale is None else scale, ws, ws_bytes, _stream(dev)), hold


def skipffn_attn_decode(q, prefix_k, prefix_v, prefix_seg, group_off, suffix_k, suffix_v, suffix_len, out, *, scale=None,
                        workspace=None):
    """q, out bf16 [n_seq, Hq, D]; prefix_k, prefix_v bf16 [Tp, Hkv, D] with prefix_seg, group_off i32 [n_groups + 1], or all
    four None; suffix_k, suffix_v bf16 [n_seq, capacity, Hkv, D] with suffix_len i32 [n_seq], or all three None.
    scale: None is 1 / sqrt(D)."""
    where = "skipffn_attn_decode"
    args, hold = _decode(where, q, prefix_k, prefix_v, prefix_seg, group_off, suffix_k, suffix_v, suffix_len, out, scale, workspace)
    _check(lib().skipffn_attn_decode(*args), where)


def skipffn_attn_decode_weights_workspace_bytes(n_seq, n_groups, Hq, Hkv, D, Tp, suffix_capacity, most_shared) -> int:
    return lib().skipffn_attn_decode_weights_workspace_bytes(n_seq, n_groups, Hq, Hkv, D, Tp, suffix_capacity, most_shared)


def skipffn_attn_decode_weights(q, prefix_k, prefix_v, prefix_seg, group_off, suffix_k, suffix_v, suffix_len, out, prefix_weights,
                                suffix_weights, *, most_shared=1, scale=None, workspace=None, flags=0):
    """skipffn_attn_decode, and what the rows receive: prefix_weights f32 [Hkv, Tp] and suffix_weights f32 [n_seq, Hkv, capacity] (None with
    the rows they belong to).  most_shared: most sequences of a group.  flags: FLAG_DW_ACCUMULATE."""
    where = "skipffn_attn_decode_weights"
    args, hold = _decode(where, q, prefix_k, prefix_v, prefix_seg, group_off, suffix_k, suffix_v, suffix_len, out, scale, workspace)
    (n_seq, _, _, Hkv, _, Tp, cap), dev = args[:7], q.get_device()
    if (prefix_k is None) != (prefix_weights is None) or (suffix_k is None) != (suffix_weights is None):
        raise ValueError(f"{where}: a prefix, or own rows, come with their weights")
    pw, sw = (None, 0), (None, 0, 0)
    if prefix_weights is not None:
        pw = _weights(prefix_weights, (Hkv, Tp), where, dev)
    if suffix_weights is not None and n_seq > 0:
        sw = _weights(suffix_weights, (n_seq, Hkv, cap), where, dev)
    _check(lib().skipffn_attn_decode_weights(*args[:19], most_shared, *pw, *sw, *args[19:21], flags, args[21]), where)


def _weights(t, shape, where, device, dtype=torch.float32):
    """(address, strides) of weights (or numbers) [..., heads, rows] whose rows lie together, and of what is before them."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or (t.stride(-1) != 1 and t.numel() > 0 and shape[-1] > 1):
        raise ValueError(f"{where}: a {dtype} tensor {tuple(shape)} on the device of the call, with contiguous rows, is wanted")
    return (t.data_ptr(),) + tuple(st if t.numel() > 0 and n > 1 else 0 for st, n in zip(t.stride()[:-1], shape[:-1]))


def skipffn_attn_key_weights_workspace_bytes(Tq, Tk, n_seq, Hq, Hkv, D, last=None) -> int:
    return lib().skipffn_attn_key_weights_workspace_bytes(Tq, Tk, n_seq, Hq, Hkv, D, -1 if last is None else last)


def skipffn_attn_key_weights(q, k, seg_q, seg_k, saved, weights, *, causal=True, scale=None, last=None, workspace=None, flags=0):
    """q, k, seg_q, seg_k, causal, scale: the forward call's, saved: what it wrote; weights f32 [Hkv, Tk] (any head stride).
    last: queries of a sequence that count, the last ones (None: all).  flags: FLAG_DW_ACCUMULATE."""
    where = "skipffn_attn_key_weights"
    dev = _device(q, where)
    (Tq, Hq, D), (Tk, Hkv, _) = q.shape, k.shape
    hold, (hq, hk) = _heads(where, dev, (q, q.shape), (k, (Tk, Hkv, D)))
    n1 = seg_q.numel()
    if last is not None and last < 0:
        raise ValueError(f"{where}: a number of queries, or None for all, is wanted")
    w, w_head = _weights(weights, (Hkv, Tk), where, dev)
    ws, ws_bytes = _buffer(workspace, 0, where, dev)
    _check(lib().skipffn_attn_key_weights(Tq, Tk, n1 - 1, Hq, Hkv, D, hq, hk, _ints(seg_q, n1, where, dev),
                                          None if seg_k is None else _ints(seg_k, n1, where, dev), 1 if causal else 0,
                                          D ** -0.5 if scale is None else scale, _buffer(saved, Tq * Hq * 4, where, dev)[0],
                                          -1 if last is None else last, w, w_head, ws, ws_bytes, flags, _stream(dev)), where)


def skipffn_kv_evict(k, v, weights, seg, n_keep, k_out, v_out, weights_out, keep, seg_out, *, first=0, recent=0):
    """Packed rows: k, v bf16 [T, Hkv, D], weights f32 [Hkv, T], seg i32 [n_seq + 1] -> k_out, v_out [T_out, Hkv, D], weights_out (or None) and keep i32
    [Hkv, T_out], seg_out i32 [n_seq + 1].  Own rows: k, v [n_seq, T, Hkv, D], weights [n_seq, Hkv, T], seg i32 [n_seq] -> k_out, v_out
    [n_seq, T_out, Hkv, D], weights_out, keep [n_seq, Hkv, T_out], seg_out i32 [n_seq].  n_keep: int, or an i32 [n_seq] device tensor."""
    where = "skipffn_kv_evict"
    dev = _device(k, where)
    packed = k.dim() == 3
    *_, T, Hkv, D = k.shape
    T_out = k_out.shape[-3]
    n_seq = seg.numel() - 1 if packed else k.shape[0]
    lead = () if packed else (n_seq,)
    src, dst, put = (*lead, T, Hkv, D), (*lead, T_out, Hkv, D), (*lead, Hkv, T_out)
    hold, at = _heads(where, dev, (k, src), (v, src), (k_out, dst), (v_out, dst))
    seq = [0] * 4 if packed or n_seq <= 1 else [t.stride(0) if t.numel() > 0 else 0 for t in (k, v, k_out, v_out)]

    def strides(t, shape, dtype=torch.float32):          # address, of heads, of sequences
        a, *st = _weights(t, shape, where, dev, dtype)
        return (a, st[-1], 0 if packed else st[0])
    w, kp = strides(weights, (*lead, Hkv, T)), strides(keep, put, torch.int32)
    wo = (None, 0, 0) if weights_out is None else strides(weights_out, put)
    nk, nkd = (0, _ints(n_keep, n_seq, where, dev)) if isinstance(n_keep, torch.Tensor) else (int(n_keep), None)
    n = n_seq + 1 if packed else n_seq
    _check(lib().skipffn_kv_evict(n_seq, Hkv, D, T, T_out, 1 if packed else 0, at[0], at[1], seq[0], seq[1], *w, _ints(seg, n, where, dev), nk, nkd,
                                  first, recent, at[2], at[3], seq[2], seq[3], *wo, *kp, _ints(seg_out, n, where, dev), _stream(dev)), where)


def _floats(t, n, where, device):
    """Address of a contiguous float32 tensor of n values on the device, or None."""
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != n or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{where}: a contiguous float32 tensor of {n} values on the device of the call is wanted")
    return t.data_ptr()


def _gain(t, D, where, device):
    if t is None:
        return None
    if t.dtype is not torch.bfloat16 or t.numel() != D or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{where}: a contiguous bfloat16 tensor of {D} values on the device of the call is wanted")
    return t.data_ptr()


def _rope(where, dev, T, pos, inv_freq, axis):
    """rot, n_axes, and the addresses of pos, inv_freq and axis"""
    rot, n_axes = 2 * inv_freq.numel(), pos.shape[0] if pos.dim() == 2 else 1
    at = _ints(pos, n_axes * T, where, dev)
    if axis is not None:
        axis = bytes(axis)
        if len(axis) != rot // 2:
            raise ValueError(f"{where}: an axis for each of {rot // 2} frequencies is wanted")
    return rot, n_axes, at, _floats(inv_freq, rot // 2, where, dev), axis


def skipffn_qk_rope_forward(q, k, q_out, k_out, pos, inv_freq, *, axis=None, v=None, v_out=None, row=None, gain_q=None, gain_k=None,
                            eps=1e-6, flags=0):
    """q, q_out bf16 [T, Hq, D]; k, v bf16 [T, Hkv, D]; k_out, v_out the same, or with row (i32 [T]) a cache [rows, Hkv, D] (any token and
    head strides); pos i32 [T] or [axes, T]; inv_freq f32 [rot / 2]; axis: bytes or a host sequence of rot / 2 axes.
    flags: FLAG_QK_NORM, FLAG_ROPE_PAIRS."""
    where = "skipffn_qk_rope_forward"
    dev = _device(q, where)
    (T, Hq, D), Hkv = q.shape, k.shape[1]
    if (v is None) != (v_out is None):
        raise ValueError(f"{where}: v and v_out come together")
    rows = T if row is None else k_out.shape[0]
    kv, out = (T, Hkv, D), (rows, Hkv, D)
    given = [(q, q.shape), (k, kv), (q_out, q.shape), (k_out, out)]
    if v is not None:
        given += [(v, kv), (v_out, out)]
    hold, at = _heads(where, dev, *given)
    rot, n_axes, hp, hf, ax = _rope(where, dev, T, pos, inv_freq, axis)
    _check(lib().skipffn_qk_rope_forward(T, Hq, Hkv, D, rot, n_axes, at[0], at[1], at[4] if v is not None else None, hp, hf, ax,
                                         _gain(gain_q, D, where, dev), _gain(gain_k, D, where, dev), eps,
                                         None if row is None else _ints(row, T, where, dev), rows, at[2], at[3],
                                         at[5] if v is not None else None, flags, _stream(dev)), where)


def skipffn_qk_rope_backward_workspace_bytes(T, Hq, Hkv, D) -> int:
    return lib().skipffn_qk_rope_backward_workspace_bytes(T, Hq, Hkv, D)


def skipffn_qk_rope_backward(grad_q_out, grad_k_out, grad_q, grad_k, pos, inv_freq, *, axis=None, q=None, k=None, gain_q=None, gain_k=None,
                             eps=1e-6, d_gain_q=None, d_gain_k=None, workspace=None, flags=0):
    """The forward call's pos, inv_freq, axis, gains, eps and flags, with FLAG_QK_NORM its q and k too; grad_* as q and k;
    d_gain_q, d_gain_k f32 [D] (FLAG_DW_ACCUMULATE: added to), which take a workspace."""
    where = "skipffn_qk_rope_backward"
    dev = _device(grad_q_out, where)
    (T, Hq, D), Hkv = grad_q_out.shape, grad_k_out.shape[1]
    qs, kv = grad_q_out.shape, (T, Hkv, D)
    given = [(grad_q_out, qs), (grad_k_out, kv), (grad_q, qs), (grad_k, kv)]
    norm = (flags & FLAG_QK_NORM) != 0
    if norm:
        if q is None or k is None:
            raise ValueError(f"{where}: the norm's gradient takes the forward call's q and k")
        given += [(q, qs), (k, kv)]
    hold, at = _heads(where, dev, *given)
    rot, n_axes, hp, hf, ax = _rope(where, dev, T, pos, inv_freq, axis)
    ws, ws_bytes = _buffer(workspace, 0, where, dev)
    _check(lib().skipffn_qk_rope_backward(T, Hq, Hkv, D, rot, n_axes, at[4] if norm else None, at[5] if norm else None, at[0], at[1], hp, hf,
                                          ax, _gain(gain_q, D, where, dev), _gain(gain_k, D, where, dev), eps, at[2], at[3],
                                          _floats(d_gain_q, D, where, dev), _floats(d_gain_k, D, where, dev), ws, ws_bytes, flags,
                                          _stream(dev)), where)


def skipffn_probe_mfma(blocks, iters, random_operands, out, clocks):
    """out f32 [blocks * 256]; clocks i64 [2 * blocks] (shader cycles, 100 MHz ticks per workgroup)."""
    _check(lib().skipffn_probe_mfma(blocks, iters, int(bool(random_operands)), _ptr(out), _ptr(clocks),
                                    _stream()), "skipffn_probe_mfma")


def skipffn_version() -> int:
    return lib().skipffn_version()


def skipffn_profile_begin():
    _check(lib().skipffn_profile_begin(), "skipffn_profile_begin")


def skipffn_profile_end():
    """-> {kernel class: (total ms, launches)} for classes that ran."""
    cap = 40
    names = (c_char_p * cap)()
    ms = (c_double * cap)()
    cnt = (c_int64 * cap)()
    n = lib().skipffn_profile_end(names, ms, cnt, cap)
    return {names[i].decode(): (ms[i], cnt[i]) for i in range(min(n, cap)) if cnt[i] > 0}


# --------------------------------------------------------------------------------------
class SkipFFNBuffers:
    """Device buffers for one (T, R_max, C, I) problem: index list, saved
    activations and workspaces, allocated once through PyTorch."""

    def __init__(self, T, R_max, C, I, device="cuda", training=True):
        self.T, self.R_max, self.C, self.I = T, R_max, C, I
        u8 = dict(dtype=torch.uint8, device=device)
        self.idx = torch.empty(max(T, 1), dtype=torch.int32, device=device)
        self.num_retained = torch.zeros(1, dtype=torch.int32, device=device)
        self.compact_ws = torch.empty(max(skipffn_compact_workspace_bytes(T), 16), **u8)
        self.saved = torch.empty(skipffn_saved_bytes(R_max, C, I), **u8) if training else None
        self.fwd_ws = torch.empty(skipffn_forward_workspace_bytes(R_max, C, I, training), **u8)
        self.bwd_ws = torch.empty(skipffn_backward_workspace_bytes(R_max, C, I), **u8) \
            if training else None

    def saved_views(self, R):
        """bf16 / f32 tensor views of the saved sections, for stage-wise checks."""
        off = skipffn_saved_layout(self.R_max, self.C, self.I)
        C, I = self.C, self.I
        s = self.saved

        def sect(o, nbytes, dtype, shape):
            return s[o:o + nbytes].view(dtype).view(shape)
        return {
            "xrows": sect(off[0], R * C * 2, torch.bfloat16, (R, C)),
            "xn": sect(off[1], R * C * 2, torch.bfloat16, (R, C)),
            "rstd": sect(off[2], R * 4, torch.float32, (R,)),
            "G": sect(off[3], R * I * 2, torch.bfloat16, (R, I)),
            "U": sect(off[4], R * I * 2, torch.bfloat16, (R, I)),
            "H": sect(off[5], R * I * 2, torch.bfloat16, (R, I)),
            "xnT": sect(off[6], C * ((self.R_max + 63) // 64 * 64) * 2, torch.bfloat16,
                        (C, (self.R_max + 63) // 64 * 64)),
            "HT": sect(off[7], I * ((self.R_max + 63) // 64 * 64) * 2, torch.bfloat16,
                       (I, (self.R_max + 63) // 64 * 64)),
        }
