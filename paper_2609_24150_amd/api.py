"""Python face of libaal: the C entry points under the same names, taking torch
tensors.  Each function checks shapes and dtypes, allocates its outputs and
workspace with torch, passes raw device pointers and the current HIP stream,
and returns.  It computes nothing itself.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import functools
import itertools
import operator
import struct

import torch

from . import _lib
from ._lib import (  # noqa: F401
    AAL_BF16, AAL_F32, AAL_FLAG_COOPERATIVE, AAL_FLAG_STREAMING, AAL_LAYOUT_SEQUENCES, AAL_LAYOUT_WINDOWS,
    AAL_BEAM_MAX, AAL_BEAM_SELECT_MAX, AAL_FP8_BLOCK, AAL_TOPK_MAX, AAL_VP_EAL, AAL_VP_WTV,
)

_DT = {torch.bfloat16: AAL_BF16, torch.float32: AAL_F32}
_FP8 = {torch.float8_e4m3fn: _lib.AAL_FP8_E4M3, torch.float8_e5m2: _lib.AAL_FP8_E5M2}
_SCALE = {torch.float32: _lib.AAL_SCALE_F32, torch.float8_e8m0fnu: _lib.AAL_SCALE_E8M0}


def _dtype_code(t: torch.dtype) -> int:
    if t not in _DT:
        raise TypeError(f"unsupported dtype {t}; use torch.bfloat16 or torch.float32")
    return _DT[t]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(device, stream):
    s = stream if stream is not None else torch.cuda.current_stream(device)
    return s.cuda_stream


def aal_workspace_bytes(rows: int, windows: int) -> int:
    return int(_lib.lib().aal_workspace_bytes(rows, windows))


def workspace(rows: int, windows: int, device) -> torch.Tensor:
    """A workspace tensor sized for `rows` logit rows and `windows` windows."""
    return torch.empty(aal_workspace_bytes(rows, windows), dtype=torch.uint8, device=device)


def _check_logits(z_draft: torch.Tensor, z_target: torch.Tensor, ndim: int):
    if z_draft.shape != z_target.shape or z_draft.dim() != ndim:
        raise ValueError(f"z_draft and z_target must both have {ndim} dims and equal shapes; got "
                         f"{tuple(z_draft.shape)} and {tuple(z_target.shape)}")
    if z_draft.dtype != z_target.dtype:
        raise TypeError("z_draft and z_target must share a dtype")
    if not (z_draft.is_cuda and z_target.is_cuda):
        raise ValueError("logits must be device tensors")
    if not (z_draft.is_contiguous() and z_target.is_contiguous()):
        raise ValueError("logits must be contiguous")


def _loss_outputs(N, K, V, dev, grad, grad_dtype, ref_dtype):
    out = {
        "loss": torch.empty(1, dtype=torch.float32, device=dev),
        "E": torch.empty(N, dtype=torch.float32, device=dev),
        "accept": torch.empty(N, K, dtype=torch.float32, device=dev),
    }
    out["grad"] = (torch.empty(N, K, V, dtype=grad_dtype or ref_dtype, device=dev) if grad else None)
    return out


def aal_eal_fwd_bwd(z_draft: torch.Tensor, z_target: torch.Tensor, temp_draft: float = 1.0, *,
                    grad: bool = True, grad_dtype: torch.dtype | None = None,
                    grad_scale: torch.Tensor | None = None, flags: int = 0,
                    ws: torch.Tensor | None = None, stream=None) -> dict:
    """Greedy EAL loss forward + backward on [N, K, V] logits.

    Returns a dict: loss [1], E [N], accept [N, K], xstar [N, K] int32 and
    grad [N, K, V] (None when grad=False)."""
    _check_logits(z_draft, z_target, 3)
    N, K, V = z_draft.shape
    dev = z_draft.device
    out = _loss_outputs(N, K, V, dev, grad, grad_dtype, z_draft.dtype)
    out["xstar"] = torch.empty(N, K, dtype=torch.int32, device=dev)
    g = out["grad"]
    if ws is None:
        ws = workspace(N * K, N, dev)
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.device != dev):
        raise TypeError("grad_scale must be a float32 device tensor")
    args = [_ptr(z_draft), _ptr(z_target), _dtype_code(z_draft.dtype), N, K, V, float(temp_draft),
            _ptr(out["loss"]), _ptr(out["E"]), _ptr(out["accept"]), _ptr(out["xstar"]),
            _ptr(g), _dtype_code(g.dtype) if g is not None else AAL_F32, _ptr(grad_scale)]
    tail = [_ptr(ws), ws.numel(), _stream(dev, stream)]
    if flags:
        st = _lib.lib().aal_eal_fwd_bwd_ex(*args, int(flags), *tail)
    else:
        st = _lib.lib().aal_eal_fwd_bwd(*args, *tail)
    _lib.check(st, "aal_eal_fwd_bwd")
    return out


def aal_wtv_fwd_bwd(z_draft: torch.Tensor, z_target: torch.Tensor, temp_draft: float = 1.0,
                    temp_target: float = 1.0, *, grad: bool = True, grad_dtype: torch.dtype | None = None,
                    grad_scale: torch.Tensor | None = None, flags: int = 0,
                    ws: torch.Tensor | None = None, stream=None) -> dict:
    """Window-TV loss forward + backward on [N, K, V] logits.

    Returns a dict: loss [1], E [N], accept [N, K] (= sum min(p, q)) and
    grad [N, K, V] (None when grad=False)."""
    _check_logits(z_draft, z_target, 3)
    N, K, V = z_draft.shape
    dev = z_draft.device
    out = _loss_outputs(N, K, V, dev, grad, grad_dtype, z_draft.dtype)
    g = out["grad"]
    if ws is None:
        ws = workspace(N * K, N, dev)
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.device != dev):
        raise TypeError("grad_scale must be a float32 device tensor")
    args = [_ptr(z_draft), _ptr(z_target), _dtype_code(z_draft.dtype), N, K, V,
            float(temp_draft), float(temp_target),
            _ptr(out["loss"]), _ptr(out["E"]), _ptr(out["accept"]),
            _ptr(g), _dtype_code(g.dtype) if g is not None else AAL_F32, _ptr(grad_scale)]
    tail = [_ptr(ws), ws.numel(), _stream(dev, stream)]
    if flags:
        st = _lib.lib().aal_wtv_fwd_bwd_ex(*args, int(flags), *tail)
    else:
        st = _lib.lib().aal_wtv_fwd_bwd(*args, *tail)
    _lib.check(st, "aal_wtv_fwd_bwd")
    return out


def aal_sim_accept_grpo(z_draft: torch.Tensor, z_target: torch.Tensor, u1: torch.Tensor, u2: torch.Tensor,
                        temperature: float = 1.0, *, eps: float = 1e-6, std_ddof: int = 0,
                        adv_clip: float = 0.0, accept: bool = True, ws: torch.Tensor | None = None,
                        stream=None) -> dict:
    """Simulated acceptance length and group advantages on [P, G, K, V] logits
    with uniforms u1, u2 of shape [P, G, K].

    Returns a dict: token [P, G, K] int32, accept [P, G, K] int32 (None with
    accept=False, which calls the entry point without that output),
    reward [P, G] int32, advantage [P, G] float32."""
    _check_logits(z_draft, z_target, 4)
    P, G, K, V = z_draft.shape
    dev = z_draft.device
    for u in (u1, u2):
        if u.shape != (P, G, K) or u.dtype != torch.float32 or u.device != dev or not u.is_contiguous():
            raise ValueError("u1 and u2 must be contiguous float32 device tensors of shape [P, G, K]")
    out = {
        "token": torch.empty(P, G, K, dtype=torch.int32, device=dev),
        "accept": torch.empty(P, G, K, dtype=torch.int32, device=dev) if accept else None,
        "reward": torch.empty(P, G, dtype=torch.int32, device=dev),
        "advantage": torch.empty(P, G, dtype=torch.float32, device=dev),
    }
    if ws is None:
        ws = workspace(P * G * K, P * G, dev)
    head = [_ptr(z_draft), _ptr(z_target), _dtype_code(z_draft.dtype), P, G, K, V, float(temperature),
            _ptr(u1), _ptr(u2), _ptr(out["token"])]
    tail = [_ptr(out["reward"]), _ptr(out["advantage"]), float(eps), int(std_ddof), float(adv_clip),
            _ptr(ws), ws.numel(), _stream(dev, stream)]
    if accept:
        st = _lib.lib().aal_sim_accept_grpo_ex(*head, _ptr(out["accept"]), *tail)
    else:
        st = _lib.lib().aal_sim_accept_grpo(*head, *tail)
    _lib.check(st, "aal_sim_accept_grpo")
    return out


def aal_loss_workspace_bytes(layout: int, B: int, S: int, K: int) -> int:
    return int(_lib.lib().aal_loss_workspace_bytes(int(layout), int(B), int(S), int(K)))


def aal_loss_fwd_bwd(z_draft: torch.Tensor, z_target: torch.Tensor | None, K: int, *,
                     weights=(0.0, 0.0, 0.0, 0.0), temp_draft: float = 1.0, temp_target: float = 1.0,
                     layout: int = AAL_LAYOUT_WINDOWS, labels: torch.Tensor | None = None,
                     grad: bool = True, grad_dtype: torch.dtype | None = None,
                     grad_scale: torch.Tensor | None = None, flags: int = 0, outputs: bool = True,
                     ws: torch.Tensor | None = None, stream=None) -> dict:
    """Combined objective forward + backward (weights = (wtv, eal, kl, tv)).

    Windows layout: logits [N, K, V] (N disjoint windows).  Sequences layout:
    logits [B, S, V]; a window of K positions starts at every t <= S - K.
    labels: int32 [rows] (or the logits' leading shape) replacing the greedy
    target token of the EAL term, or None.  z_target may be None only when
    the EAL term alone is asked for with labels.

    Returns a dict: loss [1], terms [4] (L_WTV, L_EAL, L_KL, L_TV), E_tv [W],
    E_eal [W], accept_tv [R], accept_eal [R], xstar [R] int32, grad (the
    logits' shape, or None).  With outputs=False the per-window and per-row
    arrays are not requested (None in the dict)."""
    if z_draft.dim() != 3 or not z_draft.is_cuda or not z_draft.is_contiguous():
        raise ValueError("z_draft must be a contiguous [B, S or K, V] device tensor")
    if z_target is not None:
        if z_target.shape != z_draft.shape or z_target.dtype != z_draft.dtype or not z_target.is_contiguous():
            raise ValueError("z_target must match z_draft in shape, dtype and layout")
    B, S, V = z_draft.shape
    if layout == AAL_LAYOUT_WINDOWS and S != K:
        raise ValueError("windows layout needs logits of shape [N, K, V]")
    R = B * S
    W = B if layout == AAL_LAYOUT_WINDOWS else B * max(0, S - K + 1)
    dev = z_draft.device
    if labels is not None and (labels.dtype != torch.int32 or labels.numel() != R or not labels.is_contiguous()
                               or labels.device != dev):
        raise ValueError("labels must be a contiguous int32 device tensor with one entry per row")
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.device != dev):
        raise TypeError("grad_scale must be a float32 device tensor")
    out = {
        "loss": torch.empty(1, dtype=torch.float32, device=dev),
        "terms": torch.empty(4, dtype=torch.float32, device=dev),
        "E_tv": torch.empty(W, dtype=torch.float32, device=dev) if outputs else None,
        "E_eal": torch.empty(W, dtype=torch.float32, device=dev) if outputs else None,
        "accept_tv": torch.empty(R, dtype=torch.float32, device=dev) if outputs else None,
        "accept_eal": torch.empty(R, dtype=torch.float32, device=dev) if outputs else None,
        "xstar": torch.empty(R, dtype=torch.int32, device=dev) if outputs else None,
        "grad": torch.empty(B, S, V, dtype=grad_dtype or z_draft.dtype, device=dev) if grad else None,
    }
    if ws is None:
        ws = torch.empty(aal_loss_workspace_bytes(layout, B, S, K), dtype=torch.uint8, device=dev)
    g = out["grad"]
    w = _lib.LossWeights(*(float(x) for x in weights))
    st = _lib.lib().aal_loss_fwd_bwd(
        _ptr(z_draft), _ptr(z_target), _ptr(labels), _dtype_code(z_draft.dtype), int(layout), B, S, K, V,
        float(temp_draft), float(temp_target), w, _ptr(out["loss"]), _ptr(out["terms"]),
        _ptr(out["E_tv"]) if W and outputs else None, _ptr(out["E_eal"]) if W and outputs else None,
        _ptr(out["accept_tv"]), _ptr(out["accept_eal"]), _ptr(out["xstar"]),
        _ptr(g), _dtype_code(g.dtype) if g is not None else AAL_F32, _ptr(grad_scale), int(flags),
        _ptr(ws), ws.numel(), _stream(dev, stream))
    _lib.check(st, "aal_loss_fwd_bwd")
    return out


def aal_grpo_workspace_bytes(layout: int, B: int, S: int, G: int, m: int, K: int) -> int:
    return int(_lib.lib().aal_grpo_workspace_bytes(int(layout), int(B), int(S), int(G), int(m), int(K)))


def aal_grpo_fwd_bwd(z_theta: torch.Tensor, z_ref: torch.Tensor, z_target: torch.Tensor | None, m: int, K: int, *,
                     layout: int = AAL_LAYOUT_WINDOWS, anchors: torch.Tensor | None = None,
                     labels: torch.Tensor | None = None, temperature: float = 1.0, eps: float = 1e-6,
                     adv_clip: float = 0.0, eps_clip: float = 0.2, rho_min: float = 0.0,
                     rho_max: float = float("inf"), grad: bool = True, grad_dtype: torch.dtype | None = None,
                     grad_scale: torch.Tensor | None = None, ws: torch.Tensor | None = None, stream=None) -> dict:
    """GRPO loss on the debiased greedy acceptance length, forward + backward
    w.r.t. z_theta.

    Windows layout: logits [B, m*K, V] (B groups of m windows of K rows).
    Sequences layout: logits [B, S, V] and anchors int32 [B, G].
    Returns a dict: loss [1], tau_theta, tau_ref [groups, m] int32,
    advantage, log_rho [groups, m], grad (the logits' shape, or None)."""
    for t in (z_theta, z_ref) + ((z_target,) if z_target is not None else ()):
        if t.dim() != 3 or not t.is_cuda or not t.is_contiguous() or t.shape != z_theta.shape or t.dtype != z_theta.dtype:
            raise ValueError("logits must be contiguous device tensors of one shape [B, rows, V] and dtype")
    B, S, V = z_theta.shape
    dev = z_theta.device
    if layout == AAL_LAYOUT_WINDOWS:
        if S != m * K:
            raise ValueError("windows layout needs logits of shape [groups, m*K, V]")
        G, groups = 1, B
    else:
        if anchors is None or anchors.dim() != 2 or anchors.shape[0] != B or anchors.dtype != torch.int32:
            raise ValueError("sequences layout needs int32 anchors of shape [B, G]")
        G = anchors.shape[1]
        groups = B * G
        anchors = anchors.contiguous()
    if labels is not None and (labels.dtype != torch.int32 or labels.numel() != B * S or labels.device != dev):
        raise ValueError("labels must be an int32 device tensor with one entry per row")
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.device != dev):
        raise TypeError("grad_scale must be a float32 device tensor")
    out = {
        "loss": torch.empty(1, dtype=torch.float32, device=dev),
        "tau_theta": torch.empty(groups, m, dtype=torch.int32, device=dev),
        "tau_ref": torch.empty(groups, m, dtype=torch.int32, device=dev),
        "advantage": torch.empty(groups, m, dtype=torch.float32, device=dev),
        "log_rho": torch.empty(groups, m, dtype=torch.float32, device=dev),
        "grad": torch.empty(B, S, V, dtype=grad_dtype or z_theta.dtype, device=dev) if grad else None,
    }
    if ws is None:
        ws = torch.empty(aal_grpo_workspace_bytes(layout, B, S, G, m, K), dtype=torch.uint8, device=dev)
    g = out["grad"]
    prm = _lib.GrpoParams(float(eps), float(adv_clip), float(eps_clip), float(rho_min), float(rho_max))
    st = _lib.lib().aal_grpo_fwd_bwd(
        _ptr(z_theta), _ptr(z_ref), _ptr(z_target), _ptr(labels), _dtype_code(z_theta.dtype), int(layout),
        B, S, G, m, K, V, _ptr(anchors), float(temperature), prm, _ptr(out["loss"]), _ptr(out["tau_theta"]),
        _ptr(out["tau_ref"]), _ptr(out["advantage"]), _ptr(out["log_rho"]),
        _ptr(g), _dtype_code(g.dtype) if g is not None else AAL_F32, _ptr(grad_scale),
        _ptr(ws), ws.numel(), _stream(dev, stream))
    _lib.check(st, "aal_grpo_fwd_bwd")
    return out


# ----------------------------------------------------------------------------
# Vocabulary-parallel pieces (one rank's share of a vocabulary-split LM head).
# Records are uint8 device tensors of shape [rows, record bytes]; view them as
# float32 / int32 to read fields.  The caller gathers the records over ranks.

def _vp_slice(z_draft, z_target, need_target=True):
    if z_draft.dim() != 2:
        raise ValueError("vocabulary slices are [rows, V_slice]")
    if need_target or z_target is not None:
        _check_logits(z_draft, z_target, 2)
    elif not (z_draft.is_cuda and z_draft.is_contiguous()):
        raise ValueError("z_draft must be a contiguous device tensor")
    return z_draft.shape[0], z_draft.shape[1], z_draft.device


def _records(t: torch.Tensor, nbytes: int, name: str, lead: int):
    if t.dtype != torch.uint8 or t.dim() != lead + 1 or t.shape[-1] != nbytes or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous uint8 tensor of records of {nbytes} bytes")


def aal_vp_row_partials(z_draft: torch.Tensor, z_target: torch.Tensor | None, v0: int, mode: int,
                        temp_draft: float = 1.0, temp_target: float = 1.0, *, V_total: int,
                        labels: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Step 1: partial row statistics of the slice [v0, v0 + V_slice) of a
    vocabulary of V_total entries.  EAL may take int32 labels [rows] (global
    token ids, clamped into [0, V_total)) in place of the target's greedy
    token; the target slice may then be None.  Returns [rows, 32] records."""
    rows, vs, dev = _vp_slice(z_draft, z_target, need_target=labels is None)
    if labels is not None and (labels.dtype != torch.int32 or labels.numel() != rows or labels.device != dev
                               or not labels.is_contiguous()):
        raise ValueError("labels must be a contiguous int32 device tensor with one entry per row")
    parts = torch.empty(rows, _lib.VP_PART_BYTES, dtype=torch.uint8, device=dev)
    st = _lib.lib().aal_vp_row_partials(_ptr(z_draft), _ptr(z_target), _ptr(labels), _dtype_code(z_draft.dtype),
                                        rows, vs, int(v0), int(V_total), int(mode), float(temp_draft),
                                        float(temp_target),
                                        _ptr(parts), _stream(dev, stream))
    _lib.check(st, "aal_vp_row_partials")
    return parts


def aal_vp_merge_rows(parts_all: torch.Tensor, mode: int, temp_draft: float = 1.0, temp_target: float = 1.0, *,
                      stream=None) -> torch.Tensor:
    """Step 2: merge gathered partials [R, rows, 32] in rank order.  Returns [rows, 32] row records."""
    _records(parts_all, _lib.VP_PART_BYTES, "parts_all", 2)
    R, rows = parts_all.shape[0], parts_all.shape[1]
    dev = parts_all.device
    row = torch.empty(rows, _lib.VP_ROW_BYTES, dtype=torch.uint8, device=dev)
    st = _lib.lib().aal_vp_merge_rows(_ptr(parts_all), R, rows, int(mode), float(temp_draft), float(temp_target),
                                      _ptr(row), _stream(dev, stream))
    _lib.check(st, "aal_vp_merge_rows")
    return row


def aal_vp_accept_partials(z_draft: torch.Tensor, z_target: torch.Tensor, row: torch.Tensor,
                           temp_draft: float = 1.0, temp_target: float = 1.0, *, stream=None) -> torch.Tensor:
    """Step 3 (WTV): the slice's sum min(p, q) and Q< partials.  Returns [rows, 8] records."""
    rows, vs, dev = _vp_slice(z_draft, z_target)
    _records(row, _lib.VP_ROW_BYTES, "row", 1)
    if row.shape[0] != rows:
        raise ValueError("row must hold one record per logit row")
    acc = torch.empty(rows, _lib.VP_ACC_BYTES, dtype=torch.uint8, device=dev)
    st = _lib.lib().aal_vp_accept_partials(_ptr(z_draft), _ptr(z_target), _dtype_code(z_draft.dtype), rows, vs,
                                           float(temp_draft), float(temp_target), _ptr(row), _ptr(acc),
                                           _stream(dev, stream))
    _lib.check(st, "aal_vp_accept_partials")
    return acc


def aal_vp_window_scan(row: torch.Tensor, acc_all: torch.Tensor | None, N: int, K: int, mode: int,
                       temp_draft: float = 1.0, *, grad_scale: torch.Tensor | None = None, stream=None) -> dict:
    """Step 4: window scan over the merged rows (updated in place with a, qlt
    and coef).  acc_all [R, N*K, 8] in WTV mode.  Returns loss [1], E [N],
    accept [N, K] and, in EAL mode, xstar [N, K]."""
    _records(row, _lib.VP_ROW_BYTES, "row", 1)
    if row.shape[0] != N * K:
        raise ValueError("row must hold N*K records")
    dev = row.device
    R = 0
    if mode == _lib.AAL_VP_WTV:
        if acc_all is None:
            raise ValueError("acc_all is required in WTV mode")
        _records(acc_all, _lib.VP_ACC_BYTES, "acc_all", 2)
        if acc_all.shape[1] != N * K:
            raise ValueError("acc_all must be [R, N*K, 8]")
        R = acc_all.shape[0]
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.device != dev):
        raise TypeError("grad_scale must be a float32 device tensor")
    out = {
        "loss": torch.empty(1, dtype=torch.float32, device=dev),
        "E": torch.empty(N, dtype=torch.float32, device=dev),
        "accept": torch.empty(N, K, dtype=torch.float32, device=dev),
    }
    if mode == _lib.AAL_VP_EAL:
        out["xstar"] = torch.empty(N, K, dtype=torch.int32, device=dev)
    st = _lib.lib().aal_vp_window_scan(_ptr(row), _ptr(acc_all) if R else None, R, N, K, int(mode),
                                       float(temp_draft), _ptr(grad_scale), _ptr(out["loss"]), _ptr(out["E"]),
                                       _ptr(out["accept"]), _ptr(out.get("xstar")), _stream(dev, stream))
    _lib.check(st, "aal_vp_window_scan")
    return out


def aal_vp_sequence_scan(row: torch.Tensor, acc_all: torch.Tensor | None, B: int, S: int, K: int, mode: int,
                         temp_draft: float = 1.0, *, grad_scale: torch.Tensor | None = None, stream=None) -> dict:
    """Step 4 for B sequences of S positions with windows of K sliding by one
    (rows updated in place).  Returns loss [1], E [B*(S-K+1)], accept [B, S]
    and, in EAL mode, xstar [B, S]."""
    _records(row, _lib.VP_ROW_BYTES, "row", 1)
    if row.shape[0] != B * S:
        raise ValueError("row must hold B*S records")
    dev = row.device
    R = 0
    if mode == _lib.AAL_VP_WTV:
        if acc_all is None:
            raise ValueError("acc_all is required in WTV mode")
        _records(acc_all, _lib.VP_ACC_BYTES, "acc_all", 2)
        if acc_all.shape[1] != B * S:
            raise ValueError("acc_all must be [R, B*S, 8]")
        R = acc_all.shape[0]
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.device != dev):
        raise TypeError("grad_scale must be a float32 device tensor")
    out = {
        "loss": torch.empty(1, dtype=torch.float32, device=dev),
        "E": torch.empty(B * max(0, S - K + 1), dtype=torch.float32, device=dev),
        "accept": torch.empty(B, S, dtype=torch.float32, device=dev),
    }
    if mode == _lib.AAL_VP_EAL:
        out["xstar"] = torch.empty(B, S, dtype=torch.int32, device=dev)
    st = _lib.lib().aal_vp_sequence_scan(_ptr(row), _ptr(acc_all) if R else None, R, B, S, K, int(mode),
                                         float(temp_draft), _ptr(grad_scale), _ptr(out["loss"]), _ptr(out["E"]),
                                         _ptr(out["accept"]), _ptr(out.get("xstar")), _stream(dev, stream))
    _lib.check(st, "aal_vp_sequence_scan")
    return out


def aal_vp_grad(z_draft: torch.Tensor, z_target: torch.Tensor | None, row: torch.Tensor, v0: int, mode: int,
                temp_draft: float = 1.0, temp_target: float = 1.0, *, grad_dtype: torch.dtype | None = None,
                stream=None) -> torch.Tensor:
    """Step 5: the slice [v0, v0 + V_slice) of dloss/dz_draft.  Returns [rows, V_slice]."""
    rows, vs, dev = _vp_slice(z_draft, z_target, need_target=(mode == _lib.AAL_VP_WTV))
    _records(row, _lib.VP_ROW_BYTES, "row", 1)
    if row.shape[0] != rows:
        raise ValueError("row must hold one record per logit row")
    g = torch.empty(rows, vs, dtype=grad_dtype or z_draft.dtype, device=dev)
    st = _lib.lib().aal_vp_grad(_ptr(z_draft), _ptr(z_target), _dtype_code(z_draft.dtype), rows, vs, int(v0),
                                int(mode), float(temp_draft), float(temp_target), _ptr(row), _ptr(g),
                                _dtype_code(g.dtype), _stream(dev, stream))
    _lib.check(st, "aal_vp_grad")
    return g


# ----------------------------------------------------------------------------
# Training against a target's top logits, and the processing of logits.

def _guard(device, stream):
    """Allocations and launches of a call: on the device of its tensors and in the stream's own pool."""
    if stream is not None:
        return torch.cuda.stream(stream)
    if device.index != torch.cuda.current_device():
        return torch.cuda.device(device)
    return contextlib.nullcontext()


def _raw_stream(device, stream) -> int:
    """The handle of `stream`, or of the device's current one (torch.cuda.current_stream builds an
    object for it, 2 us of a call that takes 10)."""
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(device.index)


def _device_array(t, name: str, dtype, numel: int | None, device):
    if t.dtype != dtype or t.device != device or not t.is_contiguous() or (numel is not None and t.numel() != numel):
        size = "" if numel is None else f" of {numel} entries"
        raise ValueError(f"{name} must be a contiguous {dtype} tensor{size} on {device}")


def _check_rows(z: torch.Tensor, name: str):
    if z.dim() < 1 or z.numel() == 0:
        raise ValueError(f"{name} must be [..., V] with at least one row")
    if not z.is_cuda or not z.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    V = z.shape[-1]
    return z.numel() // V, V


def aal_topk_logits(z: torch.Tensor, k: int, temperature: float = 1.0, *, rest: bool = True, stream=None) -> dict:
    """The k largest logits of each row of z [..., V] (larger first, the lower
    id first among equal ones) and the log-sum-exp of all others at
    `temperature`: what a data set keeps of a target's logits.

    Returns a dict: logits [..., k] of z's dtype, ids [..., k] int32 and rest
    [...] float32 (None with rest=False)."""
    rows, V = _check_rows(z, "z")
    code, dev, lead = _dtype_code(z.dtype), z.device, z.shape[:-1]
    if not 1 <= k <= min(V, AAL_TOPK_MAX):
        raise ValueError(f"k must be in [1, min(V, {AAL_TOPK_MAX})]; got {k}")
    with _guard(dev, stream):
        out = {
            "logits": torch.empty(*lead, k, dtype=z.dtype, device=dev),
            "ids": torch.empty(*lead, k, dtype=torch.int32, device=dev),
            "rest": torch.empty(lead, dtype=torch.float32, device=dev) if rest else None,
        }
        st = _lib.lib().aal_topk_logits(_ptr(z), code, rows, V, int(k), float(temperature), _ptr(out["logits"]),
                                        _ptr(out["ids"]), _ptr(out["rest"]), _raw_stream(dev, stream))
    _lib.check(st, "aal_topk_logits")
    return out


def aal_topk_loss_workspace_bytes(layout: int, B: int, S: int, K: int) -> int:
    return int(_lib.lib().aal_topk_loss_workspace_bytes(int(layout), int(B), int(S), int(K)))


def aal_topk_loss_fwd_bwd(z_draft: torch.Tensor, top_logits: torch.Tensor, top_ids: torch.Tensor, K: int, *,
                          rest: torch.Tensor | None = None, weights=(0.0, 0.0, 0.0, 0.0), temp_draft: float = 1.0,
                          temp_target: float = 1.0, layout: int = AAL_LAYOUT_WINDOWS, grad: bool = True,
                          grad_dtype: torch.dtype | None = None, grad_scale: torch.Tensor | None = None,
                          flags: int = 0, outputs: bool = True, ws: torch.Tensor | None = None, stream=None) -> dict:
    """The objectives of aal_loss_fwd_bwd (weights = (wtv, eal, kl, tv)) with
    the target known by its top logits, forward + backward.

    z_draft: [N, K, V] (windows layout) or [B, S, V] (sequences).  top_logits
    [N or B, K or S, k] and int32 top_ids of that shape: each row's list, as
    from aal_topk_logits; an entry with an id outside [0, V) or a logit of
    -inf is no part of it.  rest: [N or B, K or S] float32, the log-sum-exp of
    the target's other logits at temp_target, counted as one more entry; None:
    the list is renormalised.  A row without any target gets no gradient.

    Returns the dict of aal_loss_fwd_bwd: loss [1], terms [4], E_tv [W],
    E_eal [W], accept_tv [R], accept_eal [R], xstar [R] int32, grad."""
    if z_draft.dim() != 3:
        raise ValueError("z_draft must be a contiguous [B, S or K, V] device tensor")
    R, V = _check_rows(z_draft, "z_draft")
    B, S = z_draft.shape[:2]
    dev = z_draft.device
    if layout == AAL_LAYOUT_WINDOWS and S != K:
        raise ValueError("windows layout needs logits of shape [N, K, V]")
    if top_logits.dim() != 3 or top_logits.shape[:2] != z_draft.shape[:2]:
        raise ValueError("top_logits must be [B, S or K, k]")
    k = top_logits.shape[-1]
    if not 1 <= k <= min(V, AAL_TOPK_MAX):
        raise ValueError(f"lists must have 1 to min(V, {AAL_TOPK_MAX}) entries; got {k}")
    _device_array(top_logits, "top_logits", top_logits.dtype, R * k, dev)
    if top_ids.shape != top_logits.shape:
        raise ValueError("top_ids must have the shape of top_logits")
    _device_array(top_ids, "top_ids", torch.int32, R * k, dev)
    if rest is not None:
        _device_array(rest, "rest", torch.float32, R, dev)
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.device != dev):
        raise TypeError("grad_scale must be a float32 device tensor")
    if grad_scale is not None and grad_scale.numel() == 0:
        raise ValueError("grad_scale must have an element")
    if ws is not None and (ws.device != dev or not ws.is_contiguous()):
        raise ValueError(f"ws must be a contiguous tensor on {dev}")
    code, top_code = _dtype_code(z_draft.dtype), _dtype_code(top_logits.dtype)
    gcode = _dtype_code(grad_dtype or z_draft.dtype) if grad else AAL_F32
    W = B if layout == AAL_LAYOUT_WINDOWS else B * max(0, S - K + 1)
    with _guard(dev, stream):
        # the small outputs are pieces of one allocation (seven of them take 9 us)
        sizes = (1, 4, W, W, R, R, R) if outputs else (1, 4, 0, 0, 0, 0, 0)
        parts = torch.empty(sum(sizes), dtype=torch.float32, device=dev).split_with_sizes(sizes)
        out = dict(zip(("loss", "terms", "E_tv", "E_eal", "accept_tv", "accept_eal", "xstar"), parts))
        if outputs:
            out["xstar"] = out["xstar"].view(torch.int32)
        else:
            out.update(E_tv=None, E_eal=None, accept_tv=None, accept_eal=None, xstar=None)
        out["grad"] = torch.empty(B, S, V, dtype=grad_dtype or z_draft.dtype, device=dev) if grad else None
        if ws is None:
            ws = torch.empty(aal_topk_loss_workspace_bytes(layout, B, S, K), dtype=torch.uint8, device=dev)
        st = _lib.lib().aal_topk_loss_fwd_bwd(
            _ptr(z_draft), code, _ptr(top_logits), top_code, _ptr(top_ids), _ptr(rest), int(layout), B, S, int(K), V, k,
            float(temp_draft), float(temp_target), _lib.LossWeights(*(float(x) for x in weights)), _ptr(out["loss"]),
            _ptr(out["terms"]), _ptr(out["E_tv"]) if W and outputs else None,
            _ptr(out["E_eal"]) if W and outputs else None, _ptr(out["accept_tv"]), _ptr(out["accept_eal"]),
            _ptr(out["xstar"]), _ptr(out["grad"]), gcode, _ptr(grad_scale), int(flags), _ptr(ws), ws.numel(),
            _raw_stream(dev, stream))
    _lib.check(st, "aal_topk_loss_fwd_bwd")
    return out


def _logits_rules(rows, V, dev, tokens, hist_start, hist_len, prompt_len, repetition, frequency, presence,
                  bias_offsets, bias_ids, bias_values, mask, mask_row) -> _lib.LogitsRules:
    r = _lib.LogitsRules()
    history = (hist_start, hist_len, prompt_len, repetition, frequency, presence)
    if tokens is None:
        if any(t is not None for t in history):
            raise ValueError("penalties need tokens")
    else:
        if hist_start is None or hist_len is None:
            raise ValueError("tokens need hist_start and hist_len")
        _device_array(tokens, "tokens", torch.int32, None, dev)
        for t, name, dtype in zip(history, ("hist_start", "hist_len", "prompt_len", "repetition", "frequency",
                                            "presence"),
                                  (torch.int64, torch.int32, torch.int32) + (torch.float32,) * 3):
            if t is not None:
                _device_array(t, name, dtype, rows, dev)
        if tokens.numel():  # without a token every history is empty
            r.tokens, r.n_tokens, r.hist_start, r.hist_len = _ptr(tokens), tokens.numel(), _ptr(hist_start), _ptr(hist_len)
            r.prompt_len, r.repetition = _ptr(prompt_len), _ptr(repetition)
            r.frequency, r.presence = _ptr(frequency), _ptr(presence)
    if bias_offsets is None:
        if bias_ids is not None or bias_values is not None:
            raise ValueError("biases need bias_offsets")
    else:
        if bias_ids is None or bias_values is None:
            raise ValueError("bias_offsets need bias_ids and bias_values")
        _device_array(bias_offsets, "bias_offsets", torch.int64, rows + 1, dev)
        _device_array(bias_ids, "bias_ids", torch.int32, None, dev)
        _device_array(bias_values, "bias_values", torch.float32, bias_ids.numel(), dev)
        if bias_ids.numel():
            r.bias_offsets, r.bias_ids = _ptr(bias_offsets), _ptr(bias_ids)
            r.bias_values, r.n_bias = _ptr(bias_values), bias_ids.numel()
    if mask is None:
        if mask_row is not None:
            raise ValueError("mask_row needs mask")
    else:
        words = (V + 31) // 32
        if mask.dim() < 1 or mask.shape[-1] != words or mask.numel() == 0:
            raise ValueError(f"mask must be [..., {words}]: a bit for each entry of the vocabulary")
        _device_array(mask, "mask", torch.int32, None, dev)
        r.mask, r.n_masks = _ptr(mask), mask.numel() // words
        if mask_row is not None:
            _device_array(mask_row, "mask_row", torch.int32, rows, dev)
            r.mask_row = _ptr(mask_row)
        elif r.n_masks not in (1, rows):
            raise ValueError("without mask_row there must be one mask, or one for each row")
    return r


def aal_logits_process(z: torch.Tensor, *, tokens: torch.Tensor | None = None, hist_start: torch.Tensor | None = None,
                       hist_len: torch.Tensor | None = None, prompt_len: torch.Tensor | None = None,
                       repetition: torch.Tensor | None = None, frequency: torch.Tensor | None = None,
                       presence: torch.Tensor | None = None, bias_offsets: torch.Tensor | None = None,
                       bias_ids: torch.Tensor | None = None, bias_values: torch.Tensor | None = None,
                       mask: torch.Tensor | None = None, mask_row: torch.Tensor | None = None,
                       out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Biases, penalties for repeated tokens and grammar masks on the rows of
    z [..., V], in that order; blocked entries become -inf.

    tokens: int32, the histories of all rows; row r's is the hist_len[r]
    (int32) tokens from hist_start[r] (int64) on, the first prompt_len[r]
    (int32; None: none) of them the prompt.  repetition, frequency, presence:
    float32 per row, or None (1, 0, 0).  bias_offsets int64 [rows + 1],
    bias_ids int32, bias_values float32: the rows' biases one after the other.
    mask: int32 [..., ceil(V / 32)], bit v % 32 of word v / 32 allows entry v;
    mask_row: int32 per row, -1 for none (None: the one mask, or one per row).
    out: where the result goes (z itself for in place), or None.

    Returns out, [..., V] of z's dtype."""
    rows, V = _check_rows(z, "z")
    code, dev = _dtype_code(z.dtype), z.device
    rules = _logits_rules(rows, V, dev, tokens, hist_start, hist_len, prompt_len, repetition, frequency, presence,
                          bias_offsets, bias_ids, bias_values, mask, mask_row)
    if out is not None:
        if out.shape != z.shape:
            raise ValueError("out must have the shape of z")
        _device_array(out, "out", z.dtype, z.numel(), dev)
    with _guard(dev, stream):
        if out is None:
            out = torch.empty_like(z)
        st = _lib.lib().aal_logits_process(_ptr(z), code, rows, V, C.byref(rules), _ptr(out), _raw_stream(dev, stream))
    _lib.check(st, "aal_logits_process")
    return out


def aal_logits_process_bwd(grad_out: torch.Tensor, z: torch.Tensor, *, tokens: torch.Tensor | None = None,
                           hist_start: torch.Tensor | None = None, hist_len: torch.Tensor | None = None,
                           prompt_len: torch.Tensor | None = None, repetition: torch.Tensor | None = None,
                           frequency: torch.Tensor | None = None, presence: torch.Tensor | None = None,
                           bias_offsets: torch.Tensor | None = None, bias_ids: torch.Tensor | None = None,
                           bias_values: torch.Tensor | None = None, mask: torch.Tensor | None = None,
                           mask_row: torch.Tensor | None = None, grad_z: torch.Tensor | None = None,
                           stream=None) -> torch.Tensor:
    """The gradient through aal_logits_process: from grad_out (with respect to
    its result) to the gradient with respect to z, the logits that went in.
    The rules are those of that call.  grad_z: where the gradient goes
    (grad_out itself for in place), or None.

    Returns grad_z, of grad_out's shape and dtype."""
    rows, V = _check_rows(z, "z")
    code, gcode, dev = _dtype_code(z.dtype), _dtype_code(grad_out.dtype), z.device
    if grad_out.shape != z.shape:
        raise ValueError("grad_out must have the shape of z")
    _device_array(grad_out, "grad_out", grad_out.dtype, z.numel(), dev)
    rules = _logits_rules(rows, V, dev, tokens, hist_start, hist_len, prompt_len, repetition, frequency, presence,
                          bias_offsets, bias_ids, bias_values, mask, mask_row)
    if grad_z is not None:
        if grad_z.shape != z.shape:
            raise ValueError("grad_z must have the shape of z")
        _device_array(grad_z, "grad_z", grad_out.dtype, z.numel(), dev)
    with _guard(dev, stream):
        if grad_z is None:
            grad_z = torch.empty_like(grad_out)
        st = _lib.lib().aal_logits_process_bwd(_ptr(grad_out), gcode, _ptr(z), code, rows, V, C.byref(rules),
                                               _ptr(grad_z), _raw_stream(dev, stream))
    _lib.check(st, "aal_logits_process_bwd")
    return grad_z


# ----------------------------------------------------------------------------
# A language-model head in 8-bit floating point.

def _code(table: dict, t: torch.dtype, name: str) -> int:
    if t not in table:
        raise TypeError(f"unsupported {name} {t}; use one of {', '.join(str(k) for k in table)}")
    return table[t]


def _pitch(n: int) -> int:
    return (n + 15) // 16 * 16


def aal_fp8_quantize(x: torch.Tensor, *, block_rows: int = 1, rows: bool = True, columns: bool = False,
                     dtype: torch.dtype = torch.float8_e4m3fn, scale_dtype: torch.dtype = torch.float32,
                     stream=None) -> dict:
    """x [R, C] in 8-bit floating point, over a power of two for each block of
    block_rows x 128 (block_rows 1 or 128): the least that brings the block's
    largest finite value into the format's range, 1 for a block of zeros.

    x: bf16 or fp32, its columns contiguous, its rows at any distance.  dtype: float8_e4m3fn or float8_e5m2;
    scale_dtype: float32 or float8_e8m0fnu.  rows: quantise x, its blocks along the columns; columns:
    quantise x transposed, its blocks along x's rows (both in one pass over x).

    Returns a dict: q [R, C] and scale [ceil(R / block_rows), ceil(C / 128)], qt [C, R] and
    scale_t [ceil(C / block_rows), ceil(R / 128)] (None where not asked for).  q and qt are views
    whose rows start at multiples of 16 bytes, as aal_fp8_matmul takes them."""
    if x.dim() != 2 or x.numel() == 0:
        raise ValueError("x must be [R, C] with at least one entry")
    R, Cn = x.shape
    if not x.is_cuda or (Cn > 1 and x.stride(1) != 1) or (R > 1 and x.stride(0) < Cn):
        raise ValueError("x must be a device tensor of contiguous rows")
    if not (rows or columns):
        raise ValueError("rows or columns must be asked for")
    if block_rows not in (1, AAL_FP8_BLOCK):
        raise ValueError(f"block_rows must be 1 or {AAL_FP8_BLOCK}")
    code, fmt, st = _dtype_code(x.dtype), _code(_FP8, dtype, "dtype"), _code(_SCALE, scale_dtype, "scale_dtype")
    dev = x.device
    out = {"q": None, "scale": None, "qt": None, "scale_t": None}
    with _guard(dev, stream):
        for want, q, s, n, m in ((rows, "q", "scale", R, Cn), (columns, "qt", "scale_t", Cn, R)):
            if want:
                out[q] = torch.empty(n, _pitch(m), dtype=dtype, device=dev)
                out[s] = torch.empty((m + AAL_FP8_BLOCK - 1) // AAL_FP8_BLOCK, (n + block_rows - 1) // block_rows,
                                     dtype=scale_dtype, device=dev)
        st = _lib.lib().aal_fp8_quantize(_ptr(x), code, R, Cn, x.stride(0) if R > 1 else Cn, fmt, st, int(block_rows),
                                         _ptr(out["q"]), _pitch(Cn), _ptr(out["scale"]), _ptr(out["qt"]), _pitch(R),
                                         _ptr(out["scale_t"]), _raw_stream(dev, stream))
    _lib.check(st, "aal_fp8_quantize")
    for want, q, s, m in ((rows, "q", "scale", Cn), (columns, "qt", "scale_t", R)):
        if want:
            out[s] = out[s].t()
            if m % 16:
                out[q] = out[q][:, :m]
    return out


def _fp8_operand(v: torch.Tensor, s: torch.Tensor, name: str, dev) -> tuple:
    if v.dim() != 2 or v.numel() == 0 or s.dim() != 2:
        raise ValueError(f"{name} must be [rows, K] with a 2-d scale")
    R, K = v.shape
    if not v.is_cuda or v.device != dev or s.device != dev:
        raise ValueError(f"{name} and its scale must be on one device with the others")
    ld = v.stride(0) if R > 1 else _pitch(K)
    if (K > 1 and v.stride(1) != 1) or ld < K or ld % 16 or v.data_ptr() % 16:
        raise ValueError(f"{name}: values must be contiguous in a row, rows at multiples of 16 bytes")
    if v.untyped_storage().nbytes() - v.storage_offset() < R * ld:
        raise ValueError(f"{name}: the last row's memory must reach to its full stride")
    blocks = (K + AAL_FP8_BLOCK - 1) // AAL_FP8_BLOCK
    square = (R + AAL_FP8_BLOCK - 1) // AAL_FP8_BLOCK
    if s.shape[1] != blocks or s.shape[0] not in (R, square):
        raise ValueError(f"{name}: its scale must be [{R} or {square}, {blocks}]; got {tuple(s.shape)}")
    at, scale, (row, block) = v.data_ptr(), s.data_ptr(), s.stride()
    o = _lib.Fp8Operand(at, scale, ld, row, block, _code(_FP8, v.dtype, "dtype"), _code(_SCALE, s.dtype, "scale dtype"),
                        1 if s.shape[0] == R else AAL_FP8_BLOCK)
    # and the memory that it is, values and scale
    return o, ((at, at + R * ld), (scale, scale + s.element_size() * (1 + (s.shape[0] - 1) * row + (blocks - 1) * block)))


def _check_apart(at: int, end: int, read: tuple):
    for other, other_end in read:
        if at < other_end and other < end:
            raise ValueError("out and ws must share no memory with each other, an operand or its scale")


def aal_fp8_matmul(a: torch.Tensor, a_scale: torch.Tensor, b: torch.Tensor, b_scale: torch.Tensor, *,
                   out_dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None,
                   ws: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """a [M, K] times the transpose of b [N, K], 8-bit values with a scale for
    each block of 128 along K and of 1 or 128 rows (which of them, the scale's
    shape tells): a_scale [M or ceil(M / 128), ceil(K / 128)], b_scale alike, both
    float32 or both float8_e8m0fnu, any strides.  Values: float8_e4m3fn or float8_e5m2, rows at multiples
    of 16 bytes (as aal_fp8_quantize makes them).  M and N up to 2^28, M N below 2^37, K and the rows'
    distances below 2^24.  out, if given, and ws share no memory with the operands.

    out_dtype fp32: sums in fp32.  bf16: sums of 8-bit matrix instructions, which cut each eight
    neighbours' products below 2^-13 of the largest: off by up to 7 2^-13 of sum |a b| with the scales where large
    products cancel (1.5e-5 of it, root mean square, for random values), then rounded to bf16.

    Returns out, [M, N]."""
    dev = a.device
    (oa, read_a), (ob, read_b) = _fp8_operand(a, a_scale, "a", dev), _fp8_operand(b, b_scale, "b", dev)
    (M, K), N = a.shape, b.shape[0]
    if b.shape[1] != K:
        raise ValueError(f"a and b must agree in K; got {K} and {b.shape[1]}")
    if oa.scale_type != ob.scale_type:
        raise TypeError("a_scale and b_scale must be of one dtype")
    if out is not None:
        if out.shape != (M, N):
            raise ValueError(f"out must be [{M}, {N}]")
        _device_array(out, "out", out.dtype, M * N, dev)
        out_dtype = out.dtype
    code = _dtype_code(out_dtype)
    need = aal_fp8_matmul_workspace_bytes(M, N, K)
    if ws is not None and (ws.device != dev or not ws.is_contiguous()):
        raise ValueError(f"ws must be a contiguous tensor on {dev}")
    if out is not None or ws is not None:
        read = (*read_a, *read_b)
        if ws is not None:
            at, end = ws.data_ptr(), ws.data_ptr() + ws.nbytes
            _check_apart(at, end, read)
            read += ((at, end),)
        if out is not None:
            _check_apart(out.data_ptr(), out.data_ptr() + out.nbytes, read)
    with _guard(dev, stream):
        if out is None:
            out = torch.empty(M, N, dtype=out_dtype, device=dev)
        if ws is None and need:
            ws = torch.empty(need, dtype=torch.uint8, device=dev)
        st = _lib.lib().aal_fp8_matmul(C.byref(oa), C.byref(ob), M, N, K, _ptr(out), code, _ptr(ws),
                                       0 if ws is None else ws.numel() * ws.element_size(), _raw_stream(dev, stream))
    _lib.check(st, "aal_fp8_matmul")
    return out


@functools.lru_cache(maxsize=4096)
def aal_fp8_matmul_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(_lib.lib().aal_fp8_matmul_workspace_bytes(int(M), int(N), int(K)))


def _matrix(t: torch.Tensor, stream) -> torch.Tensor:
    """t as rows of its last dimension, contiguous: a copy of it, where there has to be one, is the call's own work,
    on its stream."""
    if not t.is_cuda:
        raise ValueError("tensors must be on a device")
    with _guard(t.device, stream):
        flat = t.reshape(-1, t.shape[-1])
        if flat.shape[1] > 1 and flat.stride(1) != 1 or flat.shape[0] > 1 and flat.stride(0) < flat.shape[1]:
            flat = flat.contiguous()
    return flat


def _blocks(n: int) -> int:
    return (n + AAL_FP8_BLOCK - 1) // AAL_FP8_BLOCK


def _check_head(head: dict, *names: str):
    for name in names:
        if head.get(name) is None:
            raise ValueError(f"head must hold {name}: aal_fp8_quantize(W, block_rows=128, columns=True)")


def aal_head_logits(x: torch.Tensor, head: dict, *, out_dtype: torch.dtype | None = None, stream=None) -> torch.Tensor:
    """Logits of hidden states x [..., D] (bf16 or fp32) through a head whose
    weights [V, D] are held in 8 bits: head["q"] and head["scale"], as from
    aal_fp8_quantize(W, block_rows=128, columns=True).  x is quantised here, in
    blocks of 1 x 128, to e4m3 with scales of the head's type.

    Returns [..., V] of out_dtype (x's dtype if None), as exact as aal_fp8_matmul's results of it are."""
    _check_head(head, "q", "scale")
    D = x.shape[-1] if x.dim() else 0
    if x.dim() < 1 or x.numel() == 0 or head["q"].shape[-1] != D:
        raise ValueError(f"x must be [..., {head['q'].shape[-1]}] with at least one row")
    r = aal_fp8_quantize(_matrix(x, stream), scale_dtype=head["scale"].dtype, stream=stream)
    z = aal_fp8_matmul(r["q"], r["scale"], head["q"], head["scale"], out_dtype=out_dtype or x.dtype, stream=stream)
    return z.view(*x.shape[:-1], z.shape[1])


def aal_head_logits_bwd(grad: torch.Tensor, x: torch.Tensor, head: dict, *, x_grad: bool = True,
                        weight_grad: bool = True, weight_dtype: torch.dtype = torch.float32, stream=None) -> dict:
    """The gradients through aal_head_logits, from grad [..., V] (with respect
    to the logits) and its x [..., D]: both products in 8 bits as well, grad and
    x quantised to e4m3 in blocks of 128 along the dimension that is summed over
    (x's gradient: V, against head["qt"] and head["scale_t"]; the weights': the rows).

    Returns a dict: grad_x [..., D] of x's dtype and grad_w [V, D] of
    weight_dtype (None where not asked for), as exact as aal_fp8_matmul's results of those are."""
    if not (x_grad or weight_grad):
        raise ValueError("x_grad or weight_grad must be asked for")
    _check_head(head, *(("qt", "scale_t") if x_grad else ("scale",)))
    if x.dim() < 1 or x.numel() == 0 or grad.dim() < 1 or grad.shape[:-1] != x.shape[:-1] or grad.numel() == 0:
        raise ValueError("grad must be [..., V] and x [..., D] of the same rows, one at least")
    D, V = x.shape[-1], grad.shape[-1]
    for values, scale, rows, cols in (("q", "scale", V, D), ("qt", "scale_t", D, V)):
        v, s = head.get(values), head.get(scale)
        if v is not None and tuple(v.shape) != (rows, cols):
            raise ValueError(f"grad and x of {V} and {D} columns do not fit a head whose {values} is {tuple(v.shape)}")
        if s is not None and (s.shape[0] not in (rows, _blocks(rows)) or s.shape[1] != _blocks(cols)):
            raise ValueError(f"grad and x of {V} and {D} columns do not fit a head whose {scale} is {tuple(s.shape)}")
    scale = (head["scale_t"] if x_grad else head["scale"]).dtype
    g = aal_fp8_quantize(_matrix(grad, stream), rows=x_grad, columns=weight_grad, scale_dtype=scale, stream=stream)
    out = {"grad_x": None, "grad_w": None}
    if x_grad:
        out["grad_x"] = aal_fp8_matmul(g["q"], g["scale"], head["qt"], head["scale_t"], out_dtype=x.dtype,
                                       stream=stream).view(x.shape)
    if weight_grad:
        xt = aal_fp8_quantize(_matrix(x, stream), rows=False, columns=True, scale_dtype=scale, stream=stream)
        out["grad_w"] = aal_fp8_matmul(g["qt"], g["scale_t"], xt["qt"], xt["scale_t"], out_dtype=weight_dtype,
                                       stream=stream)
    return out


# ----------------------------------------------------------------------------
# Beam search.

@functools.lru_cache(maxsize=4096)
def aal_beam_select_workspace_bytes(dtype: torch.dtype, B: int, W: int, V: int, n: int) -> int:
    return int(_lib.lib().aal_beam_select_workspace_bytes(_dtype_code(dtype), int(B), int(W), int(V), int(n)))


def aal_beam_select(z: torch.Tensor, scores: torch.Tensor, n: int, *, temperature: float = 1.0,
                    finished: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                    length_penalty: float = 0.0, eos: int = -1, pad: int = 0, ws: torch.Tensor | None = None,
                    stream=None) -> dict:
    """The n best continuations of each request's beams, over all its beams and
    the vocabulary.

    z [B, W, V]: logits (bf16 or fp32), W up to 64, V up to 2^18.  scores [B, W] float32: the beams' cumulative
    log-probabilities, -inf for one that is not to go on.  finished [B, W] bool: beams that have
    ended, each of which stands for itself with token pad and its own score.  lengths [B, W] int32: tokens so
    far.  Candidates are ordered by (score + log softmax(z / temperature)) / (lengths + 1) **
    length_penalty; among equal ones the lower beam, the larger logit, the lower token come first.

    Returns a dict of [B, n]: scores and rank float32, parents and tokens int32, finished bool, lengths
    int32.  Where a request has fewer candidates: -inf, -inf, -1, pad, True, 0."""
    if z.dim() != 3 or z.numel() == 0 or not z.is_cuda or not z.is_contiguous():
        raise ValueError("z must be a contiguous [B, W, V] device tensor with at least one entry")
    B, W, V = z.shape
    code, dev = _dtype_code(z.dtype), z.device
    if W > AAL_BEAM_MAX:
        raise ValueError(f"at most {AAL_BEAM_MAX} beams; got {W}")
    if not 1 <= n <= min(AAL_BEAM_SELECT_MAX, W * V):
        raise ValueError(f"n must be in [1, min({AAL_BEAM_SELECT_MAX}, W * V)]; got {n}")
    for t, name, dtype in ((scores, "scores", torch.float32), (finished, "finished", torch.bool),
                           (lengths, "lengths", torch.int32)):
        if t is not None:
            if t.shape != (B, W):
                raise ValueError(f"{name} must be [{B}, {W}]")
            _device_array(t, name, dtype, B * W, dev)
    if ws is not None and (ws.device != dev or not ws.is_contiguous()):
        raise ValueError(f"ws must be a contiguous tensor on {dev}")
    with _guard(dev, stream):
        # the outputs of 32 bits are pieces of one allocation
        scores_, rank, parents, tokens, lengths_ = torch.empty((5, B, n), dtype=torch.int32, device=dev).unbind(0)
        out = {"scores": scores_.view(torch.float32), "rank": rank.view(torch.float32), "parents": parents,
               "tokens": tokens, "finished": torch.empty((B, n), dtype=torch.bool, device=dev), "lengths": lengths_}
        if ws is None:
            ws = torch.empty(aal_beam_select_workspace_bytes(z.dtype, B, W, V, n), dtype=torch.uint8, device=dev)
        o = _lib.BeamOut(*[t.data_ptr() for t in out.values()])
        st = _lib.lib().aal_beam_select(
            _ptr(z), code, B, W, V, int(n), float(temperature), _ptr(scores), _ptr(finished), _ptr(lengths),
            float(length_penalty), int(eos), int(pad), C.byref(o), _ptr(ws), ws.numel() * ws.element_size(),
            _raw_stream(dev, stream))
    _lib.check(st, "aal_beam_select")
    return out


@functools.lru_cache(maxsize=4096)
def _segments(shape: tuple, stride: tuple):
    """The memory of a tensor of that shape and those strides behind its first two dimensions: (segments,
    elements of one, elements from one to the next) and the elements that all of it spans, None if it is not that regular."""
    size = 1  # of the contiguous end
    dims = [(n, s) for n, s in zip(shape[2:], stride[2:]) if n != 1]
    while dims and dims[-1][1] == size:
        size *= dims.pop()[0]
    count, step = 1, 0
    for n, s in reversed(dims):
        if count == 1:
            count, step = n, s
        elif s == step * count:
            count *= n
        else:
            return None
    return count, size, step, 1 + sum((n - 1) * s for n, s in zip(shape, stride))


@functools.lru_cache(maxsize=4096)
def _apart(shape: tuple, stride: tuple) -> bool:
    """Whether no two entries share memory (dimensions nested by their strides)."""
    end = 1
    for step, n in sorted((s, n) for n, s in zip(shape, stride) if n > 1):
        if step < end:
            return False
        end += step * (n - 1)
    return True


def _meet(d: int, a: list, na: int, b: list, nb: int, budget: list | None = None) -> bool:
    """Whether two regular sets of bytes share one: pieces of na and nb bytes, at (stride, count)s that nest, the
    largest first, the second set's first byte d behind the first's.  Sets of different strides are looked through step
    by step; True as well where that takes more steps than budget, a list of one number, has left."""
    budget = [_STEPS] if budget is None else budget
    budget[0] -= 1
    if budget[0] < 0:
        return True
    end_a, end_b = (n + sum(s * (c - 1) for s, c in dims) for dims, n in ((a, na), (b, nb)))
    if d >= end_a or -d >= end_b:
        return False
    if not a and not b:
        return True
    if a and b and a[0][0] == b[0][0]:
        (s, ca), cb = a[0], b[0][1]
        rest_a, rest_b = end_a - s * (ca - 1), end_b - s * (cb - 1)
        steps = range(max(1 - ca, -((d + rest_b - 1) // s)), min(cb - 1, (rest_a - 1 - d) // s) + 1)
        return any(_meet(d + k * s, a[1:], na, b[1:], nb, budget) for k in steps)
    if not a or (b and b[0][0] > a[0][0]):
        return _meet(-d, b, nb, a, na, budget)
    s, ca = a[0]
    rest = end_a - s * (ca - 1)
    steps = range(max(0, -((rest - 1 - d) // s)), min(ca - 1, (d + end_b - 1) // s) + 1)
    return any(_meet(d - k * s, a[1:], na, b, nb, budget) for k in steps)


_STEPS = 1 << 14  # for two sets; some 20 ms


@functools.lru_cache(maxsize=4096)
def _nested(cut: tuple, lead: tuple) -> tuple:
    """The (stride, count)s of a state's pieces, the largest first."""
    return tuple(sorted(((s, c) for s, c in (*lead, (cut[2], cut[0])) if c > 1 and s), reverse=True))


def _runs(sets: list) -> list:
    """Sets (first byte, bytes to the last one's end, ...) in order of their first bytes, as runs of those whose ranges meet."""
    sets.sort(key=_first)
    runs, last = [], None
    for x in sets:
        if last is None or x[0] >= last:
            runs.append([])
            last = x[0]
        runs[-1].append(x)
        last = max(last, x[0] + x[1])
    return runs


def _apart_by_steps(sets: list) -> bool:
    """Whether regular sets of bytes, (first byte, bytes to the last one's end, (stride, count)s, ...), are seen to be apart by what
    is left of them in one step of the stride that they all have: views of one tensor are, in one sort a stride.  False
    where they are not, or may not be."""
    if len(sets) < 2:
        return True
    if not all(x[2] for x in sets) or len({x[2][0][0] for x in sets}) > 1:
        return False
    step, base, inner = sets[0][2][0][0], min(x[0] for x in sets), []
    for at, size, dims, *_ in sets:
        inner.append(((at - base) % step, size - step * (dims[0][1] - 1), dims[1:]))
    runs = _runs(inner)
    end = max(x[0] + x[1] for x in runs[-1])
    if end - runs[0][0][0] > step:  # the last of a step reach into the next one's first
        return False
    return all(_apart_by_steps(run) for run in runs)


def _check_memory(spans: list):
    """What is written shares no memory with anything else of a call.  spans: (first byte, bytes to the last one's
    end, whether it is written, (segments, bytes of one, bytes between them), (stride, count) of requests and of beams)."""
    spans.sort(key=_first)
    if all(x[0] + x[1] <= y[0] for x, y in zip(spans, spans[1:])):
        return
    for run in _runs([(x[0], x[1], _nested(x[3], x[4]), x[3][1], x[2]) for x in spans]):
        alike = {}  # by their largest stride
        for x in run:
            alike.setdefault(x[2][0][0] if x[2] else 0, []).append(x)
        groups = list(alike.values())
        pairs = [itertools.combinations(sets, 2) for sets in groups if not _apart_by_steps(sets)]
        pairs += [itertools.product(x, y) for x, y in itertools.combinations(groups, 2)]
        for x, y in itertools.chain.from_iterable(pairs):
            if (x[4] or y[4]) and _meet(y[0] - x[0], x[2], x[3], y[2], y[3]):
                raise ValueError("what is written must share no memory with another state or output, nor with parents")


_first = operator.itemgetter(0)


def aal_beam_reorder(states, parents: torch.Tensor, *, out=None, stream=None) -> list:
    """Each state's beams after a selection: state[b, j] becomes what
    state[b, parents[b, j]] was, for tensors [B, W, ...] of any dtype (caches,
    token histories, last states), all in one call.

    parents: [B, n] int32, as from aal_beam_select; a parent outside [0, W) leaves its slot as it
    was.  out: None, for in place (n = W; beams that keep their slot move nothing), or tensors
    [B, n, ...].  What is written shares no memory with another state or output, nor with parents (views of
    one memory at different strides are refused as well where it would take long to tell that they are
    apart).  Behind its first two dimensions a state may be any view that is contiguous pieces at one
    distance (state[:, :, :, t0:t1] of a [B, W, heads, length, dim] cache), and so may its output: the
    same pieces, or as a whole contiguous in one of the two.

    Returns out, or the states."""
    states = list(states)
    outs = states if out is None else list(out)
    if parents.dim() != 2 or parents.numel() == 0:
        raise ValueError("parents must be [B, n]")
    B, n = parents.shape
    dev = parents.device
    if not parents.is_cuda:
        raise ValueError("parents must be a device tensor")
    _device_array(parents, "parents", torch.int32, B * n, dev)
    if len(outs) != len(states):
        raise ValueError("out must have a tensor for each state")
    if not states:
        return outs
    W = states[0].shape[1] if states[0].dim() >= 2 else 0
    if not 1 <= n <= AAL_BEAM_SELECT_MAX or (out is None and (n != W or n > AAL_BEAM_MAX)):
        raise ValueError(f"n must be in [1, {AAL_BEAM_SELECT_MAX}], in place W and at most {AAL_BEAM_MAX}; got {n}")
    table, spans = [], []  # what aal_beam_state_t holds, one state after the other
    for s, o in zip(states, outs):
        shape, stride = tuple(s.shape), s.stride()
        if len(shape) < 2 or shape[0] != B or shape[1] != W or s.device != dev:
            raise ValueError(f"states must be [{B}, {W}, ...] on {dev}; got {shape} on {s.device}")
        cut = _segments(shape, stride)
        if cut is None:
            raise ValueError("a state must be contiguous pieces at one distance behind its first two dimensions")
        e = s.element_size()
        count, size, step, span = cut
        moves = count and size
        at, request, beam, step, piece = s.data_ptr(), stride[0] * e, stride[1] * e, step * e, size * e
        if moves:
            spans.append((at, span * e, out is None, (count, piece, step), ((request, B), (beam, W))))
        if out is None:
            row = (at, 0, request, beam, step, 0, 0, 0, count, piece)
        else:
            if o.shape != (B, n, *shape[2:]) or o.dtype != s.dtype or o.device != dev:
                raise ValueError(f"out must be [{B}, {n}, ...] of the states' shapes and dtypes on {dev}")
            shape, stride = tuple(o.shape), o.stride()
            to = _segments(shape, stride)
            if to is None or (to[0] != count and 1 not in (to[0], count)):
                raise ValueError("an output must be contiguous as a whole or the same contiguous pieces as its state, unless that is")
            to_at, to_request, to_beam, to_step, to_piece = o.data_ptr(), stride[0] * e, stride[1] * e, to[2] * e, to[1] * e
            if moves:
                spans.append((to_at, to[3] * e, True, (to[0], to_piece, to_step), ((to_request, B), (to_beam, n))))
            # what is contiguous as a whole goes by the pieces of the other
            if to[0] < count:
                to_step = piece
            elif to[0] > count:
                count, piece, step = to[0], to_piece, to_piece
            row = (at, to_at, request, beam, step, to_request, to_beam, to_step, count, piece)
        if not _apart(shape, stride):
            raise ValueError("the entries of what is written must not share memory")
        if moves:
            table += row
    if spans:
        spans.append((parents.data_ptr(), 4 * B * n, False, (1, 4 * B * n, 0), ()))
        _check_memory(spans)
    with _guard(dev, stream):
        st = _lib.lib().aal_beam_reorder(struct.pack(f"{len(table)}q", *table), len(table) // 10, B, W, n, _ptr(parents),
                                         _raw_stream(dev, stream))
    _lib.check(st, "aal_beam_reorder")
    return outs


def aal_stream_probe(srcs, dst: torch.Tensor | None = None, flag: torch.Tensor | None = None, stream=None):
    """Measurement aid: stream 1-3 equally sized device tensors (16-byte
    nontemporal loads) and, with dst, write their 32-bit wrapping sum there;
    without dst, flag ([1] int32/uint32) is set only where a sum is all ones.
    Enqueues and returns; time it with events on `stream`."""
    srcs = list(srcs)
    if not 1 <= len(srcs) <= 3:
        raise ValueError("one to three sources")
    nbytes = srcs[0].numel() * srcs[0].element_size()
    for t in srcs + ([dst] if dst is not None else []):
        if not t.is_cuda or not t.is_contiguous() or t.numel() * t.element_size() != nbytes:
            raise ValueError("sources and dst must be contiguous device tensors of one size")
    if dst is None and flag is None:
        raise ValueError("flag is required without dst")
    ptrs = [_ptr(t) for t in srcs] + [None] * (3 - len(srcs))
    st = _lib.lib().aal_stream_probe(ptrs[0], ptrs[1], ptrs[2], _ptr(dst), nbytes, _ptr(flag),
                                     _stream(srcs[0].device, stream))
    _lib.check(st, "aal_stream_probe")
