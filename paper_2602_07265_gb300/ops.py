"""ctypes binding of the operators of include/xshare_ops.h: expert gating from
router logits, float8 quantisation, block-scaled float8 products and float8
experts.

Argument marshalling only, as in `xshare`: tensors are checked for device,
type, contiguity and size, a non-zero return code raises `XShareError`.  Outputs
and workspaces are the caller's.  The operators serve; none has a backward pass.
"""

from __future__ import annotations

import ctypes
from typing import Optional

import torch

from .xshare import LIB, STATS_WORDS, XShareError, _ptr as _checked_ptr, _stream as _any_stream

FP8 = torch.float8_e4m3fn
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
SCORING = {"softmax": 0, "sigmoid": 1}


class GateParams(ctypes.Structure):
    """xs_gate_params."""
    _fields_ = [("scoring", ctypes.c_int32), ("n_groups", ctypes.c_int32), ("top_groups", ctypes.c_int32),
                ("group_top", ctypes.c_int32), ("renorm", ctypes.c_int32), ("scale", ctypes.c_float)]


def gate_params(scoring: str = "softmax", n_groups: int = 1, top_groups: Optional[int] = None,
                group_top: int = 2, renorm: bool = True, scale: float = 1.0) -> GateParams:
    """`scoring`: "softmax" or "sigmoid"; `top_groups` defaults to all groups."""
    if scoring not in SCORING:
        raise ValueError(f"scoring must be one of {sorted(SCORING)}, got {scoring!r}")
    return GateParams(SCORING[scoring], n_groups, n_groups if top_groups is None else top_groups, group_top,
                      int(renorm), scale)


class _Fp8ExpertsStruct(ctypes.Structure):
    """xs_fp8_experts."""
    _fields_ = [("gate", ctypes.c_void_p), ("up", ctypes.c_void_p), ("down", ctypes.c_void_p),
                ("gate_s", ctypes.c_void_p), ("up_s", ctypes.c_void_p), ("down_s", ctypes.c_void_p),
                ("n", ctypes.c_int32)]


def _declare() -> None:
    P, I, Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    for name, restype, args in (
            ("xshare_gate_workspace_size", Z, [I, I, I]),
            ("xshare_gate", I, [P, I, P, P, P, I, I, I, ctypes.POINTER(GateParams), P, P, P, P, P, P, P, Z, P]),
            ("xshare_quant_fp8_rows", I, [P, I, I, I, P, P, P]),
            ("xshare_quant_fp8_blocks", I, [P, I, I, I, I, P, P, P]),
            ("xshare_matmul_fp8_workspace_size", Z, [I, I, I, I]),
            ("xshare_matmul_fp8", I, [P, P, P, P, P, I, I, I, I, P, I, P, P, Z, P]),
            ("xshare_experts_fp8_workspace_size", Z, [I, I, I, I, I]),
            ("xshare_experts_fp8", I, [P, P, P, ctypes.POINTER(_Fp8ExpertsStruct), I, I, I, I, P, P, P, Z, P])):
        fn = getattr(LIB, name)
        fn.restype, fn.argtypes = restype, args


_declare()
_gate, _matmul, _experts = LIB.xshare_gate, LIB.xshare_matmul_fp8, LIB.xshare_experts_fp8


def _ptr(t: Optional[torch.Tensor], dtype, name: str, numel: Optional[int], device: int) -> Optional[int]:
    """t's device pointer.  These calls take a few microseconds, most of them here:
    a tensor that passes costs four attribute reads, the rest is for the error."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == device and t.is_contiguous() and (numel is None or t.numel() >= numel):
        return t.data_ptr()
    return _checked_ptr(t, dtype, name, numel)


def _current_device(t: torch.Tensor) -> int:
    if not t.is_cuda:
        raise ValueError("the operators take CUDA tensors")
    return torch.cuda.current_device()


def _stream(stream, device: int) -> Optional[int]:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device)
    return _any_stream(stream)


def _check(rc: int, where: str) -> None:
    if rc != 0:
        raise XShareError(rc, where)


def _type_of(t: torch.Tensor, name: str) -> int:
    code = DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return code


def _shaped(t: torch.Tensor, name: str, *shape: int) -> None:
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


def _ws(workspace: Optional[torch.Tensor], dev: int):
    """Pointer and size of a nullable workspace."""
    if workspace is None:
        return None, 0
    return _ptr(workspace, torch.uint8, "workspace", None, dev), workspace.numel()


def _ceil128(n: int) -> int:
    return (n + 127) // 128


def xshare_gate_workspace_size(B: int, N: int, k: int) -> int:
    """Bytes of workspace for expert_counts, expert_offsets and perm; 0 if invalid."""
    return int(LIB.xshare_gate_workspace_size(B, N, k))


def xshare_gate(logits: torch.Tensor, k: int, params: GateParams, topk_ids: torch.Tensor, topk_w: torch.Tensor,
                bias: Optional[torch.Tensor] = None, expert_mask: Optional[torch.Tensor] = None,
                token_mask: Optional[torch.Tensor] = None, scores_out: Optional[torch.Tensor] = None,
                expert_counts: Optional[torch.Tensor] = None, expert_offsets: Optional[torch.Tensor] = None,
                perm: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Routes tokens by their router logits [B, N] into topk_ids and topk_w [B, k] and scores_out
    [B, N]; see xshare_ops.h.  The buffers of one dimension may be longer than is needed."""
    B, N = logits.shape
    _shaped(topk_ids, "topk_ids", B, k)
    _shaped(topk_w, "topk_w", B, k)
    if scores_out is not None:
        _shaped(scores_out, "scores_out", B, N)
    dev = _current_device(logits)
    ws = ws_bytes = bias_p = emask_p = tmask_p = scores_p = counts_p = offsets_p = perm_p = None
    if workspace is not None:
        ws, ws_bytes = _ws(workspace, dev)
    if bias is not None:
        bias_p = _ptr(bias, torch.float32, "bias", N, dev)
    if expert_mask is not None:
        emask_p = _ptr(expert_mask, torch.uint8, "expert_mask", N, dev)
    if token_mask is not None:
        tmask_p = _ptr(token_mask, torch.uint8, "token_mask", B, dev)
    if scores_out is not None:
        scores_p = _ptr(scores_out, torch.float32, "scores_out", B * N, dev)
    if expert_counts is not None:
        counts_p = _ptr(expert_counts, torch.int32, "expert_counts", N, dev)
    if expert_offsets is not None:
        offsets_p = _ptr(expert_offsets, torch.int32, "expert_offsets", N + 1, dev)
    if perm is not None:
        perm_p = _ptr(perm, torch.int32, "perm", B * k, dev)
    rc = _gate(_ptr(logits, logits.dtype, "logits", None, dev), _type_of(logits, "logits"), bias_p, emask_p, tmask_p,
               B, N, k, params, _ptr(topk_ids, torch.int32, "topk_ids", B * k, dev),
               _ptr(topk_w, torch.float32, "topk_w", B * k, dev), scores_p, counts_p, offsets_p, perm_p, ws,
               ws_bytes or 0, _stream(stream, dev))
    if rc:
        _check(rc, "xshare_gate")


def xshare_quant_fp8_rows(x: torch.Tensor, q: torch.Tensor, scales: torch.Tensor, stream=None) -> None:
    """x [M, K] into q [M, K] e4m3 and scales [M, ceil(K / 128)]; see xshare_ops.h."""
    M, K = x.shape
    dev = _current_device(x)
    _shaped(q, "q", M, K)
    _shaped(scales, "scales", M, _ceil128(K))
    rc = LIB.xshare_quant_fp8_rows(_ptr(x, x.dtype, "x", None, dev), _type_of(x, "x"), M, K,
                                   _ptr(q, FP8, "q", None, dev), _ptr(scales, torch.float32, "scales", None, dev),
                                   _stream(stream, dev))
    _check(rc, "xshare_quant_fp8_rows")


def xshare_quant_fp8_blocks(x: torch.Tensor, q: torch.Tensor, scales: torch.Tensor, stream=None) -> None:
    """x [R, K] or [n, R, K] into q of its shape and scales [(n,) ceil(R / 128),
    ceil(K / 128)]; see xshare_ops.h."""
    lead = tuple(x.shape[:-2])
    if x.dim() not in (2, 3):
        raise ValueError(f"x must have two or three dimensions, got {list(x.shape)}")
    R, K = x.shape[-2:]
    dev = _current_device(x)
    _shaped(q, "q", *x.shape)
    _shaped(scales, "scales", *lead, _ceil128(R), _ceil128(K))
    rc = LIB.xshare_quant_fp8_blocks(_ptr(x, x.dtype, "x", None, dev), _type_of(x, "x"), lead[0] if lead else 1, R, K,
                                     _ptr(q, FP8, "q", None, dev),
                                     _ptr(scales, torch.float32, "scales", None, dev), _stream(stream, dev))
    _check(rc, "xshare_quant_fp8_blocks")


def xshare_matmul_fp8_workspace_size(M: int, N: int, K: int, E: int = 1) -> int:
    """Bytes of workspace of xshare_matmul_fp8; 0 if invalid."""
    return int(LIB.xshare_matmul_fp8_workspace_size(M, N, K, E))


def xshare_matmul_fp8(a: torch.Tensor, a_scale: torch.Tensor, b: torch.Tensor, b_scale: torch.Tensor,
                      y: torch.Tensor, workspace: torch.Tensor, offsets: Optional[torch.Tensor] = None,
                      stats: Optional[torch.Tensor] = None, stream=None) -> None:
    """y [M, N] = a [M, K] b^T for b [N, K] or [1, N, K]; with `offsets` [E + 1]
    rows offsets[e] .. offsets[e + 1] - 1 times b[e] of b [E, N, K]; see xshare_ops.h."""
    M, K = a.shape
    size = tuple(b.shape)
    if len(size) == 2:
        E, N, lead = 1, size[0], ()
    elif len(size) == 3:
        E, N, lead = size[0], size[1], size[:1]
    else:
        raise ValueError(f"b must be [N, K] or [E, N, K], got {list(size)}")
    dev = _current_device(a)
    kb = (K + 127) // 128
    if size[-1] != K:
        raise ValueError(f"b must be {[*size[:-1], K]}, got {list(size)}")
    _shaped(a_scale, "a_scale", M, kb)
    _shaped(b_scale, "b_scale", *lead, (N + 127) // 128, kb)
    _shaped(y, "y", M, N)
    if offsets is not None:
        _shaped(offsets, "offsets", E + 1)
    elif E != 1:
        raise ValueError(f"{E} matrices need offsets")
    ws, ws_bytes = _ws(workspace, dev)
    rc = _matmul(
        _ptr(a, FP8, "a", None, dev), _ptr(a_scale, torch.float32, "a_scale", None, dev), _ptr(b, FP8, "b", None, dev),
        _ptr(b_scale, torch.float32, "b_scale", None, dev),
        None if offsets is None else _ptr(offsets, torch.int32, "offsets", None, dev),
        M, N, K, E, _ptr(y, y.dtype, "y", None, dev), _type_of(y, "y"),
        None if stats is None else _ptr(stats, torch.int32, "stats", STATS_WORDS, dev), ws, ws_bytes, _stream(stream, dev))
    if rc:
        _check(rc, "xshare_matmul_fp8")


class Fp8Experts:
    """The weights of n float8 experts: values gate, up [n, F, d] and down [n, d, F]
    (float8_e4m3fn) and the scales of their 128 x 128 blocks, [n, F / 128, d / 128]
    and [n, d / 128, F / 128].  Keeps references; copies nothing."""

    def __init__(self, gate: torch.Tensor, gate_s: torch.Tensor, up: torch.Tensor, up_s: torch.Tensor,
                 down: torch.Tensor, down_s: torch.Tensor):
        n, F, d = gate.shape
        if d % 128 or F % 128:
            raise ValueError(f"d and F must be multiples of 128, got {d} and {F}")
        for t, s, name, rows, cols in ((gate, gate_s, "gate", F, d), (up, up_s, "up", F, d), (down, down_s, "down", d, F)):
            _shaped(t, name, n, rows, cols)
            _shaped(s, name + "_s", n, rows // 128, cols // 128)
        self.n, self.d, self.F = n, d, F
        self._parts = dict(gate=(gate, FP8), up=(up, FP8), down=(down, FP8), gate_s=(gate_s, torch.float32),
                           up_s=(up_s, torch.float32), down_s=(down_s, torch.float32))
        self._tensors = [t for t, _ in self._parts.values()]
        self._struct, self._ptrs, self._device = None, None, -1
        self.struct(_current_device(gate))

    @classmethod
    def quantise(cls, W_gate: torch.Tensor, W_up: torch.Tensor, W_down: torch.Tensor) -> "Fp8Experts":
        """From W_gate, W_up [n, F, d] and W_down [n, d, F] in float32, bfloat16 or
        float16 (once, when the weights are loaded), on the current stream, which the
        new tensors belong to."""
        parts = []
        for w in (W_gate, W_up, W_down):
            q = torch.empty(w.shape, dtype=FP8, device=w.device)
            s = torch.empty(w.shape[0], _ceil128(w.shape[1]), _ceil128(w.shape[2]), dtype=torch.float32, device=w.device)
            xshare_quant_fp8_blocks(w, q, s)
            parts += [q, s]
        return cls(*parts)

    def struct(self, device: int) -> _Fp8ExpertsStruct:
        """The C descriptor; made again where a tensor's storage has changed."""
        ptrs = [t.data_ptr() for t in self._tensors]
        if ptrs != self._ptrs or device != self._device:
            self._struct = _Fp8ExpertsStruct(n=self.n, **{name: _ptr(t, dtype, name, t.numel(), device)
                                                          for name, (t, dtype) in self._parts.items()})
            self._ptrs, self._device = ptrs, device
        return self._struct


def xshare_experts_fp8_workspace_size(B: int, N: int, k: int, d: int, F: int) -> int:
    """Bytes of workspace of xshare_experts_fp8 on N experts; 0 if invalid."""
    return int(LIB.xshare_experts_fp8_workspace_size(B, N, k, d, F))


def xshare_experts_fp8(x: torch.Tensor, topk_ids: torch.Tensor, topk_w: torch.Tensor, experts: Fp8Experts,
                       y: torch.Tensor, workspace: torch.Tensor, stats: Optional[torch.Tensor] = None,
                       stream=None) -> None:
    """The experts of a routed batch: x [B, d] bf16 into y [B, d] bf16 by ids and
    weights [B, k]; see xshare_ops.h."""
    B, d = x.shape
    dev = _current_device(x)
    if topk_ids.dim() != 2:
        raise ValueError(f"topk_ids must be [B, k], got {list(topk_ids.shape)}")
    rows, k = topk_ids.shape
    if rows != B or d != experts.d:
        raise ValueError(f"x must be [B, {experts.d}] and topk_ids [B, k], got {[B, d]} and {[rows, k]}")
    _shaped(topk_w, "topk_w", B, k)
    _shaped(y, "y", B, d)
    ex = experts.struct(dev)
    ws, ws_bytes = _ws(workspace, dev)
    rc = _experts(
        _ptr(x, torch.bfloat16, "x", None, dev), _ptr(topk_ids, torch.int32, "topk_ids", None, dev),
        _ptr(topk_w, torch.float32, "topk_w", None, dev), ctypes.byref(ex), B, k, d, experts.F,
        _ptr(y, torch.bfloat16, "y", None, dev),
        None if stats is None else _ptr(stats, torch.int32, "stats", STATS_WORDS, dev), ws, ws_bytes, _stream(stream, dev))
    if rc:
        _check(rc, "xshare_experts_fp8")
