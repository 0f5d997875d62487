"""Binding of the 4-bit floating point operators (include/cubicquant.h, last section).  Argument marshalling only."""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass

import torch

from . import binding
from .binding import CubicQuantError, _check, _stream

CQ_MXFP4, CQ_NVFP4 = 0, 1
_BLOCK = (32, 16)
_DTYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}

_L = None


def _lib():
    global _L
    if _L is None:
        L = binding.lib()
        vp, i, i64, sz = C.c_void_p, C.c_int, C.c_int64, C.c_size_t
        for name, args in (("layout_bytes", [i, i64, i64, i64]), ("routed_layout_bytes", [i, i64, i64, i64]),
                           ("workspace_bytes", [i, i64, i64]), ("routed_workspace_bytes", [i, i64, i64, i64])):
            fn = getattr(L, "cq_fp4_" + name)
            fn.restype, fn.argtypes = sz, args
        for name, args in (("pack", [vp, vp, i, i64, i64, i64, vp, vp]), ("unpack", [vp, i, i64, i64, i64, vp, vp, vp]),
                           ("quantize", [vp, i, i64, i, i64, i64, i64, vp, vp, vp]),
                           ("quantize_routed", [vp, i, i64, i64, vp, vp, i64, i64, i, i64, vp, vp, vp]),
                           ("swiglu_quantize", [vp, i, i64, i, i64, i64, vp, i64, vp, vp, vp]),
                           ("dequantize", [vp, i, i64, i64, i64, vp, vp, vp, i, vp]),
                           ("gemm", [vp, vp, vp, vp, i, vp, i, i64, i64, i64, vp, sz, vp]),
                           ("linear", [vp, vp, vp, i64, vp, i, vp, i, i64, i64, i64, vp, sz, vp]),
                           ("gemm_routed", [vp, vp, vp, vp, vp, i64, i, vp, i, i64, i64, i64, vp, sz, vp]),
                           ("linear_routed", [vp, vp, vp, i64, i64, vp, vp, vp, i64, i, vp, i, i64, i64, i64, vp, sz, vp])):
            fn = getattr(L, "cq_fp4_" + name)
            fn.restype, fn.argtypes = i, args
        L.cq_debug_fp4_plan.restype, L.cq_debug_fp4_plan.argtypes = i, [i, i64, i64, i64, i64, i, vp]
        _L = L
    return _L


def _need(ok, what: str):
    if not ok:
        raise CubicQuantError(what)


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _here(first, *others) -> int:
    """The stream to launch on.  Every tensor has to be on the current device: the call goes to that device's current stream."""
    dev = first.get_device()
    if dev < 0 or dev != _current_device():
        raise CubicQuantError(f"a tensor on {first.device}, which is not the current device: switch with torch.cuda.device")
    for t in others:
        if t is not None and t.get_device() != dev:
            raise CubicQuantError(f"tensors on {first.device} and {t.device}")
    return binding._raw_stream(dev) if binding._raw_stream is not None else _stream()


def _at(t):
    return None if t is None else t.data_ptr()


@dataclass
class Fp4Tensor:
    """Rows in the 4-bit device layout: `matrices` of M x K one after another, or (groups) M routed rows of K.  Made by cq_fp4_empty,
    cq_fp4_pack and the quantisers; calls take what it says of its layout as they find it."""
    layout: torch.Tensor
    fmt: int
    matrices: int
    M: int
    K: int
    tensor_scale: torch.Tensor | None = None     # NVFP4: fp32 on the device, one value or one for each matrix
    groups: int = 0                              # routed rows: how many groups
    expert_offset: torch.Tensor | None = None    # routed rows: int32 [groups + 1] on the device


# The checks below cost a call more than what they look at: no text is built, and no tensor asked twice, before something is wrong.
def _check_format(fmt: int, K: int):
    if fmt != CQ_MXFP4 and fmt != CQ_NVFP4:
        raise CubicQuantError("fmt is CQ_MXFP4 or CQ_NVFP4")
    if K <= 0 or K % _BLOCK[fmt]:
        raise CubicQuantError(f"K = {K} is not a multiple of the block of {_BLOCK[fmt]}")


def _check_scale(scale, fmt: int, matrices: int = 1):
    if scale is None:
        return
    if fmt != CQ_NVFP4:
        raise CubicQuantError("MXFP4 has no tensor scale")
    if not isinstance(scale, torch.Tensor) or scale.dtype != torch.float32 or scale.numel() != matrices or (matrices > 1 and not scale.is_contiguous()):
        raise CubicQuantError(f"tensor_scale is {matrices} fp32 value(s) on the device")


def _check_offset(offset, groups=None):
    if not (isinstance(offset, torch.Tensor) and offset.dtype == torch.int32 and offset.dim() == 1 and offset.is_contiguous() and
            (offset.numel() >= 2 if groups is None else offset.numel() == groups + 1)):
        raise CubicQuantError("expert_offset is an int32 tensor of one more value than there are matrices")


def _check_rows(x, name="x"):
    """(rows, values of a row, distance of rows, address, code of the dtype): rows of contiguous values, any distance of whole 16 bytes apart; a row
    by itself, any."""
    dtype = _DTYPE.get(x.dtype)
    if dtype is None:
        raise CubicQuantError(f"{name} is bfloat16, float16 or float32")
    if x.dim() != 2:
        raise CubicQuantError(f"{name} is a matrix whose rows are contiguous")
    M, K = x.shape
    ld, one = x.stride()
    if one != 1 and K > 1:
        raise CubicQuantError(f"{name} is a matrix whose rows are contiguous")
    if M <= 1:
        ld = K
    at = x.data_ptr()
    if ld < K or at % 16 or ld % (4 if dtype == 2 else 8):
        raise CubicQuantError(f"rows of {name} start on 16-byte boundaries and do not overlap")
    return M, K, ld, at, dtype


def cq_fp4_empty(fmt: int, M: int, K: int, matrices: int = 1, groups: int | None = None, device=None) -> Fp4Tensor:
    """Room for `matrices` of M x K, or for M routed rows of K in `groups` groups."""
    _check_format(fmt, K)
    if groups is None:
        n = _lib().cq_fp4_layout_bytes(fmt, matrices, M, K)
    else:
        _need(matrices == 1, "routed rows are one matrix")
        n = _lib().cq_fp4_routed_layout_bytes(fmt, groups, M, K)
    _need(n > 0 or M == 0, f"no layout for {matrices} x {M} x {K}, {groups} groups")
    return Fp4Tensor(torch.empty(n, dtype=torch.uint8, device=device or "cuda"), fmt, matrices, M, K, None, groups or 0)


def _into(out, fmt, M, K, matrices=1, groups=None, device=None) -> Fp4Tensor:
    if out is None:
        return cq_fp4_empty(fmt, M, K, matrices, groups, device)
    if out.fmt != fmt or out.M != M or out.K != K or out.matrices != matrices or out.groups != (groups or 0):
        raise CubicQuantError("out is of another format or shape")
    return out


def cq_fp4_pack(codes: torch.Tensor, scales: torch.Tensor, fmt: int, tensor_scale: torch.Tensor | None = None) -> Fp4Tensor:
    """A checkpoint's codes uint8 [.., M, K / 2] and scales uint8 [.., M, K / block] (the first axis, if there are three: matrices)."""
    _need(codes.dim() in (2, 3) and codes.dtype == torch.uint8 and scales.dtype == torch.uint8, "codes and scales are uint8, [M, K / 2] or [E, M, K / 2]")
    E, M, K = (codes.shape[0] if codes.dim() == 3 else 1), codes.shape[-2], codes.shape[-1] * 2
    _check_format(fmt, K)
    _need(tuple(scales.shape) == tuple(codes.shape[:-1]) + (K // _BLOCK[fmt],) and codes.is_contiguous() and scales.is_contiguous(), "scales are [.., M, K / block], both contiguous")
    _check_scale(tensor_scale, fmt, E)
    _here(codes, scales, tensor_scale)
    q = cq_fp4_empty(fmt, M, K, E, device=codes.device)
    q.tensor_scale = tensor_scale
    _check(_lib().cq_fp4_pack(codes.data_ptr(), scales.data_ptr(), fmt, E, M, K, q.layout.data_ptr(), _stream()), "cq_fp4_pack")
    return q


def cq_fp4_unpack(q: Fp4Tensor):
    """(codes, scales) as cq_fp4_pack takes them."""
    _need(not q.groups, "routed rows have no checkpoint form")
    _here(q.layout)
    lead = (q.matrices, q.M) if q.matrices > 1 else (q.M,)
    codes = torch.empty(lead + (q.K // 2,), dtype=torch.uint8, device=q.layout.device)
    scales = torch.empty(lead + (q.K // _BLOCK[q.fmt],), dtype=torch.uint8, device=q.layout.device)
    _check(_lib().cq_fp4_unpack(q.layout.data_ptr(), q.fmt, q.matrices, q.M, q.K, codes.data_ptr(), scales.data_ptr(), _stream()), "cq_fp4_unpack")
    return codes, scales


def cq_fp4_quantize(x: torch.Tensor, fmt: int, tensor_scale: torch.Tensor | None = None, route_token: torch.Tensor | None = None,
                    expert_offset: torch.Tensor | None = None, out: Fp4Tensor | None = None) -> Fp4Tensor:
    """x [M, K] or [E, M, K] (bfloat16, float16, float32) -> codes and block scales.  With route_token and expert_offset (int32 on the
    device): rows route_token of x, grouped by matrix, for cq_fp4_gemm_routed."""
    E = 1
    if x.dim() == 3:
        _need(x.is_contiguous() and route_token is None, "several matrices are one contiguous tensor")
        E, x = x.shape[0], x.flatten(0, 1)
        _need(E > 0, "no matrix")
    M, K, ld, at, dtype = _check_rows(x)
    _check_format(fmt, K)
    _check_scale(tensor_scale, fmt, E)
    if (route_token is None) != (expert_offset is None):
        raise CubicQuantError("route_token and expert_offset come together")
    if route_token is None:
        stream = _here(x, tensor_scale, None if out is None else out.layout)
        q = _into(out, fmt, M // E, K, E, device=x.device)
        if M:
            status = (_L or _lib()).cq_fp4_quantize(at, dtype, ld, fmt, E, q.M, K, _at(tensor_scale), q.layout.data_ptr(), stream)
            if status != 0:
                _check(status, "cq_fp4_quantize")
    else:
        _check_offset(expert_offset)
        _need(route_token.dtype == torch.int32 and route_token.dim() == 1 and route_token.is_contiguous(), "route_token is an int32 tensor")
        stream = _here(x, tensor_scale, route_token, expert_offset, None if out is None else out.layout)
        R, groups = route_token.numel(), expert_offset.numel() - 1
        q = _into(out, fmt, R, K, 1, groups, device=x.device)
        if R:
            _check((_L or _lib()).cq_fp4_quantize_routed(at, dtype, ld, M, route_token.data_ptr(), expert_offset.data_ptr(), groups, R, fmt, K, _at(tensor_scale),
                                                         q.layout.data_ptr(), stream), "cq_fp4_quantize")
    q.tensor_scale, q.expert_offset = tensor_scale, expert_offset
    return q


def cq_fp4_swiglu_quantize(h: torch.Tensor, fmt: int, tensor_scale: torch.Tensor | None = None, expert_offset: torch.Tensor | None = None,
                           out: Fp4Tensor | None = None) -> Fp4Tensor:
    """h [M, 2 I] (gate | up; bfloat16 or float16) -> silu(gate) * up, rounded to h's dtype, quantised.  expert_offset: the rows are routed."""
    M, K, ld, at, dtype = _check_rows(h, "h")
    if dtype == 2 or K % 2:
        raise CubicQuantError("h is [M, 2 I] in bfloat16 or float16")
    K //= 2
    _check_format(fmt, K)
    _check_scale(tensor_scale, fmt)
    groups = None
    if expert_offset is not None:
        _check_offset(expert_offset)
        groups = expert_offset.numel() - 1
    stream = _here(h, tensor_scale, expert_offset, None if out is None else out.layout)
    q = _into(out, fmt, M, K, 1, groups, device=h.device)
    if M:
        status = (_L or _lib()).cq_fp4_swiglu_quantize(at, dtype, ld, fmt, M, K, _at(expert_offset), groups or 0, _at(tensor_scale), q.layout.data_ptr(), stream)
        if status != 0:
            _check(status, "cq_fp4_swiglu_quantize")
    q.tensor_scale, q.expert_offset = tensor_scale, expert_offset
    return q


def cq_fp4_dequantize(q: Fp4Tensor, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values that q stands for, [M, K] or [E, M, K]; rows of no group are left as they were (new ones: zeros).  Routed rows: of
    a handle that a quantiser has filled, which carries their offsets."""
    if q.groups:
        _check_offset(q.expert_offset, q.groups)
    shape = (q.matrices, q.M, q.K) if q.matrices > 1 else (q.M, q.K)
    if out is None:
        out = (torch.zeros if q.groups else torch.empty)(shape, dtype=dtype, device=q.layout.device)
    code, at = _DTYPE.get(out.dtype), out.data_ptr()
    if code is None or out.shape != shape or at % 16 or not out.is_contiguous():
        raise CubicQuantError(f"out is a contiguous tensor of shape {shape}")
    offset = q.expert_offset if q.groups else None
    stream = _here(q.layout, q.tensor_scale, offset, out)
    if q.M:
        status = (_L or _lib()).cq_fp4_dequantize(q.layout.data_ptr(), q.fmt, q.groups or q.matrices, q.M, q.K, _at(offset), _at(q.tensor_scale), at, code, stream)
        if status != 0:
            _check(status, "cq_fp4_dequantize")
    return out


def cq_fp4_workspace(w: Fp4Tensor, M: int) -> torch.Tensor:
    """A zeroed workspace for products of up to M rows (routes) with w.  A program that keeps one saves each call its own, and can ask
    cq_gemm_status of it whether a wait on the device gave up."""
    n = _lib().cq_fp4_routed_workspace_bytes(w.fmt, w.matrices, max(M, 1), w.K)
    return torch.zeros(max(n, 512), dtype=torch.uint8, device=w.layout.device)


def _output(w, M, dtype, workspace, out, own_workspace):
    """(workspace, out, address of out, code of its dtype), made where they are not given."""
    if out is None:
        out = torch.empty((M, w.M), dtype=dtype, device=w.layout.device)
    code, at = _DTYPE.get(out.dtype), out.data_ptr()
    if out.dtype != dtype or code is None or code == 2 or out.shape != (M, w.M) or at % 16 or not out.is_contiguous():
        raise CubicQuantError(f"out is a contiguous [{M}, {w.M}] tensor of 16-byte alignment in the dtype of x, bfloat16 or float16")
    if workspace is None:
        workspace = cq_fp4_workspace(w, M) if own_workspace else torch.zeros(512, dtype=torch.uint8, device=w.layout.device)
    if workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise CubicQuantError("workspace is a contiguous uint8 tensor")
    return workspace, out, at, code


def _check_quantised(w, x, tensor_scale):
    _need(x.fmt == w.fmt and x.matrices == 1 and x.K == w.K, "x and w differ in format or K")
    _need(tensor_scale is None, "x carries its own tensor scale")


def cq_fp4_gemm(w: Fp4Tensor, x, tensor_scale: torch.Tensor | None = None, workspace: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """y[M, N] = x W^T.  x: [M, K] in the model dtype (quantised on the way, NVFP4 with tensor_scale) or an Fp4Tensor; y has the dtype of x
    (for an Fp4Tensor that of out, or bfloat16)."""
    if w.matrices != 1 or w.groups:
        raise CubicQuantError("w is one matrix of cq_fp4_pack or cq_fp4_quantize (several: cq_fp4_gemm_routed)")
    if isinstance(x, Fp4Tensor):
        _need(not x.groups, "routed rows: cq_fp4_gemm_routed")
        _check_quantised(w, x, tensor_scale)
        M = x.M
        workspace, out, at, f16 = _output(w, M, torch.bfloat16 if out is None else out.dtype, workspace, out, False)
        stream = _here(w.layout, w.tensor_scale, x.layout, x.tensor_scale, workspace, out)
        if M:
            status = (_L or _lib()).cq_fp4_gemm(w.layout.data_ptr(), _at(w.tensor_scale), x.layout.data_ptr(), _at(x.tensor_scale), w.fmt, at, f16, M, w.M, w.K,
                                                workspace.data_ptr(), workspace.numel(), stream)
            if status != 0:
                _check(status, "cq_fp4_gemm")
        return out
    M, K, ld, x_at, dtype = _check_rows(x)
    if dtype == 2 or K != w.K:
        raise CubicQuantError(f"x is [M, {w.K}] in bfloat16 or float16")
    _check_scale(tensor_scale, w.fmt)
    workspace, out, at, f16 = _output(w, M, x.dtype, workspace, out, True)
    stream = _here(w.layout, w.tensor_scale, x, tensor_scale, workspace, out)
    if M:
        status = (_L or _lib()).cq_fp4_linear(w.layout.data_ptr(), _at(w.tensor_scale), x_at, ld, _at(tensor_scale), w.fmt, at, f16, M, w.M, K, workspace.data_ptr(),
                                              workspace.numel(), stream)
        if status != 0:
            _check(status, "cq_fp4_gemm")
    return out


def cq_fp4_gemm_routed(w: Fp4Tensor, x, route_token: torch.Tensor | None, expert_offset: torch.Tensor, tensor_scale: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Route-major y[R, N]: rows [expert_offset[e], expert_offset[e + 1]) meet matrix e of w.  x: [T, K] in the model dtype with route_token
    (int32 [R] on the device), or an Fp4Tensor of R routed rows with route_token None.  expert_offset: int32 on the device; rows from
    its last value on are left as they were (in a new tensor: undefined)."""
    if w.groups:
        raise CubicQuantError("w holds the matrices of cq_fp4_pack or cq_fp4_quantize")
    _check_offset(expert_offset, w.matrices)
    if isinstance(x, Fp4Tensor):
        _need(route_token is None and x.groups == w.matrices, "x holds the routed rows of as many groups as w has matrices")
        _check_quantised(w, x, tensor_scale)
        R = x.M
        workspace, out, at, f16 = _output(w, R, torch.bfloat16 if out is None else out.dtype, workspace, out, False)
        stream = _here(w.layout, w.tensor_scale, x.layout, x.tensor_scale, expert_offset, workspace, out)
        if R:
            status = (_L or _lib()).cq_fp4_gemm_routed(w.layout.data_ptr(), _at(w.tensor_scale), x.layout.data_ptr(), _at(x.tensor_scale), expert_offset.data_ptr(), w.matrices,
                                                       w.fmt, at, f16, R, w.M, w.K, workspace.data_ptr(), workspace.numel(), stream)
            if status != 0:
                _check(status, "cq_fp4_gemm_routed")
        return out
    T, K, ld, x_at, dtype = _check_rows(x)
    if dtype == 2 or K != w.K:
        raise CubicQuantError(f"x is [T, {w.K}] in bfloat16 or float16")
    _check_scale(tensor_scale, w.fmt)
    if route_token is None or route_token.dtype != torch.int32 or route_token.dim() != 1 or not route_token.is_contiguous():
        raise CubicQuantError("route_token is an int32 tensor")
    R = route_token.numel()
    workspace, out, at, f16 = _output(w, R, x.dtype, workspace, out, True)
    stream = _here(w.layout, w.tensor_scale, x, tensor_scale, route_token, expert_offset, workspace, out)
    if R:
        status = (_L or _lib()).cq_fp4_linear_routed(w.layout.data_ptr(), _at(w.tensor_scale), x_at, ld, T, route_token.data_ptr(), _at(tensor_scale),
                                                     expert_offset.data_ptr(), w.matrices, w.fmt, at, f16, R, w.M, w.K, workspace.data_ptr(), workspace.numel(), stream)
        if status != 0:
            _check(status, "cq_fp4_gemm_routed")
    return out


def cq_debug_fp4_plan(fmt: int, M: int, N: int, K: int, matrices: int = 0, quantised: bool = False) -> dict:
    """How cq_fp4_gemm (matrices = 0) or cq_fp4_gemm_routed cuts a product of M rows on the current device."""
    out = (C.c_int64 * 4)()
    _check(_lib().cq_debug_fp4_plan(fmt, matrices, M, N, K, 1 if quantised else 0, out), "cq_debug_fp4_plan")
    return {"channels": out[0], "rows": out[1], "runs": out[2], "quantises": bool(out[3])}
