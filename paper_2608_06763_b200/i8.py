"""Binding of the operators on 8-bit integers with a scale for each row (include/cubicquant.h, last section).  Argument marshalling only."""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass

import torch

from . import binding
from .binding import CubicQuantError, _check, _stream
from .fp4 import _DTYPE, _at, _check_offset, _check_rows, _here, _need
from .route import Routes, _matrix

_L = None


def _lib():
    global _L
    if _L is None:
        L = binding.lib()
        vp, i, i64, sz = C.c_void_p, C.c_int, C.c_int64, C.c_size_t
        for name, args in (("layout_bytes", [i64, i64, i64]), ("routed_layout_bytes", [i64, i64, i64]), ("workspace_bytes", [i64, i64]),
                           ("routed_workspace_bytes", [i64, i64, i64]), ("moe_workspace_bytes", [i64, i64, i, i64, i64])):
            fn = getattr(L, "cq_i8_" + name)
            fn.restype, fn.argtypes = sz, args
        for name, args in (("pack", [vp, i64, i64, i64, vp, vp]), ("unpack", [vp, i64, i64, i64, vp, vp]), ("quantize", [vp, i, i64, i64, i64, i64, vp, vp, vp]),
                           ("quantize_routed", [vp, i, i64, i64, vp, vp, i64, i64, i64, vp, vp, vp]), ("swiglu_quantize", [vp, i, i64, i64, i64, vp, i64, vp, vp, vp]),
                           ("dequantize", [vp, vp, i64, i64, i64, vp, vp, i, vp]), ("gemm", [vp, vp, vp, vp, vp, i, i64, i64, i64, vp, sz, vp]),
                           ("linear", [vp, vp, vp, i64, vp, i, i64, i64, i64, vp, sz, vp]), ("gemm_routed", [vp, vp, vp, vp, vp, i64, vp, i, i64, i64, i64, vp, sz, vp]),
                           ("linear_routed", [vp, vp, vp, i64, i64, vp, vp, i64, vp, i, i64, i64, i64, vp, sz, vp]),
                           ("moe", [vp, vp, vp, vp, i64, vp, i64, i64, i, vp, vp, vp, vp, i64, vp, i64, i, i64, i64, vp, sz, vp])):
            fn = getattr(L, "cq_i8_" + name)
            fn.restype, fn.argtypes = i, args
        L.cq_debug_i8_plan.restype, L.cq_debug_i8_plan.argtypes = i, [i64, i64, i64, i64, i, vp]
        _L = L
    return _L


@dataclass
class I8Tensor:
    """Rows of 8-bit codes in the device layout and the scale of each: `matrices` of M x K one after another, or (groups) M routed rows of K.  Made by cq_i8_empty,
    cq_i8_pack and the quantisers; calls take what it says of its layout as they find it."""
    layout: torch.Tensor
    scale: torch.Tensor                          # fp32 [matrices * M]
    matrices: int
    M: int
    K: int
    groups: int = 0                              # routed rows: how many groups
    expert_offset: torch.Tensor | None = None    # routed rows: int32 [groups + 1] on the device


def _check_k(K: int):
    if K <= 0 or K % 16:
        raise CubicQuantError(f"K = {K} is not a multiple of 16")


def cq_i8_empty(M: int, K: int, matrices: int = 1, groups: int | None = None, device=None) -> I8Tensor:
    """Room for `matrices` of M x K, or for M routed rows of K in `groups` groups."""
    _check_k(K)
    if groups is None:
        n = _lib().cq_i8_layout_bytes(matrices, M, K)
    else:
        _need(matrices == 1, "routed rows are one matrix")
        n = _lib().cq_i8_routed_layout_bytes(groups, M, K)
    _need(n > 0 or M == 0, f"no layout for {matrices} x {M} x {K}, {groups} groups")
    device = device or "cuda"
    return I8Tensor(torch.empty(n, dtype=torch.uint8, device=device), torch.empty(matrices * M, dtype=torch.float32, device=device), matrices, M, K, groups or 0)


def _into(out, M, K, matrices=1, groups=None, device=None) -> I8Tensor:
    if out is None:
        return cq_i8_empty(M, K, matrices, groups, device)
    if out.M != M or out.K != K or out.matrices != matrices or out.groups != (groups or 0):
        raise CubicQuantError("out is of another shape")
    return out


def cq_i8_pack(codes: torch.Tensor, scale: torch.Tensor) -> I8Tensor:
    """A checkpoint's codes int8 [.., M, K] and scales fp32 [.., M] (the first axis, if there are three: matrices).  The handle keeps `scale` itself."""
    _need(codes.dim() in (2, 3) and codes.dtype == torch.int8 and codes.is_contiguous(), "codes are int8, [M, K] or [E, M, K], contiguous")
    E, M, K = (codes.shape[0] if codes.dim() == 3 else 1), codes.shape[-2], codes.shape[-1]
    _check_k(K)
    _need(scale.dtype == torch.float32 and scale.is_contiguous() and scale.shape == codes.shape[:-1], "scales are fp32 [.., M], contiguous")
    _here(codes, scale)
    q = cq_i8_empty(M, K, E, device=codes.device)
    q.scale = scale.view(-1)
    _check(_lib().cq_i8_pack(codes.data_ptr(), E, M, K, q.layout.data_ptr(), _stream()), "cq_i8_pack")
    return q


def cq_i8_unpack(q: I8Tensor):
    """(codes, scales) as cq_i8_pack takes them."""
    _need(not q.groups, "routed rows have no checkpoint form")
    _here(q.layout, q.scale)
    lead = (q.matrices, q.M) if q.matrices > 1 else (q.M,)
    codes = torch.empty(lead + (q.K,), dtype=torch.int8, device=q.layout.device)
    _check(_lib().cq_i8_unpack(q.layout.data_ptr(), q.matrices, q.M, q.K, codes.data_ptr(), _stream()), "cq_i8_unpack")
    return codes, q.scale.view(lead)


def cq_i8_quantize(x: torch.Tensor, route_token: torch.Tensor | None = None, expert_offset: torch.Tensor | None = None, out: I8Tensor | None = None) -> I8Tensor:
    """x [M, K] or [E, M, K] (bfloat16, float16, float32) -> codes and the scale of each row.  With route_token and expert_offset (int32 on the device): rows route_token of
    x, grouped by matrix, for cq_i8_gemm_routed."""
    E = 1
    if x.dim() == 3:
        _need(x.is_contiguous() and route_token is None, "several matrices are one contiguous tensor")
        E, x = x.shape[0], x.flatten(0, 1)
        _need(E > 0, "no matrix")
    M, K, ld, at, dtype = _check_rows(x)
    _check_k(K)
    if (route_token is None) != (expert_offset is None):
        raise CubicQuantError("route_token and expert_offset come together")
    if route_token is None:
        stream = _here(x, None if out is None else out.layout, None if out is None else out.scale)
        q = _into(out, M // E, K, E, device=x.device)
        if M:
            status = (_L or _lib()).cq_i8_quantize(at, dtype, ld, E, q.M, K, q.layout.data_ptr(), q.scale.data_ptr(), stream)
            if status != 0:
                _check(status, "cq_i8_quantize")
        q.expert_offset = None
    else:
        _check_offset(expert_offset)
        _need(route_token.dtype == torch.int32 and route_token.dim() == 1 and route_token.is_contiguous(), "route_token is an int32 tensor")
        stream = _here(x, route_token, expert_offset, None if out is None else out.layout, None if out is None else out.scale)
        R, groups = route_token.numel(), expert_offset.numel() - 1
        q = _into(out, R, K, 1, groups, device=x.device)
        if R:
            _check((_L or _lib()).cq_i8_quantize_routed(at, dtype, ld, M, route_token.data_ptr(), expert_offset.data_ptr(), groups, R, K, q.layout.data_ptr(), q.scale.data_ptr(),
                                                        stream), "cq_i8_quantize")
        q.expert_offset = expert_offset
    return q


def cq_i8_swiglu_quantize(h: torch.Tensor, expert_offset: torch.Tensor | None = None, out: I8Tensor | None = None) -> I8Tensor:
    """h [M, 2 I] (gate | up; bfloat16 or float16) -> silu(gate) * up, rounded to h's dtype, quantised.  expert_offset: the rows are routed."""
    M, K, ld, at, dtype = _check_rows(h, "h")
    if dtype == 2 or K % 2:
        raise CubicQuantError("h is [M, 2 I] in bfloat16 or float16")
    K //= 2
    _check_k(K)
    groups = None
    if expert_offset is not None:
        _check_offset(expert_offset)
        groups = expert_offset.numel() - 1
    stream = _here(h, expert_offset, None if out is None else out.layout, None if out is None else out.scale)
    q = _into(out, M, K, 1, groups, device=h.device)
    if M:
        status = (_L or _lib()).cq_i8_swiglu_quantize(at, dtype, ld, M, K, _at(expert_offset), groups or 0, q.layout.data_ptr(), q.scale.data_ptr(), stream)
        if status != 0:
            _check(status, "cq_i8_swiglu_quantize")
    q.expert_offset = expert_offset
    return q


def cq_i8_dequantize(q: I8Tensor, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values that q stands for, [M, K] or [E, M, K]; rows of no group are left as they were (new ones: zeros).  Routed rows: of a handle that a quantiser has filled,
    which carries their offsets."""
    if q.groups:
        _check_offset(q.expert_offset, q.groups)
    shape = (q.matrices, q.M, q.K) if q.matrices > 1 else (q.M, q.K)
    if out is None:
        out = (torch.zeros if q.groups else torch.empty)(shape, dtype=dtype, device=q.layout.device)
    code, at = _DTYPE.get(out.dtype), out.data_ptr()
    if code is None or out.shape != shape or at % 16 or not out.is_contiguous():
        raise CubicQuantError(f"out is a contiguous tensor of shape {shape}")
    offset = q.expert_offset if q.groups else None
    stream = _here(q.layout, q.scale, offset, out)
    if q.M:
        status = (_L or _lib()).cq_i8_dequantize(q.layout.data_ptr(), q.scale.data_ptr(), q.groups or q.matrices, q.M, q.K, _at(offset), at, code, stream)
        if status != 0:
            _check(status, "cq_i8_dequantize")
    return out


def _workspace(n: int, device) -> torch.Tensor:
    """n bytes, zeroed where the device reports a wait that gave up; what else is read of them is written first."""
    if n <= 1 << 22:   # one call for the host, which is slower than the device up to there
        return torch.zeros(n, dtype=torch.uint8, device=device)
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    ws[:512].zero_()
    return ws


def cq_i8_workspace(w: I8Tensor, M: int) -> torch.Tensor:
    """A workspace for products of up to M rows (routes) with w, ready to use.  A program that keeps one saves each call its own, and can ask cq_gemm_status of it whether a wait
    on the device gave up."""
    n = _lib().cq_i8_routed_workspace_bytes(w.matrices, max(M, 1), w.K)
    return _workspace(max(n, 512), w.layout.device)


def _output(w, M, dtype, workspace, out, own_workspace):
    """(workspace, out, address of out, code of its dtype), made where they are not given."""
    if out is None:
        out = torch.empty((M, w.M), dtype=dtype, device=w.layout.device)
    code, at = _DTYPE.get(out.dtype), out.data_ptr()
    if out.dtype != dtype or code is None or code == 2 or out.shape != (M, w.M) or at % 16 or not out.is_contiguous():
        raise CubicQuantError(f"out is a contiguous [{M}, {w.M}] tensor of 16-byte alignment in the dtype of x, bfloat16 or float16")
    if workspace is None:
        workspace = cq_i8_workspace(w, M) if own_workspace else torch.zeros(512, dtype=torch.uint8, device=w.layout.device)
    if workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise CubicQuantError("workspace is a contiguous uint8 tensor")
    return workspace, out, at, code


def cq_i8_gemm(w: I8Tensor, x, workspace: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """y[M, N] = x W^T.  x: [M, K] in the model dtype (quantised on the way) or an I8Tensor; y has the dtype of x (for an I8Tensor that of out, or bfloat16)."""
    if w.matrices != 1 or w.groups:
        raise CubicQuantError("w is one matrix of cq_i8_pack or cq_i8_quantize (several: cq_i8_gemm_routed)")
    if isinstance(x, I8Tensor):
        _need(not x.groups, "routed rows: cq_i8_gemm_routed")
        _need(x.matrices == 1 and x.K == w.K, "x and w differ in K")
        M = x.M
        workspace, out, at, f16 = _output(w, M, torch.bfloat16 if out is None else out.dtype, workspace, out, False)
        stream = _here(w.layout, w.scale, x.layout, x.scale, workspace, out)
        if M:
            status = (_L or _lib()).cq_i8_gemm(w.layout.data_ptr(), w.scale.data_ptr(), x.layout.data_ptr(), x.scale.data_ptr(), at, f16, M, w.M, w.K, workspace.data_ptr(),
                                               workspace.numel(), stream)
            if status != 0:
                _check(status, "cq_i8_gemm")
        return out
    M, K, ld, x_at, dtype = _check_rows(x)
    if dtype == 2 or K != w.K:
        raise CubicQuantError(f"x is [M, {w.K}] in bfloat16 or float16")
    workspace, out, at, f16 = _output(w, M, x.dtype, workspace, out, True)
    stream = _here(w.layout, w.scale, x, workspace, out)
    if M:
        status = (_L or _lib()).cq_i8_linear(w.layout.data_ptr(), w.scale.data_ptr(), x_at, ld, at, f16, M, w.M, K, workspace.data_ptr(), workspace.numel(), stream)
        if status != 0:
            _check(status, "cq_i8_gemm")
    return out


def cq_i8_gemm_routed(w: I8Tensor, x, route_token: torch.Tensor | None, expert_offset: torch.Tensor, workspace: torch.Tensor | None = None,
                      out: torch.Tensor | None = None) -> torch.Tensor:
    """Route-major y[R, N]: rows [expert_offset[e], expert_offset[e + 1]) meet matrix e of w.  x: [T, K] in the model dtype with route_token (int32 [R] on the device), or an
    I8Tensor of R routed rows with route_token None.  expert_offset: int32 on the device; rows from its last value on are left as they were (in a new tensor: undefined)."""
    if w.groups:
        raise CubicQuantError("w holds the matrices of cq_i8_pack or cq_i8_quantize")
    _check_offset(expert_offset, w.matrices)
    if isinstance(x, I8Tensor):
        _need(route_token is None and x.groups == w.matrices, "x holds the routed rows of as many groups as w has matrices")
        _need(x.K == w.K, "x and w differ in K")
        R = x.M
        workspace, out, at, f16 = _output(w, R, torch.bfloat16 if out is None else out.dtype, workspace, out, False)
        stream = _here(w.layout, w.scale, x.layout, x.scale, expert_offset, workspace, out)
        if R:
            status = (_L or _lib()).cq_i8_gemm_routed(w.layout.data_ptr(), w.scale.data_ptr(), x.layout.data_ptr(), x.scale.data_ptr(), expert_offset.data_ptr(), w.matrices, at,
                                                      f16, R, w.M, w.K, workspace.data_ptr(), workspace.numel(), stream)
            if status != 0:
                _check(status, "cq_i8_gemm_routed")
        return out
    T, K, ld, x_at, dtype = _check_rows(x)
    if dtype == 2 or K != w.K:
        raise CubicQuantError(f"x is [T, {w.K}] in bfloat16 or float16")
    if route_token is None or route_token.dtype != torch.int32 or route_token.dim() != 1 or not route_token.is_contiguous():
        raise CubicQuantError("route_token is an int32 tensor")
    R = route_token.numel()
    workspace, out, at, f16 = _output(w, R, x.dtype, workspace, out, True)
    stream = _here(w.layout, w.scale, x, route_token, expert_offset, workspace, out)
    if R:
        status = (_L or _lib()).cq_i8_linear_routed(w.layout.data_ptr(), w.scale.data_ptr(), x_at, ld, T, route_token.data_ptr(), expert_offset.data_ptr(), w.matrices, at, f16, R,
                                                    w.M, w.K, workspace.data_ptr(), workspace.numel(), stream)
        if status != 0:
            _check(status, "cq_i8_gemm_routed")
    return out


def cq_i8_moe_workspace(gate_up: I8Tensor, down: I8Tensor, T: int, top: int) -> torch.Tensor:
    """A workspace for cq_i8_moe of up to T tokens with `top` routes each, ready to use."""
    n = _lib().cq_i8_moe_workspace_bytes(down.matrices, max(T, 1), top, down.M, down.K)
    _need(n > 0, f"no experts of {down.matrices} x {down.M} x {down.K} for {T} tokens of {top} routes")
    return _workspace(n, down.layout.device)


def cq_i8_moe(gate_up: I8Tensor, down: I8Tensor, x: torch.Tensor, routes: Routes, add: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
              out: torch.Tensor | None = None) -> torch.Tensor:
    """The experts of a layer: y[T, H] = add + the weighted sum over routes of down(silu(gate) * up).  gate_up: E matrices of 2 I x H (gate above up); down: E matrices of H x I;
    x [T, H] in bfloat16 or float16; routes of cq_route.  Equal to cq_i8_gemm_routed, cq_i8_swiglu_quantize, cq_i8_gemm_routed, cq_combine."""
    E, H, I = down.matrices, down.M, down.K  # noqa: E741
    if gate_up.groups or down.groups or gate_up.matrices != E or gate_up.M != 2 * I or gate_up.K != H:
        raise CubicQuantError("gate_up holds a 2 I x H matrix for each H x I matrix of down")
    T, K, ld, x_at, dtype = _check_rows(x)
    if dtype == 2 or K != H:
        raise CubicQuantError(f"x is [T, {H}] in bfloat16 or float16")
    top = routes.top
    if routes.tokens != T or routes.experts != E:
        raise CubicQuantError(f"routes are those of {T} tokens to {E} experts")
    if out is None:
        out = torch.empty((T, H), dtype=x.dtype, device=x.device)
    ldy, lda = _matrix(out, "out", T, H, x.dtype), 0 if add is None else _matrix(add, "add", T, H, x.dtype)
    if workspace is None:
        workspace = cq_i8_moe_workspace(gate_up, down, T, top)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise CubicQuantError("workspace is a contiguous uint8 tensor")
    stream = _here(x, gate_up.layout, gate_up.scale, down.layout, down.scale, add, workspace, out)
    if routes._device != x.get_device():
        raise CubicQuantError(f"tensors on {x.device} and {routes.row.device}")
    if T:
        status = (_L or _lib()).cq_i8_moe(gate_up.layout.data_ptr(), gate_up.scale.data_ptr(), down.layout.data_ptr(), down.scale.data_ptr(), E, x_at, ld, T, top,
                                          routes.offset.data_ptr(), routes.row.data_ptr(), routes.weight.data_ptr(), _at(add), lda, out.data_ptr(), ldy, dtype,
                                          H, I, workspace.data_ptr(), workspace.numel(), stream)
        if status != 0:
            _check(status, "cq_i8_moe")
    return out


def cq_debug_i8_plan(M: int, N: int, K: int, matrices: int = 0, quantised: bool = False) -> dict:
    """How cq_i8_gemm (matrices = 0) or cq_i8_gemm_routed cuts a product of M rows on the current device."""
    out = (C.c_int64 * 4)()
    _check(_lib().cq_debug_i8_plan(matrices, M, N, K, 1 if quantised else 0, out), "cq_debug_i8_plan")
    return {"channels": out[0], "rows": out[1], "runs": out[2], "quantises": bool(out[3])}
