"""Binding of routing to experts (include/cubicquant.h): the choice of experts with its route map, and the sum of a token's routes.  Argument marshalling only."""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass

import torch

from . import binding
from .binding import CubicQuantError, _check
from .fp4 import _DTYPE, _at, _here, _need

CQ_SOFTMAX, CQ_SIGMOID = 0, 1

_L = None


def _lib():
    global _L
    if _L is None:
        L = binding.lib()
        vp, i, i64, sz, f = C.c_void_p, C.c_int, C.c_int64, C.c_size_t, C.c_float
        L.cq_route_workspace_bytes.restype, L.cq_route_workspace_bytes.argtypes = sz, [i64, i64]
        L.cq_route.restype, L.cq_route.argtypes = i, [vp, i, i64, i64, i64, i, i, vp, i, i, i, i, f, vp, vp, vp, vp, vp, vp, sz, vp]
        L.cq_combine.restype, L.cq_combine.argtypes = i, [vp, i64, i64, vp, vp, i64, i, i64, vp, i64, vp, i64, i, vp]
        _L = L
    return _L


@dataclass(frozen=True, eq=False)
class Routes:
    """Where tokens go: `expert` and `weight` [T, top], and the map of the routes grouped by expert: `token` [T top], `offset` [E + 1], `row`
    [T, top], the row of each choice.  -1: no choice, no route.  All int32 but `weight`, fp32; contiguous, on one device.  Looked over once, when it is made."""
    expert: torch.Tensor
    weight: torch.Tensor
    token: torch.Tensor
    offset: torch.Tensor
    row: torch.Tensor

    def __post_init__(self):
        ints = (self.expert, self.token, self.offset, self.row)
        if not all(isinstance(t, torch.Tensor) and t.dtype == torch.int32 and t.is_contiguous() for t in ints):
            raise CubicQuantError("routes are contiguous int32 tensors")
        if not isinstance(self.weight, torch.Tensor) or self.weight.dtype != torch.float32 or not self.weight.is_contiguous():
            raise CubicQuantError("the weights of routes are a contiguous fp32 tensor")
        if self.expert.dim() != 2 or self.weight.shape != self.expert.shape or self.row.shape != self.expert.shape or self.token.shape != (self.expert.numel(),):
            raise CubicQuantError("routes are expert, weight and row [T, top] and token [T top]")
        if self.offset.dim() != 1 or self.offset.numel() < 2:
            raise CubicQuantError("the offsets of routes are a value more than there are experts")
        if any(t.device != self.weight.device for t in ints):
            raise CubicQuantError("routes are on one device")
        for name, value in (("tokens", self.expert.shape[0]), ("top", self.expert.shape[1]), ("experts", self.offset.numel() - 1), ("_device", self.weight.get_device())):
            object.__setattr__(self, name, value)


def cq_routes_empty(T: int, E: int, top: int, device=None) -> Routes:
    """Room for the routes of T tokens to `top` of E experts."""
    new = lambda *shape, dtype=torch.int32: torch.empty(shape, dtype=dtype, device=device or "cuda")  # noqa: E731
    return Routes(new(T, top), new(T, top, dtype=torch.float32), new(T * top), new(E + 1), new(T, top))


def cq_route_workspace(T: int, E: int, device=None) -> torch.Tensor:
    """Scratch of cq_route for up to T tokens; one call at a time."""
    n = _lib().cq_route_workspace_bytes(max(T, 1), E)
    _need(n > 0, f"no routing of {T} tokens to {E} experts")
    return torch.empty(n, dtype=torch.uint8, device=device or "cuda")


def cq_route(logits: torch.Tensor, top: int, score: int = CQ_SOFTMAX, bias: torch.Tensor | None = None, groups: int = 1, groups_kept: int | None = None, group_best: int = 2,
             renormalise: bool = True, scale: float = 1.0, workspace: torch.Tensor | None = None, out: Routes | None = None) -> Routes:
    """The `top` experts of each row of logits [T, E] (bfloat16, float16, float32), their weights and the map of their routes.  bias: fp32 [E], for the choice alone.
    groups, groups_kept, group_best: experts of the best groups alone, by the sum of a group's best one or two.
    cq_fp4_gemm_routed, cq_i8_gemm_routed and cq_i8_moe take the map as it is; cq_gemm_routed takes offsets on the host and no tokens behind the last route:
    offset = routes.offset.tolist(); cq_gemm_routed(experts, x, routes.token[:offset[-1]], offset)."""
    dtype = _DTYPE.get(logits.dtype)
    if dtype is None or logits.dim() != 2:
        raise CubicQuantError("logits are [T, E] in bfloat16, float16 or float32")
    T, E = logits.shape
    ldl, one = logits.stride()
    if T <= 1:
        ldl = E
    if (one != 1 and E > 1) or ldl < E:
        raise CubicQuantError("rows of logits are contiguous and do not overlap")
    if bias is not None and (bias.dtype != torch.float32 or bias.shape != (E,) or not bias.is_contiguous()):
        raise CubicQuantError("bias is a contiguous fp32 tensor of a value for each expert")
    if top < 1:
        raise CubicQuantError("top is 1 or more")
    if out is None:
        out = cq_routes_empty(T, E, top, logits.device)
    elif out.tokens != T or out.top != top or out.experts != E:
        raise CubicQuantError(f"out is for {out.tokens} tokens to {out.top} of {out.experts} experts")
    if workspace is None:
        workspace = cq_route_workspace(T, E, logits.device)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise CubicQuantError("workspace is a contiguous uint8 tensor")
    stream = _here(logits, bias, workspace)
    if out._device != logits.get_device():
        raise CubicQuantError(f"tensors on {logits.device} and {out.expert.device}")
    if not T:
        out.offset.zero_()
        return out
    status = (_L or _lib()).cq_route(logits.data_ptr(), dtype, ldl, T, E, top, score, _at(bias), groups, groups if groups_kept is None else groups_kept, group_best,
                                     1 if renormalise else 0, scale, out.expert.data_ptr(), out.weight.data_ptr(), out.token.data_ptr(), out.offset.data_ptr(), out.row.data_ptr(),
                                     workspace.data_ptr(), workspace.numel(), stream)
    if status != 0:
        _check(status, "cq_route")
    return out


def _matrix(t, name, T, N, dtype):
    """Distance of the rows of a [T, N] matrix in `dtype` whose rows are contiguous."""
    if t.dtype != dtype or t.shape != (T, N):
        raise CubicQuantError(f"{name} is [{T}, {N}] in the dtype of the routes")
    ld, one = t.stride()
    if T <= 1:
        ld = N
    if (one != 1 and N > 1) or ld < N:
        raise CubicQuantError(f"rows of {name} are contiguous and do not overlap")
    return ld


def cq_combine(y_routes: torch.Tensor, routes: Routes, add: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """y[t] = add[t] + sum over j of routes.weight[t, j] y_routes[routes.row[t, j]]: [T, N] in the dtype of y_routes [R, N], bfloat16 or float16.  add: [T, N] or
    None; it may be out."""
    code = _DTYPE.get(y_routes.dtype)
    if code is None or code == 2 or y_routes.dim() != 2:
        raise CubicQuantError("y_routes is [R, N] in bfloat16 or float16")
    R, N = y_routes.shape
    T, top, dtype = routes.tokens, routes.top, y_routes.dtype
    ldr = _matrix(y_routes, "y_routes", R, N, dtype)
    if out is None:
        out = torch.empty((T, N), dtype=dtype, device=y_routes.device)
    ldy = _matrix(out, "out", T, N, dtype)
    lda = 0 if add is None else _matrix(add, "add", T, N, dtype)
    stream = _here(y_routes, add, out)
    if routes._device != y_routes.get_device():
        raise CubicQuantError(f"tensors on {y_routes.device} and {routes.row.device}")
    if T and N and R:
        status = (_L or _lib()).cq_combine(y_routes.data_ptr(), ldr, R, routes.weight.data_ptr(), routes.row.data_ptr(), T, top, N, _at(add), lda, out.data_ptr(), ldy, code, stream)
        if status != 0:
            _check(status, "cq_combine")
    elif T and N:   # no route at all
        out.zero_() if add is None else out.copy_(add)
    return out
