"""Routing and 8-bit integers, without a GPU: the oracles against brute force, sizes, and every refusal of the C entries and of the Python calls (found on the
host before anything is launched)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2608_06763_b200 as cq
from i8_shapes import PRODUCTS
from oracle import i8 as ref
from oracle import route as ref_route
from paper_2608_06763_b200 import i8, route

ONE, ODD, TWO = ctypes.c_void_p(16), ctypes.c_void_p(24), ctypes.c_void_p(18)   # never dereferenced: validation fails first


# ---------------------------------------------------------------- oracles
def test_oracle_choice_is_brute_force():
    r = np.random.default_rng(0)
    for score in ("softmax", "sigmoid"):
        for _ in range(50):
            E, top = int(r.integers(2, 12)), 2
            l, b = r.standard_normal((1, E)), 0.3 * r.standard_normal(E)
            s = np.exp(l[0]) / np.exp(l[0]).sum() if score == "softmax" else 1 / (1 + np.exp(-l[0]))
            want = sorted(range(E), key=lambda e: -(s[e] + b[e]))[:top]
            expert, weight = ref_route.choose(l, top, score, b)
            assert expert[0].tolist() == want
            assert np.allclose(weight[0], s[want] / s[want].sum(), rtol=1e-12)
            assert np.allclose(ref_route.choose(l, top, score, b, renormalise=False, scale=3.0)[1][0], 3 * s[want], rtol=1e-12)


def test_oracle_groups_masks_and_equals():
    l = np.array([[5.0, -9.0, 3.0, 3.0, 4.0, -9.0]])
    assert ref_route.choose(l, 2, "sigmoid", groups=3, kept=1)[0].tolist() == [[2, 3]]        # two good ones beat one better
    assert ref_route.choose(l, 2, "sigmoid", groups=3, kept=1, best=1)[0].tolist() == [[0, 1]]
    assert ref_route.choose(np.zeros((1, 6)), 3, "softmax", groups=3, kept=2)[0].tolist() == [[0, 1, 2]]
    l = np.array([[-np.inf, 1.0, np.nan, -np.inf]])
    expert, weight = ref_route.choose(l, 3, "softmax")
    assert expert.tolist() == [[1, -1, -1]] and weight.tolist() == [[1.0, 0.0, 0.0]]
    token, offset, row = ref_route.routes(np.array([[1, 0], [-1, -1], [1, -1]]), 3)
    assert token.tolist() == [0, 0, 2, -1, -1, -1] and offset.tolist() == [0, 1, 3, 3] and row.tolist() == [[1, 0], [-1, -1], [2, -1]]
    y, _ = ref_route.combine(np.array([[1.0], [10.0]]), np.array([[2.0, 3.0]]), np.array([[1, 0]]), np.array([[0.5]]))
    assert y.tolist() == [[23.5]]


def test_oracle_codes():
    c, d = ref.quantize(np.array([[127.0, 0.5, -0.5, 1.49, -1.5, 126.5, 0, 0], [0] * 8, [np.nan] + [1] * 7]))
    assert c[0].tolist() == [127, 1, -1, 1, -2, 127, 0, 0] and d[0] == 1.0
    assert not c[1].any() and d[1] == np.float32(1e-10) / np.float32(127)
    assert not c[2].any() and np.isnan(d[2])
    assert ref.gated(np.array([0.0, 1e3, -1e3]), np.array([1.0, 2.0, 2.0])).tolist() == [0.0, 2000.0, 0.0]


# ---------------------------------------------------------------- sizes
def test_sizes():
    L = i8._lib()
    assert L.cq_i8_layout_bytes(1, 128, 128) == 16384 and L.cq_i8_layout_bytes(3, 129, 144) == 3 * 2 * 2 * 16384
    assert L.cq_i8_layout_bytes(1, 128, 136) == 0 and L.cq_i8_layout_bytes(0, 1, 128) == 0 and L.cq_i8_layout_bytes(1, 1, (1 << 17) + 16) == 0
    assert L.cq_i8_routed_layout_bytes(4, 2, 128) == 2 * 16384 and L.cq_i8_routed_layout_bytes(4, 512, 128) == 7 * 16384
    assert L.cq_i8_routed_layout_bytes(513, 512, 128) == 0
    assert L.cq_i8_workspace_bytes(1, 128) == 512 + 256 + 16384 and L.cq_i8_workspace_bytes(65, 128) == 512 + 512 + 16384
    assert L.cq_i8_moe_workspace_bytes(4, 8, 2, 128, 64) == 512 + 256 + 256 + 4 * 16384 + 4 * 16384 + 16 * 128 * 2
    assert L.cq_i8_moe_workspace_bytes(4, 8, 33, 128, 64) == 0 and L.cq_i8_moe_workspace_bytes(4, 8, 2, 120, 64) == 0
    R = route._lib()
    assert R.cq_route_workspace_bytes(1, 64) > 0 and R.cq_route_workspace_bytes(0, 64) == 0 and R.cq_route_workspace_bytes(1, 513) == 0


def test_workspaces_for_more_tokens_serve_fewer():
    R, L = route._lib(), i8._lib()
    for E in (1, 64, 512):
        sizes = [R.cq_route_workspace_bytes(T, E) for T in range(1, 9000, 7)]
        assert sizes == sorted(sizes)
    for E in (1, 16):
        sizes = [L.cq_i8_moe_workspace_bytes(E, T, 2, 256, 128) for T in range(1, 900)]
        assert sizes == sorted(sizes)


# ---------------------------------------------------------------- refusals of the C entries
def with_changes(fn, names, good):
    def call(**kw):
        a = list(good)
        for k, v in kw.items():
            a[names.index(k)] = v
        return fn(*a)
    return call


def test_route_refuses():
    L = route._lib()
    names = "logits dtype ldl T E top score bias groups kept best renormalise scale expert weight token offset row workspace bytes stream".split()
    go = with_changes(L.cq_route, names, [ONE, 0, 64, 4, 64, 4, 0, None, 1, 1, 2, 1, 1.0, ONE, ONE, ONE, ONE, ONE, ONE, 1 << 20, None])
    for null in ("logits", "expert", "weight", "token", "offset", "row", "workspace"):
        assert go(**{null: None}) == -1
    assert go(dtype=3) == -1 and go(dtype=-1) == -1 and go(score=2) == -1 and go(T=0) == -1 and go(E=0) == -1 and go(top=0) == -1 and go(ldl=63) == -1
    assert go(groups=0) == -1 and go(groups=3) == -1 and go(kept=0) == -1 and go(kept=2) == -1 and go(best=0) == -1 and go(best=3) == -1
    assert go(top=65) == -1 and go(groups=8, kept=2, top=17) == -1
    assert go(E=513, ldl=513) == -2 and go(groups=64, kept=64) == -2 and go(top=33) == -2 and go(T=1 << 29) == -2
    assert go(logits=ctypes.c_void_p(17)) == -3 and go(dtype=2, logits=TWO) == -3 and go(bias=TWO) == -3 and go(row=TWO) == -3 and go(workspace=ODD) == -3
    assert go(bytes=255) == -4


def test_combine_refuses():
    L = route._lib()
    names = "y_routes ldr R weight row T top N add lda y ldy f16 stream".split()
    go = with_changes(L.cq_combine, names, [ONE, 64, 8, ONE, ONE, 4, 2, 64, None, 0, ONE, 64, 0, None])
    for null in ("y_routes", "weight", "row", "y"):
        assert go(**{null: None}) == -1
    assert go(R=0) == -1 and go(T=0) == -1 and go(top=0) == -1 and go(N=0) == -1 and go(ldr=63) == -1 and go(ldy=63) == -1 and go(add=ONE, lda=63) == -1
    assert go(top=33) == -2 and go(T=1 << 30) == -2 and go(N=1 << 31, ldr=1 << 31, ldy=1 << 31) == -2
    assert go(y=ctypes.c_void_p(17)) == -3 and go(weight=TWO) == -3 and go(add=ctypes.c_void_p(17), lda=64) == -3


def test_products_refuse():
    L = i8._lib()
    names = "w ws x ldx y f16 M N K workspace bytes stream".split()
    go = with_changes(L.cq_i8_linear, names, [ONE, ONE, ONE, 256, ONE, 0, 4, 128, 256, ONE, 1 << 20, None])
    for null in ("w", "ws", "x", "y", "workspace"):
        assert go(**{null: None}) == -1
    assert go(M=0) == -1 and go(N=0) == -1 and go(K=0) == -1 and go(ldx=-1) == -1 and go(ldx=255) == -1 and go(ldx=260) == -3
    assert go(K=264, ldx=264) == -2 and go(K=(1 << 17) + 16, ldx=1 << 18) == -2 and go(M=1 << 31) == -2 and go(N=1 << 30, M=1 << 30) == -2
    assert go(x=ODD) == -3 and go(y=ODD) == -3 and go(w=ODD) == -3 and go(workspace=ODD) == -3 and go(ws=TWO) == -3
    assert go(bytes=511) == -4
    assert L.cq_i8_gemm(ONE, ONE, ONE, ONE, ONE, 0, 4, 128, 256, ONE, 511, None) == -4
    assert L.cq_i8_gemm(ONE, ONE, ONE, None, ONE, 0, 4, 128, 256, ONE, 512, None) == -1
    assert L.cq_i8_gemm_routed(ONE, ONE, ONE, ONE, None, 4, ONE, 0, 4, 128, 256, ONE, 1 << 20, None) == -1
    assert L.cq_i8_gemm_routed(ONE, ONE, ONE, ONE, ONE, 513, ONE, 0, 4, 128, 256, ONE, 1 << 20, None) == -2
    assert L.cq_i8_gemm_routed(ONE, ONE, ONE, ONE, ONE, 0, ONE, 0, 4, 128, 256, ONE, 1 << 20, None) == -1
    assert L.cq_i8_linear_routed(ONE, ONE, ONE, 256, 8, None, ONE, 4, ONE, 0, 4, 128, 256, ONE, 1 << 20, None) == -1
    assert L.cq_i8_linear_routed(ONE, ONE, ONE, 256, 0, ONE, ONE, 4, ONE, 0, 4, 128, 256, ONE, 1 << 20, None) == -1
    assert L.cq_i8_quantize(ONE, 3, 256, 1, 4, 256, ONE, ONE, None) == -1 and L.cq_i8_quantize(ONE, 2, 258, 1, 4, 256, ONE, ONE, None) == -3
    assert L.cq_i8_quantize(ONE, 0, 256, 1, 4, 256, ODD, ONE, None) == -3 and L.cq_i8_quantize(ONE, 0, 256, 1, 4, 256, ONE, None, None) == -1
    assert L.cq_i8_quantize_routed(ONE, 0, 256, 8, None, ONE, 4, 4, 256, ONE, ONE, None) == -1
    assert L.cq_i8_swiglu_quantize(ONE, 2, 512, 4, 256, None, 0, ONE, ONE, None) == -1 and L.cq_i8_swiglu_quantize(ONE, 0, 511, 4, 256, None, 0, ONE, ONE, None) == -1
    assert L.cq_i8_swiglu_quantize(ONE, 0, 512, 4, 256, ONE, 513, ONE, ONE, None) == -2
    assert L.cq_i8_dequantize(ONE, ONE, 1, 4, 256, None, ODD, 0, None) == -3 and L.cq_i8_dequantize(ONE, None, 1, 4, 256, None, ONE, 0, None) == -1
    assert L.cq_i8_pack(ONE, 1, 4, 250, ONE, None) == -2 and L.cq_i8_pack(None, 1, 4, 256, ONE, None) == -1 and L.cq_i8_unpack(ONE, 1, 4, 256, ODD, None) == -3


def test_moe_refuses():
    L = i8._lib()
    names = "gu gus dn dns E x ldx T top offset row weight add lda y ldy f16 H I workspace bytes stream".split()
    go = with_changes(L.cq_i8_moe, names, [ONE, ONE, ONE, ONE, 4, ONE, 256, 8, 2, ONE, ONE, ONE, None, 0, ONE, 256, 0, 256, 128, ONE, 1 << 24, None])
    for null in ("gu", "gus", "dn", "dns", "x", "offset", "row", "weight", "y", "workspace"):
        assert go(**{null: None}) == -1
    assert go(T=0) == -1 and go(top=0) == -1 and go(H=0) == -1 and go(I=0) == -1 and go(E=0) == -1 and go(ldx=255) == -1 and go(ldy=255) == -1 and go(add=ONE, lda=255) == -1
    assert go(top=33) == -2 and go(T=1 << 30) == -2 and go(E=513) == -2 and go(H=264, ldx=264, ldy=264) == -2 and go(I=72) == -2
    assert go(ldx=260) == -3 and go(x=ODD) == -3 and go(workspace=ODD) == -3 and go(weight=TWO) == -3
    assert go(bytes=L.cq_i8_moe_workspace_bytes(4, 8, 2, 256, 128) - 1) == -4


# ---------------------------------------------------------------- refusals of the Python calls
def test_python_route_refuses():
    E = cq.CubicQuantError
    l = torch.zeros((4, 64))
    r = cq.cq_routes_empty(4, 64, 2, device="cpu")
    for bad in (lambda: cq.cq_route(l.double(), 2), lambda: cq.cq_route(l[0], 2), lambda: cq.cq_route(l.T, 2), lambda: cq.cq_route(l[:1].expand(4, 64), 2), lambda: cq.cq_route(l, 0),
                lambda: cq.cq_route(l, 2, bias=torch.zeros(63)), lambda: cq.cq_route(l, 2, bias=torch.zeros(64, dtype=torch.float64)), lambda: cq.cq_route(l, 3, out=r),
                lambda: cq.cq_route(torch.zeros((4, 32)), 2, out=r), lambda: cq.cq_route(l, 2, workspace=torch.zeros(4096)), lambda: cq.cq_route(l, 2, out=r, workspace=torch.zeros(1 << 16, dtype=torch.uint8)),
                lambda: cq.cq_route_workspace(4, 513)):
        with pytest.raises(E):
            bad()
    z = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    cq.Routes(z(4, 2), torch.zeros((4, 2)), z(8), z(5), z(4, 2))
    for bad in (lambda: cq.Routes(z(4, 2).long(), torch.zeros((4, 2)), z(8), z(5), z(4, 2)), lambda: cq.Routes(z(4, 2), z(4, 2), z(8), z(5), z(4, 2)),
                lambda: cq.Routes(z(4, 2), torch.zeros((4, 3)), z(8), z(5), z(4, 2)), lambda: cq.Routes(z(4, 2), torch.zeros((4, 2)), z(7), z(5), z(4, 2)),
                lambda: cq.Routes(z(4, 2), torch.zeros((4, 2)), z(8), z(1), z(4, 2)), lambda: cq.Routes(z(2, 4).T, torch.zeros((4, 2)), z(8), z(5), z(4, 2)),
                lambda: cq.Routes(z(4, 2), torch.zeros((4, 2)), z(8), [0, 8], z(4, 2)), lambda: cq.Routes(z(8), torch.zeros(8), z(8), z(5), z(8))):
        with pytest.raises(E):
            bad()
    y = torch.zeros((8, 16), dtype=torch.bfloat16)
    for bad in (lambda: cq.cq_combine(y.float(), r), lambda: cq.cq_combine(y[0], r), lambda: cq.cq_combine(y.T, r), lambda: cq.cq_combine(y, r, add=torch.zeros((4, 15), dtype=torch.bfloat16)),
                lambda: cq.cq_combine(y, r, add=torch.zeros((4, 16))), lambda: cq.cq_combine(y, r, out=torch.zeros((4, 16), dtype=torch.float16)),
                lambda: cq.cq_combine(y, r, out=torch.zeros((1, 16), dtype=torch.bfloat16).expand(4, 16)), lambda: cq.cq_combine(y, r)):
        with pytest.raises(E):
            bad()


def test_python_i8_refuses():
    E = cq.CubicQuantError
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    layout, scale = torch.zeros(512, dtype=torch.uint8), torch.zeros(512)
    w, w4, off, tok = cq.I8Tensor(layout, scale, 1, 128, 256), cq.I8Tensor(layout, scale, 4, 128, 256), torch.zeros(5, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    routed = cq.I8Tensor(layout, scale, 1, 3, 256, 3, off)
    for bad in (lambda: cq.cq_i8_quantize(x[:, :40]), lambda: cq.cq_i8_quantize(x.double()), lambda: cq.cq_i8_quantize(x.T), lambda: cq.cq_i8_quantize(x.expand(3, 4, 256)),
                lambda: cq.cq_i8_quantize(x[:1].expand(4, 256)), lambda: cq.cq_i8_quantize(x, route_token=tok), lambda: cq.cq_i8_quantize(x), lambda: cq.cq_i8_swiglu_quantize(x.float()),
                lambda: cq.cq_i8_swiglu_quantize(x[:, :48]), lambda: cq.cq_i8_pack(torch.zeros((4, 128), dtype=torch.uint8), torch.zeros(4)),
                lambda: cq.cq_i8_pack(torch.zeros((4, 128), dtype=torch.int8), torch.zeros(3)), lambda: cq.cq_i8_pack(torch.zeros((4, 130), dtype=torch.int8), torch.zeros(4)),
                lambda: cq.cq_i8_gemm(w, x[:, :128]), lambda: cq.cq_i8_gemm(w, x.float()), lambda: cq.cq_i8_gemm(w4, x), lambda: cq.cq_i8_gemm(w, routed),
                lambda: cq.cq_i8_gemm(w, cq.I8Tensor(layout, scale, 1, 4, 128)), lambda: cq.cq_i8_gemm(w, x, out=torch.zeros((4, 127), dtype=torch.bfloat16)),
                lambda: cq.cq_i8_gemm(w, x, out=torch.zeros((4, 128), dtype=torch.float16)), lambda: cq.cq_i8_gemm(w, x, workspace=torch.zeros(512)), lambda: cq.cq_i8_gemm(w, x, workspace=layout),
                lambda: cq.cq_i8_gemm(w, cq.I8Tensor(layout, scale, 1, 4, 256), out=torch.zeros((4, 128))),
                lambda: cq.cq_i8_gemm_routed(w4, x, tok, off[:4]), lambda: cq.cq_i8_gemm_routed(w4, x, tok, off.long()), lambda: cq.cq_i8_gemm_routed(w4, x, tok.long(), off),
                lambda: cq.cq_i8_gemm_routed(w4, x, None, off), lambda: cq.cq_i8_gemm_routed(w4, routed, None, off), lambda: cq.cq_i8_unpack(routed)):
        with pytest.raises(E):
            bad()
    gu, dn = cq.I8Tensor(layout, scale, 4, 256, 256), cq.I8Tensor(layout, scale, 4, 256, 128)
    r = cq.cq_routes_empty(4, 4, 2, device="cpu")
    for bad in (lambda: cq.cq_i8_moe(w4, dn, x, r), lambda: cq.cq_i8_moe(gu, dn, x[:, :128], r), lambda: cq.cq_i8_moe(gu, dn, x.float(), r), lambda: cq.cq_i8_moe(gu, dn, x[:3], r),
                lambda: cq.cq_i8_moe(gu, dn, x, cq.cq_routes_empty(4, 5, 2, device="cpu")), lambda: cq.cq_i8_moe(gu, dn, x, r, out=x[:, :128]), lambda: cq.cq_i8_moe(gu, dn, x, r, add=x.half()),
                lambda: cq.cq_i8_moe(gu, dn, x, r, workspace=layout)):
        with pytest.raises(E):
            bad()


def test_values_of_routed_rows_need_their_offsets():
    layout, scale = torch.zeros(3 * 16384, dtype=torch.uint8), torch.zeros(3)
    for offset in (None, torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int64), [0, 1, 2, 3]):
        with pytest.raises(cq.CubicQuantError, match="expert_offset"):
            cq.cq_i8_dequantize(cq.I8Tensor(layout, scale, 1, 3, 256, 3, offset))


@pytest.mark.parametrize("routed", [False, True])
def test_a_refused_quantiser_leaves_the_given_handle_as_it_was(monkeypatch, routed):
    class Refusing:
        def __getattr__(self, name):
            return lambda *a: -2

    monkeypatch.setattr(i8, "_here", lambda *a: None)
    monkeypatch.setattr(i8, "_L", Refusing())
    layout, scale, offset = torch.zeros(3 * 16384, dtype=torch.uint8), torch.zeros(3), torch.zeros(4, dtype=torch.int32)
    x, h, token = torch.zeros((3, 128), dtype=torch.bfloat16), torch.zeros((3, 256), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    for call in (lambda q: cq.cq_i8_quantize(x, *((token, offset.clone()) if routed else (None, None)), out=q),
                 lambda q: cq.cq_i8_swiglu_quantize(h, offset.clone() if routed else None, out=q)):
        q = cq.I8Tensor(layout, scale, 1, 3, 128, 3 if routed else 0, offset if routed else None)
        with pytest.raises(cq.CubicQuantError):
            call(q)
        assert q.expert_offset is (offset if routed else None)


def test_debug_plan_refuses():
    L, plan = i8._lib(), (ctypes.c_int64 * 4)()
    assert L.cq_debug_i8_plan(0, 4, 128, 256, 0, plan) == 0
    assert L.cq_debug_i8_plan(0, 4, 128, 256, 0, None) == -1 and L.cq_debug_i8_plan(-1, 4, 128, 256, 0, plan) == -1 and L.cq_debug_i8_plan(0, 0, 128, 256, 0, plan) == -1
    assert L.cq_debug_i8_plan(0, 4, 128, 264, 0, plan) == -2 and L.cq_debug_i8_plan(513, 4, 128, 256, 0, plan) == -2
    assert L.cq_debug_i8_plan(0, 1 << 30, 1 << 30, 256, 0, plan) == -2


def _cut(M, N, K, **how):
    return tuple(cq.cq_debug_i8_plan(M, N, K, **how).values())


def test_every_kind_of_tile_is_among_the_tested_shapes():
    """The shapes that the GPU tests multiply reach each way of cutting a product, and no drawn size reaches another."""
    rng = np.random.default_rng(5)
    for plan, M, N, K in PRODUCTS:
        assert _cut(M, N, K) == plan, (M, N, K)
    kinds = {(p, N % 8 == 0) for p, _, N, _ in PRODUCTS}
    for _ in range(6000):
        M, N, K = int(2 ** rng.uniform(0, 12.5)), int(2 ** rng.uniform(0, 16)), 16 * int(2 ** rng.uniform(0, 11))
        p = _cut(M, N, K)
        assert (p, N % 8 == 0) in kinds, (M, N, K, p)
        assert _cut(M, N, K, quantised=True) == ((128, 64, p[2], False) if p[3] else p)
    assert all(_cut(R, 512, 512, matrices=E) == (256, 256, 1, False) for E in (1, 3, 16, 512) for R in (1, 60, 800, 5000, 200000))


def test_few_rows_are_quantised_by_the_product():
    """At most sixteen rows whose codes fit beside the ring, and few enough that each block may quantise them."""
    own = lambda M, N, K: cq.cq_debug_i8_plan(M, N, K)["quantises"]  # noqa: E731
    assert own(1, 4096, 4096) and own(4, 4096, 4096) and not own(5, 4096, 4096) and own(16, 4096, 1024) and not own(17, 4096, 128)
    assert own(1, 264, 16384) and not own(1, 264, 16400) and not own(1, 30000, 8192) and not own(2, 4096, 14336)
