"""4-bit floating point, without a GPU: the oracle against tables and brute force, sizes, and every refusal of the C entries and of
the Python calls (found on the host before anything is launched)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2608_06763_b200 as cq
from fp4_shapes import PRODUCTS, ROUTED
from oracle import fp4 as ref
from paper_2608_06763_b200.fp4 import _lib

ONE, ODD = ctypes.c_void_p(16), ctypes.c_void_p(24)   # never dereferenced: validation fails first


def test_oracle_rounds_to_the_nearest_code():
    mids = {0.25: 0, 0.75: 2, 1.25: 2, 1.75: 4, 2.5: 4, 3.5: 6, 5.0: 6}   # ties: the even code
    for v, c in mids.items():
        assert ref.nearest_even(np.array([v]), ref.GRID)[0] == c
        assert ref.nearest_even(np.array([np.nextafter(v, 0)]), ref.GRID)[0] <= c
        assert ref.nearest_even(np.array([np.nextafter(v, 9)]), ref.GRID)[0] >= c
    assert ref.nearest_even(np.array([1e30, 6.0, 0.0]), ref.GRID).tolist() == [7, 7, 0]


def test_oracle_e4m3_table_is_that_of_torch():
    assert np.array_equal(ref.E4M3, torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_oracle_error_is_within_half_a_step(fmt):
    x = np.random.default_rng(0).standard_normal((16, 256)).astype(np.float32).astype(np.float64)
    c, b = ref.quantize(x, fmt)
    y, s = ref.values(c, b, fmt), ref.scale_values(b, fmt)
    step = np.repeat(s, ref.BLOCK[fmt], axis=-1)
    a = np.abs(x) / step
    # half of the grid's step where a lies; MXFP4 cuts at 6 what may reach 8, NVFP4 rounds its scale by 2^-4 at most
    half = np.where(a < 2, 0.25, np.where(a < 4, 0.5, np.maximum(1.0, a - 6)))
    assert np.all(np.abs(x - y) <= half * step * (1 + 1e-6))


def test_oracle_scales():
    x = np.zeros((1, 64))
    x[0, 0], x[0, 32] = 7.9, 8.0
    assert ref.quantize(x, "mx")[1].tolist() == [[127, 128]]
    assert ref.quantize(np.zeros((1, 32)), "mx")[1].tolist() == [[0]]
    assert ref.quantize(np.zeros((1, 16)), "nv")[1].tolist() == [[1]]      # 2^-9
    x = np.full((1, 16), 6.0)
    assert ref.quantize(x, "nv")[1].tolist() == [[0x38]]                   # 1.0
    x[0, 3] = np.nan
    c, b = ref.quantize(x, "nv")
    assert b.tolist() == [[127]] and not c.any() and np.isnan(ref.values(c, b, "nv")).all()


def test_sizes():
    L = _lib()
    assert L.cq_fp4_layout_bytes(0, 1, 128, 256) == 16384 + 1024
    assert L.cq_fp4_layout_bytes(1, 1, 128, 256) == 16384 + 2048
    assert L.cq_fp4_layout_bytes(1, 3, 129, 272) == 3 * 2 * 2 * 18432
    assert L.cq_fp4_layout_bytes(0, 1, 128, 48) == 0 and L.cq_fp4_layout_bytes(1, 1, 128, 48) > 0
    assert L.cq_fp4_layout_bytes(2, 1, 128, 256) == 0 and L.cq_fp4_layout_bytes(1, 0, 1, 256) == 0
    assert L.cq_fp4_routed_layout_bytes(1, 4, 2, 256) == 2 * 18432            # two rows fill two groups at most
    assert L.cq_fp4_routed_layout_bytes(1, 4, 512, 256) == 7 * 18432          # 512 = 128 + 1 + 1 + 382: 1 + 1 + 1 + 3 blocks, seven at most
    assert L.cq_fp4_routed_layout_bytes(1, 513, 512, 256) == 0
    assert L.cq_fp4_workspace_bytes(1, 1, 256) == 512 + 18432


def test_routed_layout_has_room_for_any_loads():
    rng = np.random.default_rng(1)
    for _ in range(300):
        E, R = int(rng.integers(1, 20)), int(rng.integers(1, 2000))
        cut = np.sort(rng.integers(0, R + 1, E - 1)) if rng.random() < 0.8 else np.minimum(np.arange(1, E), R)
        m = np.diff(np.concatenate([[0], cut, [R]]))
        assert ((m + 127) // 128).sum() * 18432 <= _lib().cq_fp4_routed_layout_bytes(1, E, R, 256)


def test_c_entries_refuse():
    L = _lib()
    ws = 1 << 20
    good = [ONE, None, ONE, 256, None, 1, ONE, 0, 4, 128, 256, ONE, ws, None]   # cq_fp4_linear

    def linear(**kw):
        names = ["w", "ws_", "x", "ldx", "xs", "fmt", "y", "f16", "M", "N", "K", "workspace", "bytes", "stream"]
        a = list(good)
        for k, v in kw.items():
            a[names.index(k)] = v
        return L.cq_fp4_linear(*a)

    assert linear(w=None) == -1 and linear(x=None) == -1 and linear(y=None) == -1 and linear(workspace=None) == -1
    assert linear(fmt=2) == -1 and linear(M=0) == -1 and linear(N=0) == -1 and linear(K=0) == -1 and linear(ldx=-1) == -1
    assert linear(K=264) == -2 and linear(fmt=0, K=272) == -2 and linear(M=1 << 31) == -2 and linear(N=1 << 30, M=1 << 30) == -2
    assert linear(ldx=255) == -1 and linear(ldx=260) == -3
    assert linear(x=ODD) == -3 and linear(y=ODD) == -3 and linear(w=ODD) == -3 and linear(workspace=ODD) == -3
    assert linear(bytes=511) == -4
    assert linear(fmt=0, xs=ONE) == -1 and linear(fmt=0, ws_=ONE) == -1      # MXFP4 has no tensor scale
    assert L.cq_fp4_gemm(ONE, None, ONE, None, 1, ONE, 0, 4, 128, 256, ONE, 511, None) == -4
    assert L.cq_fp4_gemm_routed(ONE, None, ONE, None, None, 4, 1, ONE, 0, 4, 128, 256, ONE, ws, None) == -1
    assert L.cq_fp4_gemm_routed(ONE, None, ONE, None, ONE, 513, 1, ONE, 0, 4, 128, 256, ONE, ws, None) == -2
    assert L.cq_fp4_gemm_routed(ONE, None, ONE, None, ONE, 0, 1, ONE, 0, 4, 128, 256, ONE, ws, None) == -1
    assert L.cq_fp4_linear_routed(ONE, None, ONE, 256, 8, None, None, ONE, 4, 1, ONE, 0, 4, 128, 256, ONE, ws, None) == -1
    assert L.cq_fp4_linear_routed(ONE, None, ONE, 256, 0, ONE, None, ONE, 4, 1, ONE, 0, 4, 128, 256, ONE, ws, None) == -1
    assert L.cq_fp4_quantize(ONE, 3, 256, 1, 1, 4, 256, None, ONE, None) == -1
    assert L.cq_fp4_quantize(ONE, 2, 258, 1, 1, 4, 256, None, ONE, None) == -3
    assert L.cq_fp4_quantize(ONE, 0, 256, 1, 1, 4, 256, None, ODD, None) == -3
    assert L.cq_fp4_swiglu_quantize(ONE, 2, 512, 1, 4, 256, None, 0, None, ONE, None) == -1   # h in the model dtype
    assert L.cq_fp4_swiglu_quantize(ONE, 0, 511, 1, 4, 256, None, 0, None, ONE, None) == -1   # rows of gate and up
    assert L.cq_fp4_dequantize(ONE, 1, 1, 4, 256, None, None, ODD, 0, None) == -3
    assert L.cq_fp4_pack(ONE, None, 1, 1, 4, 256, ONE, None) == -1 and L.cq_fp4_unpack(ONE, 1, 1, 4, 250, ONE, ONE, None) == -2


def test_python_refuses():
    E = cq.CubicQuantError
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    for bad in (lambda: cq.cq_fp4_quantize(x, 7), lambda: cq.cq_fp4_quantize(x[:, :40], cq.CQ_MXFP4), lambda: cq.cq_fp4_quantize(x.double(), 0),
                lambda: cq.cq_fp4_quantize(x.T, 0), lambda: cq.cq_fp4_quantize(x.expand(3, 4, 256), 0), lambda: cq.cq_fp4_quantize(x[:1].expand(4, 256), 0),
                lambda: cq.cq_fp4_quantize(x, cq.CQ_MXFP4, torch.ones(1)), lambda: cq.cq_fp4_quantize(x, cq.CQ_NVFP4, torch.ones(2)),
                lambda: cq.cq_fp4_quantize(x, cq.CQ_NVFP4, torch.ones(1, dtype=torch.float64)),
                lambda: cq.cq_fp4_quantize(x, cq.CQ_NVFP4, route_token=torch.zeros(3, dtype=torch.int32)),
                lambda: cq.cq_fp4_quantize(x, cq.CQ_NVFP4),                                       # not on a GPU
                lambda: cq.cq_fp4_swiglu_quantize(x.float(), 0), lambda: cq.cq_fp4_swiglu_quantize(x[:, :96], 0),
                lambda: cq.cq_fp4_pack(torch.zeros((4, 128), dtype=torch.uint8), torch.zeros((4, 7), dtype=torch.uint8), 0)):
        with pytest.raises(E):
            bad()
    # handles on the CPU stand in: every check below comes before a device is asked for
    layout = torch.zeros(512, dtype=torch.uint8)
    w = cq.Fp4Tensor(layout, cq.CQ_NVFP4, 1, 128, 256)
    w4 = cq.Fp4Tensor(layout, cq.CQ_NVFP4, 4, 128, 256)
    off = torch.zeros(5, dtype=torch.int32)
    tok = torch.zeros(3, dtype=torch.int32)
    routed = cq.Fp4Tensor(layout, cq.CQ_NVFP4, 1, 3, 256, None, 3, off)
    for bad in (lambda: cq.cq_fp4_gemm(w, x[:, :128]), lambda: cq.cq_fp4_gemm(w, x.float()), lambda: cq.cq_fp4_gemm(w4, x), lambda: cq.cq_fp4_gemm(w, routed),
                lambda: cq.cq_fp4_gemm(w, cq.Fp4Tensor(layout, cq.CQ_MXFP4, 1, 4, 256)), lambda: cq.cq_fp4_gemm(w, w, torch.ones(1)),
                lambda: cq.cq_fp4_gemm(w, x, out=torch.zeros((4, 127), dtype=torch.bfloat16)), lambda: cq.cq_fp4_gemm(w, x, out=torch.zeros((4, 128), dtype=torch.float16)),
                lambda: cq.cq_fp4_gemm(w, x, workspace=torch.zeros(512)), lambda: cq.cq_fp4_gemm(w, x, workspace=layout),
                lambda: cq.cq_fp4_gemm_routed(w4, x, tok, off[:4]), lambda: cq.cq_fp4_gemm_routed(w4, x, tok, off.long()), lambda: cq.cq_fp4_gemm_routed(w4, x, tok.long(), off),
                lambda: cq.cq_fp4_gemm_routed(w4, x, None, off), lambda: cq.cq_fp4_gemm_routed(w4, routed, None, off), lambda: cq.cq_fp4_unpack(routed)):
        with pytest.raises(E):
            bad()


def test_values_of_routed_rows_need_their_offsets():
    """A handle that no quantiser has filled has no offsets; without them the rows would be taken for whole matrices, one for each group."""
    layout = torch.zeros(3 * 18432, dtype=torch.uint8)
    for offset in (None, torch.zeros(3, dtype=torch.int32), torch.zeros(5, dtype=torch.int32), torch.zeros(4, dtype=torch.int64), [0, 1, 2, 3]):
        q = cq.Fp4Tensor(layout, cq.CQ_NVFP4, 1, 3, 256, None, 3, offset)
        for out in (None, torch.zeros((3, 256), dtype=torch.bfloat16)):
            with pytest.raises(cq.CubicQuantError, match="expert_offset"):
                cq.cq_fp4_dequantize(q, out=out)
    q = cq.cq_fp4_empty(cq.CQ_NVFP4, 3, 256, groups=3, device="cpu")
    with pytest.raises(cq.CubicQuantError, match="expert_offset"):
        cq.cq_fp4_dequantize(q)


@pytest.mark.parametrize("routed", [False, True])
def test_a_refused_quantiser_leaves_the_given_handle_as_it_was(monkeypatch, routed):
    """What a handle says of its rows changes with the rows, not before the call that writes them may still refuse."""
    from paper_2608_06763_b200 import fp4

    class Refusing:
        def __getattr__(self, name):
            return lambda *a: -2

    monkeypatch.setattr(fp4, "_here", lambda *a: None)
    monkeypatch.setattr(fp4, "_L", Refusing())
    layout = torch.zeros(3 * 18432, dtype=torch.uint8)
    scale, offset = torch.ones(1), torch.zeros(4, dtype=torch.int32)
    token = torch.zeros(3, dtype=torch.int32)
    x, h = torch.zeros((3, 256), dtype=torch.bfloat16), torch.zeros((3, 512), dtype=torch.bfloat16)
    for call in (lambda q: cq.cq_fp4_quantize(x, cq.CQ_NVFP4, torch.full((1,), 2.0), *((token, offset.clone()) if routed else (None, None)), out=q),
                 lambda q: cq.cq_fp4_swiglu_quantize(h, cq.CQ_NVFP4, torch.full((1,), 2.0), offset.clone() if routed else None, out=q)):
        q = cq.Fp4Tensor(layout, cq.CQ_NVFP4, 1, 3, 256, scale, 3 if routed else 0, offset if routed else None)
        with pytest.raises(cq.CubicQuantError):
            call(q)
        assert q.tensor_scale is scale and q.expert_offset is (offset if routed else None)


@pytest.mark.parametrize("dtype", [torch.float64, torch.int32, torch.uint8, torch.float32])
def test_products_of_quantised_rows_refuse_an_out_of_another_type(dtype):
    layout = torch.zeros(18432, dtype=torch.uint8)
    w = cq.Fp4Tensor(layout, cq.CQ_NVFP4, 1, 128, 256)
    x = cq.Fp4Tensor(layout, cq.CQ_NVFP4, 1, 4, 256)
    off = torch.zeros(2, dtype=torch.int32)
    routed = cq.Fp4Tensor(layout, cq.CQ_NVFP4, 1, 4, 256, None, 1, off)
    out = torch.zeros((4, 128), dtype=dtype)
    for bad in (lambda: cq.cq_fp4_gemm(w, x, out=out), lambda: cq.cq_fp4_gemm_routed(w, routed, None, off, out=out)):
        with pytest.raises(cq.CubicQuantError, match="out is"):
            bad()


def _cut(fmt, M, N, K, **how):
    return tuple(cq.cq_debug_fp4_plan(fmt, M, N, K, **how).values())


def test_tested_products_reach_every_kind_of_tile():
    """What the sizes of the GPU tests are for: no kind that a product of any size takes is left out."""
    rng = np.random.default_rng(4)
    for fmt in (0, 1):
        for plan, M, N, K in PRODUCTS:
            assert _cut(fmt, M, N, K) == plan, (fmt, M, N, K)
        kinds = {(p, N % 8 == 0) for p, _, N, _ in PRODUCTS}
        for _ in range(6000):
            M, N, K = int(2 ** rng.uniform(0, 12.5)), int(2 ** rng.uniform(0, 16)), 32 * int(2 ** rng.uniform(0, 10))
            p = _cut(fmt, M, N, K)
            assert (p, N % 8 == 0) in kinds, (fmt, M, N, K, p)
            if not p[3]:
                assert _cut(fmt, M, N, K, quantised=True) == p
            else:
                assert _cut(fmt, M, N, K, quantised=True) == (128, 64, p[2], False)
        for plan, counts, N, K in ROUTED:
            assert _cut(fmt, sum(counts), N, K, matrices=len(counts)) == plan + (1, False)
        routed = {p for p, _, _, _ in ROUTED}
        assert all(_cut(fmt, R, 512, 512, matrices=E)[:2] in routed for E in (1, 3, 16, 512) for R in (1, 60, 800, 5000, 200000))


def test_debug_plan_refuses():
    L, plan = _lib(), (ctypes.c_int64 * 4)()
    assert L.cq_debug_fp4_plan(1, 0, 4, 128, 256, 0, plan) == 0
    assert L.cq_debug_fp4_plan(1, 0, 4, 128, 256, 0, None) == -1 and L.cq_debug_fp4_plan(2, 0, 4, 128, 256, 0, plan) == -1
    assert L.cq_debug_fp4_plan(1, -1, 4, 128, 256, 0, plan) == -1 and L.cq_debug_fp4_plan(1, 0, 0, 128, 256, 0, plan) == -1
    assert L.cq_debug_fp4_plan(1, 0, 4, 128, 264, 0, plan) == -2 and L.cq_debug_fp4_plan(1, 513, 4, 128, 256, 0, plan) == -2
    assert L.cq_debug_fp4_plan(1, 0, 1 << 30, 1 << 30, 256, 0, plan) == -2


def test_products_quantise_themselves_where_that_was_measured_faster():
    own = lambda M, N, K: [cq.cq_debug_fp4_plan(fmt, M, N, K)["quantises"] for fmt in (0, 1)]  # noqa: E731
    for M, N, K in ((12, 4096, 4096), (16, 1024, 2048), (4, 28672, 4096), (4, 4096, 14336), (8, 2048, 8192), (12, 8192, 2048), (6, 6144, 4096)):
        assert own(M, N, K) == [True, True], (M, N, K)
    for M, N, K in ((13, 4096, 4096), (16, 4096, 4096), (13, 8192, 2048), (16, 8192, 2048), (5, 28672, 4096), (6, 4096, 14336), (11, 2048, 8192)):
        assert own(M, N, K) == [False, False], (M, N, K)
