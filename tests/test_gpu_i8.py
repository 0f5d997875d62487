"""8-bit integers with a scale for each row on the GPU against the oracle (oracle/i8.py).

Quantisers and exchanges: equal byte for byte (every decision is exact).  Products: sums are whole numbers, so the fp32 operations that follow have one result, and the
output is that, rounded once: equal bit for bit; and within half a step of the output type and three roundings to fp32 (the sum, the scales' product, theirs) of the
formula in 64 bits.
"""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2608_06763_b200 as cq
from i8_shapes import PRODUCTS, ROUTED
from oracle import i8 as ref
from oracle import route as ref_route

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def rows(M, K, dtype, seed, spread=1.0):
    """Normal values with a few large columns and magnitudes that differ from row to row."""
    r = np.random.default_rng(seed)
    x = r.standard_normal((M, K)) * np.exp(spread * r.standard_normal((M, 1)))
    x[:, r.integers(0, K, max(1, K // 100))] *= 20
    return torch.from_numpy(x).float().to(DTYPE[dtype])


def as64(t):
    return t.detach().double().cpu().numpy()


def check_codes(q, codes, scale):
    c, s = cq.cq_i8_unpack(q)
    assert np.array_equal(s.cpu().numpy(), scale, equal_nan=True), "scales"
    assert np.array_equal(c.cpu().numpy(), codes), "codes"


def bits(t):
    return t.view(torch.int16)


def check_product(got, exact, in32):
    """in32: fp32 before the last rounding."""
    want = torch.from_numpy(np.ascontiguousarray(in32)).to(got.dtype)
    same = bits(got.cpu()) == bits(want)
    assert bool((same | (torch.isnan(got.cpu()) & torch.isnan(want))).all()), int((~same).sum())
    err, fine = np.abs(as64(got) - exact), np.isfinite(as64(want))
    allowed = (torch.finfo(got.dtype).eps / 2 + 3.01 * 2.0 ** -24) * np.abs(exact) + torch.finfo(got.dtype).tiny
    assert np.all(err[fine] <= allowed[fine])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,K", [(1, 16), (3, 64), (5, 352), (128, 128), (130, 4096), (257, 1408), (400, 304), (2, 70000 // 16 * 16), (300, 20000), (1, 131072)])
def test_quantize(M, K, dtype):
    x = rows(M, K, dtype, seed=M + K)
    q = cq.cq_i8_quantize(x.cuda())
    codes, scale = ref.quantize(as64(x))
    check_codes(q, codes, scale)
    for out in (torch.bfloat16, torch.float16, torch.float32):
        want = torch.from_numpy(codes.astype(np.float32) * scale[:, None]).to(out)
        assert torch.equal(cq.cq_i8_dequantize(q, out).cpu(), want)


def test_quantize_ties_extremes_and_non_finite():
    K = 256
    x = torch.zeros((20, K))
    half = torch.arange(-127, 127).float() + 0.5
    for j, top in enumerate((127.0, 254.0, 127.0 * 2.0 ** -20, 127.0 * 2.0 ** 30)):     # the scale is a power of two, every border exactly hit
        x[j, :254] = half * (top / 127)
        x[j, 255] = top
    x[4] = torch.nextafter(x[0], torch.tensor(1e9))
    x[4, 255] = 127.0
    x[5] = torch.nextafter(x[0], torch.tensor(-1e9))
    x[5, 255] = 127.0
    x[6, 5], x[7, 40], x[8, 0] = float("inf"), float("nan"), -float("inf")
    x[9], x[10], x[11], x[12, ::3] = 1e-12, 2.0 ** -149, 3.3e38, 1e-10
    x[13, 100] = 1.0
    x[14] = torch.linspace(-1, 1, K)
    x[15] = torch.linspace(-3.0, 0.1, K)
    for dtype in ("f32", "bf16", "f16"):
        xd = x.to(DTYPE[dtype])
        q = cq.cq_i8_quantize(xd.cuda())
        check_codes(q, *ref.quantize(as64(xd)))
        values = as64(cq.cq_i8_dequantize(q, torch.float32))
        assert np.isnan(values[6:9]).all() and np.isfinite(values[9]).all()


def test_quantize_near_borders():
    """Quotients within a few units of a half, scales of every kind: the decision is that of the quotient in fp32."""
    r = np.random.default_rng(7)
    M, K = 600, 512
    top = np.exp(r.uniform(-20, 20, (M, 1))).astype(np.float32)
    d = (top / np.float32(127)).astype(np.float64)
    x = ((r.integers(-126, 126, (M, K)) + 0.5) * d).astype(np.float32)
    x = (x.view(np.int32) + r.integers(-3, 4, (M, K)).astype(np.int32)).view(np.float32)
    x[:, :1] = top
    q = cq.cq_i8_quantize(torch.from_numpy(x).cuda())
    check_codes(q, *ref.quantize(x.astype(np.float64)))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_quantize_all_16bit_values(dtype):
    p = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(DTYPE[dtype])
    x = torch.zeros((65536, 16), dtype=DTYPE[dtype])
    x[:, 3] = p
    x[:, 4] = p.flip(0)
    x[:, 9] = p.roll(77)
    check_codes(cq.cq_i8_quantize(x.cuda()), *ref.quantize(as64(x)))


def test_the_quantiser_is_that_of_dynamic_a8():
    x = rows(40, 2048, "bf16", 3).cuda()
    x8, dx = cq.cq_quantize_a8(x)
    c, s = cq.cq_i8_unpack(cq.cq_i8_quantize(x))
    assert torch.equal(c, x8) and torch.equal(s, dx.view(-1))


def test_strided_rows_several_matrices_and_checkpoints():
    wide = rows(70, 512, "bf16", 5).cuda()
    x = wide[:, 64:64 + 320]
    check_codes(cq.cq_i8_quantize(x), *ref.quantize(as64(x)))
    w = torch.stack([rows(130, 288, "f32", 6 + e) for e in range(3)])
    q = cq.cq_i8_quantize(w.cuda())
    parts = [ref.quantize(as64(w[e])) for e in range(3)]
    check_codes(q, np.stack([p[0] for p in parts]), np.stack([p[1] for p in parts]))
    codes = torch.from_numpy(np.random.default_rng(0).integers(-128, 128, (3, 130, 288)).astype(np.int8)).cuda()
    scale = torch.rand((3, 130), device="cuda")
    c, s = cq.cq_i8_unpack(cq.cq_i8_pack(codes, scale))
    assert torch.equal(c, codes) and torch.equal(s, scale)
    assert torch.equal(cq.cq_i8_dequantize(cq.cq_i8_pack(codes, scale), torch.float32), codes.float() * scale[..., None])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,I", [(1, 16), (7, 1408), (300, 4096), (2, 40000), (400, 17008), (13, 14336)])
def test_swiglu_quantize(M, I, dtype):
    h = rows(M, 2 * I, dtype, seed=M + I, spread=0.5)
    v = as64(h)
    act = torch.from_numpy(ref.gated(v[:, :I], v[:, I:])).to(DTYPE[dtype])
    check_codes(cq.cq_i8_swiglu_quantize(h.cuda()), *ref.quantize(as64(act)))


def test_swiglu_far_gates_subnormal_and_non_finite():
    I = 64
    for dtype in ("bf16", "f16"):
        top = 300.0 if dtype == "bf16" else 100.0
        gate = torch.linspace(-top, top, 16 * I).reshape(16, I)
        up = torch.tensor([1.0, -2.0, 1e-6, 3e4]).repeat(4)[:, None].expand(16, I)
        h = torch.cat([gate, up], dim=1).to(DTYPE[dtype])
        if dtype == "bf16":
            h[1, 0], h[2, 1], h[1, I], h[2, I + 1] = 3.3e38, 2.4e38, 0.5, 1e-20
            h[4, :I] = -50.0
            h[4, I:] = 1e37                                   # gate * up leaves fp32, the activation does not
        h[3, 7], h[5, I + 9], h[6, 2] = float("nan"), float("inf"), -float("inf")
        v = as64(h)
        act = torch.from_numpy(ref.gated(v[:, :I], v[:, I:])).to(DTYPE[dtype])
        check_codes(cq.cq_i8_swiglu_quantize(h.cuda()), *ref.quantize(as64(act)))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,I", [(6000, 32), (3000, 272), (20, 100000)])
def test_swiglu_roundings_that_32_bits_leave_open(M, I, dtype):
    """Short rows, whose largest value is open often, rows beyond what is kept of them, and activations about the least half."""
    h = rows(M, 2 * I, dtype, seed=M, spread=0.5)
    h[M // 3: M // 2] *= 1e-3 if dtype == "f16" else 1e-18
    h[M // 2: M // 2 + 5] *= 2e-4 if dtype == "f16" else 1e-19
    h[-1] = 0
    v = as64(h)
    act = torch.from_numpy(ref.gated(v[:, :I], v[:, I:])).to(DTYPE[dtype])
    check_codes(cq.cq_i8_swiglu_quantize(h.cuda()), *ref.quantize(as64(act)))


@pytest.mark.parametrize("K", [8192, 14336 + 16, 40000])
def test_few_long_routed_rows(K):
    """Rows that several blocks share, of groups: as the same rows by themselves, tokens out of range as zeros, rows behind the last left alone."""
    x = rows(5, 2 * K, "bf16", K, 1.0).cuda()
    token = torch.tensor([4, 0, 9, 4, 2, -1, 1, 3], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 3, 3, 7], dtype=torch.int32, device="cuda")
    live, t = 7, token.clamp(0, 4).long()
    inside = ((token >= 0) & (token < 5))[:, None]
    taken = torch.where(inside, x[:, :K][t], torch.zeros((), dtype=x.dtype, device="cuda")).contiguous()
    q, one = cq.cq_i8_quantize(x[:, :K], route_token=token, expert_offset=off), cq.cq_i8_quantize(taken)
    left = torch.full((8, K), 7.0, dtype=torch.bfloat16, device="cuda")
    cq.cq_i8_dequantize(q, out=left)
    assert torch.equal(left[:live], cq.cq_i8_dequantize(one)[:live]) and torch.all(left[live:] == 7.0) and torch.equal(q.scale[:live], one.scale[:live])
    h = x[t].contiguous()
    a, b = cq.cq_i8_swiglu_quantize(h, expert_offset=off), cq.cq_i8_swiglu_quantize(h)
    assert torch.equal(cq.cq_i8_dequantize(a)[:live], cq.cq_i8_dequantize(b)[:live]) and torch.equal(a.scale[:live], b.scale[:live])
    check_codes(b, *ref.quantize(torch.from_numpy(ref.gated(as64(h[:, :K]), as64(h[:, K:]))).bfloat16().double().numpy()))


def product_case(M, N, K, dtype, seed=0):
    r = np.random.default_rng(seed)
    wc, wd = r.integers(-128, 128, (N, K)).astype(np.int8), (0.001 * np.exp(0.5 * r.standard_normal(N))).astype(np.float32)
    x = rows(M, K, dtype, seed + 1, 0.3)
    xc, xd = ref.quantize(as64(x))
    w = cq.cq_i8_pack(torch.from_numpy(wc).cuda(), torch.from_numpy(wd).cuda())
    return w, x.cuda(), *ref.product(xc, xd, wc, wd)


SMALL = [(1, 128, 16), (1, 128, 128), (1, 128, 256), (16, 128, 128), (5, 200, 528), (128, 256, 1024), (129, 128, 304), (256, 130, 768)]


@pytest.mark.parametrize("M,N,K", SMALL)
def test_gemm_small(M, N, K):
    w, x, y, y32 = product_case(M, N, K, "bf16")
    check_product(cq.cq_i8_gemm(w, x), y, y32)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (2, 1001, 2816), (13, 6144, 4096), (16, 4096, 14336), (17, 513, 5632), (40, 1024, 1024), (100, 2816, 2048), (200, 4096, 1408),
                                   (300, 700, 4096), (513, 1024, 512), (1000, 2050, 288), (65, 300, 1024), (449, 1100, 2048), (1024, 6144, 512), (1, 28672, 2048), (9, 20100, 1312)])
def test_gemm(M, N, K, dtype):
    w, x, y, y32 = product_case(M, N, K, dtype)
    ws = cq.cq_i8_workspace(w, M)
    got = cq.cq_i8_gemm(w, x, workspace=ws)
    assert got.dtype == DTYPE[dtype]
    check_product(got, y, y32)
    assert torch.equal(cq.cq_i8_gemm(w, x, workspace=ws), got)          # the same bits again
    q = cq.cq_i8_quantize(x)
    assert torch.equal(cq.cq_i8_gemm(w, q, out=torch.full_like(got, 7.0)), got)
    assert cq.cq_gemm_status(ws) == 0


@pytest.mark.parametrize("M,N", [(70, n) for n in (1, 2, 3, 5, 6, 7, 8, 9, 15, 121, 122, 123, 124, 125, 126, 127, 129, 135, 249, 250)] + [(700, 259), (700, 381), (33, 1003), (300, 1134)])
def test_rows_of_y_of_any_length(M, N):
    """Rows of y that start at any value of a sixteen-byte piece, last row blocks of any width; nothing behind y is touched."""
    w, x, y, y32 = product_case(M, N, 48, "bf16", seed=N)
    room = torch.full((M * N + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    got = cq.cq_i8_gemm(w, x, out=room[:M * N].view(M, N))
    check_product(got, y, y32)
    assert torch.all(room[M * N:] == 7.0)


@pytest.mark.parametrize("M", [2, 40, 200])
def test_gemm_of_the_largest_sums(M):
    """All products -128 * 127 (or that with another sign) over the longest K: the sums stay within 32 bits."""
    K, N = 131072, 128
    wc = np.full((N, K), -128, np.int8)
    wc[1::2] = 127
    x = torch.ones((M, K), dtype=torch.bfloat16)
    x[1::2] = -1.0
    wd = np.full(N, 2.0 ** -20, np.float32)
    xc, xd = ref.quantize(as64(x))
    y, y32 = ref.product(xc, xd, wc, wd)
    check_product(cq.cq_i8_gemm(cq.cq_i8_pack(torch.from_numpy(wc).cuda(), torch.from_numpy(wd).cuda()), x.cuda()), y, y32)


@pytest.mark.parametrize("M", [4, 20, 200])
def test_gemm_non_finite_rows_stay_alone(M):
    w, x, y, y32 = product_case(M, 256, 512, "bf16")
    x[1, 100] = float("nan")
    x[3, 500] = float("inf")
    got = cq.cq_i8_gemm(w, x)
    bad = np.isin(np.arange(M), (1, 3))
    assert torch.isnan(got[torch.from_numpy(bad).cuda()]).all()
    keep = torch.from_numpy(~bad).cuda()
    check_product(got[keep], y[~bad], y32[~bad])
    x.zero_()
    assert torch.all(cq.cq_i8_gemm(w, x) == 0)


def routed_case(counts, N, K, dtype, seed=0, T=50):
    E, R = len(counts), sum(counts)
    r = np.random.default_rng(seed)
    x = rows(T, K, dtype, seed + 1, 0.3)
    token = r.integers(0, T, R).astype(np.int32)
    off = np.concatenate([[0], np.cumsum(counts)])
    wc, wd = r.integers(-128, 128, (E, N, K)).astype(np.int8), (0.001 * np.exp(0.5 * r.standard_normal((E, N)))).astype(np.float32)
    xc, xd = ref.quantize(as64(x))
    y, y32 = np.zeros((R, N)), np.zeros((R, N), np.float32)
    for e in range(E):
        t, part = token[off[e]:off[e + 1]], slice(off[e], off[e + 1])
        if len(t):
            y[part], y32[part] = ref.product(xc[t], xd[t], wc[e], wd[e])
    w = cq.cq_i8_pack(torch.from_numpy(wc).cuda(), torch.from_numpy(wd).cuda())
    return w, x.cuda(), torch.from_numpy(token).cuda(), torch.tensor(off, dtype=torch.int32).cuda(), y, y32


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("counts", [[1], [3, 0, 5, 1], [0, 0, 7], [128, 1, 129, 0, 300, 16], [1] * 40, [700, 2], [100, 3, 0, 65, 1, 1, 1, 1, 129, 1], [300, 0, 700, 257, 1000]])
def test_gemm_routed(counts, dtype):
    N, K = 260, 544
    w, x, token, off, y, y32 = routed_case(counts, N, K, dtype)
    ws = cq.cq_i8_workspace(w, sum(counts))
    got = cq.cq_i8_gemm_routed(w, x, token, off, workspace=ws)
    check_product(got, y, y32)
    q = cq.cq_i8_quantize(x, route_token=token, expert_offset=off)
    assert torch.equal(cq.cq_i8_gemm_routed(w, q, None, off, out=torch.empty_like(got)), got)
    assert cq.cq_gemm_status(ws) == 0
    codes, scale = ref.quantize(as64(x))
    values = codes.astype(np.float32) * scale[:, None]
    assert np.array_equal(cq.cq_i8_dequantize(q, torch.float32).cpu().numpy(), values[token.cpu().numpy()])


@pytest.mark.parametrize("plan,M,N,K", PRODUCTS)
def test_every_kind_of_tile(plan, M, N, K):
    """bfloat16 and binary16 in turn; from rows in the model dtype and from quantised ones, which have the same bits."""
    assert tuple(cq.cq_debug_i8_plan(M, N, K).values()) == plan
    w, x, y, y32 = product_case(M, N, K, "bf16" if M % 2 else "f16", seed=M)
    ws = cq.cq_i8_workspace(w, M)
    got = cq.cq_i8_gemm(w, x, workspace=ws)
    check_product(got, y, y32)
    out = torch.full_like(got, 7.0)
    assert torch.equal(cq.cq_i8_gemm(w, cq.cq_i8_quantize(x), workspace=ws, out=out), got)
    assert cq.cq_gemm_status(ws) == 0


@pytest.mark.parametrize("counts,N,K", ROUTED)
def test_every_kind_of_routed_tile(counts, N, K):
    w, x, token, off, y, y32 = routed_case(counts, N, K, "bf16" if N % 2 else "f16", seed=N, T=150)
    ws = cq.cq_i8_workspace(w, sum(counts))
    got = cq.cq_i8_gemm_routed(w, x, token, off, workspace=ws)
    check_product(got, y, y32)
    q = cq.cq_i8_quantize(x, route_token=token, expert_offset=off)
    assert torch.equal(cq.cq_i8_gemm_routed(w, q, None, off, workspace=ws, out=torch.full_like(got, 7.0)), got)
    assert cq.cq_gemm_status(ws) == 0


def repaired(offset, R):
    """Offsets as the calls take them: the largest so far, within [0, R]."""
    return np.maximum.accumulate(np.clip(offset, 0, R))


ASTRAY = {"descends": [0, 10, 5, 28], "behind the rows": [0, 10, 22, 99], "negative": [-3, 10, 22, 28], "starts late": [4, 10, 12, 28], "starts behind": [41, 0, 0, 0],
          "all at once": [9, -5, 200, 3], "none": [0, 0, 0, 0], "descends at 32": list(range(33)) + [7] * 4 + [38]}


@pytest.mark.parametrize("name", ASTRAY)
def test_offsets_that_go_astray_and_tokens_out_of_range(name):
    """Every row against the matrix that it belongs to; rows of no group are left as they were: by product, quantiser, gated activation and inverse."""
    offset, R, N, K, I = ASTRAY[name], 40, 136, 256, 64
    E = len(offset) - 1
    r = np.random.default_rng(E)
    wc, wd = r.integers(-128, 128, (E, N, K)).astype(np.int8), np.full((E, N), 0.001, np.float32)
    w = cq.cq_i8_pack(torch.from_numpy(wc).cuda(), torch.from_numpy(wd).cuda())
    x, token = rows(50, K, "bf16", 7, 0.3), r.integers(0, 50, R).astype(np.int32)
    token[[6, 25]] = -1, 50
    off = torch.tensor(offset, dtype=torch.int32, device="cuda")
    true = repaired(offset, R)
    mine = np.zeros(R, bool)
    mine[true[0]:true[-1]] = True
    xr = np.where(((token >= 0) & (token < 50))[:, None], as64(x)[np.clip(token, 0, 49)], 0.0)
    xc, xd = ref.quantize(xr)
    y, y32 = np.zeros((R, N)), np.zeros((R, N), np.float32)
    for e in range(E):
        part = slice(true[e], true[e + 1])
        if true[e] < true[e + 1]:
            y[part], y32[part] = ref.product(xc[part], xd[part], wc[e], wd[e])
    out = torch.full((R, N), 7.0, dtype=torch.bfloat16, device="cuda")
    tok = torch.from_numpy(token).cuda()
    q = cq.cq_i8_empty(R, K, groups=E)
    q.scale.fill_(7.0)
    cq.cq_i8_quantize(x.cuda(), route_token=tok, expert_offset=off, out=q)
    keep, rest = torch.from_numpy(mine).cuda(), torch.from_numpy(~mine).cuda()
    assert torch.all(q.scale[rest] == 7.0)
    for call in (lambda: cq.cq_i8_gemm_routed(w, x.cuda(), tok, off, out=out), lambda: cq.cq_i8_gemm_routed(w, q, None, off, out=out)):
        out.fill_(7.0)
        call()
        check_product(out[keep], y[mine], y32[mine])
        assert torch.all(out[rest] == 7.0)
    back = cq.cq_i8_dequantize(q, out=torch.full((R, K), 7.0, device="cuda"))
    assert np.array_equal(back.cpu().numpy(), np.where(mine[:, None], xc.astype(np.float32) * xd[:, None], 7.0))
    h = rows(R, 2 * I, "bf16", 8, 0.3)
    v = as64(h)
    ac, ad = ref.quantize(as64(torch.from_numpy(ref.gated(v[:, :I], v[:, I:])).to(torch.bfloat16)))
    a = cq.cq_i8_swiglu_quantize(h.cuda(), expert_offset=off)
    back = cq.cq_i8_dequantize(a, out=torch.full((R, I), 7.0, device="cuda"))
    assert np.array_equal(back.cpu().numpy(), np.where(mine[:, None], ac.astype(np.float32) * ad[:, None], 7.0))


@pytest.mark.parametrize("M,N,K", [(3, 130, 288), (20, 300, 1056), (100, 200, 512), (300, 900, 800)])
def test_what_lies_behind_the_last_row_reaches_nothing(M, N, K):
    """Layouts and workspaces full of other codes beforehand: the same results, and not a byte of the rows behind the last written."""
    w, x, y, y32 = product_case(M, N, K, "bf16")
    codes, scale = cq.cq_i8_unpack(w)
    q = cq.cq_i8_empty(N, K)
    q.layout.fill_(0x55)
    from paper_2608_06763_b200.i8 import _check, _lib, _stream
    _check(_lib().cq_i8_pack(codes.data_ptr(), 1, N, K, q.layout.data_ptr(), _stream()), "pack")
    q.scale = scale
    ws = cq.cq_i8_workspace(w, M)
    ws[512:].fill_(255)
    check_product(cq.cq_i8_gemm(q, x, workspace=ws), y, y32)
    xq = cq.cq_i8_empty(M, K)
    xq.layout.fill_(0x55)
    xq.scale.fill_(float("nan"))
    cq.cq_i8_quantize(x, out=xq)
    check_product(cq.cq_i8_gemm(q, xq), y, y32)
    last = xq.layout.view(-1, (K + 127) // 128, 16384)[-1]
    used = (M - 1) % 128 + 1
    assert torch.all(last[:, used * 128:] == 0x55)


@pytest.mark.parametrize("M,N,K", [(1, 300, 512), (9, 300, 512), (16, 600, 8192), (70, 300, 512), (300, 9843, 864)])
def test_rows_apart(M, N, K):
    """x as columns of a wider matrix, a single row at any distance: the bits of a copy."""
    w, x, y, y32 = product_case(M, N, K, "bf16")
    wide = torch.full((M, K + 96), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, 64:64 + K] = x
    part = wide[:, 64:64 + K]
    check_product(cq.cq_i8_gemm(w, part), y, y32)
    token, off = torch.arange(M, dtype=torch.int32, device="cuda"), torch.tensor([0, M], dtype=torch.int32, device="cuda")
    check_product(cq.cq_i8_gemm_routed(w, part, token, off), y, y32)
    if M == 1:
        odd = torch.zeros((3, K + 8), dtype=x.dtype, device="cuda")
        odd[1, :K] = x[0]
        check_product(cq.cq_i8_gemm(w, odd[1:2, :K].as_strided((1, K), (3, 1), odd[1].storage_offset())), y, y32)


def test_two_streams_and_two_graphs():
    """Two products at once on two streams, two captured graphs over one workspace replayed in turn, operands that another stream makes."""
    cases = [product_case(M, 2048, 1024, "bf16", seed=50 + M) for M in (4, 40, 200)]
    want = [cq.cq_i8_gemm(w, x) for w, x, _, _ in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], []
    for _ in range(20):
        for st, (w, x, _, _) in zip(streams, cases):
            with torch.cuda.stream(st):
                got.append(cq.cq_i8_gemm(w, x))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[i % 3]) for i, a in enumerate(got))
    ws = cq.cq_i8_workspace(cases[2][0], 200)
    graphs, outs = [], []
    for w, x, _, _ in cases:
        out = torch.empty((x.shape[0], 2048), dtype=x.dtype, device="cuda")
        cq.cq_i8_gemm(w, x, workspace=ws, out=out)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            cq.cq_i8_gemm(w, x, workspace=ws, out=out)
        graphs.append(graph)
        outs.append(out)
    for _ in range(10):
        for graph, out, y in zip(graphs, outs, want):
            out.zero_()
            graph.replay()
            assert torch.equal(out, y)
    assert cq.cq_gemm_status(ws) == 0
    side = torch.cuda.Stream()
    for w, x, _, _ in cases:
        y = cq.cq_i8_gemm(w, x)
        for _ in range(10):
            late = torch.full_like(x, float("nan"))
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                torch.cuda._sleep(200000)
                late.copy_(x)
            torch.cuda.current_stream().wait_stream(side)
            assert torch.equal(cq.cq_i8_gemm(w, late), y)


@pytest.mark.parametrize("M,N,K", [(5, 24000, 200), (2, 20100, 1312), (40, 20100, 1312), (60, 24000, 144), (200, 24000, 400), (600, 9600, 272)])
def test_many_output_tiles_called_often(M, N, K):
    """Several output tiles to a CTA, an odd number of stages each: called often, always the same bits."""
    K = K // 16 * 16
    w, x, y, y32 = product_case(M, N, K, "bf16")
    ws = cq.cq_i8_workspace(w, M)
    want = cq.cq_i8_gemm(w, x, workspace=ws)
    check_product(want, y, y32)
    out = torch.empty_like(want)
    for i in range(200):
        cq.cq_i8_gemm(w, x, workspace=ws, out=out)
        if i % 20 == 0:
            assert torch.equal(out, want)
    assert torch.equal(out, want) and cq.cq_gemm_status(ws) == 0


def test_long_rows_and_a_layout_beyond_two_gigabytes():
    M, K = 540000, 8192
    x = torch.randn((256, K), generator=torch.Generator("cuda").manual_seed(3), device="cuda").bfloat16().repeat(M // 256 + 1, 1)[:M]
    q = cq.cq_i8_quantize(x)
    assert q.layout.numel() > 2 ** 32 and x.numel() > 2 ** 32
    few = cq.cq_i8_quantize(x[:256])
    v, ref_v = cq.cq_i8_dequantize(q), cq.cq_i8_dequantize(few)
    for lo in (0, 262144, 2 ** 32 // K // 256 * 256, M // 256 * 256 - 256):
        assert torch.equal(v[lo:lo + 256], ref_v)
    assert torch.equal(v[M // 256 * 256:], ref_v[:M % 256])
    small = torch.randn((40, K), device="cuda").bfloat16()
    y, part = cq.cq_i8_gemm(q, small), cq.cq_i8_gemm(few, small)
    for lo in (0, 2 ** 32 // K // 256 * 256, M // 256 * 256 - 256):
        assert torch.equal(y[:, lo:lo + 256], part)


# ---------------------------------------------------------------- as they are used
def moe_oracle(x, expert, weight, up, down, dtype):
    """The expert block from codes, in the order of the definition: every product and the activation rounded to the model dtype."""
    T, H = x.shape
    E, I = down[0].shape[0], down[0].shape[2]
    token, off, row = ref_route.routes(expert, E)
    y = np.zeros((T * expert.shape[1], H))
    xc, xd = ref.quantize(x)
    for e in range(E):
        t = token[off[e]:off[e + 1]]
        if not len(t):
            continue
        h = torch.from_numpy(ref.product(xc[t], xd[t], up[0][e], up[1][e])[1]).to(dtype).double().numpy()
        act = torch.from_numpy(ref.gated(h[:, :I], h[:, I:])).to(dtype).double().numpy()
        y[off[e]:off[e + 1]] = torch.from_numpy(ref.product(*ref.quantize(act), down[0][e], down[1][e])[1]).to(dtype).double().numpy()
    return ref_route.combine(y, weight, row)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T", [1, 24, 600])
def test_expert_block_from_logits(T, dtype):
    """Routing, experts and combining from a captured graph that follows new tokens and loads; padded rows; equal to the calls one after another."""
    E, H, I, top = 6, 512, 288, 3
    r = np.random.default_rng(11)
    up = (r.integers(-127, 128, (E, 2 * I, H)).astype(np.int8), (0.0005 * np.exp(0.3 * r.standard_normal((E, 2 * I)))).astype(np.float32))
    down = (r.integers(-127, 128, (E, H, I)).astype(np.int8), (0.0005 * np.exp(0.3 * r.standard_normal((E, H)))).astype(np.float32))
    wu, wd = (cq.cq_i8_pack(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()) for c, s in (up, down))
    x = torch.zeros((T, H), dtype=DTYPE[dtype], device="cuda")
    l, bias = torch.zeros((T, E), device="cuda"), torch.from_numpy(0.05 * r.standard_normal(E)).float().cuda()
    shared, y = torch.zeros_like(x), torch.zeros_like(x)
    routes, ws, rws = cq.cq_routes_empty(T, E, top), cq.cq_i8_moe_workspace(wu, wd, T, top), cq.cq_route_workspace(T, E)

    def block():
        cq.cq_route(l, top, cq.CQ_SIGMOID, bias=bias, scale=1.5, workspace=rws, out=routes)
        cq.cq_i8_moe(wu, wd, x, routes, add=shared, workspace=ws, out=y)

    block()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    for seed in range(3):
        xs, ls = rows(T, H, dtype, 100 + seed, 0.3), torch.from_numpy(np.random.default_rng(seed).standard_normal((T, E))).float()
        ls[:, 4] -= 20.0 * seed                                        # a matrix without rows
        if T > 1:
            ls[T - T // 4:] = -float("inf")                            # padding
        add = rows(T, H, dtype, 200 + seed, 0.1)
        x.copy_(xs)
        l.copy_(ls)
        shared.copy_(add)
        y.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        expert, _ = ref_route.choose(as64(ls), top, "sigmoid", as64(bias))
        assert np.array_equal(routes.expert.cpu().numpy(), expert)
        want, size = moe_oracle(as64(xs), expert, as64(routes.weight), up, down, DTYPE[dtype])
        want, size = want + as64(add), size + np.abs(as64(add))
        err = np.abs(as64(y) - want)
        allowed = torch.finfo(y.dtype).eps / 2 * np.abs(want) * (1 + 2.0 ** -10) + (top + 1) * 2.0 ** -24 * size + torch.finfo(y.dtype).tiny
        assert np.all(err <= allowed), float((err / allowed).max())
        h = cq.cq_i8_gemm_routed(wu, x, routes.token, routes.offset)
        a = cq.cq_i8_swiglu_quantize(h, expert_offset=routes.offset)
        yr = cq.cq_i8_gemm_routed(wd, a, None, routes.offset, out=torch.empty((T * top, H), dtype=x.dtype, device="cuda"))
        assert torch.equal(cq.cq_combine(yr, routes, add=shared), y)
        assert torch.equal(cq.cq_i8_moe(wu, wd, x, routes, add=shared), y)
    assert cq.cq_gemm_status(ws) == 0


@pytest.mark.parametrize("T,E,top,H,I", [(1, 1, 1, 16, 16), (5, 512, 32, 48, 80), (64, 512, 1, 144, 16), (33, 60, 4, 272, 336), (700, 3, 2, 1040, 144), (300, 2, 2, 16, 1296)])
def test_expert_block_of_odd_sizes(T, E, top, H, I):
    """Most matrices without rows, one matrix with all, lengths that end inside a tile, tokens with fewer choices than asked for or none."""
    r = np.random.default_rng(T + E)
    up = (r.integers(-127, 128, (E, 2 * I, H)).astype(np.int8), (0.002 * np.exp(0.3 * r.standard_normal((E, 2 * I)))).astype(np.float32))
    down = (r.integers(-127, 128, (E, H, I)).astype(np.int8), (0.002 * np.exp(0.3 * r.standard_normal((E, H)))).astype(np.float32))
    wu, wd = (cq.cq_i8_pack(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()) for c, s in (up, down))
    x, l = rows(T, H, "bf16", T, 0.3), torch.from_numpy(r.standard_normal((T, E))).float()
    if T > 1:
        l[torch.from_numpy(r.random((T, E)) < 0.4)] = -float("inf")
        l[T // 2] = -float("inf")
    routes = cq.cq_route(l.cuda(), top, cq.CQ_SOFTMAX)
    expert, _ = ref_route.choose(as64(l), top, "softmax")
    assert np.array_equal(routes.expert.cpu().numpy(), expert)
    y = cq.cq_i8_moe(wu, wd, x.cuda(), routes)
    want, size = moe_oracle(as64(x), expert, as64(routes.weight), up, down, torch.bfloat16)
    err = np.abs(as64(y) - want)
    allowed = torch.finfo(y.dtype).eps / 2 * np.abs(want) * (1 + 2.0 ** -10) + (top + 1) * 2.0 ** -24 * size + torch.finfo(y.dtype).tiny
    assert np.all(err <= allowed), float((err / allowed).max())
    if T > 1:
        assert torch.all(y[T // 2] == 0)


def test_two_expert_blocks_at_once():
    """Two blocks on two streams with workspaces of their own, and two captured ones that share one, replayed in turn."""
    E, H, I, top = 8, 512, 256, 2
    g = torch.Generator("cuda").manual_seed(9)
    wu = cq.cq_i8_quantize(torch.randn((E, 2 * I, H), generator=g, device="cuda") * 0.05)
    wd = cq.cq_i8_quantize(torch.randn((E, H, I), generator=g, device="cuda") * 0.05)
    cases = []
    for T in (3, 200, 900):
        x = torch.randn((T, H), generator=g, device="cuda").bfloat16()
        cases.append((x, cq.cq_route(torch.randn((T, E), generator=g, device="cuda"), top)))
    want = [cq.cq_i8_moe(wu, wd, x, r) for x, r in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], []
    for _ in range(15):
        for st, (x, r) in zip(streams, cases):
            with torch.cuda.stream(st):
                got.append(cq.cq_i8_moe(wu, wd, x, r))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[i % 3]) for i, a in enumerate(got))
    ws = cq.cq_i8_moe_workspace(wu, wd, 900, top)
    graphs, outs = [], []
    for x, r in cases:
        out = torch.empty_like(x)
        cq.cq_i8_moe(wu, wd, x, r, workspace=ws, out=out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cq.cq_i8_moe(wu, wd, x, r, workspace=ws, out=out)
        graphs.append(graph)
        outs.append(out)
    for _ in range(10):
        for graph, out, y in zip(graphs, outs, want):
            out.zero_()
            graph.replay()
            assert torch.equal(out, y)
    assert cq.cq_gemm_status(ws) == 0


def test_routes_lead_the_other_routed_products():
    """The same map in front of 4-bit products (offsets on the device) and of cubic ones (offsets on the host)."""
    from util import logical_case
    T, E, top, K, N = 60, 4, 2, 512, 256
    x = rows(T, K, "bf16", 1, 0.3).cuda()
    r = cq.cq_route(torch.randn((T, E), generator=torch.Generator("cuda").manual_seed(1), device="cuda"), top)
    w = torch.stack([rows(N, K, "f32", 30 + e, 0.3) * 0.05 for e in range(E)]).cuda()
    q4 = cq.cq_fp4_quantize(w, cq.CQ_MXFP4)
    y = cq.cq_fp4_gemm_routed(q4, x, r.token, r.offset)
    off = r.offset.tolist()
    for e in range(E):
        t = r.token[off[e]:off[e + 1]].long()
        one = cq.cq_fp4_gemm(cq.cq_fp4_quantize(w[e], cq.CQ_MXFP4), x[t])
        assert torch.allclose(y[off[e]:off[e + 1]].float(), one.float(), rtol=2.0 ** -7, atol=1e-3)
    assert cq.cq_combine(y, r).shape == (T, N)
    cases = [logical_case(N, K, 4, 128, seed=70 + e) for e in range(E)]
    yc = cq.cq_gemm_routed([c.pw for c in cases], x, r.token, off)
    assert torch.isfinite(cq.cq_combine(yc.view(T * top, N), r)).all()


def test_the_first_call_of_a_process_may_be_captured():
    """What the library asks the device once (places for clusters, room for shared memory) is asked inside a capture here."""
    code = """
import torch, paper_2608_06763_b200 as cq
w = cq.cq_i8_pack(torch.ones((1024, 512), dtype=torch.int8, device="cuda"), torch.full((1024,), 0.5, device="cuda"))
x, out, ws = torch.ones((40, 512), device="cuda").bfloat16(), torch.zeros((40, 1024), dtype=torch.bfloat16, device="cuda"), cq.cq_i8_workspace(w, 40)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    cq.cq_i8_gemm(w, x, workspace=ws, out=out)
graph.replay()
assert torch.all(out == 256)
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=ROOT, timeout=300)


def test_workspaces_may_hold_anything_but_for_their_front():
    """Products and expert blocks in workspaces full of NaN patterns behind the status words."""
    E, H, I, T, top = 5, 528, 272, 150, 2
    g = torch.Generator("cuda").manual_seed(4)
    wu, wd = (cq.cq_i8_quantize(torch.randn((E, n, k), generator=g, device="cuda") * 0.05) for n, k in ((2 * I, H), (H, I)))
    one = cq.cq_i8_quantize(torch.randn((700, H), generator=g, device="cuda"))
    x, r = torch.randn((T, H), generator=g, device="cuda").bfloat16(), cq.cq_route(torch.randn((T, E), generator=g, device="cuda"), top)
    results = []
    for fill in (0, 0xFF):
        ws, wm = cq.cq_i8_workspace(one, T), cq.cq_i8_moe_workspace(wu, wd, T, top)
        ws[512:] = fill
        wm[512:] = fill
        results.append((cq.cq_i8_gemm(one, x, workspace=ws), cq.cq_i8_moe(wu, wd, x, r, workspace=wm)))
        assert cq.cq_gemm_status(ws) == 0 and cq.cq_gemm_status(wm) == 0
    assert all(torch.equal(a, b) and torch.isfinite(a).all() for a, b in zip(*results))
