"""4-bit floating point with block scales on the GPU against the 64-bit oracle (oracle/fp4.py).

Quantisers and exchanges: equal byte for byte (every decision is exact).  Products: what the tensor core adds up, then one
rounding to the model dtype.  Tolerance, derived: half a step of the output type of |y|, and for each 64-wide step at most three
roundings (or cuts) to fp32 of partial sums that never exceed the sum of the magnitudes S: K / 64 * 3 * 2^-23 * S.
"""
import numpy as np
import pytest
import torch

import paper_2608_06763_b200 as cq
from fp4_shapes import PRODUCTS, ROUTED
from oracle import fp4 as ref

pytestmark = pytest.mark.gpu

FMT = {"mx": cq.CQ_MXFP4, "nv": cq.CQ_NVFP4}
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def rows(M, K, dtype, seed, spread=1.0):
    """Normal values with a few large columns and magnitudes that differ from row to row."""
    r = np.random.default_rng(seed)
    x = r.standard_normal((M, K)) * np.exp(spread * r.standard_normal((M, 1)))
    x[:, r.integers(0, K, max(1, K // 100))] *= 20
    return torch.from_numpy(x).float().to(DTYPE[dtype])


def g_of(fmt, value):
    return None if fmt == "mx" else torch.tensor(value, dtype=torch.float32, device="cuda")


def as64(t):
    return t.detach().double().cpu().numpy()


def nan_equal(a, b):
    return np.array_equal(a, b, equal_nan=True)


def check_bytes(q, c, b):
    codes, scales = cq.cq_fp4_unpack(q)
    got = codes.cpu().numpy()
    low, high = got & 15, got >> 4
    both = np.stack([low, high], axis=-1).reshape(c.shape)
    assert np.array_equal(scales.cpu().numpy(), b), "scales"
    # a zero has no sign that counts
    assert np.array_equal(np.where(both & 7, both, 0), np.where(c & 7, c, 0)), "codes"


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,K", [(1, 32), (3, 64), (5, 352), (128, 256), (130, 4096), (257, 1408)])
def test_quantize(M, K, fmt, dtype):
    x = rows(M, K, dtype, seed=M + K)
    g = 0.0131
    q = cq.cq_fp4_quantize(x.cuda(), FMT[fmt], g_of(fmt, g))
    c, b = ref.quantize(as64(x), fmt, g)
    check_bytes(q, c, b)
    for out in (torch.bfloat16, torch.float16, torch.float32):
        want = torch.from_numpy(ref.values(c, b, fmt, g)).float().to(out)
        assert torch.equal(cq.cq_fp4_dequantize(q, out).cpu(), want)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_quantize_ties_extremes_and_non_finite(fmt):
    """Every border between codes exactly hit, zeros, subnormal values, values beyond the scales, blocks with an infinity or a NaN."""
    K = 256
    x = torch.zeros((16, K), dtype=torch.float32)
    mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    for j, s in enumerate((1.0, 2.0 ** -30, 2.0 ** 40, 1.5, 1.125, 1.875)):
        x[j] = (mids * s).repeat(K // 8) * torch.tensor([1.0, -1.0]).repeat_interleave(8).repeat(K // 16)
    x[6, 5] = float("inf")
    x[7, 40] = float("nan")
    x[8, 0] = -float("inf")
    x[9] = 2.0 ** -130
    x[10] = 2.0 ** -149
    x[11] = 3.3e38
    x[12, ::3] = 1e-20
    x[13] = -448.0 * 6 * 4
    x[14, 100] = 1.0
    for dtype in ("f32", "bf16"):
        xd = x.to(DTYPE[dtype])
        q = cq.cq_fp4_quantize(xd.cuda(), FMT[fmt])
        c, b = ref.quantize(as64(xd), fmt)
        check_bytes(q, c, b)
        assert nan_equal(as64(cq.cq_fp4_dequantize(q, torch.float32)), ref.values(c, b, fmt).astype(np.float32).astype(np.float64))


def test_quantize_all_bf16_values():
    """Each of the 65536 patterns, alone in a block with a fixed neighbour and among others."""
    p = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = torch.zeros((65536, 32), dtype=torch.bfloat16)
    x[:, 3] = p
    x[:, 4] = p.flip(0)
    x[:, 20] = p.roll(77)
    for fmt in ("mx", "nv"):
        q = cq.cq_fp4_quantize(x.cuda(), FMT[fmt])
        check_bytes(q, *ref.quantize(as64(x), fmt))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_strided_rows_and_several_matrices(fmt):
    wide = rows(70, 512, "bf16", 5).cuda()
    x = wide[:, 64:64 + 320]
    check_bytes(cq.cq_fp4_quantize(x, FMT[fmt]), *ref.quantize(as64(x), fmt))
    w = torch.stack([rows(130, 288, "f32", 6 + e) for e in range(3)])
    g = None if fmt == "mx" else torch.tensor([0.01, 0.5, 1.0], device="cuda")
    q = cq.cq_fp4_quantize(w.cuda(), FMT[fmt], g)
    parts = [ref.quantize(as64(w[e]), fmt, 1.0 if g is None else float(g[e])) for e in range(3)]
    check_bytes(q, np.stack([p[0] for p in parts]), np.stack([p[1] for p in parts]))
    codes, scales = cq.cq_fp4_unpack(q)
    again = cq.cq_fp4_pack(codes, scales, FMT[fmt], g)
    for e in range(3):
        want = torch.from_numpy(ref.values(*parts[e], fmt, 1.0 if g is None else float(g[e]))).float()
        assert torch.equal(cq.cq_fp4_dequantize(again, torch.float32)[e].cpu(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,I", [(1, 32), (7, 1408), (300, 4096)])
def test_swiglu_quantize(M, I, fmt, dtype):
    h = rows(M, 2 * I, dtype, seed=M + I, spread=0.5)
    g = 0.11
    q = cq.cq_fp4_swiglu_quantize(h.cuda(), FMT[fmt], g_of(fmt, g))
    v = as64(h)
    act = torch.from_numpy(ref.gated(v[:, :I], v[:, I:])).to(DTYPE[dtype])
    check_bytes(q, *ref.quantize(as64(act), fmt, g))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_swiglu_far_gates_and_subnormal_activations(fmt):
    I = 64
    for dtype in ("bf16", "f16"):
        top = 300.0 if dtype == "bf16" else 100.0
        gate = torch.linspace(-top, top, 16 * I).reshape(16, I)
        up = torch.tensor([1.0, -2.0, 1e-6, 3e4]).repeat(4)[:, None].expand(16, I)
        h = torch.cat([gate, up], dim=1).to(DTYPE[dtype])
        if dtype == "bf16":
            h[1, 0], h[2, 1], h[1, I], h[2, I + 1] = 3.3e38, 2.4e38, 0.5, 1e-20
        h[3, 7], h[5, I + 9], h[6, 2] = float("nan"), float("inf"), -float("inf")
        q = cq.cq_fp4_swiglu_quantize(h.cuda(), FMT[fmt])
        v = as64(h)
        act = torch.from_numpy(ref.gated(v[:, :I], v[:, I:])).to(DTYPE[dtype])
        check_bytes(q, *ref.quantize(as64(act), fmt))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_swiglu_products_of_gate_and_up_beyond_fp32(fmt):
    """gate * up leaves fp32 where silu(gate) * up does not: finite values, and an infinity only where the activation itself is one."""
    I, M = 64, 40
    r = np.random.default_rng(21)
    gate = r.uniform(-60, 60, (M, I)) * r.choice([1.0, 0.05], (M, I))
    up = 10.0 ** r.uniform(36.5, 38.5, (M, I)) * r.choice([-1.0, 1.0], (M, I))
    gate[0, :3], up[0, :3] = (-2.0, -50.0, 1.5), (3e38, 1e37, 2.4e38)
    gate[1:20] = -np.abs(gate[1:20])              # whole blocks of finite activations
    up[20:30, ::2] = 1.0                           # among ordinary ones
    h = torch.from_numpy(np.concatenate([gate, up], axis=1)).float().to(torch.bfloat16)
    v = as64(h)
    act = torch.from_numpy(ref.gated(v[:, :I], v[:, I:])).to(torch.bfloat16)
    assert torch.isfinite(act[1:20]).all() and not torch.isfinite(act).all()
    assert (np.abs(v[:, :I] * v[:, I:]) > torch.finfo(torch.float32).max).any(axis=1)[1:20].all()
    g = 1e34
    q = cq.cq_fp4_swiglu_quantize(h.cuda(), FMT[fmt], g_of(fmt, g))
    check_bytes(q, *ref.quantize(as64(act), fmt, g))


def product_case(M, N, K, fmt, dtype, seed=0):
    gw, gx = (1.0, 1.0) if fmt == "mx" else (0.0007, 0.021)
    w, x = rows(N, K, "f32", seed, 0.3) * 0.05, rows(M, K, dtype, seed + 1, 0.3)
    wc, wb = ref.quantize(as64(w), fmt, gw)
    xc, xb = ref.quantize(as64(x), fmt, gx)
    wq = cq.cq_fp4_pack(torch.from_numpy(ref.pack(wc)).cuda(), torch.from_numpy(wb).cuda(), FMT[fmt], g_of(fmt, gw))
    y, S = ref.product(xc, xb, wc, wb, fmt, gx, gw)
    return wq, x.cuda(), g_of(fmt, gx), y, S


def check_product(got, y, S, K):
    t = got.dtype
    err = np.abs(as64(got) - y)
    allowed = torch.finfo(t).eps / 2 * np.abs(y) + (K / 64 + 1) * 3 * 2.0 ** -23 * S + torch.finfo(t).tiny
    assert np.all(err <= allowed), (float((err / allowed).max()), np.argwhere(err > allowed)[:4].tolist())


SMALL = [(1, 128, 64), (1, 128, 256), (16, 128, 128), (5, 200, 512), (128, 256, 1024), (129, 128, 320), (256, 130, 768)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", SMALL)
def test_gemm_small(M, N, K, fmt):
    w, x, g, y, S = product_case(M, N, K, fmt, "bf16")
    check_product(cq.cq_fp4_gemm(w, x, g), y, S, K)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (2, 1001, 2816), (13, 6144, 4096), (17, 513, 5632), (40, 1024, 1024), (100, 2816, 2048), (200, 4096, 1408),
                                   (300, 700, 4096), (513, 1024, 512), (1000, 2050, 288), (65, 300, 1024), (449, 1100, 2048), (1024, 6144, 512)])
def test_gemm(M, N, K, fmt, dtype):
    w, x, g, y, S = product_case(M, N, K, fmt, dtype)
    ws = cq.cq_fp4_workspace(w, M)
    got = cq.cq_fp4_gemm(w, x, g, workspace=ws)
    assert got.dtype == DTYPE[dtype]
    check_product(got, y, S, K)
    assert torch.equal(cq.cq_fp4_gemm(w, x, g, workspace=ws), got)          # the same bits again
    q = cq.cq_fp4_quantize(x, FMT[fmt], g)
    assert torch.equal(cq.cq_fp4_gemm(w, q, out=torch.empty_like(got)), got)
    assert cq.cq_gemm_status(ws) == 0


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_gemm_exact_integers(fmt):
    """Codes that are whole numbers under scales of one: every sum is exact."""
    M, N, K = 33, 260, 1024
    r = np.random.default_rng(3)
    xc, wc = (r.choice([0, 2, 4, 5, 10, 12, 13], size=s).astype(np.uint8) for s in ((M, K), (N, K)))
    one = 127 if fmt == "mx" else 0x38
    blk = ref.BLOCK[fmt]
    xb, wb = np.full((M, K // blk), one, np.uint8), np.full((N, K // blk), one, np.uint8)
    # one block of each row under another power of two, so that scales of the wrong block show
    xb[np.arange(M), np.arange(M) % (K // blk)] += 1 if fmt == "mx" else 8
    wb[np.arange(N), np.arange(N) * 7 % (K // blk)] -= 1 if fmt == "mx" else 8
    pack = lambda c, b: cq.cq_fp4_pack(torch.from_numpy(ref.pack(c)).cuda(), torch.from_numpy(b).cuda(), FMT[fmt])  # noqa: E731
    y, _ = ref.product(xc, xb, wc, wb, fmt)
    got = cq.cq_fp4_gemm(pack(wc, wb), pack(xc, xb))
    assert torch.equal(got.cpu(), torch.from_numpy(y).float().to(torch.bfloat16))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_gemm_non_finite_rows_stay_alone(fmt):
    w, x, g, y, S = product_case(20, 256, 512, fmt, "bf16")
    x[3, 100] = float("nan")
    x[11, 500] = float("inf")
    got = as64(cq.cq_fp4_gemm(w, x, g))
    bad = np.isin(np.arange(20), (3, 11))
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()
    check_product(torch.from_numpy(got[~bad]).to(torch.bfloat16), y[~bad], S[~bad], 512)


def routed_case(counts, N, K, fmt, dtype, seed=0, T=50):
    E, R = len(counts), sum(counts)
    r = np.random.default_rng(seed)
    x = rows(T, K, dtype, seed + 1, 0.3)
    gx = 1.0 if fmt == "mx" else 0.03
    gw = np.linspace(0.0005, 0.002, E).astype(np.float32)
    token = torch.from_numpy(r.integers(0, T, R).astype(np.int32))
    off = np.concatenate([[0], np.cumsum(counts)])
    W = [ref.quantize(as64(rows(N, K, "f32", seed + 2 + e, 0.3) * 0.05), fmt, float(gw[e])) for e in range(E)]
    w = cq.cq_fp4_pack(torch.from_numpy(np.stack([ref.pack(c) for c, _ in W])).cuda(), torch.from_numpy(np.stack([b for _, b in W])).cuda(), FMT[fmt],
                       None if fmt == "mx" else torch.from_numpy(gw).cuda())
    xc, xb = ref.quantize(as64(x), fmt, gx)
    y, S = np.zeros((R, N)), np.zeros((R, N))
    for e in range(E):
        t = token[off[e]:off[e + 1]].numpy()
        if len(t):
            y[off[e]:off[e + 1]], S[off[e]:off[e + 1]] = ref.product(xc[t], xb[t], *W[e], fmt, gx, float(gw[e]) if fmt == "nv" else 1.0)
    return w, x.cuda(), token.cuda(), torch.tensor(off, dtype=torch.int32).cuda(), g_of(fmt, gx), y, S


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("counts", [[1], [3, 0, 5, 1], [0, 0, 7], [128, 1, 129, 0, 300, 16], [1] * 40, [700, 2], [100, 3, 0, 65, 1, 1, 1, 1, 129, 1]])
def test_gemm_routed(counts, fmt):
    N, K = 260, 544
    w, x, token, off, g, y, S = routed_case(counts, N, K, fmt, "bf16")
    ws = cq.cq_fp4_workspace(w, sum(counts))
    got = cq.cq_fp4_gemm_routed(w, x, token, off, g, workspace=ws)
    check_product(got, y, S, K)
    q = cq.cq_fp4_quantize(x, FMT[fmt], g, route_token=token, expert_offset=off)
    assert torch.equal(cq.cq_fp4_gemm_routed(w, q, None, off), got)
    assert cq.cq_gemm_status(ws) == 0
    values = as64(cq.cq_fp4_dequantize(q, torch.float32))
    xc, xb = ref.quantize(as64(x), fmt, 0.03 if fmt == "nv" else 1.0)
    want = ref.values(xc, xb, fmt, 0.03 if fmt == "nv" else 1.0).astype(np.float32)   # rounded once to the type asked for
    assert np.array_equal(values, want[token.cpu().numpy()].astype(np.float64))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_routed_rows_of_nobody_and_tokens_out_of_range(fmt):
    N, K, R = 136, 256, 40
    w, x, token, off, g, y, S = routed_case([10, 12, 6], N, K, fmt, "bf16", T=30)   # 28 of 40 rows
    token = torch.cat([token, torch.zeros(R - 28, dtype=torch.int32, device="cuda")])
    token[4], token[20] = -1, 30
    out = torch.full((R, N), 7.0, dtype=torch.bfloat16, device="cuda")
    got = cq.cq_fp4_gemm_routed(w, x, token, off, g, out=out)
    assert torch.all(got[28:] == 7.0)
    assert torch.all(got[[4, 20]] == 0)
    keep = [r for r in range(28) if r not in (4, 20)]
    check_product(got[keep], y[keep], S[keep], K)
    # offsets that descend or leave the rows are brought back, and no group takes rows that are not there
    for bad in ([0, 10, 5, 28], [0, 10, 22, 99], [-3, 10, 22, 28]):
        out.fill_(7.0)
        got = cq.cq_fp4_gemm_routed(w, x, token, torch.tensor(bad, dtype=torch.int32, device="cuda"), g, out=out)
        check_product(got[keep[:9]], y[keep[:9]], S[keep[:9]], K)
    empty = cq.cq_fp4_gemm_routed(w, x, token, torch.zeros(4, dtype=torch.int32, device="cuda"), g, out=out.fill_(7.0))
    assert torch.all(empty == 7.0)
    none = cq.cq_fp4_gemm_routed(w, x, token[:0], torch.zeros(4, dtype=torch.int32, device="cuda"), g)
    assert none.shape == (0, N)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_expert_block_as_it_is_used(fmt, dtype):
    """Routed gate | up, gated activation, routed down, from a captured graph that follows new tokens, routes and loads."""
    E, H, I, T, top = 6, 512, 288, 24, 2
    R = T * top
    r = np.random.default_rng(11)
    g1, g2 = (1.0, 1.0) if fmt == "mx" else (0.03, 0.09)
    up = [ref.quantize(r.standard_normal((2 * I, H)) * 0.06, fmt, 0.001) for _ in range(E)]
    down = [ref.quantize(r.standard_normal((H, I)) * 0.06, fmt, 0.001) for _ in range(E)]
    gw = None if fmt == "mx" else torch.full((E,), 0.001, device="cuda")
    stack = lambda W: cq.cq_fp4_pack(torch.from_numpy(np.stack([ref.pack(c) for c, _ in W])).cuda(), torch.from_numpy(np.stack([b for _, b in W])).cuda(), FMT[fmt], gw)  # noqa: E731
    wu, wd = stack(up), stack(down)
    x = torch.zeros((T, H), dtype=DTYPE[dtype], device="cuda")
    token, off = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    ws, ws2 = cq.cq_fp4_workspace(wu, R), cq.cq_fp4_workspace(wd, R)
    h = torch.zeros((R, 2 * I), dtype=x.dtype, device="cuda")
    a = cq.cq_fp4_empty(FMT[fmt], R, I, groups=E)
    y = torch.zeros((R, H), dtype=x.dtype, device="cuda")
    s1, s2 = g_of(fmt, g1), g_of(fmt, g2)

    def block():
        cq.cq_fp4_gemm_routed(wu, x, token, off, s1, workspace=ws, out=h)
        cq.cq_fp4_swiglu_quantize(h, FMT[fmt], s2, expert_offset=off, out=a)
        cq.cq_fp4_gemm_routed(wd, a, None, off, workspace=ws2, out=y)

    block()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    for seed in range(3):
        xs = rows(T, H, dtype, 100 + seed, 0.3)
        chosen = np.random.default_rng(seed).random((T, E)).argsort(axis=1)[:, :top].reshape(-1)
        chosen = np.minimum(chosen, E - 1 - seed)   # uneven, and matrices without rows
        order = chosen.argsort(kind="stable")
        offs = np.concatenate([[0], np.bincount(chosen, minlength=E).cumsum()])
        x.copy_(xs)
        token.copy_(torch.from_numpy((order // top).astype(np.int32)))
        off.copy_(torch.from_numpy(offs.astype(np.int32)))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        xc, xb = ref.quantize(as64(xs), fmt, g1)
        for e in range(E):
            part = slice(offs[e], offs[e + 1])
            t = order[part] // top
            if not len(t):
                continue
            hy, hS = ref.product(xc[t], xb[t], *up[e], fmt, g1, 0.001)
            check_product(h[part], hy, hS, H)
            hv = as64(h[part])   # from here on by what the first product returned
            act = torch.from_numpy(ref.gated(hv[:, :I], hv[:, I:])).to(x.dtype)
            ac, ab = ref.quantize(as64(act), fmt, g2)
            yy, yS = ref.product(ac, ab, *down[e], fmt, g2, 0.001)
            check_product(y[part], yy, yS, I)
    assert cq.cq_gemm_status(ws) == 0 and cq.cq_gemm_status(ws2) == 0


def test_another_stream_and_refusals_on_the_gpu():
    w, x, g, y, S = product_case(40, 1024, 2048, "nv", "bf16")
    want = cq.cq_fp4_gemm(w, x, g)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = cq.cq_fp4_gemm(w, x, g)
    s.synchronize()
    assert torch.equal(got, want)
    with pytest.raises(cq.CubicQuantError):
        cq.cq_fp4_gemm(w, x[:, 1:], g)
    with pytest.raises(cq.CubicQuantError):
        cq.cq_fp4_gemm(w, x.cpu(), g)
    with pytest.raises(cq.CubicQuantError):
        cq.cq_fp4_gemm(w, x, g, workspace=torch.zeros(512, dtype=torch.uint8, device="cuda"))
    assert cq.cq_fp4_gemm(w, x[:0], g).shape == (0, 1024)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", [(3, 130, 288), (20, 300, 1056), (100, 200, 512), (300, 900, 800)])
def test_what_lies_behind_the_last_row_reaches_nothing(M, N, K, fmt):
    """Layouts and workspaces full of NaN scales beforehand: the same results, and not a byte of the rows behind the last written."""
    w, x, g, y, S = product_case(M, N, K, fmt, "bf16")
    want = cq.cq_fp4_gemm(w, x, g)
    q = cq.cq_fp4_empty(FMT[fmt], N, K)
    codes, scales = cq.cq_fp4_unpack(w)
    q.layout.fill_(255)
    from paper_2608_06763_b200.fp4 import _check, _lib, _stream
    _check(_lib().cq_fp4_pack(codes.data_ptr(), scales.data_ptr(), FMT[fmt], 1, N, K, q.layout.data_ptr(), _stream()), "pack")
    q.tensor_scale = w.tensor_scale
    ws = cq.cq_fp4_workspace(w, M)
    ws[512:].fill_(255)
    got = cq.cq_fp4_gemm(q, x, g, workspace=ws)
    assert torch.equal(got, want)
    check_product(got, y, S, K)
    xq = cq.cq_fp4_empty(FMT[fmt], M, K)
    xq.layout.fill_(255)
    cq.cq_fp4_quantize(x, FMT[fmt], g, out=xq)
    assert torch.equal(cq.cq_fp4_gemm(q, xq), want)
    KT, tile = (K + 255) // 256, 16384 + (1024 if fmt == "mx" else 2048)
    last = xq.layout.view(-1, KT, tile)[-1]
    used = (M - 1) % 128 + 1
    assert torch.all(last[:, used * 128:16384] == 255)


def test_two_streams_and_two_graphs_with_workspaces_of_their_own():
    """Two products at once on two streams, and two captured graphs over one workspace replayed in turn."""
    cases = [product_case(M, 2048, 1024, "nv", "bf16", seed=50 + M) for M in (40, 200)]
    want = [cq.cq_fp4_gemm(w, x, g) for w, x, g, _, _ in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], []
    for _ in range(20):
        for st, (w, x, g, _, _) in zip(streams, cases):
            with torch.cuda.stream(st):
                got.append(cq.cq_fp4_gemm(w, x, g))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[i % 2]) for i, a in enumerate(got))
    ws = cq.cq_fp4_workspace(cases[1][0], 200)
    graphs, outs = [], []
    for w, x, g, _, _ in cases:
        out = torch.empty((x.shape[0], 2048), dtype=x.dtype, device="cuda")
        cq.cq_fp4_gemm(w, x, g, workspace=ws, out=out)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            cq.cq_fp4_gemm(w, x, g, workspace=ws, out=out)
        graphs.append(graph)
        outs.append(out)
    for _ in range(10):
        for graph, out, y in zip(graphs, outs, want):
            out.zero_()
            graph.replay()
            assert torch.equal(out, y)
    assert cq.cq_gemm_status(ws) == 0


def test_long_rows_and_a_layout_beyond_two_gigabytes():
    """Offsets past 32 bits: the last rows of a matrix of 2.4 GB in the layout, and of 8.6 GB before it."""
    M, K = 540000, 8192
    x = torch.randn((256, K), generator=torch.Generator("cuda").manual_seed(3), device="cuda").bfloat16().repeat(M // 256 + 1, 1)[:M]
    q = cq.cq_fp4_quantize(x, cq.CQ_MXFP4)
    assert q.layout.numel() > 2 ** 31 and x.numel() > 2 ** 32
    few = cq.cq_fp4_quantize(x[:256], cq.CQ_MXFP4)
    v, ref_v = cq.cq_fp4_dequantize(q), cq.cq_fp4_dequantize(few)
    for lo in (0, 262144, M // 256 * 256 - 256):
        assert torch.equal(v[lo:lo + 256], ref_v)
    assert torch.equal(v[M // 256 * 256:], ref_v[:M % 256])
    small = cq.cq_fp4_quantize(torch.randn((40, K), device="cuda").bfloat16(), cq.CQ_MXFP4)
    y = cq.cq_fp4_gemm(q, small)
    a, b = as64(cq.cq_fp4_dequantize(small, torch.float32)), as64(cq.cq_fp4_dequantize(few, torch.float32))
    for lo in (0, M // 256 * 256 - 256):
        check_product(y[:, lo:lo + 256], a @ b.T, np.abs(a) @ np.abs(b).T, K)


@pytest.mark.parametrize("M,N,K", [(5, 24000, 200), (5, 24000, 700), (2, 20100, 1312), (40, 20100, 1312), (60, 24000, 144)])
@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_odd_numbers_of_k_tiles_over_many_output_tiles(M, N, K, fmt):
    """Several output tiles to a CTA, an odd number of stages each, so that the ring's stages fall to other k tiles from one to the next:
    called often enough for the two issuing warps to drift apart, always the same bits."""
    K = K // 32 * 32
    w, x, g, y, S = product_case(M, N, K, fmt, "bf16")
    ws = cq.cq_fp4_workspace(w, M)
    want = cq.cq_fp4_gemm(w, x, g, workspace=ws)
    check_product(want, y, S, K)
    out = torch.empty_like(want)
    for i in range(200):
        cq.cq_fp4_gemm(w, x, g, workspace=ws, out=out)
        if i % 20 == 0:
            assert torch.equal(out, want)
    assert torch.equal(out, want) and cq.cq_gemm_status(ws) == 0


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("plan,M,N,K", PRODUCTS)
def test_every_kind_of_tile(plan, M, N, K, fmt):
    """bfloat16 and binary16 in turn; from rows in the model dtype and from quantised ones, which have the same bits."""
    assert tuple(cq.cq_debug_fp4_plan(FMT[fmt], M, N, K).values()) == plan
    w, x, g, y, S = product_case(M, N, K, fmt, "bf16" if (M + (fmt == "nv")) % 2 else "f16", seed=M)
    ws = cq.cq_fp4_workspace(w, M)
    got = cq.cq_fp4_gemm(w, x, g, workspace=ws)
    check_product(got, y, S, K)
    q = cq.cq_fp4_quantize(x, FMT[fmt], g)
    out = torch.full_like(got, 7.0)
    assert torch.equal(cq.cq_fp4_gemm(w, q, workspace=ws, out=out), got)
    assert cq.cq_gemm_status(ws) == 0


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("plan,counts,N,K", ROUTED)
def test_every_kind_of_routed_tile(plan, counts, N, K, fmt):
    R = sum(counts)
    assert tuple(cq.cq_debug_fp4_plan(FMT[fmt], R, N, K, matrices=len(counts)).values()) == plan + (1, False)
    w, x, token, off, g, y, S = routed_case(counts, N, K, fmt, "bf16" if fmt == "nv" else "f16", seed=N, T=150)
    ws = cq.cq_fp4_workspace(w, R)
    got = cq.cq_fp4_gemm_routed(w, x, token, off, g, workspace=ws)
    check_product(got, y, S, K)
    q = cq.cq_fp4_quantize(x, FMT[fmt], g, route_token=token, expert_offset=off)
    assert torch.equal(cq.cq_fp4_gemm_routed(w, q, None, off, workspace=ws, out=torch.full_like(got, 7.0)), got)
    assert cq.cq_gemm_status(ws) == 0


def repaired(offset, R):
    """Offsets as the calls take them: the largest so far, within [0, R]."""
    return np.maximum.accumulate(np.clip(offset, 0, R))


ASTRAY = {
    "descends": [0, 10, 5, 28], "behind the rows": [0, 10, 22, 99], "negative": [-3, 10, 22, 28], "starts late": [4, 10, 12, 28], "starts behind": [41, 0, 0, 0],
    "all at once": [9, -5, 200, 3],
    # over the 32 offsets that one step of the scan takes, and over 64 of them
    "descends at 31": list(range(32)) + [3, 4] + [35] * 6, "descends at 32": list(range(33)) + [7] * 4 + [38], "falls behind 31": [5] * 31 + [39] + list(range(10)),
    "long": [3] + [2 * i if i % 5 else -i for i in range(1, 20)] + [38] * 30 + [0] * 15 + [40] * 10, "thirty-two": list(range(0, 33)), "thirty-one": list(range(0, 32)),
}


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("name", ASTRAY)
def test_offsets_that_go_astray(name, fmt):
    """Every row against the matrix that it belongs to by the rule in the header; rows of no group are left as they were: by product, quantiser,
    gated activation and inverse."""
    offset, R, N, K, I = ASTRAY[name], 40, 136, 256, 64
    E = len(offset) - 1
    r = np.random.default_rng(E)
    gw = np.linspace(0.0005, 0.002, E).astype(np.float32)
    gx = 0.03 if fmt == "nv" else 1.0
    W = [ref.quantize(r.standard_normal((N, K)) * 0.05, fmt, float(gw[e])) for e in range(E)]
    w = cq.cq_fp4_pack(torch.from_numpy(np.stack([ref.pack(c) for c, _ in W])).cuda(), torch.from_numpy(np.stack([b for _, b in W])).cuda(), FMT[fmt],
                       None if fmt == "mx" else torch.from_numpy(gw).cuda())
    x, token = rows(50, K, "bf16", 7, 0.3), r.integers(0, 50, R).astype(np.int32)
    off = torch.tensor(offset, dtype=torch.int32, device="cuda")
    true = repaired(offset, R)
    mine = np.zeros(R, bool)
    mine[true[0]:true[-1]] = True
    xc, xb = ref.quantize(as64(x), fmt, gx)
    y, S = np.zeros((R, N)), np.zeros((R, N))
    for e in range(E):
        part = slice(true[e], true[e + 1])
        if true[e] < true[e + 1]:
            y[part], S[part] = ref.product(xc[token[part]], xb[token[part]], *W[e], fmt, gx, float(gw[e]) if fmt == "nv" else 1.0)
    ws = cq.cq_fp4_workspace(w, R)
    out = torch.full((R, N), 7.0, dtype=torch.bfloat16, device="cuda")
    q = cq.cq_fp4_quantize(x.cuda(), FMT[fmt], g_of(fmt, gx), route_token=torch.from_numpy(token).cuda(), expert_offset=off)
    for call in (lambda: cq.cq_fp4_gemm_routed(w, x.cuda(), torch.from_numpy(token).cuda(), off, g_of(fmt, gx), workspace=ws, out=out),
                 lambda: cq.cq_fp4_gemm_routed(w, q, None, off, workspace=ws, out=out)):
        out.fill_(7.0)
        call()
        if mine.any():
            check_product(out[torch.from_numpy(mine).cuda()], y[mine], S[mine], K)
        assert torch.all(out[torch.from_numpy(~mine).cuda()] == 7.0)
    assert cq.cq_gemm_status(ws) == 0
    back = cq.cq_fp4_dequantize(q, out=torch.full((R, K), 7.0, device="cuda"))
    want = np.where(mine[:, None], ref.values(xc, xb, fmt, gx).astype(np.float32)[token].astype(np.float64), 7.0)
    assert np.array_equal(as64(back), want)
    h = rows(R, 2 * I, "bf16", 8, 0.3)
    v = as64(h)
    act = torch.from_numpy(ref.gated(v[:, :I], v[:, I:])).to(torch.bfloat16)
    g2 = 0.11 if fmt == "nv" else 1.0
    a = cq.cq_fp4_swiglu_quantize(h.cuda(), FMT[fmt], g_of(fmt, g2), expert_offset=off)
    back = cq.cq_fp4_dequantize(a, out=torch.full((R, I), 7.0, device="cuda"))
    want = np.where(mine[:, None], ref.values(*ref.quantize(as64(act), fmt, g2), fmt, g2).astype(np.float32).astype(np.float64), 7.0)
    assert np.array_equal(as64(back), want)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,dtype", [(1, "bf16"), (5, "f16"), (200, "bf16")])
def test_mlp_as_it_is_used(M, dtype, fmt):
    """gate | up, gated activation, down of a dense layer from a captured graph, one workspace for both products."""
    H, I = 512, 1376
    g1, g2 = (1.0, 1.0) if fmt == "mx" else (0.03, 0.09)
    r = np.random.default_rng(31)
    up, down = ref.quantize(r.standard_normal((2 * I, H)) * 0.06, fmt, 0.001), ref.quantize(r.standard_normal((H, I)) * 0.06, fmt, 0.001)
    load = lambda c, b: cq.cq_fp4_pack(torch.from_numpy(ref.pack(c)).cuda(), torch.from_numpy(b).cuda(), FMT[fmt], g_of(fmt, 0.001))  # noqa: E731
    wu, wd = load(*up), load(*down)
    x = torch.zeros((M, H), dtype=DTYPE[dtype], device="cuda")
    ws = cq.cq_fp4_workspace(wu, M)
    h, a, y = torch.zeros((M, 2 * I), dtype=x.dtype, device="cuda"), cq.cq_fp4_empty(FMT[fmt], M, I), torch.zeros((M, H), dtype=x.dtype, device="cuda")
    s1, s2 = g_of(fmt, g1), g_of(fmt, g2)

    def mlp():
        cq.cq_fp4_gemm(wu, x, s1, workspace=ws, out=h)
        cq.cq_fp4_gemm(wd, cq.cq_fp4_swiglu_quantize(h, FMT[fmt], s2, out=a), workspace=ws, out=y)

    mlp()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mlp()
    for seed in range(3):
        xs = rows(M, H, dtype, 200 + seed, 0.3)
        x.copy_(xs)
        graph.replay()
        torch.cuda.synchronize()
        check_product(h, *ref.product(*ref.quantize(as64(xs), fmt, g1), *up, fmt, g1, 0.001), H)
        hv = as64(h)   # from here on by what the first product returned
        act = torch.from_numpy(ref.gated(hv[:, :I], hv[:, I:])).to(x.dtype)
        check_product(y, *ref.product(*ref.quantize(as64(act), fmt, g2), *down, fmt, g2, 0.001), I)
    assert cq.cq_gemm_status(ws) == 0


def test_quantize_all_f16_values():
    p = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.float16)
    x = torch.zeros((65536, 32), dtype=torch.float16)
    x[:, 3] = p
    x[:, 4] = p.flip(0)
    x[:, 20] = p.roll(77)
    for fmt in ("mx", "nv"):
        q = cq.cq_fp4_quantize(x.cuda(), FMT[fmt])
        check_bytes(q, *ref.quantize(as64(x), fmt))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", [(1, 300, 512), (9, 300, 512), (16, 600, 8192), (70, 300, 512), (300, 9843, 864)])
def test_rows_apart(M, N, K, fmt):
    """x as columns of a wider matrix, a single row at any distance, the factor with and without an axis: the bits of a copy."""
    w, x, g, y, S = product_case(M, N, K, fmt, "bf16")
    want = cq.cq_fp4_gemm(w, x, g)
    check_product(want, y, S, K)
    wide = torch.full((M, K + 96), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, 64:64 + K] = x
    part = wide[:, 64:64 + K]
    assert part.stride(0) == K + 96
    assert torch.equal(cq.cq_fp4_gemm(w, part, None if g is None else g.reshape(1)), want)
    token, off = torch.arange(M, dtype=torch.int32, device="cuda"), torch.tensor([0, M], dtype=torch.int32, device="cuda")
    routed = cq.cq_fp4_gemm_routed(w, part, token, off, g)
    check_product(routed, y, S, K)
    assert torch.equal(cq.cq_fp4_gemm_routed(w, x, token, off, g), routed)
    if M == 1:
        odd = torch.zeros((3, K + 8), dtype=x.dtype, device="cuda")
        odd[1, :K] = x[0]
        assert torch.equal(cq.cq_fp4_gemm(w, odd[1:2, :K].as_strided((1, K), (3, 1), odd[1].storage_offset()), g), want)
    I = K // 64 * 32
    h = torch.full((M, 2 * I + 32), float("nan"), dtype=x.dtype, device="cuda")
    h[:, 16:16 + 2 * I] = x[:, :2 * I]
    a, b = cq.cq_fp4_swiglu_quantize(h[:, 16:16 + 2 * I], FMT[fmt], g), cq.cq_fp4_swiglu_quantize(x[:, :2 * I], FMT[fmt], g)
    assert all(torch.equal(s, t) for s, t in zip(cq.cq_fp4_unpack(a), cq.cq_fp4_unpack(b)))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_as_many_groups_as_there_may_be(fmt):
    r = np.random.default_rng(12)
    counts = r.integers(0, 4, 512)
    counts[[0, 31, 32, 511]] = 0, 140, 1, 2
    w, x, token, off, g, y, S = routed_case(counts.tolist(), 40, 96, fmt, "bf16")
    ws = cq.cq_fp4_workspace(w, int(counts.sum()))
    check_product(cq.cq_fp4_gemm_routed(w, x, token, off, g, workspace=ws), y, S, 96)
    assert cq.cq_gemm_status(ws) == 0
    with pytest.raises(cq.CubicQuantError):
        cq.cq_fp4_quantize(x, FMT[fmt], g, route_token=token, expert_offset=torch.zeros(514, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("M,N,K", [(4, 300, 512), (100, 300, 512)])
def test_rows_of_zeros_under_their_own_factor(M, N, K):
    """max|x| / 2688 of a matrix of zeros is zero: so are its values and its products."""
    w, x, _, _, _ = product_case(M, N, K, "nv", "bf16")
    x.zero_()
    g = x.abs().amax().float() / 2688
    assert torch.all(cq.cq_fp4_gemm(w, x, g) == 0)
    assert torch.all(cq.cq_fp4_dequantize(cq.cq_fp4_quantize(x, cq.CQ_NVFP4, g)) == 0)


@pytest.mark.parametrize("M", [4, 100])
def test_captured_without_a_workspace_and_between_streams(M):
    """What a call allocates for itself lives as long as the graph; operands that another stream makes are waited for by an event alone."""
    w, x, g, y, S = product_case(M, 1024, 2048, "nv", "bf16")
    want = cq.cq_fp4_gemm(w, x, g)
    static = torch.zeros_like(x)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = cq.cq_fp4_gemm(w, static, g)
    static.copy_(x)
    for _ in range(3):
        out.zero_()
        graph.replay()
        assert torch.equal(out, want)
    side = torch.cuda.Stream()
    for _ in range(20):
        late = torch.full_like(x, float("nan"))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(200000)
            late.copy_(x)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(cq.cq_fp4_gemm(w, late, g), want)
        q = cq.cq_fp4_quantize(late, cq.CQ_NVFP4, g)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = cq.cq_fp4_gemm(w, q)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)
