"""The map of cq_route in front of the other routed products, with padded rows, value by value: 4-bit products, which take its offsets on the device, and cubic ones, which
take them on the host and exactly as many tokens as there are routes.  Tolerances are those of each product's own tests."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_06763_b200 as cq
from oracle import fp4 as ref_fp4
from oracle import route as ref_route
from test_gpu_fp4 import FMT, check_product, g_of
from test_gpu_i8 import rows
from test_gpu_route import as64, check, check_combine
from util import check_y, logical_case, y_to_numpy

pytestmark = pytest.mark.gpu

T, E, TOP, K, N = 60, 4, 2, 512, 256


def routes_of(padded, seed):
    """Logits with rows of padding, one token that may go to one matrix alone, a matrix without routes; their routes and those of the oracle."""
    l = torch.from_numpy(np.random.default_rng(seed).standard_normal((T, E))).float()
    l[T - padded:] = -float("inf")
    l[3, :E - 1] = -float("inf")
    l[:, 1] -= 50.0
    got = cq.cq_route(l.cuda(), TOP)
    check(got, l, TOP, "softmax")
    expert, _ = ref_route.choose(as64(l), TOP, "softmax")
    return got, ref_route.routes(expert, E)


@pytest.mark.parametrize("padded", [0, 15])
@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_in_front_of_4_bit_products(fmt, padded):
    r, (token, off, _) = routes_of(padded, 1)
    x = rows(T, K, "bf16", 1, 0.3)
    gx, gw = 1.0 if fmt == "mx" else 0.03, np.linspace(0.0005, 0.002, E).astype(np.float32)
    W = [ref_fp4.quantize(as64(rows(N, K, "f32", 30 + e, 0.3) * 0.05), fmt, float(gw[e])) for e in range(E)]
    w = cq.cq_fp4_pack(torch.from_numpy(np.stack([ref_fp4.pack(c) for c, _ in W])).cuda(), torch.from_numpy(np.stack([b for _, b in W])).cuda(), FMT[fmt],
                       None if fmt == "mx" else torch.from_numpy(gw).cuda())
    y = cq.cq_fp4_gemm_routed(w, x.cuda(), r.token, r.offset, g_of(fmt, gx))
    xc, xb = ref_fp4.quantize(as64(x), fmt, gx)
    for e in range(E):
        t = token[off[e]:off[e + 1]]
        if len(t):
            check_product(y[off[e]:off[e + 1]], *ref_fp4.product(xc[t], xb[t], *W[e], fmt, gx, float(gw[e]) if fmt == "nv" else 1.0), K)
    out = cq.cq_combine(y, r)
    check_combine(out, y.nan_to_num(), r.row.cpu(), r.weight.cpu(), None)
    assert torch.all(out[T - padded:] == 0)


@pytest.mark.parametrize("padded", [0, 15])
@pytest.mark.parametrize("mode", [cq.CQ_MODEL_DTYPE, cq.CQ_DYN_A8])
def test_in_front_of_cubic_products(mode, padded):
    r, (token, off, _) = routes_of(padded, 2)
    x = rows(T, K, "bf16", 1, 0.3)
    cases = [logical_case(N, K, 4, 128, seed=70 + e) for e in range(E)]
    offset = r.offset.tolist()                                     # on the host: waits
    y = cq.cq_gemm_routed([c.pw for c in cases], x.cuda(), r.token[:offset[-1]], offset, mode)
    want = oracle.gemm_routed([dict(codes=c.codes, s=c.s, a=c.a, b=c.b, B=4, G=128, K=K) for c in cases], x.view(torch.int16).numpy().view(np.uint16), token[:off[-1]], off,
                              "model" if mode == cq.CQ_MODEL_DTYPE else "a8")
    for e in range(E):
        if off[e] < off[e + 1]:
            check_y(y_to_numpy(y[off[e]:off[e + 1]]), want[off[e]:off[e + 1]], f"matrix {e}")
    out = cq.cq_combine(y, r)
    check_combine(out, y, r.row.cpu(), r.weight.cpu(), None)
    assert torch.all(out[T - padded:] == 0)
