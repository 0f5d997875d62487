"""The largest sum that packed codes have: -128 on both sides over the longest K, 2^17 * 2^14 = 2^31, which is no signed 32-bit integer.  Rows of one code each, so that the
sums are products of whole numbers: y = float(sum) * (w_scale * x_scale), rounded once, bit for bit."""
import pytest
import torch

import paper_2608_06763_b200 as cq

pytestmark = pytest.mark.gpu

K = 131072
CODES = (-128, 127, -128, -127, 0, 1)
# (channels, rows of x to a tile, runs of K, whether the product quantises x itself), M, N
PLANS = [((128, 64, 1, False), 3, 10000), ((128, 64, 2, False), 13, 4500), ((128, 64, 4, False), 1, 100), ((128, 64, 4, False), 40, 301), ((128, 128, 1, False), 70, 10000),
         ((128, 128, 2, False), 1000, 1000), ((128, 128, 4, False), 300, 1000), ((128, 240, 2, False), 1500, 1000), ((128, 240, 4, False), 700, 1001),
         ((256, 128, 1, False), 1000, 2000), ((256, 192, 1, False), 1500, 2001), ((256, 256, 1, False), 400, 7000)]


def constant_rows(n, k):
    """Codes [n, k] of one value a row, and the values."""
    value = torch.tensor(CODES, dtype=torch.int8, device="cuda").repeat(n // len(CODES) + 1)[:n]
    return value[:, None].expand(n, k).contiguous(), value


def check(M, N, k, plan=None, dtype=torch.bfloat16):
    if plan is not None:
        assert tuple(cq.cq_debug_i8_plan(M, N, k, quantised=True).values()) == plan
    (wc, wv), (xc, xv) = constant_rows(N, k), constant_rows(M, k)
    wd = torch.exp2(torch.randint(-24, -20, (N,), generator=torch.Generator("cuda").manual_seed(N), device="cuda").float())
    xd = torch.exp2(-torch.rand(M, generator=torch.Generator("cuda").manual_seed(M), device="cuda")) * 1e-3
    out = torch.empty((M, N), dtype=dtype, device="cuda")
    got = cq.cq_i8_gemm(cq.cq_i8_pack(wc, wd), cq.cq_i8_pack(xc, xd), out=out)
    total = xv.double()[:, None] * wv.double()[None, :] * k
    assert total.max() == 16384 * k
    want = (total.float() * (wd[None, :] * xd[:, None])).to(dtype)
    assert torch.equal(got, want), (int((got != want).sum()), got.flatten()[:4].tolist(), want.flatten()[:4].tolist())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("plan,M,N", PLANS)
def test_minus_128_on_both_sides(plan, M, N, dtype):
    """Every kind of tile, whole K and runs of it."""
    check(M, N, K, plan, dtype)


def test_one_piece_less():
    for M in (3, 40):
        check(M, 300, K - 16)
