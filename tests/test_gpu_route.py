"""Routing to experts and combining on the GPU against the 64-bit oracle (oracle/route.py).

Choices and the map: equal.  Weights, in units u = 2^-24 of the value: logits apart by z round by z, expf 4, 1 + exp and the division under a sigmoid 2, sums of at most 512
terms in order 37 and their terms' own errors as large as the value's, the last division and the factor 2: (2 z + 64) u with z the spread of the row, and
2^-126 where values are subnormal.  Sums of routes: half a step of the output type and a rounding to fp32 for each term.
"""
import numpy as np
import pytest
import torch

import paper_2608_06763_b200 as cq
from oracle import route as ref

pytestmark = pytest.mark.gpu

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SCORE = {"softmax": cq.CQ_SOFTMAX, "sigmoid": cq.CQ_SIGMOID}


def as64(t):
    return t.detach().double().cpu().numpy()


def some_logits(T, E, dtype, seed, spread=1.5):
    r = np.random.default_rng(seed)
    return torch.from_numpy(spread * r.standard_normal((T, E)) + r.standard_normal(E)).float().to(DTYPE[dtype])


def some_bias(E, seed, size=0.1):
    return torch.from_numpy(size * np.random.default_rng(seed + 999).standard_normal(E)).float()


def check(got, l, top, score, bias=None, **how):
    """got: Routes for logits l (on the CPU)."""
    T, E = l.shape
    l64, b64 = as64(l), None if bias is None else as64(bias)
    expert, weight = ref.choose(l64, top, score, b64, **how)
    assert np.array_equal(got.expert.cpu().numpy(), expert), "experts"
    c = ref.cleaned(l64)
    with np.errstate(invalid="ignore"):
        z = np.minimum(np.nan_to_num(c.max(axis=1) - np.where(c > -np.inf, c, np.inf).min(axis=1), posinf=0.0, neginf=0.0, nan=0.0), 200.0)   # beyond, weights are zeros
    w = as64(got.weight)
    allowed = np.abs(weight) * ((2 * z + 64) * 2.0 ** -24)[:, None] + 2.0 ** -126 * max(1.0, how.get("scale", 1.0))
    assert np.all(np.abs(w - weight) <= allowed), float((np.abs(w - weight) / allowed).max())
    token, offset, row = ref.routes(expert, E)
    assert np.array_equal(got.offset.cpu().numpy(), offset), "offsets"
    assert np.array_equal(got.token.cpu().numpy(), token), "tokens"
    assert np.array_equal(got.row.cpu().numpy(), row), "rows"


def call(l, top, score, bias=None, groups=1, kept=1, best=2, renormalise=True, scale=1.0, **more):
    return cq.cq_route(l if l.is_cuda else l.cuda(), top, SCORE[score], bias=None if bias is None else bias.cuda(), groups=groups, groups_kept=kept, group_best=best,
                       renormalise=renormalise, scale=scale, **more)


def both(l, top, score, bias=None, **how):
    got = call(l, top, score, bias, **how)
    check(got, l, top, score, bias, **how)
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,top", [(1, 1, 1), (1, 64, 4), (3, 2, 2), (31, 7, 3), (64, 8, 2), (65, 30, 6), (200, 60, 4), (129, 72, 8), (1000, 256, 8), (33, 500, 32), (700, 512, 31), (5000, 16, 2)])
def test_plain(T, E, top, score, dtype):
    l = some_logits(T, E, dtype, T + E)
    both(l, top, score)
    both(l, top, score, renormalise=False, scale=2.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,top", [(1, 64, 4), (31, 7, 3), (65, 30, 6), (200, 60, 32), (1000, 256, 8), (40, 512, 32), (300, 33, 32)])
def test_bias(T, E, top, score, dtype):
    l = some_logits(T, E, dtype, T + E + 1)
    both(l, top, score, some_bias(E, T))
    both(l, top, score, torch.zeros(E), renormalise=False)
    both(l, top, score, some_bias(E, T, 1e-6), scale=0.5)
    both(l, top, score, some_bias(E, T, 1e3))


@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,top,groups,kept,best", [(1, 256, 8, 8, 4, 2), (300, 256, 8, 8, 4, 2), (77, 160, 6, 8, 3, 1), (65, 30, 5, 3, 1, 2), (64, 12, 2, 6, 2, 2), (50, 32, 16, 32, 16, 2),
                                                      (200, 510, 32, 17, 8, 2), (90, 72, 9, 2, 1, 1), (1500, 64, 4, 4, 4, 2), (40, 512, 32, 32, 2, 2), (64, 14, 3, 7, 3, 1)])
def test_groups(T, E, top, groups, kept, best, score, with_bias):
    for dtype in ("bf16", "f32"):
        l = some_logits(T, E, dtype, T + E + 2)
        both(l, top, score, some_bias(E, T) if with_bias else None, groups=groups, kept=kept, best=best)


@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_groups_of_which_one_or_none_is_left(score, best):
    r = np.random.default_rng(3)
    l = some_logits(400, 48, "f32", 11)
    l[torch.from_numpy(r.random((400, 48)) < np.linspace(0.3, 1.0, 400)[:, None])] = float("-inf")
    for bias in (None, some_bias(48, 3, 0.5)):
        both(l, 6, score, bias, groups=12, kept=5, best=best)


@pytest.mark.parametrize("E,top,groups,kept", [(64, 8, 1, 1), (64, 6, 8, 3), (512, 32, 1, 1), (256, 30, 8, 4)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_lowest_and_infinite_biases(score, E, top, groups, kept):
    """The type's lowest value is a bias like any other, and so is infinity: experts with it go by their logits."""
    l = some_logits(70, E, "f32", E + top)
    least, most = torch.finfo(torch.float32).min, float("inf")
    for value in (least, most):
        for share in (0.05, 0.5, 0.97, 1.0):
            b = some_bias(E, int(100 * share))
            b[torch.from_numpy(np.random.default_rng(E).random(E) < share)] = value
            both(l, top, score, b, groups=groups, kept=kept)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_scores_closer_than_32_bits_tell(score):
    """Biases that bring all choice scores of a row within a few units of fp32: decided in 64 bits."""
    for E, top, groups in ((64, 8, 1), (256, 8, 1), (256, 8, 8), (60, 31, 1), (33, 32, 1)):
        l = some_logits(1, E, "f32", E).repeat(20, 1)
        l += 1e-7 * torch.from_numpy(np.random.default_rng(E).standard_normal((20, E))).float()
        b = torch.from_numpy(0.5 - ref.scores(as64(l[:1]), score)[0]).float()
        c = ref.scores(as64(l), score) + as64(b)
        assert (c.max() - c.min()) < 1e-6 and len(np.unique(c[0])) > E // 2
        both(l, top, score, b, groups=groups, kept=max(1, groups // 2))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_equals_go_to_the_lowest_index(score):
    E = 96
    l = torch.zeros((70, E), dtype=torch.bfloat16)
    l[10:40] = torch.from_numpy(np.random.default_rng(0).integers(-2, 3, (30, E))).to(torch.bfloat16)
    l[40:50, 1::2] = -0.0                                        # the same number as 0
    for bias in (None, torch.zeros(E), torch.full((E,), 0.25)):
        for groups in (1, 8):
            got = both(l, 6, score, bias, groups=groups, kept=max(1, groups // 4))
            assert got.expert[0].tolist() == list(range(6))
    l = torch.tensor([[40.0, 41.0, 42.0, 41.0]])                  # a sigmoid in 64 bits is 1 for all of them: the larger logit first
    assert both(l, 4, "sigmoid").expert[0].tolist() == [2, 1, 3, 0]
    assert both(l, 4, "sigmoid", torch.zeros(4)).expert[0].tolist() == [2, 1, 3, 0]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_masks(score, dtype):
    """Rows that mask all, all but some, all but fewer than `top`; masks of the type's lowest value; NaN; infinities."""
    E, top = 40, 6
    l = some_logits(90, E, dtype, 3)
    inf = float("inf")
    l[0] = -inf
    l[1, :] = -inf
    l[1, 17] = 2.0
    l[2, 3:] = -inf
    l[3] = float("nan")
    l[4, ::2] = float("nan")
    l[5] = torch.finfo(l.dtype).min
    l[6, 5:] = torch.finfo(l.dtype).min
    l[7, 9] = inf
    l[8, [3, 9, 30]] = inf
    l[9] = inf
    l[70:] = -inf
    bias = some_bias(E, 4)
    how = [dict(), dict(renormalise=False), dict(groups=5, kept=2), dict(groups=8, kept=8, best=1)]
    for h in how:
        both(l, top, score, None, **h)
        got = both(l, top, score, bias, **h)
        assert torch.all(got.expert[70:] == -1) and torch.all(got.weight[70:] == 0) and torch.all(got.row[70:] == -1)
    bias[[2, 17]] = -inf
    bias[3] = float("nan")
    bias[30] = inf
    bias[31] = inf
    for h in how:
        got = both(l, top, score, bias, **h)
        assert not torch.isin(got.expert, torch.tensor([2, 3, 17], dtype=torch.int32, device="cuda")).any()
    got = both(torch.full((100, E), -inf, dtype=DTYPE[dtype]), top, score, bias)
    assert got.offset.eq(0).all() and got.token.eq(-1).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_far_logits(score):
    """Scores that vanish in 32 bits: weights over the sum of the chosen are still theirs."""
    l = torch.from_numpy(np.random.default_rng(5).standard_normal((40, 24)) * 3).float()
    l[:10] -= 300.0
    l[10:20] += 300.0
    l[20:30] *= 100.0
    bias = torch.zeros(24)
    bias[20:] = 5.0                                               # chosen against far larger scores
    l[30:, 20:] -= 200.0
    for b in (None, bias):
        for renormalise in (True, False):
            both(l, 4, score, b, renormalise=renormalise)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_apart_and_at_odd_addresses(dtype):
    base = torch.full((90, 300), float("nan"), dtype=DTYPE[dtype]).cuda()
    for E, at in ((64, 3), (64, 8), (256, 1), (60, 16), (8, 5)):
        l = some_logits(90, E, dtype, E)
        base.fill_(float("nan"))
        base[:, at:at + E] = l.cuda()
        got = call(base[:, at:at + E], 4, "softmax", some_bias(E, 1))
        check(got, l, 4, "softmax", some_bias(E, 1))
        one = base[5:6, at:at + E]
        check(call(one, 4, "sigmoid"), l[5:6], 4, "sigmoid")


@pytest.mark.parametrize("T", [1, 64, 65, 3000, 40000])
def test_many_tokens_twice(T):
    """The map of counts of every size, the same bits again, and into the same buffers."""
    l = some_logits(T, 24, "bf16", T).cuda()
    l[T // 3: T // 2] = l[0]                                       # runs of tokens to the same experts
    out, ws = cq.cq_routes_empty(T, 24, 5), cq.cq_route_workspace(T, 24)
    first = call(l, 5, "sigmoid", workspace=ws, out=out)
    check(first, l.cpu(), 5, "sigmoid")
    keep = [t.clone() for t in (first.expert, first.weight, first.token, first.offset, first.row)]
    for t in (out.expert, out.token, out.offset, out.row):
        t.fill_(77)
    out.weight.fill_(float("nan"))
    ws.fill_(255)
    again = call(l, 5, "sigmoid", workspace=ws, out=out)
    assert again is out
    assert all(torch.equal(a, b) for a, b in zip(keep, (again.expert, again.weight, again.token, again.offset, again.row)))


def test_logits_beyond_32_bits():
    """4.3 M rows of 512 logits: offsets past 2^31 values."""
    T, E = 4300000, 512
    few = some_logits(256, E, "bf16", 8)
    l = few.cuda().repeat(T // 256 + 1, 1)[:T]
    got, small = call(l, 2, "softmax"), call(few, 2, "softmax")
    for lo in (0, 2 ** 31 // E // 256 * 256, T // 256 * 256 - 256):
        assert torch.equal(got.expert[lo:lo + 256], small.expert) and torch.equal(got.weight[lo:lo + 256], small.weight)
    assert int(got.offset[-1]) == 2 * T
    assert torch.equal(got.offset.diff(), torch.bincount(got.expert.flatten(), minlength=E).int())
    of = torch.repeat_interleave(torch.arange(E, device="cuda"), got.offset.diff().long())
    assert torch.equal(of[got.row.flatten().long()], got.expert.flatten().long())
    assert torch.equal(got.token[got.row.flatten().long()], torch.arange(T, device="cuda", dtype=torch.int32).repeat_interleave(2))
    same = of[1:] == of[:-1]
    assert torch.all(got.token.diff()[same] > 0)


def test_captured_and_on_other_streams():
    T, E, top = 300, 64, 4
    l = torch.zeros((T, E), dtype=torch.bfloat16, device="cuda")
    bias = some_bias(E, 2).cuda()
    out, ws = cq.cq_routes_empty(T, E, top), cq.cq_route_workspace(T, E)
    cq.cq_route(l, top, bias=bias, workspace=ws, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cq.cq_route(l, top, bias=bias, workspace=ws, out=out)
    for seed in range(3):
        new = some_logits(T, E, "bf16", seed)
        if seed == 2:
            new[100:] = -float("inf")
        l.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        check(out, new, top, "softmax", bias.cpu())
    side = torch.cuda.Stream()
    a, b = some_logits(200, 256, "f32", 10), some_logits(50, 30, "f32", 11)
    ga, gb = a.cuda(), b.cuda()
    torch.cuda.synchronize()
    for _ in range(10):
        with torch.cuda.stream(side):
            first = cq.cq_route(ga, 8)
        second = cq.cq_route(gb, 3)
    torch.cuda.synchronize()
    check(first, a, 8, "softmax")
    check(second, b, 3, "softmax")


# ---------------------------------------------------------------- combine
def combine_case(T, N, top, R, dtype, seed, add):
    r = np.random.default_rng(seed)
    y = torch.from_numpy(r.standard_normal((R, N))).float().to(DTYPE[dtype])
    row = torch.from_numpy(r.integers(-1, R, (T, top)).astype(np.int32))
    weight = torch.from_numpy(r.random((T, top))).float()
    return y, row, weight, torch.from_numpy(r.standard_normal((T, N))).float().to(DTYPE[dtype]) if add else None


def as_routes(row, weight):
    z = torch.zeros(max(2, row.numel()), dtype=torch.int32, device="cuda")
    return cq.Routes(row.cuda(), weight.cuda(), z[:row.numel()], z[:2], row.cuda())


def check_combine(got, y, row, weight, add):
    want, size = ref.combine(as64(y), as64(weight), row.numpy(), None if add is None else as64(add))
    t = got.dtype
    allowed = torch.finfo(t).eps / 2 * np.abs(want) * (1 + 2.0 ** -10) + (row.shape[1] + 1) * 2.0 ** -24 * size + torch.finfo(t).tiny
    err = np.abs(as64(got) - want)
    assert np.all(err <= allowed), float((err / allowed).max())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("T,N,top,R", [(1, 1, 1, 1), (1, 2048, 4, 4), (13, 2056, 4, 50), (7, 333, 3, 9), (130, 4096, 8, 1000), (300, 1000, 32, 77), (5, 8, 5, 2), (2, 70000, 2, 3)])
def test_combine(T, N, top, R, add, dtype):
    y, row, weight, a = combine_case(T, N, top, R, dtype, T + N, add)
    got = cq.cq_combine(y.cuda(), as_routes(row, weight), add=None if a is None else a.cuda())
    assert got.dtype == y.dtype
    check_combine(got, y, row, weight, a)


@pytest.mark.parametrize("N", [2, 3, 6, 255, 510, 1022, 1025, 2046, 4095, 4100])
@pytest.mark.parametrize("shift", [0, 1, 2])
def test_combine_of_any_length_and_alignment(N, shift):
    """One, two or eight values to a load, by the alignment of all rows; values beside the rows are left alone."""
    T, top, R = 37, 5, 60
    y, row, weight, add = combine_case(T, N, top, R, "bf16", N + shift, True)
    apart = torch.full((T, N + shift), 7.0, dtype=y.dtype, device="cuda")
    cq.cq_combine(y.cuda(), as_routes(row, weight), add=add.cuda(), out=apart[:, :N])
    check_combine(apart[:, :N], y, row, weight, add)
    assert torch.all(apart[:, N:] == 7.0)


def test_combine_rows_apart_in_place_and_unread_rows():
    T, N, top, R = 40, 512, 4, 60
    y, row, weight, a = combine_case(T, N, top, R, "bf16", 1, True)
    row[3] = -1
    row[4, 1:] = -1
    row[5, 2] = R                                                  # outside
    wide = torch.full((R + 5, N + 40), float("nan"), dtype=y.dtype, device="cuda")
    wide[:R, 8:8 + N] = y.cuda()
    used = np.unique(row.numpy()[(row.numpy() >= 0) & (row.numpy() < R)])
    unused = np.setdiff1d(np.arange(R), used)
    wide[torch.from_numpy(unused).cuda()] = float("nan")           # what no choice names may hold anything
    big = torch.zeros((T, N + 24), dtype=y.dtype, device="cuda")
    out = big[:, 16:16 + N]
    out.copy_(a)
    got = cq.cq_combine(wide[:R, 8:8 + N], as_routes(row, weight), add=out, out=out)
    assert got is out and torch.isfinite(got).all()
    check_combine(got, y, row, weight, a)
    assert torch.all(big[:, :16] == 0) and torch.all(big[:, 16 + N:] == 0)
    odd = torch.empty((R, N + 3), dtype=y.dtype, device="cuda")[:, 1:1 + N]
    odd.copy_(y)
    check_combine(cq.cq_combine(odd, as_routes(row, weight), add=a.cuda()), y, row, weight, a)
    assert torch.all(cq.cq_combine(y.cuda(), as_routes(row, weight))[3] == 0)
    none = cq.cq_combine(y[:0].cuda(), as_routes(torch.full((T, top), -1, dtype=torch.int32), weight), add=a.cuda())
    assert torch.equal(none.cpu(), a)


def test_combine_takes_back_what_routing_gave():
    """Each token's own row as the output of each of its routes: the token again, times the sum of its weights."""
    T, E, top, N = 500, 40, 6, 264
    x = torch.from_numpy(np.random.default_rng(2).standard_normal((T, N))).float().to(torch.bfloat16).cuda()
    r = call(some_logits(T, E, "f32", 9), top, "sigmoid", some_bias(E, 3))
    y = x[r.token.long()]
    got = cq.cq_combine(y, r)
    check_combine(got, y, r.row.cpu(), r.weight.cpu(), None)
    assert (got.float() - x.float()).abs().max() <= 2.0 ** -7 * x.float().abs().max()


def test_combine_beyond_32_bits():
    """Rows past 2^31 values."""
    R, N = 300000, 8192
    y = torch.zeros((R, N), dtype=torch.bfloat16, device="cuda")
    y[-3:] = torch.tensor([1.0, 2.0, 3.0], device="cuda")[:, None].bfloat16()
    row = torch.tensor([[R - 1, R - 3], [0, R - 2]], dtype=torch.int32)
    got = cq.cq_combine(y, as_routes(row, torch.tensor([[1.0, 2.0], [7.0, 0.5]])))
    assert torch.all(got[0] == 5.0) and torch.all(got[1] == 1.0)
