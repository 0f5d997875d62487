"""Equals on the border of the choice: the last expert that is chosen and the first that is not have the same logit and bias, and another one, which 32 bits cannot
tell from them, lies in front of both in 64.  Against the 64-bit oracle (oracle/route.py): choices, weights and the map as in test_gpu_route.py."""
import itertools

import numpy as np
import pytest
import torch

from test_gpu_route import DTYPE, both, call, check

pytestmark = pytest.mark.gpu

# Large logits under sigmoids; small scores beside a large one, or beside a common bias, under a softmax.
ROWS = {"sigmoid": [[41, 41, 42], [20, 20, 30, -1], [41, 41, 41, 42, 43], [18, 18, 18.0625, -2, 50], [30, 30, 31, 31, 32]],
        "softmax": [[20, 0, 0, 1], [30, -2, -2, -1, 3], [9, -9, -9, -8.9375, -9.0625], [25, 1, 1, 2, 2]]}


def orders(row):
    return torch.tensor(sorted(set(itertools.permutations(row))), dtype=torch.float32)


@pytest.mark.parametrize("value", [0.0, 0.25, -3.0])
@pytest.mark.parametrize("score,which", [(s, i) for s in ROWS for i in range(len(ROWS[s]))])
def test_in_every_order(score, which, value):
    l = orders(ROWS[score][which])
    n = l.shape[1]
    apart = torch.full((len(l), 40), -float("inf"))
    apart[:, torch.arange(n) * 9 + 2] = l                      # a lane each, with experts that may not be chosen between them
    for some in (l, apart):
        for top in range(1, n + 1):
            for dtype in ("f32", "bf16"):
                both(some.to(DTYPE[dtype]), top, score, torch.full((some.shape[1],), value))
    few = l[:9]
    for top in range(1, n + 1):
        both(few, top, score, torch.full((n,), value), renormalise=False)   # one block has all tokens


@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_in_groups(score, best):
    for row in ROWS[score]:
        l = orders(row)
        n = l.shape[1]
        two = torch.cat([l, l.flip(0)], dim=1)
        for value in (0.0, 0.25):
            for kept in (1, 2):
                for top in range(1, n + 1):
                    both(two, top, score, torch.full((2 * n,), value), groups=2, kept=kept, best=best)


@pytest.mark.parametrize("top", [1, 2, 7, 8, 31, 32])
@pytest.mark.parametrize("E,equals", [(64, 20), (64, 40), (96, 60), (256, 200), (512, 500)])
def test_many_equals(E, equals, top):
    """Up to all experts equal but a few that only 64 bits tell from them, anywhere; more of them than there is room for."""
    r = np.random.default_rng(E + equals + top)
    for score, same, larger, rest in (("sigmoid", 41.0, 42.0, -1.0), ("sigmoid", 25.0, 26.0, 26.0), ("softmax", 0.0, 0.0625, 20.0)):
        l = np.full((60, E), rest if score == "sigmoid" else -30.0)
        for t in range(len(l)):
            at = r.permutation(E)
            l[t, at[:equals]] = same
            l[t, at[equals:equals + t % 4]] = larger
            if score == "softmax":
                l[t, at[-1]] = rest
        for value in (0.0, 0.25):
            both(torch.from_numpy(l).float(), top, score, torch.full((E,), value))
            both(torch.from_numpy(l).float(), min(top, E // 8), score, torch.full((E,), value), groups=4, kept=2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_biases_that_are_equal_in_parts(score):
    """Integer logits of a few values, biases of two: equal pairs of every kind on the border."""
    r = np.random.default_rng(17)
    for E, top in ((16, 3), (64, 8), (256, 8), (256, 30)):
        l = torch.from_numpy(r.integers(17, 24, (300, E)) * 1.0).float() if score == "sigmoid" else torch.from_numpy(r.integers(-3, 1, (300, E)) * 1.0).float()
        if score == "softmax":
            l[:, 5] = 18.0
        b = torch.from_numpy(np.where(r.random(E) < 0.5, 0.25, 0.25 + 2.0 ** -20)).float()
        for dtype in ("bf16", "f32"):
            both(l.to(DTYPE[dtype]), top, score, b)


def test_the_excluded_are_not_compared():
    """Experts without a logit or a bias beside equals on the border."""
    l = torch.tensor([[41.0, 41.0, 42.0, -float("inf"), float("nan"), 43.0]]).repeat(20, 1)
    b = torch.tensor([0.5, 0.5, 0.5, 0.5, 0.5, -float("inf")])
    for top in range(1, 6):
        got = call(l, top, "sigmoid", b)
        check(got, l, top, "sigmoid", b)
        assert got.expert[0].tolist() == [2, 0, 1, -1, -1][:top]
