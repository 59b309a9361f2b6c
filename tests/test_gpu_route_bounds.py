"""Routing at the edges of what 32 bits can decide and of what one launch holds, against tests/blocks_ref.py.

Tolerances as in tests/test_gpu_experts.py: ids, offsets and order equal, weights within one rounding to fp32.
"""

import numpy as np
import pytest

from tests import blocks_ref as ref
from tests.test_gpu_experts import _check_route, _say, sd, torch  # noqa: F401  (the last two are fixtures)

pytestmark = pytest.mark.gpu

LOWEST = float(np.finfo(np.float32).min)


@pytest.mark.parametrize("T", [8, 1500])
@pytest.mark.parametrize("groups,size", [(4, 2), (8, 3), (8, 4), (4, 150)])
@pytest.mark.parametrize("B", [100.0, 1000.0])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_groups_whose_two_best_cancel(torch, sd, score, B, groups, size, T):  # noqa: F811
    """Biases of +B and -B on a group's two best experts: the choices are rounded at B's magnitude in 32 bits, and their
    sums, which decide the groups, differ by far less than that rounding."""
    rng = np.random.default_rng(int(B) + groups * size + T)
    bias = np.full((groups, size), -2 * B, np.float32)
    mine = B * (1 + np.arange(groups) / 64)  # so far apart that the experts' own order is never in doubt
    bias[:, 0], bias[:, size - 1] = mine, -mine
    near = 10.0 ** rng.uniform(-6, -3, (T, 1, 1)) * rng.standard_normal((T, groups, 1))
    l = (rng.standard_normal((T, 1, size)) + near).reshape(T, groups * size).astype(np.float32)
    _say("groups that cancel", score, B, groups, size, T)
    _check_route(torch, sd, l.astype(np.float64), torch.float32, 2, score, bias.reshape(-1), groups, 2, 2, True, 1.0)


@pytest.mark.parametrize("T", [3, 200])
@pytest.mark.parametrize("low", [LOWEST, -3e38])
@pytest.mark.parametrize("spread", [1.0, 0.75])
@pytest.mark.parametrize("best", [1, 2])
def test_groups_masked_by_a_bias_of_the_lowest_value(torch, sd, best, spread, low, T):  # noqa: F811
    """A bias of the type's lowest value puts experts last and leaves them choosable: the sum of two such choices is a
    finite 64-bit number, so their group stays where fewer others do than groups_kept, and only -inf takes it out."""
    rng = np.random.default_rng(T)
    for groups, size in ((4, 4), (8, 3)):
        bias = (rng.integers(-100, 101, (groups, size)) * np.float32(1e-3)).astype(np.float32)
        # masks of one value, and masks that differ, which 32 bits can tell apart
        bias[[0, groups - 1]] = low * np.linspace(1, spread, 2 * size, dtype=np.float32).reshape(2, size)
        bias[1, 1:] = low * np.linspace(spread, 1, size - 1, dtype=np.float32)  # an open expert beside masked ones
        bias[2] = -np.inf
        l = rng.standard_normal((T, groups * size)).astype(np.float32)
        for score in ("softmax", "sigmoid"):
            for kept in (1, groups - 2, groups - 1, groups):
                _say("groups masked", best, spread, low, T, groups, score, kept)
                with np.errstate(over="ignore"):
                    _check_route(torch, sd, l.astype(np.float64), torch.float32, min(6, size * kept), score,
                                 bias.reshape(-1), groups, kept, best, True, 1.0)


@pytest.mark.parametrize("high", [-LOWEST, 3e38, np.inf])
def test_groups_raised_by_a_bias_of_the_largest_value(torch, sd, high):  # noqa: F811
    rng = np.random.default_rng(6)
    bias = np.zeros((8, 4), np.float32)
    bias[3, 1:3] = high
    bias[5] = high
    bias[6, 2] = high
    l = rng.standard_normal((50, 32)).astype(np.float32)
    for score in ("softmax", "sigmoid"):
        for best in (1, 2):
            for kept in (1, 2, 4):
                with np.errstate(over="ignore", invalid="ignore"):
                    _check_route(torch, sd, l.astype(np.float64), torch.float32, 4, score, bias.reshape(-1), 8, kept,
                                 best, True, 1.0)


@pytest.mark.parametrize("T", [4, 70])
@pytest.mark.parametrize("E,groups", [(12, 1), (88, 1), (88, 4), (300, 1), (700, 2)])
def test_equal_logits_beside_others_of_the_same_score(torch, sd, E, groups, T):  # noqa: F811
    """More experts with the largest logit than places, and lower logits whose 64-bit scores are the same: the lowest
    experts of all of these are taken, not those of the larger logit."""
    rng = np.random.default_rng(E + T)
    for score, low, high in (("sigmoid", 50.0, np.nextafter(np.float32(50), np.float32(60))), ("sigmoid", 40.0, 300.0),
                             ("sigmoid", -5000.0, -2000.0), ("softmax", -5000.0, -2000.0), ("softmax", 1e-30, 2e-30)):
        l = np.full((T, E), low, np.float32)
        for t in range(T):
            l[t, rng.permutation(E)[:E // 3]] = high
        if score == "softmax" and low < 0:
            l[:, E // 2] = 1.0
        l[1::3, 2] = -np.inf
        l[2::3, 1] = low - abs(low) / 2  # lower still: of another score, or of the same one too
        for k in (1, 2, E // 3 - 1, E // 3):
            _say("equal logits", score, low, E, groups, T, k)
            with np.errstate(over="ignore", invalid="ignore"):
                _check_route(torch, sd, l.astype(np.float64), torch.float32, min(k, 64, E // groups), score, None, groups, 1, 1,
                             True, 1.0)


def test_more_tokens_than_one_launch_holds(torch, sd):  # noqa: F811
    """2^28 tokens and a few, at 16 lanes each: 2^32 threads and more.  Two experts, so that the definition is one
    comparison and one exponential for a token."""
    T = (1 << 28) + 5
    g = torch.Generator(device="cuda").manual_seed(9)
    logits = torch.randn(T, 2, generator=g, device="cuda", dtype=torch.bfloat16)
    logits[-3, 1] = -float("inf")
    logits[T // 2] = -float("inf")
    _say("many tokens", T)
    got = sd.route(logits, 1, normalize=False)
    part = 1 << 24
    for t in range(0, T, part):
        l = logits[t:t + part].double()
        one = l[:, 1] > l[:, 0]
        there = l.amax(dim=1) > -float("inf")
        assert torch.equal(got.ids[t:t + part, 0], torch.where(there, one.int(), -1))
        want = torch.where(there, 1 / (1 + torch.exp(-(l[:, 1] - l[:, 0]).abs())), 0.0)
        assert bool(((got.weight[t:t + part, 0].double() - want).abs() <= 2.0 ** -23 * want).all())
    ones = int((got.ids == 1).sum())
    zeros = T - 1 - ones
    assert got.offsets.tolist() == [0, zeros, T - 1] and int(got.order[-1]) == -1
    order = got.order[:T - 1].long()
    assert bool((got.ids[order[:zeros], 0] == 0).all()) and bool((got.ids[order[zeros:], 0] == 1).all())
    for run in (order[:zeros], order[zeros:]):  # ascending within an expert, so each slot once
        assert bool((run[1:] > run[:-1]).all())
