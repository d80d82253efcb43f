"""Choices by scores that are too near to 0 or 1 for fp32 or double to tell apart, against decimal arithmetic of as many digits as they need."""
import decimal

import numpy as np
import pytest
import torch

import paper_1912_02057_b200 as rtn

pytestmark = pytest.mark.gpu

D = decimal.Decimal


def choices(x, k, kind, bias, groups=1, kept=1, top=1):
    """x: fp32 [T, E]; bias: fp32 [E].  Experts [T, k], in the order of exact scores."""
    with decimal.localcontext() as ctx:
        span = np.abs(x).max() if kind == rtn.SCORE_SIGMOID else (x.max(1) - x.min(1)).max()
        ctx.prec = 80 + int(span / 2.3)                         # (the smallest score, beside 1, and 80 digits of it)
        out = []
        for row in x:
            e = [D(float(v)).exp() for v in row]
            s = [v / (1 + v) for v in e] if kind == rtn.SCORE_SIGMOID else [v / sum(e) for v in e]
            c = [a + D(float(b)) for a, b in zip(s, bias)]
            size = len(row) // groups
            value = [sum(sorted(c[g * size:(g + 1) * size], reverse=True)[:top]) for g in range(groups)]
            best = sorted(range(groups), key=lambda g: (-value[g], g))[:kept]
            free = [i for i in range(len(row)) if i // size in best]
            out.append(sorted(free, key=lambda i: (-c[i], i))[:k])
    return np.array(out, np.int32)


def check(x, k, kind, bias=None, groups=1, kept=1, top=1):
    want = choices(x, k, kind, np.zeros(x.shape[1], np.float32) if bias is None else bias, groups, kept, top)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    for renormalise in (True, False):
        got = rtn.rtn_route_experts(dev(x), k, score=kind, bias=None if bias is None else dev(bias), groups=groups, kept_groups=kept, group_top=top,
                                    renormalise=renormalise)
        assert np.array_equal(got.experts.cpu().numpy(), want)
        # their weights: the exponent's rounding (a unit for each unit of distance to the largest logit, or to 0), the exponential, sums, the quotient
        y = np.take_along_axis(x, want, 1).astype(np.float64)
        low = y if kind == rtn.SCORE_SOFTMAX else np.minimum(y, 0.0) - np.log1p(np.exp(-np.abs(y)))
        every = x.astype(np.float64)
        most = every.max(1, keepdims=True) if kind == rtn.SCORE_SOFTMAX and not renormalise else low.max(1, keepdims=True) if renormalise else 0.0
        w = np.exp(low - most)
        if renormalise:
            w /= w.sum(1, keepdims=True)
        elif kind == rtn.SCORE_SOFTMAX:
            w /= np.exp(every - most).sum(1, keepdims=True)
        off = np.abs(got.weights.cpu().numpy() - w)
        assert (off <= (np.abs(low - most) + 80) * 2.0 ** -24 * w + 1e-37).all()
        # and the plan of their rows
        start, tokens, place = (t.cpu().numpy() for t in (got.start, got.tokens, got.place))
        assert np.array_equal(np.diff(start), np.bincount(want.ravel(), minlength=x.shape[1]))
        assert np.array_equal(np.sort(place.ravel()), np.arange(want.size)) and np.array_equal(tokens[place], np.arange(len(x))[:, None] + 0 * place)


def biases(r, E):
    two = np.where(np.arange(E) % 3 == 0, np.float32(0.25), np.float32(0.25) + np.float32(2.0 ** -20)).astype(np.float32)
    return [np.zeros(E, np.float32), np.full(E, 0.3, np.float32), np.full(E, -1e6, np.float32), two, (0.1 * r.standard_normal(E)).astype(np.float32)]


@pytest.mark.parametrize("kind,low,high", [(1, 30.0, 80.0), (1, 36.0, 38.0), (1, -80.0, -30.0), (1, -1e-9, 1e-9), (0, -700.0, 0.0), (0, -40.0, 40.0), (0, -1400.0, 0.0)], ids=str)
@pytest.mark.parametrize("E,k", [(24, 24), (70, 6)], ids=str)
def test_route_by_scores_that_saturate(E, k, kind, low, high):
    r = np.random.default_rng(int(high) + E + 100)
    for bias in biases(r, E):
        x = r.uniform(low, high, (3, E)).astype(np.float32)
        x[1] = np.sort(x[1])                                    # the best last, and the best first
        x[2] = -np.sort(-x[2])
        x[0, 5], x[0, 7] = x[0, 3], x[0, 4]                     # ties go to the lowest index
        check(x, k, kind, bias)


@pytest.mark.parametrize("kind,low,high", [(1, 30.0, 60.0), (1, -60.0, -30.0), (0, -300.0, 0.0)], ids=str)
@pytest.mark.parametrize("E,groups,kept,top,k", [(32, 4, 2, 2, 6), (60, 6, 2, 3, 4), (128, 8, 4, 4, 8)], ids=str)
def test_route_by_groups_of_scores_that_saturate(E, groups, kept, top, k, kind, low, high):
    r = np.random.default_rng(E)
    for bias in [None] + biases(r, E):
        x = r.uniform(low, high, (2, E)).astype(np.float32)
        x[1] = np.sort(x[1])
        check(x, k, kind, bias, groups, kept, top)


def test_route_equal_choices_still_go_to_the_lowest_index():
    x = torch.tensor([[50.0, 40.0, 50.0, 45.0] * 4], device="cuda")
    bias = torch.zeros(16, device="cuda")
    assert rtn.rtn_route_experts(x, 4, score=rtn.SCORE_SIGMOID, bias=bias).experts.tolist() == [[0, 2, 4, 6]]
    bias[[9, 3, 12]] = float("inf")                             # (infinities are equal, whatever the logits)
    assert rtn.rtn_route_experts(x, 4, score=rtn.SCORE_SIGMOID, bias=bias).experts.tolist() == [[3, 9, 12, 0]]
